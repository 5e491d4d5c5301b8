// Host-side check that numbers of rows whose product with a row's length leaves 64 bits are refused (test infrastructure; no GPU).
// The handle is made up, and names a device that does not exist; nothing may get as far as a launch.
// Build: hipcc -std=c++17 -I include -I paper_2007_13055_amd/csrc tests/host_rows_driver.cpp libbsr_spmm.so -o driver
#include <cstdio>

#include "bsr_internal.h"

static void* at(uintptr_t v) { return reinterpret_cast<void*>(v); }

int main()
{
    bsr_matrix W;
    W.n = 4096; W.k = 2048; W.bs_r = 16; W.bs_c = 1; W.R = 256; W.C = 2048; W.nnzb = 10000;
    W.dtype = BSR_F32;
    W.device = 1 << 20;
    W.data = at(0x100000000);
    W.indices = static_cast<const int32_t*>(at(0x200000000));
    W.indptr = static_cast<const int32_t*>(at(0x300000000));
    W.row_order = static_cast<const int32_t*>(at(0x400000000));
    W.workspace_bytes = 1 << 20;
    const bsr_gated gated{BSR_ACT_SILU, BSR_F32, nullptr, nullptr};
    bsr_epilogue epilogue{};
    void *const X = at(0x600000000), *const Y = at(0x700000000), *const ws = at(0x800000000);
    int failed = 0;
    auto refused = [&](const char* what, int64_t m, bsr_status st) {
        if (st != BSR_ERR_SHAPE) { std::printf("FAILED %s, %lld rows: %d\n", what, (long long)m, (int)st); ++failed; }
    };
    // a row is 4096 long: in 64 bits the products with the first are 0, 4096 and 2^18; the last is the smallest that is refused
    for (int64_t m : {(int64_t)1 << 52, ((int64_t)1 << 52) + 1, ((int64_t)1 << 62) + 64, (int64_t)1 << 31, (int64_t)1 << 19}) {
        size_t need = 7;
        refused("workspace of a gated product", m, bsr_spmm_gated_workspace_size(&W, m, BSR_F32, &need));
        if (need) { std::printf("FAILED a size beside the refusal\n"); ++failed; }
        refused("gated product", m, bsr_spmm_gated(&W, m, X, Y, BSR_F32, &gated, ws, SIZE_MAX, nullptr));
        refused("product with an epilogue", m, bsr_spmm_epilogue(&W, m, X, Y, BSR_F32, &epilogue, nullptr));
        refused("sampled product", m, bsr_sddmm_ws(&W, m, Y, X, ws, BSR_F32, nullptr, 0, nullptr));
        refused("product", m, bsr_spmm_ex(&W, m, X, Y, BSR_F32, BSR_PATH_AUTO, nullptr));
    }
    size_t need = 0;
    if (bsr_spmm_gated_workspace_size(&W, ((int64_t)1 << 19) - 1, BSR_F32, &need) != BSR_OK) { std::printf("FAILED most rows\n"); ++failed; }
    if (failed) return 1;
    std::printf("all refused\n");
    return 0;
}
