// Host-side check of what bsr_spmm_epilogue() refuses to write over (test infrastructure; no GPU).  The handle is made up:
// every address is fake, and it names a device that does not exist, so that no call gets as far as a launch -- one whose
// buffers are apart ends with BSR_ERR_DEVICE.
// Build: hipcc -std=c++17 -I include -I paper_2007_13055_amd/csrc tests/host_epilogue_driver.cpp libbsr_spmm.so -o driver
#include <cstdio>

#include "bsr_internal.h"

static void* at(uintptr_t v) { return reinterpret_cast<void*>(v); }

int main()
{
    constexpr int64_t m = 64;
    bsr_matrix W;
    W.n = 4096; W.k = 2048; W.bs_r = 16; W.bs_c = 1; W.R = 256; W.C = 2048; W.nnzb = 10000;
    W.dtype = BSR_F32;
    W.device = 1 << 20;
    W.data = at(0x100000000);
    W.indices = static_cast<const int32_t*>(at(0x200000000));
    W.indptr = static_cast<const int32_t*>(at(0x300000000));
    W.row_order = static_cast<const int32_t*>(at(0x400000000));
    W.workspace_bytes = 1 << 20;
    W.scratch = at(0x500000000);
    W.scratch_bytes = (size_t)1 << 30;
    void* const X = at(0x600000000);
    void* const apart_y = at(0x700000000);
    void* const apart_z = at(0x800000000);
    const size_t out = (size_t)m * 4096 * 4, scratch = mfma_thin_scratch_bytes(&W, m);
    struct { const char* name; uintptr_t from; size_t bytes; } parts[] = {
        {"X", 0x600000000, (size_t)m * 2048 * 4}, {"block_data", 0x100000000, 10000 * 64}, {"block_indices", 0x200000000, 10000 * 4},
        {"index_pointer", 0x300000000, 257 * 4}, {"workspace", 0x400000000, 1 << 20}, {"scratch", 0x500000000, scratch}};
    int failed = 0;
    auto expect = [&](const char* what, const char* name, void* y, void* z, bsr_status want) {
        bsr_epilogue e{};
        e.z_dev = z;
        const bsr_status st = bsr_spmm_epilogue(&W, m, X, y, BSR_F32, &e, nullptr);
        if (st != want) { std::printf("FAILED %s %s: %d, not %d\n", what, name, (int)st, (int)want); ++failed; }
    };
    expect("apart", "", apart_y, apart_z, BSR_ERR_DEVICE);
    if (scratch == 0) { std::printf("FAILED no scratch\n"); ++failed; }
    for (const auto& p : parts) {
        const uintptr_t last = (p.from + p.bytes - 1) & ~(uintptr_t)15, behind = (p.from + p.bytes + 15) & ~(uintptr_t)15;
        for (uintptr_t y : {p.from, last, p.from - out + 16}) {
            expect("Y over", p.name, at(y), apart_z, BSR_ERR_OVERLAP);
            expect("Z over", p.name, apart_y, at(y), BSR_ERR_OVERLAP);
        }
        expect("Y behind", p.name, at(behind), nullptr, BSR_ERR_DEVICE);
        expect("Z before", p.name, apart_y, at(p.from - out), BSR_ERR_DEVICE);
    }
    W.scratch = nullptr;                                                  // none lent
    W.scratch_bytes = 0;
    expect("no scratch", "", at(0x500000000), nullptr, BSR_ERR_DEVICE);
    if (failed) return 1;
    std::printf("all refused\n");
    return 0;
}
