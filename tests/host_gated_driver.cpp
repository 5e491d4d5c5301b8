// Host-side check of what bsr_spmm_gated() refuses (test infrastructure; no GPU).  The handle is made up: every address is fake,
// and it names a device that does not exist, so that no call gets as far as a launch -- one that is in order ends with
// BSR_ERR_DEVICE.
// Build: hipcc -std=c++17 -I include -I paper_2007_13055_amd/csrc tests/host_gated_driver.cpp libbsr_spmm.so -o driver
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
    int failed = 0;
    size_t need = 0;
    if (bsr_spmm_gated_workspace_size(&W, m, BSR_F32, &need) != BSR_OK || need < (size_t)m * 4096 * 4) { std::printf("FAILED workspace\n"); return 1; }
    struct call { void* X; void* H; void* z; const void* bias; void* ws; size_t bytes; bsr_dtype t; bsr_act act; bsr_dtype bias_t; };
    const call right{at(0x600000000), at(0x700000000), at(0x800000000), at(0x900000000), at(0xA00000000), need, BSR_F32, BSR_ACT_SILU, BSR_F32};
    auto expect = [&](const char* what, const char* name, const call& c, bsr_status want) {
        const bsr_gated how{c.act, c.bias_t, c.bias, c.z};
        const bsr_status st = bsr_spmm_gated(&W, m, c.X, c.H, c.t, &how, c.ws, c.bytes, nullptr);
        if (st != want) { std::printf("FAILED %s %s: %d, not %d\n", what, name, (int)st, (int)want); ++failed; }
    };
    auto with = [&](auto set) { call c = right; set(c); return c; };
    expect("in order", "", right, BSR_ERR_DEVICE);
    expect("no Z", "", with([](call& c) { c.z = nullptr; }), BSR_ERR_DEVICE);
    expect("fp32 sums kept", "no workspace", with([](call& c) { c.ws = nullptr; c.bytes = 0; }), BSR_ERR_DEVICE);
    expect("no Z", "no workspace", with([](call& c) { c.z = nullptr; c.ws = nullptr; }), BSR_ERR_WORKSPACE);
    expect("no Z", "short workspace", with([](call& c) { c.z = nullptr; c.bytes -= 256; }), BSR_ERR_WORKSPACE);
    expect("X", "null", with([](call& c) { c.X = nullptr; }), BSR_ERR_NULL);
    expect("H", "null", with([](call& c) { c.H = nullptr; }), BSR_ERR_NULL);
    expect("H", "type", with([](call& c) { c.t = BSR_F16; }), BSR_ERR_DTYPE);
    expect("act", "", with([](call& c) { c.act = (bsr_act)5; }), BSR_ERR_DTYPE);
    expect("bias", "type", with([](call& c) { c.bias_t = BSR_BF16; }), BSR_ERR_DTYPE);
    expect("Z", "alignment", with([](call& c) { c.z = at(0x800000008); }), BSR_ERR_ALIGN);
    expect("workspace", "alignment", with([](call& c) { c.ws = at(0xA00000004); }), BSR_ERR_ALIGN);
    W.R = 255;
    expect("an odd number of block-rows", "", right, BSR_ERR_SHAPE);
    if (bsr_spmm_gated_workspace_size(&W, m, BSR_F32, &need) != BSR_ERR_SHAPE || need != 0) { std::printf("FAILED odd\n"); ++failed; }
    W.R = 256;
    const size_t h = (size_t)m * 2048 * 4, z = 2 * h, scratch = mfma_thin_scratch_bytes(&W, m);
    struct { const char* name; uintptr_t from; size_t bytes; } parts[] = {
        {"X", 0x600000000, (size_t)m * 2048 * 4}, {"bias", 0x900000000, 4096 * 4}, {"block_data", 0x100000000, 10000 * 64}, {"block_indices", 0x200000000, 10000 * 4},
        {"index_pointer", 0x300000000, 257 * 4}, {"workspace", 0x400000000, 1 << 20}, {"scratch", 0x500000000, scratch}};
    for (const auto& p : parts) {
        const uintptr_t last = (p.from + p.bytes - 1) & ~(uintptr_t)15, behind = (p.from + p.bytes + 15) & ~(uintptr_t)15;
        for (uintptr_t y : {p.from, last}) {
            expect("H over", p.name, with([&](call& c) { c.H = at(y); }), BSR_ERR_OVERLAP);
            expect("Z over", p.name, with([&](call& c) { c.z = at(y); }), BSR_ERR_OVERLAP);
            expect("workspace over", p.name, with([&](call& c) { c.z = nullptr; c.ws = at(y); }), BSR_ERR_OVERLAP);
        }
        expect("H behind", p.name, with([&](call& c) { c.H = at(behind); }), BSR_ERR_DEVICE);
        expect("Z before", p.name, with([&](call& c) { c.z = at(p.from - z); }), BSR_ERR_DEVICE);
    }
    expect("H over", "Z", with([&](call& c) { c.H = at(0x800000000 + z - 16); }), BSR_ERR_OVERLAP);
    expect("H over", "workspace", with([&](call& c) { c.z = nullptr; c.H = at(0xA00000000 - h + 16); }), BSR_ERR_OVERLAP);
    if (failed) return 1;
    std::printf("all refused\n");
    return 0;
}
