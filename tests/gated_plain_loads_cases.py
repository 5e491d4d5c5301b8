"""Gated products through every kernel that finishes them and places waits by hand: these are compiled apart from the plain ones.

Run as a script: python tests/gated_plain_loads_cases.py <library.so> <out.npz>"""
import os
import sys

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
for d in (os.path.dirname(HERE), HERE):
    if d not in sys.path:
        sys.path.insert(0, d)


def cases():
    """(name, BSR_SPMM_TUNE, gate, up, rows of X, type, result's type)"""
    import workloads as wl
    out = []

    def add(tune, bs_r, bs_c, m, dtype, h, R=10, C=16):
        rng = np.random.default_rng(bs_r + bs_c + m)
        pair = []
        for i in range(2):
            counts = rng.integers(0, 9, size=R)
            counts[2 + i], counts[5 - i] = 0, C
            pair.append(wl.make_problem("gated loads", 4, C * bs_c, R * bs_r, bs_r, bs_c, dtype, dtype, ("counts", counts), ("normal", 0.3), ("normal", 1.0), 60 + i))
        out.append((f"{tune} {bs_r}x{bs_c} {m} {dtype} {h}", tune, *pair, m, dtype, h))

    for bs_r in (32, 64):                              # tile kernel: every block shape and type, one block in flight and two
        for bs_c in (16, 32, 64):
            for dtype, h in (("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")):
                for depth in (1, 2):
                    add(f"variant=3,a={depth}", bs_r, bs_c, 300, dtype, h)
    for bs_r, bs_c in ((16, 16), (16, 64), (32, 16), (32, 32), (64, 32), (64, 64)):   # k-split kernel: both tiles, strips
        for dtype, h in (("f32", "f32"), ("f16", "f32"), ("bf16", "bf16")):
            for mt in (1,) if bs_r == 16 else (1, 2, 3):
                add(f"variant=2,mt={mt}", bs_r, bs_c, 70, dtype, h)
    for bs_r, bs_c, dtype, h in ((8, 8, "f32", "f32"), (8, 16, "bf16", "bf16"), (16, 8, "f16", "f32"), (16, 16, "bf16", "bf16")):   # sweep kernel
        for mt in (1, 2, 4):
            add(f"variant=6,mt={mt}", bs_r, bs_c, 300, dtype, h, R=32, C=40)
    return out


def run_cases():
    """{case name: [Z's halves and H side by side, in fp32]} of whichever library the binding has loaded."""
    import torch
    import paper_2007_13055_amd as lib
    from gpu_util import to_device
    results = {}
    for name, tune, gate, up, m, dtype, h in cases():
        os.environ["BSR_SPMM_TUNE"] = tune
        try:
            arrays = lib.bsr_gated_arrays(*((p.block_data, p.block_indices, p.index_pointer) for p in (gate, up)))
            W = lib.bsr_create(2 * gate.n, gate.k, *arrays, dtype=dtype)
        finally:
            os.environ.pop("BSR_SPMM_TUNE", None)
        rng = np.random.default_rng(len(name))
        X, bias = to_device(rng.normal(size=(m, gate.k)), dtype), to_device(rng.normal(size=2 * gate.n) * 0.3, "f32")
        H, Z = lib.bsr_spmm_gated(W, X, h_dtype=h, bias=bias, act="silu", keep_z=True)
        torch.cuda.synchronize()
        results[name] = torch.cat((Z, H), 1).float().cpu().numpy()
    return results


if __name__ == "__main__":
    import paper_2007_13055_amd.binding as binding
    binding._LIB_PATH = os.path.abspath(sys.argv[1])
    print("library", binding.library_path(), flush=True)
    np.savez(sys.argv[2], **run_cases())
    print("done", flush=True)
