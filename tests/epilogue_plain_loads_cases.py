"""The cases of plain_loads_cases.py with an epilogue: the same kernels are compiled a second time for it.

Run as a script: python tests/epilogue_plain_loads_cases.py <library.so> <out.npz>"""
import os
import sys

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
for d in (os.path.dirname(HERE), HERE):
    if d not in sys.path:
        sys.path.insert(0, d)


def run_cases():
    """{case name: its sums and results in fp32} of whichever library the binding has loaded."""
    import torch
    import paper_2007_13055_amd as lib
    import plain_loads_cases as plc
    from gpu_util import to_device
    results = {}
    for name, tune, p in plc.cases():
        if tune:
            os.environ["BSR_SPMM_TUNE"] = tune
        try:
            W = lib.bsr_create(p.n, p.k, p.block_data, p.block_indices, p.index_pointer, dtype=p.in_dtype)
        finally:
            os.environ.pop("BSR_SPMM_TUNE", None)
        rng = np.random.default_rng(len(name))
        bias, R = to_device(rng.normal(size=p.n), "f32"), to_device(rng.normal(size=(p.m, p.n)), "f32")
        Y, Z = lib.bsr_spmm_epilogue(W, to_device(p.X, p.in_dtype), y_dtype="f32", bias=bias, act="silu", residual=R, keep_z=True)
        torch.cuda.synchronize()
        results[name] = np.stack([Z.cpu().numpy(), Y.cpu().numpy()])
    return results


if __name__ == "__main__":
    import paper_2007_13055_amd.binding as binding
    binding._LIB_PATH = os.path.abspath(sys.argv[1])
    print("library", binding.library_path(), flush=True)
    np.savez(sys.argv[2], **run_cases())
    print("done", flush=True)
