"""Products on another stream: what happens to the tensors of a matrix that is dropped behind them."""
import numpy as np
import pytest

import workloads as wl
from gpu_util import to_device

pytestmark = pytest.mark.gpu


def _spans(tensors):
    return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors]


SQUARE, THIN = (200, 256, 512, 16, 16, "bf16"), (200, 512, 512, 16, 1, "f32")


@pytest.mark.parametrize("shape,what", [(s, w) for s in (SQUARE, THIN) for w in ("spmm", "epilogue", "sddmm")] + [(THIN, "static")],
                         ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v)))
def test_dropped_while_a_product_on_another_stream_is_still_to_run(shape, what):
    import torch
    import paper_2007_13055_amd as lib
    m, k, n, bs_r, bs_c, dtype = shape
    rng = np.random.default_rng(2)
    p = wl.make_problem("streams", m, k, n, bs_r, bs_c, dtype, dtype, ("counts", rng.binomial(k // bs_c, 0.3, size=n // bs_r)),
                        ("normal", 0.3), ("normal", 1.0), 2)
    X = to_device(p.X, dtype)
    G = torch.randn((m, n), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(X.dtype)

    def make():
        return lib.bsr_create(p.n, p.k, p.block_data, p.block_indices, p.index_pointer, dtype=dtype)

    def run(W):
        if what == "spmm":
            return lib.bsr_spmm(W, X)
        if what == "epilogue":
            return lib.bsr_spmm_epilogue(W, X, act="silu", residual=G)
        if what == "sddmm":
            return lib.bsr_sddmm(W, G, X)
        return lib.bsr_spmm_static(W, X, torch.empty((m, n), device="cuda"))

    W, one = make(), make()
    run(W)                                                                # its plans are built
    want = run(one)
    room = [torch.empty(1 << s, dtype=torch.uint8, device="cuda") for s in range(9, 22) for _ in range(6)]
    del room                                                              # so that nothing below asks the driver for memory
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                                    # a tenth of a second and more
        got = run(W)
    own = [t for t in (*W._tensors, W._scratch) if t is not None]
    sizes, held = [(t.numel(), t.dtype) for t in own], _spans(own)
    del W, own
    new = [torch.empty(c, dtype=t, device="cuda") for c, t in sizes for _ in range(2)]   # (not written to)
    still_to_run = not side.query()
    taken = [a for a in _spans(new) for b in held if a[0] < b[1] and b[0] < a[1]]
    torch.cuda.synchronize()
    assert still_to_run and not taken
    assert torch.equal(got, want)
