"""Settings of a step that are refused before the handle or any device is looked at (the handle is made up)."""
import ctypes

import pytest

SHAPE = 2


@pytest.mark.parametrize("kw", [dict(grad_scale=v) for v in (float("nan"), float("inf"), -float("inf"), 2.0 ** 41, -2.0 ** 41, 2.0 ** -41, 1e-44)] +
                         [dict(step=0), dict(step=-1), dict(beta1=1.0), dict(beta2=-0.5), dict(beta2=float("nan")), dict(eps=-1e-9),
                          dict(lr=-1e-3), dict(lr=float("nan"))])
def test_out_of_range(kw):
    import os
    from paper_2007_13055_amd import binding as b
    if not os.path.exists(b.library_path()):
        from paper_2007_13055_amd import build
        build.build()
    nowhere = ctypes.create_string_buffer(4096)
    hyper = b.AdamWHyper(**dict(dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, grad_scale=1.0), **kw))
    assert b.load_library().bsr_adamw_step(ctypes.addressof(nowhere), ctypes.byref(hyper), None) == SHAPE
