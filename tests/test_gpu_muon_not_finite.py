"""bsr_muon_step where gradients are not finite: their whole block of p ends as NaN, and no other, whatever its sides and settings."""
import numpy as np
import pytest

from gpu_util import torch_dtype

pytestmark = pytest.mark.gpu

# blocks beside one another down (bs_r <= 8) and across (bs_c <= 8), one a wavefront, and large ones, which have a workgroup each
# while there are few
SHAPES = [((16, 1), 40), ((1, 16), 40), ((61, 3), 40), ((64, 8), 40), ((5, 7), 40), ((8, 8), 40), ((3, 61), 40), ((16, 16), 40), ((24, 40), 40),
          ((64, 16), 40), ((48, 64), 40), ((33, 61), 40), ((64, 64), 40), ((64, 64), 1100), ((50, 49), 1100)]
# products of two fp16 parts; coefficients that leave them to three bf16 parts and fp32
SETTINGS = [(5, (3.4445, -4.7750, 2.0315)), (2, (0.9, -0.3, 0.1)), (0, (3.4445, -4.7750, 2.0315)), (0, (0.9, -0.3, 0.1))]


@pytest.mark.parametrize("shape,blocks", SHAPES)
@pytest.mark.parametrize("steps,abc", SETTINGS)
@pytest.mark.parametrize("nesterov", [True, False])
def test_the_whole_block_and_no_other(shape, blocks, steps, abc, nesterov):
    import torch
    import paper_2007_13055_amd as lib
    gen = torch.Generator(device="cuda").manual_seed(blocks)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    p, g = rand(blocks, *shape), rand(blocks, *shape)
    perm = np.random.default_rng(0).permutation(blocks).astype(np.int32)
    bad = g.clone()
    r, c = shape[0] - 1, shape[1] // 2
    bad[4, r, c], bad[7, 0, 0], bad[18, r, 0] = float("nan"), float("inf"), -float("inf")
    hit = [4, 7, 18]
    rest = torch.tensor([i for i in range(blocks) if i not in hit], device="cuda")
    results = []
    for grad in (g, bad):
        param, turned = p.clone(), torch.zeros((blocks, shape[1], shape[0]), device="cuda")
        opt = lib.bsr_muon_create([param], [grad.clone()], transposed=[(turned, perm)])
        lib.bsr_muon_step(opt, 1, ns_steps=steps, coefficients=abc, nesterov=nesterov)
        results.append((param, turned, opt.momentum[0].view(blocks, *shape)))
    (clean, clean_t, _), (got, got_t, momentum) = results
    assert torch.equal(got[rest], clean[rest]) and bool(clean.isfinite().all())
    assert bool(got[hit].isnan().all())
    assert torch.equal(momentum.isfinite(), bad.isfinite())              # M has them where they are
    where = torch.from_numpy(perm).cuda().long()                          # stored block q of the transpose is block perm[q]
    assert torch.equal(got_t.isnan(), got[where].transpose(1, 2).isnan()) and torch.equal(got_t[~got_t.isnan()], got[where].transpose(1, 2)[~got_t.isnan()])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("master", [True, None])
@pytest.mark.parametrize("shape", [(16, 16), (8, 8), (64, 8), (64, 64)])
def test_16_bit_parameters(shape, master, dtype):
    import torch
    import paper_2007_13055_amd as lib
    T = torch_dtype(dtype)
    p, g = torch.randn((12, *shape), device="cuda").to(T), torch.randn((12, *shape), device="cuda").to(T)
    g[5, 0, shape[1] - 1] = float("inf")
    opt = lib.bsr_muon_create([p], [g], master=master)
    for steps in (0, 5):
        lib.bsr_muon_step(opt, 1, ns_steps=steps)
        assert bool(p[5].isnan().all()) and bool(p[[0, 4, 6, 11]].isfinite().all())
        if master:
            assert bool(opt.master[0].view(12, *shape)[5].isnan().all())
