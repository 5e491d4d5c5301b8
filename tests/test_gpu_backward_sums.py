"""The bias's gradient as a sum that has one value only: whole numbers whose partial sums fp32 holds exactly, so that a row, a chunk
of rows or a lane's share that is left out or added twice shows, whatever the order of the additions."""
import pytest

pytestmark = pytest.mark.gpu


def _whole(m, n, dtype, seed):
    """Whole numbers from -8 to 8; every 16-bit type holds them."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-8, 9, (m, n), generator=gen, device="cuda", dtype=torch.int8).to(getattr(torch, dtype))


def _sum(t, rows=8192):
    """Of each column, in whole numbers."""
    import torch
    total = torch.zeros(t.shape[1], dtype=torch.int64, device="cuda")
    for i in range(0, t.shape[0], rows):
        total += t[i:i + rows].to(torch.int64).sum(0)
    return total


SHAPES = [(1, 1), (1, 2081), (2, 8), (15, 16), (16, 17), (17, 128), (63, 129), (64, 64), (127, 1000), (255, 513), (257, 3), (1000, 1), (1025, 2048),
          (4096, 31), (4097, 256), (16384, 40), (100003, 5), (65537, 136), (1000000, 1)]


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("types", [("float32", "f32"), ("float32", "f16"), ("float16", "f16"), ("bfloat16", "bf16")])
def test_every_row_once(m, n, types):
    import torch
    import paper_2007_13055_amd as lib
    dtype, out = types
    assert 8 * m < 2 ** 24                                                # no partial sum is beyond what fp32 holds exactly
    G = _whole(m, n, dtype, m + n)
    Z = torch.randn((m, n), generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").to(G.dtype)
    none, db = lib.bsr_epilogue_backward(G, need_dz=False)
    assert none is None and torch.equal(db.to(torch.int64), _sum(G))
    dz, db = lib.bsr_epilogue_backward(G, Z, "relu", dz_dtype=out)
    masked = torch.where(Z > 0, G, torch.zeros_like(G))
    assert torch.equal(dz, masked.to(dz.dtype)) and torch.equal(db.to(torch.int64), _sum(masked))
    one = torch.zeros_like(G)
    one[m - 1] = 1                                                        # the last row alone
    assert bool((lib.bsr_epilogue_backward(one, need_dz=False)[1] == 1).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_beyond_32_bits(dtype):
    """More than 2^31 elements: 263147 rows of 8192, in chunks of 4112 rows and a shorter last one."""
    import torch
    import paper_2007_13055_amd as lib
    m, n = 262144 + 1003, 8192
    G = _whole(m, n, dtype, 3)
    _, db = lib.bsr_epilogue_backward(G, need_dz=False)
    assert torch.equal(db.to(torch.int64), _sum(G))
    Z = torch.empty_like(G).normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    _, db = lib.bsr_epilogue_backward(G, Z, "relu", need_dz=False)
    G[Z <= 0] = 0
    assert torch.equal(db.to(torch.int64), _sum(G))
