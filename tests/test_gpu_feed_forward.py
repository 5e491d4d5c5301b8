"""The operators of a gated feed-forward block as a training loop runs them: norm, gated pair, projection back, norms around the
residual, all their gradients, and the step of both matrices with their transposed copies."""
import numpy as np
import pytest
import torch

import workloads as wl
from gpu_util import to_device

pytestmark = pytest.mark.gpu

M, D, HIDDEN, UNIT, EPS = 200, 128, 256, 16, 1e-6
VECTORS = ("before", "post", "gate", "after")


class Block:
    """The block's tensors in fp32, made from a seed; step() is one pass over all of it."""

    def __init__(self, seed):
        import paper_2007_13055_amd as lib
        self.lib = lib
        make = lambda k, n, s: wl.make_problem("block", 4, k, n, UNIT, UNIT, "f32", "f32", ("bernoulli", 0.4), ("normal", 0.3), ("normal", 1.0), s)  # noqa: E731
        self.halves, self.down = (make(D, HIDDEN, seed), make(D, HIDDEN, seed + 1)), make(HIDDEN, D, seed + 2)
        arrays = lib.bsr_gated_arrays(*((p.block_data, p.block_indices, p.index_pointer) for p in self.halves))
        two = (2 * HIDDEN, D, *arrays), (D, HIDDEN, self.down.block_data, self.down.block_indices, self.down.index_pointer)
        self.patterns = [(n, k, idx, ptr) for n, k, _, idx, ptr in two]
        self.W = [lib.bsr_create(*a, dtype="f32") for a in two]
        self.WT = [lib.bsr_create_transposed(*a, dtype="f32") for a in two]
        perms = [lib.bsr_transpose_pattern(n, k, UNIT, UNIT, ptr, idx)[2] for n, k, idx, ptr in self.patterns]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s, scale=1.0, shift=0.0: torch.randn(s, generator=gen, device="cuda") * scale + shift  # noqa: E731
        self.S, self.GS, self.GU = normal(M, D, scale=2.0), normal(M, D), normal(M, D)
        self.bias = normal(2 * HIDDEN, scale=0.3)
        self.vectors = {k: normal(D, scale=0.2, shift=1.0) for k in VECTORS}
        self.grads = [torch.empty_like(w.block_data) for w in self.W]
        self.opt = lib.bsr_muon_create([w.block_data for w in self.W], self.grads, weight_decay=0.1, transposed=list(zip(self.WT, perms)))
        self.number = torch.zeros(1, dtype=torch.int64, device="cuda")

    def settings(self):
        return dict(post="rms", pre="rms", post_weight=self.vectors["post"], gate=self.vectors["gate"], pre_weight=self.vectors["after"], eps=EPS,
                    branch_scale=0.5)

    def step(self, number):
        lib, (W1, W2), (T1, T2) = self.lib, self.W, self.WT
        _, U = lib.bsr_residual_norm(self.S, pre_weight=self.vectors["before"], eps=EPS, need_sum=False)
        H, Z = lib.bsr_spmm_gated(W1, U, bias=self.bias, act="silu", keep_z=True)
        B = lib.bsr_spmm(W2, H)
        total, after = lib.bsr_residual_norm(self.S, B, **self.settings())
        ds, db, sums = lib.bsr_residual_norm_backward(total, B, self.GS, self.GU, **self.settings())
        lib.bsr_sddmm(W2, db, H, self.grads[1])
        dz, dbias = lib.bsr_gated_backward(lib.bsr_spmm(T2, db), Z, UNIT, "silu")
        lib.bsr_sddmm(W1, dz, U, self.grads[0])
        ds, _, first = lib.bsr_residual_norm_backward(self.S, None, ds, lib.bsr_spmm(T1, dz), pre_weight=self.vectors["before"], eps=EPS)
        out = {"total": total, "after": after, "dS": ds, "bias": dbias, "before": first["pre_weight"], "post": sums["post_weight"], "gate": sums["gate"],
               "vafter": sums["pre_weight"], "W1": self.grads[0], "W2": self.grads[1]}
        lib.bsr_muon_step(self.opt, number, lr=0.02)
        return out

    def formulas(self, T):
        """step()'s results in T, gradients by differentiation, on the CPU."""
        S, v = self.S.to("cpu", T).requires_grad_(), {k: x.to("cpu", T).requires_grad_() for k, x in self.vectors.items()}
        bias, data, dense = self.bias.to("cpu", T).requires_grad_(), [], []
        for w, (n, k, idx, ptr) in zip(self.W, self.patterns):
            blocks = w.block_data.detach().to("cpu", T).requires_grad_()
            rows, cols = torch.from_numpy(np.repeat(np.arange(n // UNIT), np.diff(ptr))), torch.from_numpy(np.asarray(idx, dtype=np.int64))
            grid = torch.zeros((n // UNIT, k // UNIT, UNIT, UNIT), dtype=T).index_put((rows, cols), blocks)
            data.append(blocks)
            dense.append(grid.permute(0, 2, 1, 3).reshape(n, k))
        rms = lambda x, w: x / ((x * x).mean(1, keepdim=True) + EPS).sqrt() * w  # noqa: E731
        z = (rms(S, v["before"]) @ dense[0].t() + bias).view(M, -1, 2, UNIT)
        h = (z[:, :, 0] * torch.sigmoid(z[:, :, 0]) * z[:, :, 1]).reshape(M, HIDDEN)
        total = S + 0.5 * v["gate"] * rms(h @ dense[1].t(), v["post"])
        after = rms(total, v["after"])
        loss = (total * self.GS.to("cpu", T)).sum() + (after * self.GU.to("cpu", T)).sum()
        names = ("dS", "bias", "before", "post", "gate", "vafter", "W1", "W2")
        given = (S, bias, v["before"], v["post"], v["gate"], v["after"], *data)
        return {"total": total.detach(), "after": after.detach(), **dict(zip(names, torch.autograd.grad(loss, given)))}


def test_a_block_and_its_gradients():
    """As exact as the same chain in plain fp32 arithmetic: the same sums in another order and two functions (exponential,
    reciprocal) of up to four times its error, so 4 times its root mean square and 16 times its largest error."""
    block = Block(1)
    want, plain = block.formulas(torch.float64), block.formulas(torch.float32)
    copies = [w.block_data.clone() for w in block.W]
    got = block.step(1)
    for name, x in want.items():
        y, ref = got[name].cpu().double().reshape(x.shape), plain[name].double() - x
        err, floor = y - x, 2.0 ** -22 * float(x.pow(2).mean().sqrt())
        assert float(err.pow(2).mean().sqrt()) <= 4 * float(ref.pow(2).mean().sqrt()) + floor, name
        assert float(err.abs().max()) <= 16 * float(ref.abs().max()) + 4 * floor, name
    for w, t, before, pattern in zip(block.W, block.WT, copies, block.patterns):
        n, k, idx, ptr = pattern
        perm = torch.from_numpy(np.asarray(block.lib.bsr_transpose_pattern(n, k, UNIT, UNIT, ptr, idx)[2], dtype=np.int64)).cuda()
        assert not torch.equal(w.block_data, before)
        assert torch.equal(t.block_data.view(-1, UNIT, UNIT), w.block_data.view(-1, UNIT, UNIT)[perm].transpose(1, 2))


def test_steps_replayed_from_a_graph():
    """The whole step recorded once: every replay gives what the same step gives eagerly, with eager work between them."""
    block, twin = Block(2), Block(2)
    block.step(1)                                     # (plans and tables of first calls)
    twin.step(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = block.step(block.number)
    for t in range(2, 6):
        for b in (block, twin):
            b.S.add_(0.01 * t)
        block.number.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        want = twin.step(t)
        for name, x in want.items():
            assert torch.equal(held[name], x), (t, name)
        for one, other in zip(block.W + block.WT, twin.W + twin.WT):
            assert torch.equal(one.block_data, other.block_data), t
    assert bool(want["after"].isfinite().all())
