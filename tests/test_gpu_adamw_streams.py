"""AdamW steps on other streams: what happens to the buffers of a list that is dropped behind them."""
import pytest

pytestmark = pytest.mark.gpu


def _spans(tensors):
    return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("what", ["step", "moments"])
def test_dropped_while_work_on_another_stream_is_still_to_run(bits, what):
    """Its tables, moments and master copies are no one else's before that work is done."""
    import torch
    import paper_2007_13055_amd as lib
    T = torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(1)
    params = [torch.randn(c, generator=gen, device="cuda").to(T) for c in (5000, 300000)]
    grads = [torch.randn_like(p) for p in params]
    twin = [p.clone() for p in params]
    one = lib.bsr_adamw_create(twin, grads, state_bits=bits, master=True)
    opt = lib.bsr_adamw_create(params, grads, state_bits=bits, master=True)
    for o in (one, opt):
        lib.bsr_adamw_step(o, 1)
    want = lib.bsr_adamw_moments(one)
    out = [(torch.zeros_like(m), torch.zeros_like(v)) for m, v in want]
    room = [torch.empty(300000 * 4, dtype=torch.uint8, device="cuda") for _ in range(24)] + [torch.empty(4096, device="cuda") for _ in range(24)]
    del room                                                              # so that nothing below asks the driver for memory
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                                    # a tenth of a second and more
        if what == "step":
            lib.bsr_adamw_step(opt, 2)
        else:
            lib.bsr_adamw_moments(opt, out=out)
    own = [t for t in opt._keep if isinstance(t, torch.Tensor)] + opt.exp_avg + opt.exp_avg_sq + opt.master + [t for t in opt.scales if t is not None]
    sizes, held = [(t.numel(), t.dtype) for t in own], _spans(own)
    del opt, own, o
    new = [torch.empty(n, dtype=t, device="cuda") for n, t in sizes for _ in range(2)]   # (not written to)
    still_to_run = not side.query()
    taken = [a for a in _spans(new) for b in held if a[0] < b[1] and b[0] < a[1]]
    torch.cuda.synchronize()
    assert still_to_run and not taken
    if what == "step":
        lib.bsr_adamw_step(one, 2)
        assert all(torch.equal(p, q) for p, q in zip(params, twin))
    else:
        assert all(torch.equal(a, b) for pair, pair2 in zip(out, want) for a, b in zip(pair, pair2))


def test_on_two_streams_in_turn():
    """Steps on the home stream and two others, each ordered behind the one before, and captured on a fourth."""
    import torch
    import paper_2007_13055_amd as lib
    p, q = (torch.ones(10000, device="cuda") for _ in range(2))
    g = torch.full((10000,), 0.5, device="cuda")
    opt, one = lib.bsr_adamw_create([p], [g]), lib.bsr_adamw_create([q], [g])
    streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    before = streams[0]
    for t in range(1, 10):
        s = streams[t % 3]
        s.wait_stream(before)
        with torch.cuda.stream(s):
            lib.bsr_adamw_step(opt, t)
        before = s
    torch.cuda.synchronize()
    number = torch.ones(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.bsr_adamw_step(opt, number, lr=1e-3)
    for t in range(1, 10):
        lib.bsr_adamw_step(one, t)
    torch.cuda.synchronize()
    assert torch.equal(p, q)
    for t in (10, 11):
        number.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        lib.bsr_adamw_step(one, number, lr=1e-3)
        torch.cuda.synchronize()
        assert torch.equal(p, q), t
