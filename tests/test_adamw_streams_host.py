"""What a list's owner tells the allocator when its steps run on other streams than the one its buffers were made on."""
import pytest


@pytest.fixture
def recorded(monkeypatch):
    """[(tensor, stream)] of every record_stream, no GPU needed."""
    import torch
    calls = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: calls.append((id(t), s)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "side")
    return calls


def test_every_buffer_is_recorded_once_a_stream(recorded):
    import numpy as np
    import torch
    from paper_2007_13055_amd.binding import BsrAdamW
    new = lambda: torch.zeros(4)  # noqa: E731
    opt = BsrAdamW(8, [new(), new()], [new(), new()], [new(), None], [new(), new()], [new(), new()], [new(), new()])
    copy, workspace = new(), new()
    opt._keep += [copy, np.arange(3), workspace]
    opt._on_stream(77)
    want = {id(t) for held in (opt.params, opt.grads, opt.exp_avg, opt.exp_avg_sq, opt.scales) for t in held} | {id(opt.master[0]), id(copy), id(workspace)}
    assert {t for t, _ in recorded} == want and len(recorded) == len(want) and {s for _, s in recorded} == {"side"}
    opt._on_stream(77)
    assert len(recorded) == len(want)
    opt._on_stream(78)
    assert len(recorded) == 2 * len(want)
