"""What a matrix's owner tells the allocator when products run on other streams than the one its tensors were made on."""
import types


def _stream(address):
    return types.SimpleNamespace(cuda_stream=address)


def test_every_tensor_is_recorded_once_a_stream(monkeypatch):
    import torch
    from paper_2007_13055_amd.binding import BsrMatrix
    calls, now = [], [_stream(7)]
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: calls.append((id(t), s.cuda_stream)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[0])
    W = object.__new__(BsrMatrix)
    W.handle = None
    W._tensors, W._scratch, W._streams = tuple(torch.zeros(4) for _ in range(4)), None, {0: _stream(0)}
    W._on_stream(0)                                                       # the home stream
    assert calls == []
    W._on_stream(7)
    assert calls == [(id(t), 7) for t in W._tensors]
    W._on_stream(7)
    assert len(calls) == 4
    now[0], W._scratch = _stream(9), torch.zeros(4)
    W._on_stream(9)
    assert calls[4:] == [(id(t), 9) for t in (*W._tensors, W._scratch)] and list(W._streams) == [0, 7, 9]
    W._on_stream(11)                                                      # not the current stream of its device
    assert len(calls) == 9 and 11 not in W._streams


def test_scratch_is_recorded_on_every_stream_known(monkeypatch):
    import torch
    from paper_2007_13055_amd import binding
    calls, lent = [], []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: calls.append((t.numel(), s.cuda_stream)))
    monkeypatch.setattr(binding, "bsr_scratch_size", lambda W, m: 100 * m)
    monkeypatch.setattr(binding, "load_library", lambda: types.SimpleNamespace(bsr_set_scratch=lambda *a: 0))
    W = object.__new__(binding.BsrMatrix)
    W.handle, W._core = None, types.SimpleNamespace(lent=lent.append)
    W._tensors, W._scratch, W._streams = (torch.zeros(4),), None, {0: _stream(0), 7: _stream(7)}
    W.ensure_scratch(2)
    W.ensure_scratch(1)
    W.ensure_scratch(3)
    assert calls == [(200, 0), (200, 7), (300, 0), (300, 7)] and lent == [200, 300]
