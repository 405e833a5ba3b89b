"""The Python binding's own host work, without a GPU."""
import types

import pytest
import torch

from paper_2510_13161_b200 import binding


def test_accept_result_follows_its_tensors():
    """The addresses handed to the library are those of the tensors as they are now, however they came to lie elsewhere."""
    out = binding.AcceptResult(2, 3, "cpu")
    current = lambda: [getattr(out, f).data_ptr() for f, _ in binding.AcceptOut._fields_]        # noqa: E731
    passed = lambda: [getattr(out.struct(), f) for f, _ in binding.AcceptOut._fields_]           # noqa: E731
    assert passed() == current()
    out.emitted = torch.empty((2, 4), dtype=torch.int32)
    assert passed() == current()
    out.n_accepted.resize_(1 << 16)
    assert passed() == current()
    out.reuse_slot.set_(torch.empty(7, dtype=torch.int32))
    assert passed() == current()
    out.decide_row.data = torch.empty(5, dtype=torch.int32)
    assert passed() == current()


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_current_stream_without_torchs_private_names(missing, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 11 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=22))
    assert binding._stream(None) == 14 and binding._stream(types.SimpleNamespace(cuda_stream=33)) == 33
    monkeypatch.delattr(torch._C, missing)
    assert binding._stream(None) == 22


def test_a_workspace_that_a_captured_call_uses_outlives_its_successor(monkeypatch):
    """A graph goes on writing to the workspace that its calls were captured with: a larger one must not set it free.  One that no graph uses
    is given back, behind the stream that may still be using it."""
    import gc
    import weakref

    class Workspace(torch.Tensor):
        def record_stream(self, s):
            given_back.append(s)
    given_back, need, capturing = [], [100], [False]
    m = object.__new__(binding.Mirror)
    m.lib = types.SimpleNamespace(mirror_workspace_bytes=lambda ctx, tree, kv, what, out: setattr(out._obj, "value", need[0]) or 0,
                                  mirror_set_workspace=lambda ctx, p, n: 0)
    m._ctx, m.device, m._ws, m._ws_captured, m._old_ws, m._need = None, torch.device("cpu"), None, False, [], {}
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(Workspace))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "s")
    kept, left = [], []
    for step, (n, captured) in enumerate([(100, False), (300, False), (200, True), (400, False), (500, False)]):
        need[0], capturing[0] = n, captured
        m.ensure_workspace(binding.Tree(1, 1 + step, 1, 1, None, None), None, 1)
        assert m._ws.numel() >= n
        (kept if captured else left).append(weakref.ref(m._ws))
    gc.collect()
    assert [w() is not None for w in kept] == [True]                       # (300 bytes, captured in the third step)
    assert [w() is not None for w in left] == [False, True, False, True]
    assert given_back == ["s", "s"]
