"""The operators' wrappers without a GPU: tensors in host memory that say they are on a device, and a library that notes what it is told."""
import torch


class OnDevice(torch.Tensor):
    is_cuda = True


def on_device(t):
    return t.as_subclass(OnDevice)


class RecordingLibrary:
    """Takes the calls of gated units and dropout; `calls` has (name, description) of each, the description a copy of its own."""

    def __init__(self):
        self.calls, self.rules = [], []

    def pbt_gated_query_workspace(self, desc, backward, nbytes):
        return 0

    def pbt_last_error(self, handle):
        return b""

    def _note(self, name, desc, rule):
        copy = type(desc).from_buffer_copy(desc)
        self.calls.append((name, copy))
        self.rules.append(None if rule is None else type(rule).from_buffer_copy(rule))
        return 0

    def _gated(self, name, desc):
        from paper_1711_09846_b200.binding import PbtDropRule
        return self._note(name, desc, PbtDropRule.from_address(desc.drop) if desc.drop else None)

    def pbt_gated_forward(self, desc, workspace, nbytes, stream):
        return self._gated("forward", desc)

    def pbt_gated_backward(self, desc, workspace, nbytes, stream):
        return self._gated("backward", desc)

    def pbt_dropout(self, desc, stream):
        return self._note("dropout", desc, desc.rule)


class _Stream:
    def synchronize(self):
        pass


def install(monkeypatch):
    """The recording library in the place of the built one, for the test that asks."""
    from paper_1711_09846_b200 import operators
    lib = RecordingLibrary()
    monkeypatch.setattr(operators, "load_library", lambda: lib)
    monkeypatch.setattr(operators, "_current_stream", lambda index: 0)
    monkeypatch.setattr(operators, "_current_device", lambda: None)
    monkeypatch.setattr(operators, "_allocate", lambda nbytes, stream: 4096)
    monkeypatch.setattr(operators, "_release", lambda at: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: _Stream())
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    return lib
