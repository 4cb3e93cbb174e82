"""The binding asks torch for the current device and stream by its inner functions where they are, and by its public ones where they are not (no GPU)."""
import importlib.util


def test_device_and_stream_without_the_inner_functions(monkeypatch):
    import torch

    from paper_2310_05869_amd import binding as used

    spec = importlib.util.spec_from_file_location("paper_2310_05869_amd.binding_anew", used.__file__)   # (what it asks by is decided once)
    binding = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(binding)

    class Inner:   # torch._C of a version that has neither
        pass

    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch, "_C", Inner)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: Stream)

    class Tensor:
        def get_device(self):
            return 3

    assert binding._here(Tensor(), "Q", None) == (3, 77)
