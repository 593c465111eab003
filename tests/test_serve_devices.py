"""Helpers whose first argument may be None run with their tensors' device
current: on the CPU, with tensors that say they are on another device."""
import pytest
import torch


class Far(torch.Tensor):
    """A CPU tensor that says it is on device 1."""

    def get_device(self):
        return 1


def far(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Far)


@pytest.fixture
def seen(monkeypatch):
    """Devices that were current when an entry was called; 0 is where the caller is."""
    from paper_2011_14504_amd import iseg
    now, calls = [0], []

    class Device:
        def __init__(self, i):
            self.i = i

        def __enter__(self):
            now.append(self.i)

        def __exit__(self, *a):
            now.pop()

    monkeypatch.setattr(iseg, "_raw_device", lambda: now[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(iseg, "_scratch", lambda x, n: None)
    for name in ("iseg_qk_norm_rope_fwd", "iseg_qk_norm_rope_bwd"):
        monkeypatch.setattr(iseg, name, lambda *a: calls.append(now[-1]))
    return iseg, calls


def test_queries_or_keys_alone(seen):
    iseg, calls = seen
    x, pos, freq = far(3, 2, 8), far(3, dtype=torch.int32), far(4)
    iseg.qk_norm_rope_fwd(x, None, pos, freq)
    iseg.qk_norm_rope_fwd(None, x, pos, freq)
    iseg.qk_norm_rope_fwd(q=None, k=x, positions=pos, inv_freq=freq)
    iseg.qk_norm_rope_fwd(positions=pos, inv_freq=freq, k=x, q=x)
    iseg.qk_norm_rope_fwd(None, x, None, None)
    iseg.qk_norm_rope_bwd(x, None, x, None, pos, freq)
    iseg.qk_norm_rope_bwd(None, x, None, x, pos, freq)
    iseg.qk_norm_rope_bwd(dyq=None, dyk=x, q=None, k=x, positions=pos, inv_freq=freq, gamma_k=far(8))
    assert calls == [1] * 8


def test_tensors_on_two_devices_are_refused(seen):
    iseg, calls = seen
    x = far(3, 2, 8)
    for other in (dict(positions=torch.zeros(3, dtype=torch.int32), inv_freq=far(4)), dict(positions=far(3, dtype=torch.int32), inv_freq=torch.zeros(4)),
                  dict(positions=None, inv_freq=None, gamma_k=torch.zeros(8))):
        with pytest.raises(ValueError, match="expected"):
            iseg.qk_norm_rope_fwd(None, x, **other)
    assert not calls
