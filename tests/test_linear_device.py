"""The wrappers of packmamba_linear.h call the library with their tensors' GPU current, on the CPU: a call for the
current GPU as it is, one for another inside of a device guard that ends with it, also where the call fails."""
import contextlib

import pytest


@pytest.mark.parametrize("current,status", [(0, 0), (1, 0), (0, 2), (1, 2)])
def test_call_is_made_on_the_tensors_gpu(monkeypatch, current, status):
    import torch
    from paper_2408_03865_amd import PackMambaError, linear
    now, seen = [current], []

    @contextlib.contextmanager
    def guard(device):
        old, now[0] = now[0], device.index
        try:
            yield
        finally:
            now[0] = old

    class Library:
        @staticmethod
        def packmamba_test(*args):
            seen.append((now[0], args))
            return status

        @staticmethod
        def packmamba_status_string(st):
            return b"of the test"

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", guard)
    monkeypatch.setattr(linear, "load", Library)
    monkeypatch.setattr(linear._lib, "load", Library)
    with pytest.raises(PackMambaError) if status else contextlib.nullcontext():
        linear._call(torch.device("cuda", 0), "packmamba_test", 1, 2)
    assert seen == [(0, (1, 2))] and now[0] == current
