"""Sizes of workspaces that the binding makes itself: asked for the device of the tensors, with that device as the current one, whichever
device was asked about before."""
import contextlib

import pytest


class Devices:
    """Two devices of different SM counts behind the library's size functions."""

    def __init__(self):
        self.now, self.asked = 0, []

    def _cuda_getDevice(self):
        return self.now

    def __getattr__(self, name):
        def size(*args):
            self.asked.append((name, self.now, args))
            return (148, 132)[self.now] * 1000 + args[1]
        return size

    @contextlib.contextmanager
    def device(self, dev):
        before, self.now = self.now, dev
        yield
        self.now = before


@pytest.mark.parametrize("name", ["psrl_rms_norm_workspace_bytes", "psrl_linear_workspace_bytes", "psrl_token_logprob_workspace_bytes"])
def test_sizes_go_by_the_tensors_device(lib, monkeypatch, name):
    fake = Devices()
    torch = type("torch", (), {"cuda": fake})
    monkeypatch.setattr(lib, "lib", lambda: fake)
    monkeypatch.setattr(lib, "_cuda", lambda: fake)
    monkeypatch.setattr(lib, "_torch", lambda: torch)
    lib._workspace_bytes.cache_clear()
    try:
        for _ in range(2):
            assert lib._workspace_bytes(name, 0, 1, 7) == 148007      # the current device
            assert lib._workspace_bytes(name, 1, 1, 7) == 132007      # another one
        fake.now = 1
        assert lib._workspace_bytes(name, 0, 1, 7) == 148007 and lib._workspace_bytes(name, 1, 1, 7) == 132007
        assert fake.now == 1 and fake.asked == [(name, 0, (1, 7)), (name, 1, (1, 7))]
    finally:
        lib._workspace_bytes.cache_clear()


def test_the_wrappers_name_the_tensors_device(lib, monkeypatch):
    """Stand-ins for tensors on device 1 while 0 is current: what each wrapper asks for, up to the launch."""
    asked = []
    monkeypatch.setattr(lib, "_workspace_bytes", lambda name, dev, *args: asked.append((name, dev, args)) or 512)

    class Stop(Exception):
        pass

    def scratch(*args):
        raise Stop

    monkeypatch.setattr(lib, "_scratch", scratch)
    monkeypatch.setattr(lib, "Workspace", scratch)
    monkeypatch.setattr(lib, "_stream_on", lambda stream, dev: (0, None))
    import torch

    class T:
        def __init__(self, *shape, dtype=torch.float32):
            self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device("cuda", 1), True

        def dim(self):
            return len(self.shape)

        def stride(self, i=None):
            s = [1] * len(self.shape)
            for j in range(len(s) - 2, -1, -1):
                s[j] = s[j + 1] * self.shape[j + 1]
            return tuple(s) if i is None else s[i]

        def get_device(self):
            return 1

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 1 << 20

        def new_empty(self, shape):
            return T(*shape, dtype=self.dtype)

    monkeypatch.setattr(lib, "_like", lambda t, keep: T(*t.shape, dtype=t.dtype))
    monkeypatch.setattr(lib, "_new", lambda stream, shape, dtype, device: T(*(shape if isinstance(shape, tuple) else (shape,)), dtype=dtype))
    monkeypatch.setattr(lib, "_result", lambda t, rows, cols, dtype, keep, like, name: (T(rows, cols, dtype=dtype), 1 << 20, cols))
    x, w, y = T(6, 64), T(24, 64), T(6, 24)
    stream = object()
    calls = [(lambda: lib.psrl_rms_norm_bwd(x, T(64), x, stream=stream), ("psrl_rms_norm_workspace_bytes", 1, (0, 6, 1, 64))),
             (lambda: lib.psrl_linear_fwd(x, w, stream=stream), ("psrl_linear_workspace_bytes", 1, (0, 6, 64, 24, 0))),
             (lambda: lib.psrl_linear_bwd(x, w, y, stream=stream), ("psrl_linear_workspace_bytes", 1, (0, 6, 64, 24, 1))),
             (lambda: lib._logprob_workspace(None, 0, None, 0, 6, 64, 24, 6, True, torch.device("cuda", 1)), ("psrl_token_logprob_workspace_bytes", 1, (0, 6, 64, 24, 6, 1)))]
    for call, want in calls:
        asked.clear()
        with pytest.raises(Stop):
            call()
        assert asked == [want]
