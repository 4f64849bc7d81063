"""Dimensions that the library takes in 32 bits: larger ones are refused, not cut off to whatever their low bits say."""
import pytest


class Tensor:
    """What the wrappers look at before they launch."""
    is_cuda = True

    def __init__(self, *shape, dtype=None):
        import torch

        self.shape, self.dtype, self.device = torch.Size(shape), dtype or torch.bfloat16, torch.device("cuda", 0)

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def stride(self, i=None):
        s = [1] * len(self.shape)
        for j in range(len(s) - 2, -1, -1):
            s[j] = s[j + 1] * self.shape[j + 1]
        return tuple(s) if i is None else s[i]

    def data_ptr(self):
        return 1 << 20


def test_refused(lib, monkeypatch):
    import torch

    launched = []
    monkeypatch.setattr(lib, "_launch", lambda *a: launched.append(a))
    monkeypatch.setattr(lib, "_stream_on", lambda stream, dev: (0, None))
    monkeypatch.setattr(lib, "_new", lambda stream, shape, dtype, device: Tensor(*shape, dtype=dtype))
    monkeypatch.setattr(lib, "_like", lambda t, keep: Tensor(*t.shape))
    monkeypatch.setattr(lib, "_codes_rows", lambda codes, shape, keep, like, name="codes": (Tensor(*shape, dtype=torch.float8_e4m3fn), 64))
    monkeypatch.setattr(lib, "_result", lambda t, rows, cols, dtype, keep, like, name: (Tensor(rows, cols), 1 << 20, cols))
    monkeypatch.setattr(lib, "_scratch", lambda *a: (1 << 20, 1 << 30, None))
    monkeypatch.setattr(lib, "_workspace_bytes", lambda *a: 256)
    big, s = (1 << 32) + 64, object()
    rope, pos = lib.Rope(64, sections=[16, 16]), Tensor(2, 3, dtype=torch.int32)
    for call in (lambda n: lib.psrl_rms_norm_fwd(Tensor(3, n), None, stream=s), lambda n: lib.psrl_rms_norm_fwd(Tensor(3, n, 64), None, stream=s),
                 lambda n: lib.psrl_rms_norm_bwd(Tensor(3, n), None, Tensor(3, n), stream=s), lambda n: lib.psrl_quantize_rows(Tensor(3, n), stream=s),
                 lambda n: lib.psrl_linear_fwd(Tensor(3, n), Tensor(8, n), stream=s), lambda n: lib.psrl_linear_fwd(Tensor(3, 8), Tensor(n, 8), stream=s),
                 lambda n: lib.psrl_linear_bwd(Tensor(3, 8), Tensor(n, 8), Tensor(3, n), stream=s), lambda n: lib.psrl_rope_axes_rows(rope, Tensor(3, n, 64), pos, stream=s),
                 lambda n: lib._logprob_args(Tensor(3, n), Tensor(8, n), Tensor(3, dtype=torch.int32), None, []),
                 lambda n: lib._logprob_args(Tensor(3, 8), Tensor(n, 8), Tensor(3, dtype=torch.int32), None, [])):
        with pytest.raises(ValueError):
            call(big)
        assert not launched
        call(64)
        launched.clear()
