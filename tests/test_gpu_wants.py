"""A choice that is neither true nor false is refused with the error that asking it gives, whichever way the call takes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_choices_without_a_truth_value(lib):
    x, w = torch.randn(3, 64, device="cuda"), torch.randn(64, device="cuda")
    m = torch.randn(8, 64, device="cuda")
    dy = torch.randn(3, 8, device="cuda")
    both = np.array([True, False])
    rope, pos = lib.Rope(64, sections=[16, 16]), torch.zeros(2, 3, device="cuda", dtype=torch.int32)
    calls = [lambda **k: lib.psrl_rms_norm_fwd(x, w, want_y=both, **k), lambda **k: lib.psrl_rms_norm_fwd(x, w, want_codes=both, **k),
             lambda **k: lib.psrl_rms_norm_bwd(x, w, x, want_x=both, **k), lambda **k: lib.psrl_rms_norm_bwd(x, w, x, want_weight=both, **k),
             lambda **k: lib.psrl_linear_fwd(x, m, want_z=both, **k), lambda **k: lib.psrl_linear_bwd(x, m, dy, want_x=both, **k),
             lambda **k: lib.psrl_linear_bwd(x, m, dy, want_weight=both, **k), lambda **k: lib.psrl_linear_bwd(x, m, dy, want_bias=both, **k),
             lambda **k: lib.psrl_rope_axes_rows(rope, x.view(3, 1, 64), pos, inverse=both, **k)]
    for call in calls:
        for kw in ({}, {"stream": torch.cuda.current_stream()}):
            with pytest.raises(ValueError):
                call(**kw)
    # and the same calls with one that has
    for kw in ({}, {"stream": torch.cuda.current_stream()}):
        assert lib.psrl_rms_norm_fwd(x, w, want_y=np.bool_(False), want_codes=np.array([True]), **kw)[0] is None
