"""Argument checks of the 8-bit cache's calls that need no GPU, and the test reference's rounding
against torch's."""
import ctypes

import numpy as np
import torch

import qcache_reference as ref


def test_null_arguments_are_refused():
    import paper_2607_01308_gb300 as cm
    bad = cm.Status.ERR_INVALID_ARG
    n = ctypes.c_int64()
    assert cm.lib.cm_qcache_schedule(None, None, None, None, None, 0, None, 0, None, None) == bad
    assert cm.lib.cm_qcache_append(None, None, 0, 1, None, None, 0, 0, 0, None, 0, None) == bad
    assert cm.lib.cm_qcache_attend(None, None, 0, None, None, None, 0, None) == bad
    assert cm.lib.cm_qcache_workspace(None, 128, ctypes.byref(n)) == bad
    assert "context" in cm.cm_last_error_message()


def test_reference_codes_are_the_formats_own():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = np.unique(every[np.isfinite(every)])
    np.testing.assert_array_equal(ref.nearest_codes(every, "e4m3"), every)
    mid = (every[1:] + every[:-1]) / 2
    x = np.concatenate([mid, np.nextafter(mid, 1e9), np.nextafter(mid, -1e9), [447.0, -500.0, np.inf, -np.inf, np.nan]])
    want = torch.from_numpy(np.clip(np.nan_to_num(x, nan=0.0, posinf=448, neginf=-448), -448, 448))
    # fp64 -> e4m3 directly, by the nearest of all codes (the even one of two)
    got = ref.nearest_codes(x, "e4m3")
    d = np.abs(want.numpy()[:, None] - every[None])
    assert np.array_equal(np.abs(got - want.numpy()), d.min(1))
    np.testing.assert_array_equal(ref.nearest_codes(mid, "e4m3"), torch.from_numpy(mid).float().to(torch.float8_e4m3fn).double().numpy())
    np.testing.assert_array_equal(ref.nearest_codes(np.array([0.5, 1.5, -2.5, 127.5, -400.0, np.nan]), "int8"), [0, 2, -2, 127, -127, 0])


def test_reference_scales():
    for fmt, top in ref.TOP.items():
        for k in (-60, -3, 0, 17, 60):
            at = top * 2.0 ** k
            assert ref.scale_for(np.array([at, -1e-30]), fmt) == 2.0 ** k
            if k < 60:
                assert ref.scale_for(np.array([-at * (1 + 2 ** -7)]), fmt) == 2.0 ** (k + 1)
        assert ref.scale_for(np.array([np.inf, np.nan, 1.0]), fmt) == ref.scale_for(np.array([1.0]), fmt)
        assert ref.scale_for(np.array([0.0]), fmt) == 2.0 ** -60
        assert ref.scale_for(np.array([1e30]), fmt) == 2.0 ** 60
