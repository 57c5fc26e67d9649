"""What of he_i8_layer_create is decided on the host: its refusals, in the order of the other plans', without a device."""
import ctypes

import numpy as np
import pytest

from paper_1908_04172_amd import he
from paper_1908_04172_amd import workloads as wl


@pytest.fixture(scope="module")
def ctx():
    return he.Context(10, wl.modulus_chain([30, 30], 1 << 10), device=None)


def status(ctx, n_in=2, n_out=1, n_pt=2, off=(0, 2), ct=(0, 1), pt=(0, 1), w=(1, -1), scale=None):
    arr = [np.asarray(a, np.uint32) for a in (off, ct, pt)]
    weights = None if w is None else np.asarray(w, np.int8)
    channel = None if scale is None else np.asarray(scale, np.float64)
    h = ctypes.c_void_p(1)
    rc = he.lib().he_i8_layer_create(ctx._h if ctx else None, n_in, n_out, n_pt, *(a.ctypes.data for a in arr),
                                     None if weights is None else weights.ctypes.data, None if channel is None else channel.ctypes.data,
                                     1.0, ctypes.byref(h))
    assert h.value is None                                          # no layer from a refused call
    return rc


def test_refusals_of_the_arrays(ctx):
    assert status(ctx) == -5                                        # all is well but for the device
    assert status(None) == -1
    assert status(ctx, w=None) == -1
    assert status(ctx, off=(1, 2)) == -4
    assert status(ctx, n_out=2, off=(0, 2, 1)) == -4
    assert status(ctx, ct=(0, 2)) == -4
    assert status(ctx, pt=(2, 0)) == -4
    assert status(ctx, scale=[float("nan")]) == -1
    assert status(ctx, scale=[float("inf")]) == -1
    assert he.lib().he_i8_layer_create(ctx._h, 1, 1, 1, None, None, None, None, None, 1.0, None) == -1


def test_an_output_takes_131071_terms_and_no_more(ctx):
    for terms, want in ((131071, -5), (131072, -4)):
        z = np.zeros(terms, np.uint32)
        assert status(ctx, off=(0, terms), ct=z, pt=z) == want


def test_refusals_without_a_layer(ctx):
    assert he.lib().he_i8_layer_destroy(None) == -1
    b = ctypes.c_size_t()
    assert he.lib().he_i8_workspace_bytes(None, 1, 0, ctypes.byref(b)) == -1
    assert he.lib().he_ct_i8_mac(ctx._h, None, 1, None, None, None, None, 0, None, 0, None) == -1
    assert he.lib().he_ct_i8_mac32(None, None, 1, None, None, None, None, 0, None, 0, None) == -1
