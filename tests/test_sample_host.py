"""he_sample_slots' refusals, all decided on the host before anything is enqueued."""
import ctypes

import pytest

from paper_1908_04172_amd import he
from paper_1908_04172_amd import workloads as wl


@pytest.fixture(scope="module")
def ctx():
    return he.Context(10, wl.modulus_chain([30], 1 << 10), device=None)


# made-up device addresses (nothing reads them: a context without a device ends every call before a launch)
SLOTS, T, K, P, M, U, TOKENS, LOG = (0x10000000 + 0x10000000 * k for k in range(8))


def status(ctx, n=100, n_slots=512, parts=1, slots=SLOTS, t=T, k=K, p=P, m=M, u=U, tokens=TOKENS, log=LOG):
    return he.lib().he_sample_slots(ctx._h if ctx else None, slots, n, n_slots, parts, t, k, p, m, u, tokens, log, None)


def test_refusals(ctx):
    assert status(ctx) == -5                                        # all is well but for the device
    assert status(ctx, t=None, k=None, p=None, m=None, log=None) == -5
    assert status(None) == -1
    assert status(ctx, n=0) == -1
    assert status(ctx, parts=0) == -1 and status(ctx, parts=3) == -1
    assert status(ctx, n=32768) == -5 and status(ctx, n=32769) == -4
    assert status(ctx, n_slots=513) == -4
    assert status(ctx, slots=None) == -1 and status(ctx, u=None) == -1 and status(ctx, tokens=None) == -1
    assert status(ctx, n_slots=0, slots=None, u=None, tokens=None) == 0


def test_outputs_may_not_overlap(ctx):
    for name in ("slots", "t", "k", "p", "m", "u"):
        assert status(ctx, **{name: TOKENS}) == -1, name
        assert status(ctx, **{name: LOG}) == -1, name
        assert status(ctx, **{name: TOKENS + 512 * 4}) == -5, name
    assert status(ctx, tokens=LOG + 8) == -1
    assert status(ctx, tokens=SLOTS + 100 * 1024 * 8 - 4) == -1     # the last word of the logits
    assert status(ctx, tokens=SLOTS + 100 * 1024 * 8) == -5
