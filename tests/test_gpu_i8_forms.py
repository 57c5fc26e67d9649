"""The forms in which layers of 8-bit integer weights are launched, each at a size that takes it, and the form asserted: groups of up to
16, 32 and 64 outputs, in 64-bit and packed storage, written through the caches and past them, a workgroup running through
several groups of several blocks of terms.  All residues, against he_ct_pt_mac step by step (the sums, the channels' scales, the tokens
with the bias), and some outputs against the oracle."""
import numpy as np
import pytest

import oracle
from paper_1908_04172_amd import workloads as wl
from test_gpu_i8 import expected, groups_plan

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def he():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1908_04172_amd import he as he_mod
    he_mod.lib()
    return he_mod


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).cuda()


def by_steps(he, ctx, plan, x, w, s, token, b):
    """The layer as calls of he_ct_pt_mac: plaintexts w, then s_o per output, then the tokens' polynomial; the bias with the last."""
    q = np.array(ctx.moduli[:x.shape[2]], dtype=object)
    each, off = np.arange(plan.n_out, dtype=np.uint32), np.arange(plan.n_out + 1, dtype=np.uint32)
    single = ctx.plan(plan.n_out, plan.n_out, plan.n_out, off, each, each)
    alike = ctx.plan(plan.n_out, plan.n_out, 1, off, each, np.zeros_like(each))
    pt = dev((w.astype(object)[:, None] % q).astype(np.uint64))
    sums = ctx.ct_pt_mac(ctx.plan(plan.n_in, plan.n_out, plan.n_pt, plan.off, plan.term_ct, plan.term_pt), x, pt, he.PT_SCALAR)
    sums = ctx.ct_pt_mac(single, sums, s, he.PT_SCALAR, bias=b if token is None else None)
    return sums if token is None else ctx.ct_pt_mac(alike, sums, token[None], he.PT_POLY, bias=b)


# 128 KiB a ciphertext: 64-bit residues of two limbs at N = 2^12, packed ones at 2^13.  In
# either a group takes 128 workgroups, and a workgroup of the two smaller classes runs through as many groups as leave 2048.
CASES = {  # plan, outputs of a group, groups of that class, groups of a workgroup, past the caches
    # (64 of 400 inputs each: too few in common to be one group)
    "up to 16": (lambda: groups_plan([(11, 64)] * 121, 400, 500, 1), 11, 121, 8, False),
    "up to 16, past the caches": (lambda: groups_plan([(11, 64)] * 201, 400, 500, 2), 11, 201, 8, True),
    "17 to 32": (lambda: wl.conv_plan(9, 7, 4, 3, 3, 20, 1, "same"), 20, 63, 4, False),
    "17 to 32, past the caches": (lambda: wl.conv_plan(12, 12, 4, 3, 3, 20, 1, "same"), 20, 144, 8, True),
    "merged windows": (lambda: wl.conv_plan(8, 8, 4, 3, 3, 16, 1, "same"), 32, 32, 2, False),
    "merged windows, past the caches": (lambda: wl.conv_plan(14, 14, 4, 3, 3, 16, 1, "same"), 32, 98, 4, True),
    "33 to 64": (lambda: wl.dense_plan(70, 320), 64, 5, 1, False),
    "33 to 64, past the caches": (lambda: wl.dense_plan(70, 2050), 64, 32, 1, True),
}


@pytest.mark.parametrize("bits", [[62, 40], [50, 30], [30, 30]], ids=["62 40", "50 30", "packed"])
@pytest.mark.parametrize("case", CASES)
def test_forms(he, case, bits):
    make, outputs, groups, run, past = CASES[case]
    packed = bits == [30, 30]
    log2N = 13 if packed else 12
    N = 1 << log2N
    q = wl.modulus_chain(bits, N)
    ctx = he.Context(log2N, q)
    plan = make()
    rng = np.random.default_rng(plan.n_out)
    w, scale = rng.integers(-128, 128, plan.n_pt).astype(np.int8), rng.normal(0, 1, plan.n_out)
    residues = lambda outer, seed: wl.uniform_residues_torch(outer, q, N, seed, "cuda", chunk=2048)
    x, token, start = residues((plan.n_in, 2), 1), residues((), 2), residues((plan.n_out, 2), 3)
    b = wl.uniform_residues_torch((plan.n_out,), q, 1, 4, "cuda")[..., 0].contiguous()
    s = dev(oracle.encode_scalars(scale, 2.0**25, q))
    call = ctx.ct_i8_mac32 if packed else ctx.ct_i8_mac
    into = ctx.pack32 if packed else lambda t: t
    back = ctx.unpack32 if packed else lambda t: t
    moduli = torch.tensor([int(m) for m in q], dtype=torch.int64, device="cuda").view(1, 1, -1, 1)
    for has_scale, has_token, has_bias in ((True, True, True), (True, False, True), (False, True, False), (False, False, False)):
        layer = ctx.i8_layer(plan.n_in, plan.n_out, plan.n_pt, plan.off, plan.term_ct, plan.term_pt, w, scale if has_scale else None, 2.0**25)
        assert layer.form(2, outputs, packed) == (groups, run, he.FORM_PAST_CACHES if past else 0)
        tok, bias = token if has_token else None, b if has_bias else None
        want = by_steps(he, ctx, plan, x, w, s if has_scale else torch.ones_like(s), tok, bias)
        args = (layer, into(x), None if tok is None else into(tok), bias)
        assert torch.equal(back(call(*args)), want)
        added = call(*args, flags=he.ACCUMULATE, out=into(start).clone())
        total = want + start
        total -= torch.where(total >= moduli, moduli, torch.zeros_like(moduli))
        assert torch.equal(back(added), total)
        assert torch.equal(back(call(*args, flags=he.RESCALE)), ctx.rescale(want))
        if not has_token and not has_scale:
            continue
        some = [0, 1, plan.n_out // 2, plan.n_out - 1]              # against the oracle
        terms = [np.arange(plan.off[o], plan.off[o + 1]) for o in some]
        few = wl.Plan(plan.n_in, len(some), plan.n_pt, np.cumsum([0] + [len(t) for t in terms]).astype(np.uint32),
                      plan.term_ct[np.concatenate(terms)], plan.term_pt[np.concatenate(terms)])
        ours = lambda t: t.cpu().numpy().view(np.uint64)
        assert np.array_equal(ours(want[some]), expected(ours(x), q, few, w, scale[some] if has_scale else None, 2.0**25,
                                                         None if tok is None else ours(tok), None if bias is None else ours(bias[some])))


def test_as_many_workgroups_as_a_grid_holds(he):
    """Outputs without terms, each between two that have some, are groups of 2^14 workgroups here: 1023 of them fit the 2^32 threads
    of a grid, and 1024 are refused before anything is enqueued."""
    N = 1 << 15
    q = wl.modulus_chain([60] + [50] * 15, N)                       # 8 MiB a ciphertext
    ctx = he.Context(15, q)
    x = wl.uniform_residues_torch((1, 2), q, N, 3, "cuda")

    def layer(empty):
        n_out = 2 * empty - 1
        off = (np.arange(n_out + 1) // 2).astype(np.uint32)   # outputs 1, 3, 5, ... have the one term
        zeros = np.zeros(off[-1], np.uint32)
        return ctx.i8_layer(1, n_out, 1, off, zeros, zeros, np.ones(1, np.int8))

    out = torch.full((2047, 2, 16, N), -7, dtype=torch.int64, device="cuda")
    with pytest.raises(he.HeError) as e:
        ctx.ct_i8_mac(layer(1024), x, out=out)
    assert e.value.status == -4
    torch.cuda.synchronize()
    assert all(bool((out[k:k + 128] == -7).all()) for k in range(0, 2047, 128))
    ctx.ct_i8_mac(layer(1023), x, out=out[:2045])
    for k in range(0, 2045, 128):
        part = out[k:min(k + 128, 2045)]
        assert not bool(part[0::2].any()) and bool((part[1::2] == x).all())
    assert bool((out[2045:] == -7).all())


def test_what_has_no_form(he):
    ctx = he.Context(10, wl.modulus_chain([40, 30], 1 << 10))
    plan = wl.dense_plan(3, 2)
    layer = ctx.i8_layer(plan.n_in, plan.n_out, plan.n_pt, plan.off, plan.term_ct, plan.term_pt, np.ones(6, np.int8))
    assert layer.form(2, 2) == (1, 1, 0) and layer.form(1, 33) == (0, 1, 0)
    for limbs, outputs, status in ((2, 0, -1), (2, 65, -1), (0, 1, -3), (3, 1, -3)):
        with pytest.raises(he.HeError) as e:
            layer.form(limbs, outputs)
        assert e.value.status == status
