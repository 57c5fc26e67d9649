"""Layers of 8-bit integer weights (he_ct_i8_mac, he_ct_i8_mac32) at the sizes where they can go wrong: output counts around the
tiles of 32 and the groups of 64, term counts around the blocks of 32 and up to the longest sum, moduli of every width, extreme
residues and weights, and every combination of scales and bias.  Exact residues, against the oracle and Python integers."""
import numpy as np
import pytest

import oracle
from paper_1908_04172_amd import workloads as wl

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


def host(t):
    return t.cpu().numpy().view(np.uint64)


def groups_plan(groups, n_in, n_pt, seed):
    """One group of `count` outputs over `terms` random ciphertexts per (count, terms)."""
    rng = np.random.default_rng(seed)
    off, tc, tp = [0], [np.zeros(0)], [np.zeros(0)]
    for count, terms in groups:
        cts = rng.integers(0, n_in, terms)
        for _ in range(count):
            tc.append(cts)
            tp.append(rng.integers(0, n_pt, terms))
            off.append(off[-1] + terms)
    cat = lambda xs: np.concatenate(xs).astype(np.uint32)
    return wl.Plan(n_in, len(off) - 1, n_pt, np.asarray(off, np.uint32), cat(tc), cat(tp))


def operands(plan, q, N, seed, extreme=False):
    rng = np.random.default_rng(seed)
    ct = wl.uniform_residues((plan.n_in, 2), q, N, seed)
    w = rng.integers(-128, 128, plan.n_pt).astype(np.int8)
    scale = rng.normal(0, 1, plan.n_out)
    token = wl.uniform_residues((), q, N, seed + 1)
    b = wl.uniform_residues((plan.n_out,), q, 1, seed + 2)[..., 0]
    if extreme:  # the largest residues, all bits clear, bytes next to where a digit changes sign; weights at both ends
        for i, qi in enumerate(q):
            values = [qi - 1, 0, 0x8080808080808080 % (1 << (qi.bit_length() - 1)), 0x7F7F7F7F7F7F7F7F % (1 << (qi.bit_length() - 1))]
            for c in range(plan.n_in):
                if c % 5 < 4:
                    ct[c, :, i, :] = values[c % 5]
            token[i, ::2] = qi - 1
            b[:, i] = qi - 1
        w[0::3], w[1::3] = -128, 127
    return ct, w, scale, token, b


def expected(ct, q, plan, w, scale=None, delta=1.0, token=None, b=None):
    """The oracle's MAC with a plaintext s_o * w of its own for every term, then the tokens and the bias in Python integers."""
    s = np.ones((plan.n_out, len(q)), dtype=object) if scale is None else oracle.encode_scalars(scale, delta, q).astype(object)
    owner = np.repeat(np.arange(plan.n_out), np.diff(plan.off.astype(np.int64)))
    qa = np.array(q, dtype=object)[None, :]
    pt = (s[owner] * w[plan.term_pt].astype(object)[:, None] % qa).astype(np.uint64)
    if len(pt) == 0:
        pt = np.zeros((1, len(q)), np.uint64)
    out = oracle.mac(ct, q, plan.off, plan.term_ct, np.arange(plan.n_terms, dtype=np.uint32), pt, oracle.PT_SCALAR).astype(object)
    qb = np.array(q, dtype=object)[None, None, :, None]
    if token is not None:
        out = out * token.astype(object)[None, None] % qb
    if b is not None:
        out[:, 0] = (out[:, 0] + b.astype(object)[:, :, None]) % qb[:, 0]
    return out.astype(np.uint64)


def layer_of(ctx, plan, w, scale=None, delta=1.0):
    return ctx.i8_layer(plan.n_in, plan.n_out, plan.n_pt, plan.off, plan.term_ct, plan.term_pt, w, scale, delta)


GROUPS = [(c, t) for c in (1, 3, 31, 32, 33) for t in (1, 31, 32, 33)] + [(1, 0), (64, 2), (65, 7), (2, 64), (5, 65), (4, 96), (3, 97), (97, 129)]


@pytest.mark.parametrize("bits", [[14, 20, 24, 30], [31, 32, 33, 39], [40, 41, 47, 48], [49, 50, 55, 56], [57, 60, 61, 62]], ids=str)
@pytest.mark.parametrize("extreme", [False, True])
def test_group_sizes_and_term_counts_on_moduli_of_every_width(he, bits, extreme):
    N = 1 << 10
    q = wl.modulus_chain(bits, N)
    ctx = he.Context(10, q)
    plan = groups_plan(GROUPS, 40, 90, sum(bits))
    ct, w, scale, token, b = operands(plan, q, N, 7 + sum(bits), extreme)
    layer = layer_of(ctx, plan, w, scale, 2.0**30)
    want = expected(ct, q, plan, w, scale, 2.0**30, token, b)
    assert np.array_equal(host(ctx.ct_i8_mac(layer, dev(ct), dev(token), dev(b))), want)
    assert np.array_equal(host(ctx.ct_i8_mac(layer, dev(ct), dev(token), dev(b), flags=he.RESCALE)), oracle.rescale(want, q, ctx.psi))


@pytest.mark.parametrize("M", [1, 2, 31, 64, 65, 96, 97, 128, 129, 192, 257, 300])
def test_dense_layers_of_every_number_of_tiles(he, M):
    N, K = 1 << 10, 37
    q = wl.modulus_chain([60, 50, 40], N)
    ctx = he.Context(10, q)
    plan = wl.dense_plan(K, M)
    ct, w, scale, _, b = operands(plan, q, N, M)
    got = ctx.ct_i8_mac(layer_of(ctx, plan, w, scale, 2.0**25), dev(ct), bias=dev(b))
    assert np.array_equal(host(got), expected(ct, q, plan, w, scale, 2.0**25, None, b))


@pytest.mark.parametrize("has_scale", [False, True])
@pytest.mark.parametrize("has_token", [False, True])
@pytest.mark.parametrize("has_bias", [False, True])
@pytest.mark.parametrize("geometry", [(9, 9, 2, 3, 3, 5, 2, "valid"), (8, 8, 3, 3, 3, 4, 1, "same"), (6, 6, 1, 1, 1, 33, 1, "valid")], ids=str)
def test_convolutions_with_every_choice_of_scales(he, geometry, has_scale, has_token, has_bias):
    N = 1 << 11
    q = wl.modulus_chain([58, 45], N)
    ctx = he.Context(11, q)
    plan = wl.conv_plan(*geometry)
    ct, w, scale, token, b = operands(plan, q, N, 5)
    scale, token, b = scale if has_scale else None, token if has_token else None, b if has_bias else None
    got = ctx.ct_i8_mac(layer_of(ctx, plan, w, scale, 2.0**20), dev(ct), None if token is None else dev(token), None if b is None else dev(b))
    assert np.array_equal(host(got), expected(ct, q, plan, w, scale, 2.0**20, token, b))


@pytest.mark.parametrize("bits", [[62], [50], [40], [30]], ids=str)
def test_the_longest_sums(he, bits):
    """131071 terms whose digits' sums come as close to 2^31 as they can, of either sign."""
    N, K = 1 << 10, 131071
    q = wl.modulus_chain(bits, N)
    ctx = he.Context(10, q)
    rng = np.random.default_rng(3)
    ct = np.zeros((3, 2, 1, N), np.uint64)
    ct[1] = (1 << (q[0].bit_length() - 1)) - 1                      # all bytes but the highest at 255
    ct[2] = wl.uniform_residues((1, 2), q, N, 4)[0]
    lists = [np.zeros(K, np.uint32), np.ones(K, np.uint32), np.full(K, 2, np.uint32), rng.integers(0, 3, K).astype(np.uint32)]
    plan = wl.Plan(3, 4, 4, (np.arange(5) * K).astype(np.uint32), np.concatenate(lists),
                   np.concatenate([np.zeros(K), np.zeros(K), np.ones(K), rng.integers(0, 4, K)]).astype(np.uint32))
    w = np.array([-128, 127, -1, 0], np.int8)
    got = host(ctx.ct_i8_mac(layer_of(ctx, plan, w), dev(ct)))
    for o in range(4):
        counts = [[int(np.sum((lists[o] == c) & (plan.term_pt[o * K:(o + 1) * K] == k))) for k in range(4)] for c in range(3)]
        want = sum(ct[c].astype(object) * sum(int(w[k]) * counts[c][k] for k in range(4)) for c in range(3)) % q[0]
        assert np.array_equal(got[o], want.astype(np.uint64)), o


@pytest.mark.parametrize("M", [1, 33, 100, 130])
@pytest.mark.parametrize("has_token", [False, True])
def test_packed_storage(he, M, has_token):
    N, K = 1 << 10, 70
    q = wl.modulus_chain([30, 30, 25], N)
    ctx = he.Context(10, q)
    plan = wl.dense_plan(K, M)
    ct, w, scale, token, b = operands(plan, q, N, M, extreme=M == 33)
    layer = layer_of(ctx, plan, w, scale, 2.0**20)
    want = expected(ct, q, plan, w, scale, 2.0**20, token if has_token else None, b)
    packed = ctx.pack32(dev(ct))
    tok = ctx.pack32(dev(token)) if has_token else None
    got = ctx.ct_i8_mac32(layer, packed, tok, dev(b))
    assert np.array_equal(host(ctx.unpack32(got)), want)
    rescaled = ctx.ct_i8_mac32(layer, packed, tok, dev(b), flags=he.RESCALE)
    assert np.array_equal(host(ctx.unpack32(rescaled)), oracle.rescale(want, q, ctx.psi))
    twice = ctx.ct_i8_mac32(layer, packed, tok, dev(b), flags=he.ACCUMULATE, out=got.clone())
    assert np.array_equal(host(ctx.unpack32(twice)), (want * 2 % np.array(q, np.uint64)[None, None, :, None]))


@pytest.mark.parametrize("log2N", [10, 12, 13, 14, 15])
def test_ring_degrees_and_levels(he, log2N):
    """... on the chain's first limbs too: a layer serves every level."""
    N = 1 << log2N
    q = wl.modulus_chain([60, 50, 50], N)
    ctx = he.Context(log2N, q)
    plan = wl.dense_plan(40, 5)
    ct, w, scale, token, b = operands(plan, q, N, log2N)
    layer = layer_of(ctx, plan, w, scale, 2.0**25)
    for limbs in (3, 2):
        x, tok, bias = ct[:, :, :limbs].copy(), token[:limbs].copy(), b[:, :limbs].copy()
        want = expected(x, q[:limbs], plan, w, scale, 2.0**25, tok, bias)
        assert np.array_equal(host(ctx.ct_i8_mac(layer, dev(x), dev(tok), dev(bias))), want)
        got = ctx.ct_i8_mac(layer, dev(x), dev(tok), dev(bias), flags=he.RESCALE)
        assert np.array_equal(host(got), oracle.rescale(want, q[:limbs], ctx.psi[:limbs]))


def test_partial_sums_and_rows_behind_the_last_output(he):
    """A layer split over two calls; what lies behind the outputs and the accumulators stays as it was."""
    N = 1 << 11
    q = wl.modulus_chain([60, 40], N)
    ctx = he.Context(11, q)
    a, c = wl.dense_plan(45, 35), wl.dense_plan(20, 35)
    ct_a, w_a, scale, _, b = operands(a, q, N, 1)
    ct_c, w_c, _, _, _ = operands(c, q, N, 2)
    room = torch.full((40, 2, 2, N), -7, dtype=torch.int64, device="cuda")
    ctx.ct_i8_mac(layer_of(ctx, a, w_a, scale, 2.0**25), dev(ct_a), bias=dev(b), out=room[:35])
    ctx.ct_i8_mac(layer_of(ctx, c, w_c, scale, 2.0**25), dev(ct_c), flags=he.ACCUMULATE, out=room[:35])
    qa = np.array(q, dtype=object)[None, None, :, None]
    want = expected(ct_a, q, a, w_a, scale, 2.0**25, None, b).astype(object) + expected(ct_c, q, c, w_c, scale, 2.0**25).astype(object)
    assert np.array_equal(host(room[:35]).astype(object), want % qa)
    assert bool((room[35:] == -7).all())


def test_the_same_residues_as_plaintexts_of_full_width(he):
    """he_ct_i8_mac and he_ct_pt_mac with the products s_o * w as plaintexts, both rescaled."""
    N = 1 << 12
    q = wl.modulus_chain([60, 50, 50], N)
    ctx = he.Context(12, q)
    K, M = 33, 20
    plan = wl.dense_plan(K, M)
    ct, w, scale, _, b = operands(plan, q, N, 9)
    s = oracle.encode_scalars(scale, 2.0**25, q).astype(object)
    pt = s[np.tile(np.arange(M), K)] * w.astype(object)[:, None] % np.array(q, dtype=object)[None]
    hp = ctx.plan(plan.n_in, plan.n_out, plan.n_pt, plan.off, plan.term_ct, plan.term_pt)
    full = ctx.ct_pt_mac(hp, dev(ct), dev(pt.astype(np.uint64)), he.PT_SCALAR, bias=dev(b), flags=he.RESCALE)
    got = ctx.ct_i8_mac(layer_of(ctx, plan, w, scale, 2.0**25), dev(ct), bias=dev(b), flags=he.RESCALE)
    assert torch.equal(got, full)


def test_tensors_beyond_four_gigabytes(he):
    """Inputs and outputs whose byte offsets do not fit 32 bits."""
    N, n = 1 << 15, 520
    q = wl.modulus_chain([60] + [50] * 15, N)                       # 8 MiB a ciphertext
    ctx = he.Context(15, q)
    ct = wl.uniform_residues_torch((n, 2), q, N, 5, "cuda")
    rng = np.random.default_rng(6)
    off = np.arange(n + 1, dtype=np.uint32)
    plan = wl.Plan(n, n, 7, off, np.arange(n, dtype=np.uint32)[::-1].copy(), rng.integers(0, 7, n).astype(np.uint32))
    w = np.array([-128, 127, 1, -1, 50, -77, 3], np.int8)
    out = ctx.ct_i8_mac(layer_of(ctx, plan, w), ct)
    for o in (0, 1, 255, 256, 511, 512, 513, 519):
        want = ct[n - 1 - o].cpu().numpy().view(np.uint64).astype(object) * int(w[plan.term_pt[o]]) % np.array(q, dtype=object)[None, :, None]
        assert np.array_equal(host(out[o]), want.astype(np.uint64)), o


def test_two_streams_and_a_captured_graph(he):
    N = 1 << 11
    q = wl.modulus_chain([60, 40, 40], N)
    ctx = he.Context(11, q)
    plan = wl.dense_plan(50, 40)
    ct, w, scale, token, b = operands(plan, q, N, 21)
    layer = layer_of(ctx, plan, w, scale, 2.0**25)
    x, tok, bias = dev(ct), dev(token), dev(b)
    want = dev(oracle.rescale(expected(ct, q, plan, w, scale, 2.0**25, token, b), q, ctx.psi))
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for s in streams:                                               # two calls of one layer at once, workspaces of their own
        with torch.cuda.stream(s):
            outs.append(ctx.ct_i8_mac(layer, x, tok, bias, flags=he.RESCALE))
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    out = torch.zeros_like(want)
    ws = torch.empty(layer.workspace_bytes(3, he.RESCALE), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.ct_i8_mac(layer, x, tok, bias, flags=he.RESCALE, out=out, workspace=ws)
    for k in range(4):                                              # other inputs from replay to replay, eager work in between
        shifted = (x.roll(k, 0)).contiguous()
        eager = ctx.ct_i8_mac(layer, shifted, tok, bias, flags=he.RESCALE)
        keep = x.clone()
        x.copy_(shifted)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), k
        x.copy_(keep)


def test_refusals_on_a_device(he):
    N = 1 << 10
    q = wl.modulus_chain([60, 40], N)
    ctx = he.Context(10, q)
    plan = wl.dense_plan(5, 3)
    ct, w, scale, token, b = operands(plan, q, N, 1)
    layer = layer_of(ctx, plan, w, scale)
    x, tok, bias = dev(ct), dev(token), dev(b)

    def status(call):
        with pytest.raises(he.HeError) as e:
            call()
        return e.value.status

    both = torch.empty((8, 2, 2, N), dtype=torch.int64, device="cuda")
    both[:5] = x
    out = torch.empty((3, 2, 2, N), dtype=torch.int64, device="cuda")
    assert status(lambda: ctx.ct_i8_mac(layer, both[:5], out=both[4:7])) == -1             # output over an input
    assert status(lambda: ctx.ct_i8_mac(layer, x, token_scale=out.view(-1)[:2 * N].view(2, N), out=out)) == -1
    assert status(lambda: ctx.ct_i8_mac(layer, x, bias=out.view(-1)[:6].view(3, 2), out=out)) == -1
    assert status(lambda: ctx.ct_i8_mac(layer, x, flags=he.RESCALE | he.ACCUMULATE, out=out[:, :, :1].contiguous())) == -1
    assert status(lambda: ctx.ct_i8_mac(layer, x, flags=4)) == -1
    small = torch.empty(layer.workspace_bytes(2, he.RESCALE) - 256, dtype=torch.uint8, device="cuda")
    assert status(lambda: ctx.ct_i8_mac(layer, x, flags=he.RESCALE, workspace=small)) == -6
    shared = torch.empty(layer.workspace_bytes(2, he.RESCALE) // 8 + 64, dtype=torch.int64, device="cuda")
    res = shared[:3 * 2 * N].view(3, 2, 1, N)
    assert status(lambda: ctx.ct_i8_mac(layer, x, flags=he.RESCALE, out=res, workspace=shared)) == -1
    one = x[:, :, :1].contiguous()
    assert status(lambda: ctx.ct_i8_mac(layer, one, flags=he.RESCALE)) == -3      # nothing left to drop
    assert status(lambda: he.Context(10, q).ct_i8_mac(layer, x)) == -1                     # another context's layer
    assert status(lambda: ctx.ct_i8_mac32(layer, ctx.pack32(x))) == -2                     # a 60-bit limb has no packed form
    assert status(lambda: layer_of(ctx, plan, w, np.array([1.0, np.inf, 1.0]))) == -1
    empty = ctx.i8_layer(5, 0, 15, np.zeros(1, np.uint32), [], [], w)
    assert ctx.ct_i8_mac(empty, x).numel() == 0


def test_arrays_at_odd_multiples_of_eight_bytes(he):
    N = 1 << 11

    def shifted(t):
        raw = torch.empty(t.numel() * t.element_size() + 8, dtype=torch.uint8, device="cuda")
        view = raw[8:].view(t.dtype).view(t.shape)
        assert view.data_ptr() % 16 == 8
        view.copy_(t)
        return view

    for bits, M in (([60, 40], 9), ([60, 40], 50), ([30, 30], 9), ([30, 30], 50)):
        q = wl.modulus_chain(bits, N)
        ctx = he.Context(11, q)
        plan = wl.dense_plan(40, M)
        ct, w, scale, token, b = operands(plan, q, N, M)
        layer = layer_of(ctx, plan, w, scale, 2.0**20)
        x, tok, bias = dev(ct), dev(token), dev(b)
        call = ctx.ct_i8_mac
        if bits[0] == 30:
            x, tok, call = ctx.pack32(x), ctx.pack32(tok), ctx.ct_i8_mac32
        for flags in (0, he.RESCALE):
            want = call(layer, x, tok, bias, flags=flags)
            ws = torch.empty(layer.workspace_bytes(2, flags) + 8, dtype=torch.uint8, device="cuda")[8:] if flags else None
            got = call(layer, shifted(x), shifted(tok), shifted(bias), flags=flags, out=shifted(torch.zeros_like(want)), workspace=ws)
            assert torch.equal(got, want)


def test_single_outputs_share_blocks_of_terms(he):
    """An elementwise scaling and a depthwise convolution: outputs with inputs of their own, which the layer merges."""
    N, n = 1 << 10, 75
    q = wl.modulus_chain([60, 50], N)
    ctx = he.Context(10, q)
    each = np.arange(n, dtype=np.uint32)
    scaling = wl.Plan(n, n, n, np.arange(n + 1, dtype=np.uint32), each, each)
    taps = np.stack([np.clip(each.astype(int) + d, 0, n - 1) for d in (-1, 0, 1)], 1).astype(np.uint32)  # (the ends read an input twice)
    depthwise = wl.Plan(n, n, 3, np.arange(n + 1, dtype=np.uint32) * 3, taps.ravel(), np.tile(np.arange(3, dtype=np.uint32), n))
    for plan in (scaling, depthwise):
        ct, w, scale, token, b = operands(plan, q, N, 31, extreme=True)
        got = ctx.ct_i8_mac(layer_of(ctx, plan, w, scale, 2.0**25), dev(ct), dev(token), dev(b))
        assert np.array_equal(host(got), expected(ct, q, plan, w, scale, 2.0**25, token, b))


@pytest.mark.parametrize("terms", [2047, 2048, 2049, 2112, 4160])
def test_large_groups_whose_lists_are_taken_in_parts(he, terms):
    """More terms than the list in the LDS holds at a time, in both storage forms."""
    N = 1 << 10
    q = wl.modulus_chain([30, 27], N)
    ctx = he.Context(10, q)
    plan = groups_plan([(40, terms)], 60, 70, terms)
    ct, w, scale, token, b = operands(plan, q, N, terms, extreme=True)
    layer = layer_of(ctx, plan, w, scale, 2.0**20)
    want = expected(ct, q, plan, w, scale, 2.0**20, token, b)
    assert np.array_equal(host(ctx.ct_i8_mac(layer, dev(ct), dev(token), dev(b))), want)
    got = ctx.ct_i8_mac32(layer, ctx.pack32(dev(ct)), ctx.pack32(dev(token)), dev(b))
    assert np.array_equal(host(ctx.unpack32(got)), want)
    q60 = wl.modulus_chain([62], N)                                 # four digits a half, the exact estimates
    ctx60 = he.Context(10, q60)
    ct, w, scale, _, b = operands(plan, q60, N, terms + 1)
    got = ctx60.ct_i8_mac(layer_of(ctx60, plan, w, scale, 2.0**30), dev(ct), bias=dev(b))
    assert np.array_equal(host(got), expected(ct, q60, plan, w, scale, 2.0**30, None, b))
