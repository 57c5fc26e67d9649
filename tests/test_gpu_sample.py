"""he_sample_slots against a plain implementation in whole numbers: row lengths around what a thread and a workgroup hold, few and many
rows, equal logits, rows with nothing to take, and parameters at and beyond their ends."""
import math

import numpy as np
import pytest

from paper_1908_04172_amd import workloads as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ONE = 1 << 47


@pytest.fixture(scope="module")
def he():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1908_04172_amd import he as he_mod
    he_mod.lib()
    return he_mod


@pytest.fixture(scope="module")
def contexts(he):
    made = {}

    def get(log2N):
        if log2N not in made:
            made[log2N] = he.Context(log2N, wl.modulus_chain([30], 1 << log2N))
        return made[log2N]
    return get


def plain(x, u, t=1.0, k=0, p=1.0, m=0.0):
    """(token, log-probability) of one row"""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, -np.inf
    if not t > 0:
        return int(np.flatnonzero(x == top)[0]), 0.0
    with np.errstate(all="ignore"):
        inv = np.float64(1.0) / np.float64(t)
        d = (x - top) * inv
        w = np.where(x == top, float(ONE), np.rint(np.nan_to_num(np.exp(d), nan=0.0) * float(ONE))).astype(np.int64)
    order = np.argsort(-w, kind="stable")
    keep = len(x) if k == 0 else min(k, len(x))
    if p < 1:
        sums = np.cumsum(w[order[:keep]])
        need = max(1, math.ceil(float(sums[-1]) * p)) if p > 0 else 1
        keep = min(keep, int(np.searchsorted(sums, need)) + 1)
    kept = np.zeros_like(w)
    kept[order[:keep]] = w[order[:keep]]
    if m > 0:
        kept[kept < min(m, 1.0) * float(ONE)] = 0
    sums = np.cumsum(kept)
    total = int(sums[-1])
    u = 0.0 if not u > 0 else min(u, 1.0)
    at = min(math.floor(float(total) * u), total - 1)
    token = int(np.searchsorted(sums, at, side="right"))
    return token, (0.0 if x[token] == top else float(d[token])) - math.log(total / ONE)


def check(ctx, logits, u, parts, **params):
    """logits [n][half][2]; params [rows] arrays or nothing"""
    rows = len(u)
    cuda = lambda a, dtype: torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()
    types = {"temperature": np.float64, "top_k": np.int32, "top_p": np.float64, "min_p": np.float64}
    slots = torch.view_as_complex(cuda(logits, np.float64))
    tokens, log_prob = ctx.sample_slots(slots, cuda(u, np.float64), parts=parts, **{k: cuda(v, types[k]) for k, v in params.items()})
    tokens, log_prob = tokens.cpu().numpy(), log_prob.cpu().numpy()
    for r in range(rows):
        want = plain(logits[:, r // parts, r % parts], u[r], *(params[k][r] if k in params else d
                                                               for k, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))))
        assert tokens[r] == want[0], (r, tokens[r], want)
        # the exponent and the logarithm: a few roundings of 2^-53 relative to their operands' magnitudes, and a total whose weights may each be
        # off by one unit of 2^-47 where the exponential is rounded
        bound = 2.0**-50 * (1 + abs(want[1])) + len(logits) * 2.0**-46
        assert log_prob[r] == want[1] or abs(log_prob[r] - want[1]) <= bound, (r, log_prob[r], want)


def random_params(rng, rows, n, names="tkpm"):
    every = {"temperature": rng.choice([0.0, 0.3, 1.0, 1.0, 1.7], rows), "top_k": rng.choice([0, 1, 2, 7, 50, 1000, n, n + 1], rows),
             "top_p": rng.choice([1.0, 0.99, 0.9, 0.5, 0.01], rows), "min_p": rng.choice([0.0, 0.01, 0.3, 1.0], rows)}
    return {k: v for k, v in every.items() if k[0] in names or k[-1] in names}


@pytest.mark.parametrize("n", [1, 2, 3, 31, 32, 33, 64, 65, 511, 512, 513, 1000, 1025, 2049, 4096, 8191])
@pytest.mark.parametrize("n_slots,parts", [(1, 1), (5, 2), (67, 1)])
def test_row_lengths(contexts, n, n_slots, parts):
    rng = np.random.default_rng(n * 7 + n_slots)
    ctx = contexts(10)
    logits = rng.normal(0, 2.5, (n, 512, 2))
    rows = n_slots * parts
    check(ctx, logits, rng.random(rows), parts)
    check(ctx, logits, rng.random(rows), parts, **random_params(rng, rows, n))


@pytest.mark.parametrize("n", [16384, 16385, 32767, 32768])
def test_the_longest_rows(contexts, n):
    rng = np.random.default_rng(n)
    logits = np.zeros((n, 512, 2))
    logits[:, :6] = rng.normal(0, 2.5, (n, 6, 2))
    check(contexts(10), logits, rng.random(12), 2, **random_params(rng, 12, n))
    check(contexts(10), logits, rng.random(6), 1, top_p=np.full(6, 0.95))


@pytest.mark.parametrize("n,log2N,n_slots,parts", [(10, 12, 2048, 1), (10, 12, 2048, 2), (10, 12, 2047, 1), (100, 13, 4096, 2), (1000, 11, 1023, 2),
                                                   (3000, 11, 600, 1)])
def test_many_rows(contexts, n, log2N, n_slots, parts):
    rng = np.random.default_rng(n + n_slots)
    logits = rng.normal(0, 3, (n, 1 << (log2N - 1), 2))
    rows = n_slots * parts
    check(contexts(log2N), logits, rng.random(rows), parts, **random_params(rng, rows, n))


@pytest.mark.parametrize("names", ["t", "k", "p", "m", "kp", "km", "pm", "kpm"])
def test_every_choice_of_filters(contexts, names):
    rng = np.random.default_rng(11)
    logits = rng.normal(0, 2, (700, 512, 2))
    params = {k: v for k, v in random_params(rng, 600, 700).items() if k == "temperature" or k[-1] in names}
    if "t" not in names:
        params.pop("temperature")
    check(contexts(10), logits, rng.random(600), 2, **params)


@pytest.mark.parametrize("levels", [1, 2, 5, 40])
@pytest.mark.parametrize("n", [7, 640, 5000])
def test_equal_logits_are_taken_in_the_order_of_their_indices(contexts, n, levels):
    """... as those of a quantised head are: the cuts fall among tokens of one weight."""
    rng = np.random.default_rng(n + levels)
    logits = rng.integers(0, levels, (n, 512, 2)) * 0.25
    params = {"top_k": rng.integers(0, n + 2, 200), "top_p": rng.choice([1.0, 0.83, 0.31, 0.07], 200)}
    check(contexts(10), logits, rng.random(200), 2, **params)
    check(contexts(10), logits, rng.random(200), 2, top_p=params["top_p"])
    check(contexts(10), logits, rng.random(200), 2, temperature=np.zeros(200), top_k=params["top_k"])


def test_flat_and_far_rows(contexts):
    """Weights that differ in their last bits only, that span every power of two, and rows of one token far above the rest."""
    rng = np.random.default_rng(3)
    n, rows = 4000, 64
    logits = np.zeros((n, 512, 2))
    logits[:, :16] = rng.normal(0, 1e-12, (n, 16, 2))
    logits[:, 16:32] = -rng.random((n, 16, 2)) * 40
    logits[:, 32:48] = rng.normal(0, 1, (n, 16, 2)) * 1e300
    logits[:, 48:64] = rng.normal(0, 0.3, (n, 16, 2))
    logits[17, 48:64] += 25
    u = rng.random(2 * rows)
    k, p = rng.integers(1, 300, 2 * rows), rng.choice([0.9, 0.6, 0.999], 2 * rows)
    # of logits 1e-12 apart the weights differ by a few hundred units, and a token's place in the order may hang on the exponential's last
    # bit: for those rows only that the token has one of the k largest weights or a neighbouring one
    near = slice(0, 32)
    ctx = contexts(10)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    tokens, _ = ctx.sample_slots(torch.view_as_complex(cuda(logits)), cuda(u), parts=2, top_k=cuda(k.astype(np.int32)), top_p=cuda(p))
    tokens = tokens.cpu().numpy()
    for r in range(near.start, near.stop):
        x = logits[:, r // 2, r % 2]
        least = np.sort(x)[-k[r]]
        assert x[tokens[r]] >= least - 2.0**-45, r
    for r in range(near.stop, 2 * rows):
        assert tokens[r] == plain(logits[:, r // 2, r % 2], u[r], 1.0, k[r], p[r])[0], r


def test_nothing_to_take_infinities_and_nan(contexts):
    n = 300
    rng = np.random.default_rng(8)
    logits = rng.normal(0, 1, (n, 512, 2))
    logits[:, 0, 0] = -np.inf                                       # nothing left
    logits[:, 0, 1] = np.nan
    logits[:, 1, 0] = -np.inf
    logits[211, 1, 0] = -1.7e308                                    # one token, of the type's lowest values
    logits[::2, 1, 1] = np.nan
    logits[1::3, 2, 0] = -np.inf
    logits[[5, 77], 2, 1] = np.inf                                  # as good as certain, both alike
    logits[:, 3, 0] = -np.finfo(np.float64).max                     # all equal, the type's lowest value
    logits[:, 3, 1] = 0.0
    logits[3, 3, 1] = -0.0
    for temperature in (1.0, 0.0, 0.01, 1e-310, 1e300, np.inf, -1.0, np.nan):
        u = np.concatenate([rng.random(4), [0.0, 1 - 2.0**-53, 0.5, 0.999]])
        check(contexts(10), logits, u, 2, temperature=np.full(8, temperature), top_k=np.array([0, 3, 1, 5, 0, 0, 2, 299]),
              top_p=np.full(8, 0.9), min_p=np.full(8, 0.05))


def test_parameters_beyond_their_ends(contexts):
    n = 50
    rng = np.random.default_rng(9)
    logits = rng.normal(0, 1, (n, 512, 2))
    u = np.array([0.0, 1.0, 2.0, -1.0, np.nan, np.inf, -np.inf, 0.5])
    check(contexts(10), logits, u, 1)
    half = np.full(8, 0.5)
    check(contexts(10), logits, half, 1, top_p=np.array([0.0, -1.0, 2.0, np.nan, np.inf, 1e-300, 1.0, 0.5]))
    check(contexts(10), logits, half, 1, min_p=np.array([0.0, -1.0, 2.0, np.nan, np.inf, 1e-300, 1.0, 0.5]))
    check(contexts(10), logits, half, 1, top_k=np.array([0, -1, -2**31, 49, 50, 51, 2**31 - 1, 1]).astype(np.int64) % 2**32 % 2**31)


def test_the_other_slots_and_what_lies_behind_are_left_alone(contexts):
    ctx = contexts(11)
    rng = np.random.default_rng(10)
    logits = torch.view_as_complex(torch.from_numpy(rng.normal(0, 1, (20, 1024, 2))).cuda())
    before = logits.clone()
    tokens = torch.full((50,), 77, dtype=torch.int32, device="cuda")
    log_prob = torch.full((50,), 7.5, dtype=torch.float64, device="cuda")
    u = torch.rand(33, dtype=torch.float64, device="cuda")
    ctx.sample_slots(logits, u, out=tokens[:33], log_prob=log_prob[:33])
    assert bool((tokens[33:] == 77).all()) and bool((log_prob[33:] == 7.5).all()) and bool((tokens[:33] < 20).all())
    assert torch.equal(logits, before)


def test_frequencies_follow_the_weights(contexts):
    """Evenly spread numbers (k + 1/2) / rows take each token as often as its share says, to within one."""
    ctx, rows = contexts(13), 4096
    x = torch.tensor([0.3, -1.0, 2.0, 0.0, 1.1, 1.9], dtype=torch.float64, device="cuda")
    slots = x[:, None].expand(6, rows).to(torch.complex128).contiguous()
    u = (torch.arange(rows, dtype=torch.float64, device="cuda") + 0.5) / rows
    tokens, log_prob = ctx.sample_slots(slots, u)
    share = torch.softmax(x, 0)
    assert float((torch.bincount(tokens.long(), minlength=6) - share * rows).abs().max()) <= 1.0
    assert float((log_prob - torch.log(share)[tokens.long()]).abs().max()) <= 6 * 2.0**-46


def test_streams_and_a_captured_graph(contexts):
    ctx = contexts(11)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    slots = torch.view_as_complex(torch.randn((900, 1024, 2), dtype=torch.float64, device="cuda", generator=gen) * 3)
    u = torch.rand(1024, dtype=torch.float64, device="cuda", generator=gen)
    k = torch.full((1024,), 40, dtype=torch.int32, device="cuda")
    p = torch.full((1024,), 0.9, dtype=torch.float64, device="cuda")
    want = ctx.sample_slots(slots, u, top_k=k, top_p=p)
    torch.cuda.synchronize()
    outs = []
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            outs.append(ctx.sample_slots(slots, u, top_k=k, top_p=p))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in outs for a, b in zip(out, want))
    tokens, log_prob = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.sample_slots(slots, u, top_k=k, top_p=p, out=tokens, log_prob=log_prob)
    for _ in range(4):
        u.copy_(torch.rand(1024, dtype=torch.float64, device="cuda", generator=gen))
        eager = ctx.sample_slots(slots, u, top_k=k, top_p=p)
        tokens.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, eager[0]) and torch.equal(log_prob, eager[1])


def test_arrays_at_odd_multiples_of_eight_bytes(contexts):
    ctx = contexts(10)

    def shifted(t):
        raw = torch.empty(t.numel() * t.element_size() + 8, dtype=torch.uint8, device="cuda")
        view = raw[8:].view(t.dtype).view(t.shape)
        view.copy_(t)
        return view

    flat = torch.randn(200 * 1024 + 1, dtype=torch.float64, device="cuda")[1:].view(200, 512, 2)
    slots = torch.view_as_complex(flat.clone())
    odd = torch.empty(200 * 512 * 16 + 8, dtype=torch.uint8, device="cuda")[8:].view(torch.float64).view(200, 512, 2)
    odd.copy_(flat)
    u = torch.rand(1024, dtype=torch.float64, device="cuda")
    p = torch.full_like(u, 0.8)
    want = ctx.sample_slots(slots, u, parts=2, top_p=p)
    lib, ptr = ctx_lib(), lambda t: t.data_ptr()
    tokens, log_prob = shifted(torch.zeros_like(want[0])), shifted(torch.zeros_like(want[1]))
    odd_p, odd_u = shifted(p), shifted(u)
    assert all(ptr(t) % 16 == 8 for t in (odd, odd_p, odd_u, log_prob))
    status = lib.he_sample_slots(ctx._h, ptr(odd), 200, 512, 2, None, None, ptr(odd_p), None, ptr(odd_u), ptr(tokens), ptr(log_prob),
                                 torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == 0 and torch.equal(tokens, want[0]) and torch.equal(log_prob, want[1])


def ctx_lib():
    from paper_1908_04172_amd import he
    return he.lib()
