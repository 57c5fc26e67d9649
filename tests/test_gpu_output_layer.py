"""The output layer of a quantised model on encrypted data, as a server and its client run it: int8 activations with a scale per
token (slot), encrypted; he_ct_i8_mac with int8 weights, channel scales, token scales, bias and one lazy rescale; decryption;
he_decode_vector; he_sample_slots."""
import numpy as np
import pytest

import oracle
from oracle.ckks_scaffold import Scaffold
from paper_1908_04172_amd import workloads as wl
from test_gpu_sample import plain

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
def test_from_encrypted_activations_to_tokens(packed):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1908_04172_amd import he
    N, K, V = 1 << 10, 12, 33
    # packed: three 30-bit limbs; the scales of the channels and the tokens share the one rescale of 30 bits
    q = wl.modulus_chain([30, 30, 30] if packed else [60, 50, 50], N)
    d_in, d_channel, d_token = (2.0**22, 2.0**15, 2.0**15) if packed else (2.0**30, 2.0**25, 2.0**25)
    ctx = he.Context(10, q)
    sc = Scaffold(N, q, ctx.psi, 17)
    rng = np.random.default_rng(18)
    x = rng.normal(0, 1, (K, N // 2)) * rng.uniform(0.5, 2, N // 2)
    token = np.abs(x).max(0) / 127
    x8 = np.rint(x / token)
    w = rng.normal(0, 0.4, (K, V))
    channel = np.abs(w).max(0) / 127
    w8 = np.rint(w / channel).astype(np.int8)
    b = rng.normal(0, 0.5, V)
    plan = wl.dense_plan(K, V)
    layer = ctx.i8_layer(plan.n_in, plan.n_out, plan.n_pt, plan.off, plan.term_ct, plan.term_pt, w8.ravel(), channel, d_channel)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).cuda()
    ct = dev(np.stack([sc.encrypt(x8[k], d_in) for k in range(K)]))
    tok = ctx.encode_vector(torch.from_numpy(token.astype(np.complex128)[None]).cuda(), d_token)[0]
    bias = ctx.encode_scalar(torch.from_numpy(b).cuda(), d_in * d_channel * d_token)
    if packed:
        out = ctx.unpack32(ctx.ct_i8_mac32(layer, ctx.pack32(ct), ctx.pack32(tok), bias, flags=he.RESCALE))
    else:
        out = ctx.ct_i8_mac(layer, ct, tok, bias, flags=he.RESCALE)
    c = out.cpu().numpy().view(np.uint64)
    poly = np.empty((V, 2, N), np.uint64)
    for i in range(2):
        poly[:, i] = ((c[:, 0, i].astype(object) + c[:, 1, i].astype(object) * sc.s_ntt[i].astype(object)) % q[i]).astype(np.uint64)
    slots = ctx.decode_vector(dev(poly), d_in * d_channel * d_token / q[2])
    # against the float layer with the scales as they were encoded (a scalar rounded to 1 / d_channel, a polynomial's coefficients to 1 / d_token)
    channel = np.rint(channel * d_channel) / d_channel
    token = ctx.decode_vector(tok[None], d_token).cpu().numpy()[0].real
    want = (w8 * channel).T @ (x8 * token) + b[:, None]
    # The encryption's noise, below 6 * 3.2 in each of N coefficients, reaches a slot as at most 20 N, over d_in and times a row of weights.
    # The rescale's roundings (e0 + e1 s, a ternary secret s) have a standard deviation below sqrt(N / 12) per coefficient and below
    # N / sqrt(12) per slot, over the scale that is left: six of them.  2^-20: the bias's encoding and the doubles of the decoder.
    scale_out = d_in * d_channel * d_token / q[2]
    bound = 20 * N / d_in * np.abs(w8 * channel).sum(0).max() * np.abs(token).max() + 6 * N / 12**0.5 / scale_out + 2.0**-20
    got = slots.cpu().numpy()
    worst = np.abs(got.real - want).max()
    assert worst <= bound, (worst, bound)
    rows = N // 2
    u, t, k = rng.random(rows), rng.choice([0.0, 0.8, 1.2], rows), rng.choice([0, 3, 10], rows)
    p, m = np.full(rows, 0.9), np.full(rows, 0.02)
    cuda = lambda a: torch.from_numpy(a).cuda()
    tokens, log_prob = ctx.sample_slots(slots, cuda(u), temperature=cuda(t), top_k=cuda(k.astype(np.int32)), top_p=cuda(p), min_p=cuda(m))
    tokens, log_prob = tokens.cpu().numpy(), log_prob.cpu().numpy()
    for r in range(rows):
        expect = plain(got[:, r].real, u[r], t[r], k[r], p[r], m[r])
        assert tokens[r] == expect[0] and abs(log_prob[r] - expect[1]) <= 2.0**-46 * (V + abs(expect[1]))
        top = np.sort(want[:, r])
        if t[r] == 0 and top[-1] - top[-2] > 2 * bound:
            assert tokens[r] == int(np.argmax(want[:, r]))
