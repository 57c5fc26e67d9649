"""Two operators of encrypted language models, as cases to time: the matrix product in 8-bit integers over tensors of
ciphertexts, with a scale for each channel and each token, and the sampling of answers from the decoded slots.

They are the two ends of an output layer on ciphertexts.  The server multiplies the encrypted activations by int8 weights (one
scalar scale per output channel; one scale per token, that is per slot, where the client quantised its tokens one by one) and
the client, which has decrypted and decoded the logits, picks a token per slot.

Kinds:
  i8      out[o] = token * (channel[o] * sum over t of w[term_pt[t]] * ct[term_ct[t]]) + bias[o] (bias on component 0), modulo
          every limb's prime, over a dense layer or a convolution; residues in 64-bit words, or packed in 32-bit words
  sample  a token per row of decoded logits, slots [n][N/2] complex, from a given uniform number per row: temperature, top-k,
          top-p and min-p; and the logarithm of its probability among the tokens that the filters leave

A case is a dict of plain values.  "bits" is the modulus chain as text, one bit size per limb.  Residues and tokens are whole
numbers.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
WEIGHT_ONE = 47  # a row's weights are whole multiples of 2^-47 of its largest


def listed():
    return [
        # a small dense layer of 30-bit moduli: launches and latency count
        {"name": "i8_dense_64_16", "kind": "i8", "log2N": 12, "bits": "30 30", "layer": "dense", "K": 64, "M": 16, "channel": True,
         "token": False, "bias": True, "packed": False},
        # the first convolution over a 28x28 image, five filters: short sums, as many outputs as inputs
        {"name": "i8_conv_28x28x1_5", "kind": "i8", "log2N": 13, "bits": "60 40 40 40", "layer": "conv", "H": 28, "C": 1, "KH": 5,
         "OC": 5, "stride": 2, "padding": "valid", "channel": True, "token": False, "bias": True, "packed": False},
        # a dense layer of long sums and an odd number of outputs, tokens with scales of their own
        {"name": "i8_dense_845_100", "kind": "i8", "log2N": 13, "bits": "60 40 40 40", "layer": "dense", "K": 845, "M": 100,
         "channel": True, "token": True, "bias": True, "packed": False},
        # a vocabulary (or a thousand classes) from a hidden state: many outputs per input
        {"name": "i8_head_256_1000", "kind": "i8", "log2N": 12, "bits": "60 40", "layer": "dense", "K": 256, "M": 1000,
         "channel": True, "token": False, "bias": True, "packed": False},
        # the same layer in packed storage, with more of both: the matrix cores' share counts
        {"name": "i8_packed_1024_1024", "kind": "i8", "log2N": 12, "bits": "30 30", "layer": "dense", "K": 1024, "M": 1024,
         "channel": True, "token": False, "bias": True, "packed": True},
        # a padded convolution of a feature map at a larger ring: the most bytes
        {"name": "i8_conv_16x16x8_16", "kind": "i8", "log2N": 13, "bits": "60 50 50", "layer": "conv", "H": 16, "C": 8, "KH": 3,
         "OC": 16, "stride": 1, "padding": "same", "channel": True, "token": True, "bias": True, "packed": False},
        # one token of an eight-limb chain through a slim projection, no scales: the sums alone
        {"name": "i8_dense_113_37", "kind": "i8", "log2N": 14, "bits": "60 60 50 50 50 50 50 50", "layer": "dense", "K": 113, "M": 37,
         "channel": False, "token": False, "bias": False, "packed": False},
        # ten classes, every slot an image: the smallest rows
        {"name": "sample_10x2048", "kind": "sample", "log2N": 12, "n": 10, "slots": 2048, "parts": 1, "filters": ""},
        # a thousand classes, every slot an image, all filters
        {"name": "sample_1000x4096", "kind": "sample", "log2N": 13, "n": 1000, "slots": 4096, "parts": 1, "filters": "k p m"},
        # a vocabulary with two tokens per slot (complex packing)
        {"name": "sample_8192x4096", "kind": "sample", "log2N": 12, "n": 8192, "slots": 2048, "parts": 2, "filters": "k p"},
        # a small batch: few rows, of a vocabulary of an odd size
        {"name": "sample_5003x37", "kind": "sample", "log2N": 12, "n": 5003, "slots": 37, "parts": 1, "filters": "p m"},
    ]


def _log_int(rng, low, high):
    """low..high, spread over the logarithm; odd sizes as they come."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _draw_once(rng):
    if rng.random() < 0.4:
        log2N = rng.choice([11, 12, 13])
        slots = _log_int(rng, 1, 1 << (log2N - 1))
        filters = " ".join(f for f in "kpm" if rng.random() < 0.6)
        return {"kind": "sample", "log2N": log2N, "n": _log_int(rng, 2, 16000), "slots": slots, "parts": rng.choice([1, 2]),
                "filters": filters}
    packed = rng.random() < 0.25
    log2N = rng.choice([12, 13, 13, 14])
    if packed:
        bits = " ".join(["30"] * rng.randint(1, 4))
    else:
        first, rest, most = rng.choice([("30", "30", 4), ("60", "40", 5), ("60", "45", 4), ("60 60", "50", 8), ("58", "55", 4)])
        n = rng.randint(len(first.split()), most)
        bits = " ".join([first] + [rest] * (n - len(first.split())))
    case = {"kind": "i8", "log2N": log2N, "bits": bits, "channel": rng.random() < 0.8, "token": rng.random() < 0.4,
            "bias": rng.random() < 0.7, "packed": packed}
    if rng.random() < 0.6:
        return dict(case, layer="dense", K=_log_int(rng, 1, 1024), M=_log_int(rng, 1, 1024))
    KH = rng.choice([1, 3, 3, 5])
    return dict(case, layer="conv", H=rng.randint(max(6, KH), 28), C=rng.randint(1, 8), KH=KH, OC=_log_int(rng, 1, 32),
                stride=1 if KH == 1 else rng.choice([1, 2]), padding=rng.choice(["valid", "same"]))


def draw(rng):
    """One more case; none costs more than the largest of listed()."""
    while True:
        case = _draw_once(rng)
        w = work(case)
        if case["kind"] == "sample":
            if (case["n"] * 16) << (case["log2N"] - 1) <= 2.7e8:
                return case
        elif w["bytes"] <= 2.4e9 and w["flops"] <= 3.4e10:
            return case


# ------------------------------------------------------------------------------------------------ shapes


def _windows(case):
    """A convolution's windows: (number, taps of each window as (input, weight row) pairs)."""
    H, C, KH, stride = case["H"], case["C"], case["KH"], case["stride"]
    if case["padding"] == "valid":
        OH, first = (H - KH) // stride + 1, 0
    else:
        OH = -(-H // stride)
        first = max((OH - 1) * stride + KH - H, 0) // 2
    out = []
    for oh in range(OH):
        for ow in range(OH):
            taps = []
            for kh in range(KH):
                for kw in range(KH):
                    h, w = oh * stride + kh - first, ow * stride + kw - first
                    if 0 <= h < H and 0 <= w < H:
                        taps += [((h * H + w) * C + c, (kh * KH + kw) * C + c) for c in range(C)]
            out.append(taps)
    return out


def _shape(case):
    """(inputs, outputs, weights, terms)"""
    if case["layer"] == "dense":
        return case["K"], case["M"], case["K"] * case["M"], case["K"] * case["M"]
    windows = _windows(case)
    C, OC = case["C"], case["OC"]
    return case["H"] ** 2 * C, len(windows) * OC, case["KH"] ** 2 * C * OC, sum(map(len, windows)) * OC


def work(case):
    if case["kind"] == "sample":
        rows = case["slots"] * case["parts"]
        per_row = 8 + 8 + 4 + 8 + (4 if "k" in case["filters"] else 0) + 8 * (("p" in case["filters"]) + ("m" in case["filters"]))
        return {"bytes": case["n"] * rows * 8 + rows * per_row, "flops": 4 * case["n"] * rows}
    n_in, n_out, n_pt, n_terms = _shape(case)
    limbs, N = len(case["bits"].split()), 1 << case["log2N"]
    word = 4 if case["packed"] else 8
    row = 2 * limbs * N
    read = n_in * row * word + n_pt + (n_out * limbs * 8 if case["bias"] else 0) + (n_out * 8 if case["channel"] else 0)
    read += limbs * N * word if case["token"] else 0
    # one multiply-add per term and residue, and one product per scale and residue of the output
    return {"bytes": read + n_out * row * word, "flops": 2 * n_terms * row + (case["channel"] + case["token"]) * n_out * row}


# ------------------------------------------------------------------------------------------------ inputs


def _is_prime(n):
    if n < 2:
        return False
    for p in (2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37):
        if n % p == 0:
            return n == p
    d, r = n - 1, 0
    while d % 2 == 0:
        d, r = d // 2, r + 1
    for a in (2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37):
        x = pow(a, d, n)
        if x in (1, n - 1):
            continue
        for _ in range(r - 1):
            x = x * x % n
            if x == n - 1:
                break
        else:
            return False
    return True


def _primes(case):
    """The modulus chain: for each bit size the largest primes = 1 (mod 2N) below it, each once."""
    step, taken, chain = 2 << case["log2N"], {}, []
    for b in map(int, case["bits"].split()):
        p = taken.get(b, ((1 << b) - 1) // step * step + 1 + step) - step
        while p >= 1 << b or not _is_prime(p):
            p -= step
        taken[b] = p
        chain.append(p)
    return chain


def _terms(case):
    """The layer as the framework's plans describe it: off, term_ct, term_pt."""
    if case["layer"] == "dense":
        K, M = case["K"], case["M"]
        k = np.tile(np.arange(K, dtype=np.uint32), M)
        return np.arange(M + 1, dtype=np.uint32) * np.uint32(K), k, k * np.uint32(M) + np.repeat(np.arange(M, dtype=np.uint32), K)
    OC, off, ct, pt = case["OC"], [0], [], []
    for taps in _windows(case):
        taps = np.asarray(taps, dtype=np.uint32).reshape(-1, 2)
        for oc in range(OC):
            ct.append(taps[:, 0])
            pt.append(taps[:, 1] * np.uint32(OC) + np.uint32(oc))
            off.append(off[-1] + len(taps))
    return np.asarray(off, np.uint32), np.concatenate(ct), np.concatenate(pt)


def _residues(shape, q, N, gen, dtype=torch.int64):
    """[*shape][len(q)][N], limb i uniform below q[i]: what ciphertexts look like."""
    out = torch.empty(tuple(shape) + (len(q), N), dtype=dtype, device=DEVICE)
    for i, qi in enumerate(q):
        out[..., i, :] = torch.randint(0, qi, tuple(shape) + (N,), dtype=torch.int64, device=DEVICE, generator=gen).to(dtype)
    return out


def _encode(values, scale, q):
    """round(scale * value), halves away from zero, modulo each prime: [n][limbs] (magnitudes below 2^53)"""
    v = values * scale
    whole = (torch.sign(v) * torch.floor(v.abs() + 0.5)).to(torch.int64)
    return torch.stack([whole % qi for qi in q], dim=1).contiguous()


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def _inputs_i8(case, seed):
    gen = _generator(seed)
    q, N = _primes(case), 1 << case["log2N"]
    n_in, n_out, n_pt, _ = _shape(case)
    dtype = torch.int32 if case["packed"] else torch.int64
    outs = case["M"] if case["layer"] == "dense" else case["OC"]
    d = {"q": q, "N": N}
    # int8 weights of a normal distribution, the largest of a channel near 127
    d["w"] = torch.randn((n_pt // outs, outs), device=DEVICE, generator=gen).mul_(40).round_().clamp_(-128, 127).to(torch.int8)
    d["ct"] = _residues((n_in, 2), q, N, gen, dtype)
    channel = torch.rand(outs, device=DEVICE, generator=gen, dtype=torch.float64).mul_(0.01).add_(0.001)
    d["channel"] = channel.repeat(n_out // outs) if case["channel"] else None
    d["scale"] = 2.0 ** 25
    d["token"] = _residues((), q, N, gen, dtype) if case["token"] else None
    bias = torch.randn(n_out, device=DEVICE, generator=gen, dtype=torch.float64)
    d["bias"] = _encode(bias, 2.0 ** 40, q) if case["bias"] else None
    return d


def _inputs_sample(case, seed):
    gen = _generator(seed)
    n, half, rows = case["n"], 1 << (case["log2N"] - 1), case["slots"] * case["parts"]
    # logits of a normal distribution whose width differs from slot to slot, a few tokens well above the others, and what is left
    # of the encryption's noise
    width = torch.rand((1, half, 2), device=DEVICE, generator=gen, dtype=torch.float64).mul_(3).add_(0.5)
    logits = torch.randn((n, half, 2), device=DEVICE, generator=gen, dtype=torch.float64) * width
    lift = torch.rand((n, 1, 1), device=DEVICE, generator=gen, dtype=torch.float64)
    logits += torch.where(lift < 4.0 / n, 3.0, 0.0)
    d = {"slots": torch.view_as_complex(logits), "u": torch.rand(rows, device=DEVICE, generator=gen, dtype=torch.float64)}

    def pick(values, dtype):
        at = torch.randint(0, len(values), (rows,), device=DEVICE, generator=gen)
        return torch.tensor(values, dtype=dtype, device=DEVICE)[at]

    d["temperature"] = pick([0.0, 0.5, 0.7, 1.0, 1.0, 1.3], torch.float64)
    d["top_k"] = pick([0, 1, 5, 40, 50, 500], torch.int32) if "k" in case["filters"] else None
    d["top_p"] = pick([1.0, 0.95, 0.9, 0.9, 0.3], torch.float64) if "p" in case["filters"] else None
    d["min_p"] = pick([0.0, 0.02, 0.1], torch.float64) if "m" in case["filters"] else None
    return d


def prepare(case, seed):
    if case["kind"] == "sample":
        d = _inputs_sample(case, seed)
        state = {"case": case, **d, "out": torch.empty(d["u"].numel(), dtype=torch.int32, device=DEVICE),
                 "log_prob": torch.empty_like(d["u"])}
        if own:
            from paper_1908_04172_amd import he
            # (the sampler needs a ring degree and a device of the context, and no particular modulus)
            state["ctx"] = he.Context(case["log2N"], _primes(dict(case, bits="30")), device=0)
        return state
    d = _inputs_i8(case, seed)
    n_in, n_out, n_pt, _ = _shape(case)
    state = {"case": case, **d, "out": torch.empty((n_out,) + tuple(d["ct"].shape[1:]), dtype=d["ct"].dtype, device=DEVICE)}
    if own:
        from paper_1908_04172_amd import he
        ctx = he.Context(case["log2N"], d["q"], device=0)
        state["ctx"] = ctx
        state["layer"] = ctx.i8_layer(n_in, n_out, n_pt, *_terms(case), d["w"].reshape(-1).cpu().numpy(),
                                      None if d["channel"] is None else d["channel"].cpu().numpy(), d["scale"])
        return state
    state["s"] = None if d["channel"] is None else _encode(d["channel"], d["scale"], d["q"])
    if case["layer"] == "conv":
        windows = _windows(case)
        K = case["KH"] ** 2 * case["C"]
        index, there = np.zeros((K, len(windows)), np.int64), np.zeros((K, len(windows)), bool)
        for j, taps in enumerate(windows):
            for ct, row in taps:
                index[row, j], there[row, j] = ct, True
        state["index"] = torch.from_numpy(index).to(DEVICE)
        state["there"] = torch.from_numpy(there).to(DEVICE)
    return state


# ------------------------------------------------------------------------------------------------ the plain forms


def _mul_small(a, c, q):
    """a * c mod q, 0 <= a < q < 2^60, 0 <= c < 2^31 (numbers or tensors): the quotient from doubles is off by at most one"""
    k = torch.floor(a.double() * (c.double() if torch.is_tensor(c) else float(c)) / q).to(torch.int64)
    r = a * c - k * q  # wraps around 2^64, the difference does not
    r = torch.where(r < 0, r + q, r)
    return torch.where(r >= q, r - q, r)


def _mul(a, b, q):
    """a * b mod q for residues below q < 2^60"""
    high = _mul_small(_mul_small(a, b >> 30, q), 1 << 30, q)
    return (high + _mul_small(a, b & ((1 << 30) - 1), q)) % q


def _plain_i8(state):
    case, q, N, out = state["case"], state["q"], state["N"], state["out"]
    conv = case["layer"] == "conv"
    wt = state["w"].double().t().contiguous()  # [outputs of a window][K]
    n_win = state["index"].shape[1] if conv else 1
    step = max(1, (1 << 26) // (wt.shape[1] * 2 * N)) if conv else 1
    cols = 2 * N if conv else max(N // 4, min(2 * N, (1 << 26) // wt.shape[1] // 512 * 512))
    for i, qi in enumerate(q):
        for first in range(0, n_win, step):
            last = min(n_win, first + step)
            for c0 in range(0, 2 * N, cols):
                if conv:
                    x = state["ct"][:, :, i, :].reshape(-1, 2 * N)[state["index"][:, first:last]].long()
                    x = x * state["there"][:, first:last, None]
                    x = x.reshape(wt.shape[1], -1)
                else:
                    x = state["ct"][:, :, i, :].reshape(-1, 2 * N)[:, c0:c0 + cols].long()
                # two pieces of the residues, each of whose sums a double holds exactly
                low = torch.matmul(wt, (x & ((1 << 30) - 1)).double()).to(torch.int64) % qi
                high = torch.matmul(wt, (x >> 30).double()).to(torch.int64) % qi
                v = (_mul_small(high, 1 << 30, qi) + low) % qi
                # [outputs][windows][columns] -> [windows * outputs][columns]
                v = v.reshape(wt.shape[0], last - first, -1).transpose(0, 1).reshape(-1, v.shape[1] // (last - first))
                rows = slice(first * wt.shape[0], last * wt.shape[0])
                if state["s"] is not None:
                    v = _mul(v, state["s"][rows, i, None], qi)
                if state["token"] is not None:
                    v = _mul(v, state["token"][i].long().repeat(2)[None, c0:c0 + cols], qi)
                if state["bias"] is not None and c0 < N:
                    v[:, :N - c0] = (v[:, :N - c0] + state["bias"][rows, i, None]) % qi
                dst = out[rows, :, i, :]
                if cols == 2 * N:
                    dst.copy_(v.reshape(-1, 2, N))
                else:
                    for part in range(2):
                        a, b = max(c0, part * N), min(c0 + v.shape[1], (part + 1) * N)
                        if a < b:
                            dst[:, part, a - part * N:b - part * N] = v[:, a - c0:b - c0].to(out.dtype)
    return out


def _plain_sample(state):
    case = state["case"]
    n, parts, rows = case["n"], case["parts"], state["u"].numel()
    out = state["out"]
    logits = torch.view_as_real(state["slots"])[:, :case["slots"], :parts].reshape(n, rows)
    step = max(1, (1 << 25) // n)
    for a in range(0, rows, step):
        r = slice(a, min(rows, a + step))
        x = logits[:, r].t()  # [rows][n]
        top, arg = x.max(dim=1, keepdim=True).values, None
        first = torch.where(x == top, torch.arange(n, device=DEVICE), n).min(dim=1).values
        t = state["temperature"][r, None]
        one = float(1 << WEIGHT_ONE)
        w = torch.round(torch.exp((x - top) * (1.0 / t)) * one)
        w = torch.where(x == top, one, w).to(torch.int64)
        if state["top_k"] is not None or state["top_p"] is not None:
            s, order = torch.sort(w, dim=1, descending=True, stable=True)
            if state["top_k"] is not None:
                k = state["top_k"][r, None].long()
                s = torch.where((torch.arange(n, device=DEVICE) < k) | (k == 0), s, 0)
            if state["top_p"] is not None:
                p = state["top_p"][r, None]
                run = torch.cumsum(s, dim=1)
                need = torch.ceil(run[:, -1:].double() * p).to(torch.int64)
                s = torch.where((run - s < need) | (p >= 1), s, 0)
            w = torch.zeros_like(w).scatter_(1, order, s)
        if state["min_p"] is not None:
            w = torch.where(w.double() >= state["min_p"][r, None] * one, w, 0)
        run = torch.cumsum(w, dim=1)
        total = run[:, -1:]
        at = torch.minimum(torch.floor(total.double() * state["u"][r, None]).to(torch.int64), total - 1)
        token = (run <= at).sum(dim=1)
        token = torch.where(t[:, 0] > 0, token, first)
        out[r] = token.to(torch.int32)
        log_prob = ((torch.gather(x, 1, token[:, None]) - top) * (1.0 / t) - torch.log(total.double() / one))[:, 0]
        state["log_prob"][r] = torch.where(t[:, 0] > 0, log_prob, 0.0)
    return out, state["log_prob"]


def run(state):
    case = state["case"]
    if not own:
        return _plain_sample(state) if case["kind"] == "sample" else _plain_i8(state)
    ctx = state["ctx"]
    if case["kind"] == "sample":
        return ctx.sample_slots(state["slots"], state["u"], parts=case["parts"], temperature=state["temperature"],
                                top_k=state["top_k"], top_p=state["top_p"], min_p=state["min_p"], out=state["out"],
                                log_prob=state["log_prob"])
    call = ctx.ct_i8_mac32 if case["packed"] else ctx.ct_i8_mac
    return call(state["layer"], state["ct"], token_scale=state["token"], bias=state["bias"], out=state["out"])


# ------------------------------------------------------------------------------------------------ the definitions


def _exact_i8(case, seed):
    n_in, n_out, n_pt, n_terms = _shape(case)
    limbs, N = len(case["bits"].split()), 1 << case["log2N"]
    if n_out * 2 * limbs * N > 1 << 20 or n_terms * 2 * limbs * N > 1 << 31:
        return None
    d = _inputs_i8(case, seed)
    ct, w = d["ct"].cpu().numpy().astype(np.int64), d["w"].cpu().numpy().reshape(-1).astype(np.float64)
    off, term_ct, term_pt = _terms(case)
    out = np.empty((n_out, 2, limbs, N), np.int32 if case["packed"] else np.int64)
    for i, q in enumerate(d["q"]):
        low, high = (ct[:, :, i] & 0xFFFFFF).astype(np.float64), (ct[:, :, i] >> 24).astype(np.float64)
        for o in range(n_out):
            t = slice(int(off[o]), int(off[o + 1]))
            # sums of at most 2^11 products below 2^43: whole numbers that a double holds
            a = np.tensordot(w[term_pt[t]], low[term_ct[t]], 1).astype(np.int64).astype(object)
            b = np.tensordot(w[term_pt[t]], high[term_ct[t]], 1).astype(np.int64).astype(object)
            v = a + b * (1 << 24)
            if d["channel"] is not None:
                v = v * int(math.floor(float(d["channel"][o]) * d["scale"] + 0.5))
            if d["token"] is not None:
                v = v * d["token"][i].cpu().numpy().astype(object)
            if d["bias"] is not None:
                v[0] = v[0] + int(d["bias"][o, i])
            out[o, :, i] = (v % q).astype(out.dtype)
    return torch.from_numpy(out)


def _exact_sample(case, seed):
    n, rows = case["n"], case["slots"] * case["parts"]
    if n * rows > 1 << 23:
        return None
    d = {k: None if v is None else v.cpu().numpy() for k, v in _inputs_sample(case, seed).items()}
    out, log_prob = np.empty(rows, np.int32), np.zeros(rows)
    for r in range(rows):
        z = d["slots"][:, r // case["parts"]]
        x = z.real if r % case["parts"] == 0 else z.imag
        top = x.max()
        t = d["temperature"][r]
        if not t > 0:
            out[r] = int(np.flatnonzero(x == top)[0])
            continue
        w = np.rint(np.exp((x - top) * (1.0 / t)) * 2.0 ** WEIGHT_ONE).astype(np.int64)
        order = np.argsort(-w, kind="stable")
        keep = n
        if d["top_k"] is not None and d["top_k"][r] > 0:
            keep = min(keep, int(d["top_k"][r]))
        sums = np.cumsum(w[order[:keep]])
        if d["top_p"] is not None and d["top_p"][r] < 1:
            need = math.ceil(float(sums[-1]) * float(d["top_p"][r]))
            keep = min(keep, int(np.searchsorted(sums, need)) + 1)
        kept = np.zeros(n, np.int64)
        kept[order[:keep]] = w[order[:keep]]
        if d["min_p"] is not None:
            kept[kept < d["min_p"][r] * 2.0 ** WEIGHT_ONE] = 0
        sums = np.cumsum(kept)
        at = min(math.floor(float(sums[-1]) * float(d["u"][r])), int(sums[-1]) - 1)
        out[r] = int(np.searchsorted(sums, at, side="right"))
        log_prob[r] = (x[out[r]] - top) * (1.0 / t) - math.log(int(sums[-1]) / 2.0 ** WEIGHT_ONE)
    return torch.from_numpy(out), torch.from_numpy(log_prob)


def exact(case, seed):
    return _exact_sample(case, seed) if case["kind"] == "sample" else _exact_i8(case, seed)
