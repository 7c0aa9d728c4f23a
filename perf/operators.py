"""Prompt attention, the 4-bit key/value cache and token log probabilities, as a
program using this package calls them, beside their plain forms.

Four families:

  prompt         a packed batch of prompts of different lengths: queries and
                 keys rotated, keys and values appended to the fp16 caches,
                 causal grouped-query attention over them (sq_attention_prompt)
  kv4_append     the new tokens' keys and values into the 4-bit caches, and
                 read back as fp16 (sq_kv4_append, sq_kv4_unpack)
  kv4_attention  decode or verify attention over the 4-bit caches
                 (sq_attention_kv4)
  logprobs       log probabilities of given tokens with the rows' entropies and
                 top alternatives, from fp16 logits (sq_logprobs)

Head counts and vocabularies are those of shapes.STACKS, or generic.
"""
import math
import random

import torch

own = False

D = 128
THETA = 1e6
# rates behind the cost bound of drawn cases (bytes/s, flop/s); only their
# ratio matters
COST_BYTES, COST_FLOPS = 6.8e12, 1.7e15


# ---- cases ---------------------------------------------------------------------

def listed():
    return [
        # the smallest prompt: one question of 20 tokens, 1.5B heads
        {"name": "prompt_20", "family": "prompt", "B": 1, "longest": 20, "mix": 0, "prefix": 0, "pad": 0,
         "q_heads": 12, "kv_heads": 2, "max_ctx": 256},
        # a batch of prompts of mixed lengths, 7B heads, rows padded for a
        # captured graph
        {"name": "prompt_ragged_12x1000", "family": "prompt", "B": 12, "longest": 1000, "mix": 3, "prefix": 0,
         "pad": 13, "q_heads": 28, "kv_heads": 4, "max_ctx": 2048},
        # the next chunk of a long document behind 12000 cached tokens, 14B heads
        {"name": "prompt_chunk_300_behind_12k", "family": "prompt", "B": 1, "longest": 300, "mix": 0,
         "prefix": 12000, "pad": 0, "q_heads": 40, "kv_heads": 8, "max_ctx": 16384},
        # one whole prompt of 8000 tokens, 14B heads
        {"name": "prompt_8000", "family": "prompt", "B": 1, "longest": 8000, "mix": 0, "prefix": 0, "pad": 0,
         "q_heads": 40, "kv_heads": 8, "max_ctx": 8192},
        # a decode step's append: one token of each of 16 sequences
        {"name": "kv4_append_16x1", "family": "kv4_append", "B": 16, "longest": 1, "mix": 0, "prefix": 900,
         "q_heads": 40, "kv_heads": 8, "max_ctx": 1024},
        # a batch of prompts quantised into the cache
        {"name": "kv4_append_ragged_8x2000", "family": "kv4_append", "B": 8, "longest": 2000, "mix": 5, "prefix": 0,
         "q_heads": 40, "kv_heads": 8, "max_ctx": 2048},
        # the verify step of one short conversation, five tokens, 1.5B heads
        {"name": "kv4_verify_5_behind_1000", "family": "kv4_attention", "B": 1, "T": 5, "ctx": 1000, "q_heads": 12,
         "kv_heads": 2, "max_ctx": 2048},
        # a decode step of four long conversations, 14B heads
        {"name": "kv4_decode_4x8000", "family": "kv4_attention", "B": 4, "T": 1, "ctx": 8000, "q_heads": 40,
         "kv_heads": 8, "max_ctx": 16384},
        # a verify step of sixteen long documents, 7B heads
        {"name": "kv4_verify_16x5_behind_30k", "family": "kv4_attention", "B": 16, "T": 5, "ctx": 30000,
         "q_heads": 28, "kv_heads": 4, "max_ctx": 32768},
        # one decoded token's log probability and 20 alternatives
        {"name": "logprobs_1x151936_top20", "family": "logprobs", "R": 1, "vocab": 151936, "top": 20,
         "temperature": 1.0},
        # a ragged vocabulary: rows of 50021 entries, unaligned
        {"name": "logprobs_77x50021_top5", "family": "logprobs", "R": 77, "vocab": 50021, "top": 5,
         "temperature": 0.7},
        # scoring 1000 positions of a prompt
        {"name": "logprobs_1000x152064_top5", "family": "logprobs", "R": 1000, "vocab": 152064, "top": 5,
         "temperature": 1.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return w["bytes"] / COST_BYTES + w["flops"] / COST_FLOPS


def draw(rng):
    """A case of the same ranges, no dearer than the dearest listed one of its family."""
    while True:
        case = _draw_any(rng)
        alike = [c for c in listed() if c["family"] == case["family"]]
        if _cost(case) <= max(_cost(c) for c in alike) and _scores(case) <= max(_scores(c) for c in alike):
            return case


def _scores(case):
    """Scores that the plain form of prompt attention holds at once."""
    if case["family"] != "prompt":
        return 0
    return case["B"] * case["q_heads"] * case["longest"] * (case["prefix"] + case["longest"])


def _draw_any(rng):
    family = rng.choice(["prompt", "prompt", "prompt", "kv4_append", "kv4_attention", "kv4_attention", "logprobs",
                         "logprobs"])
    if family == "logprobs":
        return {"family": family, "R": _log_int(rng, 1, 2000),
                "vocab": rng.choice([32000, 151936, 152064, _log_int(rng, 1000, 300000)]),
                "top": rng.choice([0, 1, 5, 20, rng.randint(2, 32)]), "temperature": rng.choice([0.7, 1.0, 1.3])}
    kv = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 5, 6, 7, 8])
    if family == "kv4_attention":
        T = rng.choice([1, 1, 2, _log_int(rng, 2, min(32, 200 // g))])
        ctx = _log_int(rng, 1, 30000)
        return {"family": family, "B": _log_int(rng, 1, 16), "T": T, "ctx": ctx, "q_heads": kv * g, "kv_heads": kv,
                "max_ctx": (int((ctx + T) * rng.choice([1.0, 1.3, 4.0])) + 15) // 16 * 16}
    longest = _log_int(rng, 1, 8000 if family == "prompt" else 2000)
    prefix = rng.choice([0, 0, _log_int(rng, 1, 12000)])
    case = {"family": family, "B": _log_int(rng, 1, 16), "longest": longest, "mix": rng.randint(0, 99),
            "prefix": prefix, "q_heads": kv * g, "kv_heads": kv,
            "max_ctx": (longest + prefix + rng.choice([0, 5, 1000]) + 15) // 16 * 16}
    if family == "prompt":
        case["pad"] = rng.choice([0, 0, 7])
    return case


def _lengths(case):
    """Sequence lengths of a packed batch: the first the longest, the others
    down to single tokens (mix 0: all alike), and the positions they start at."""
    r = random.Random(case["mix"])
    n = case["longest"]
    lens = [n if b == 0 or case["mix"] == 0 else _log_int(r, 1, n) for b in range(case["B"])]
    return lens, [max(0, case["prefix"] - 5 * b) for b in range(case["B"])]


def work(case):
    """What a pass cannot do without: every input read once, every output
    written once, two operations a multiply-add of the products over the keys
    that a query sees."""
    if case["family"] == "logprobs":
        R, V, k = case["R"], case["vocab"], case["top"]
        # a difference, a product, an exponential, two sums and a comparison an entry
        return {"bytes": 2.0 * R * V + R * (12 + 8 * k), "flops": 6.0 * R * V}
    Hq, Hkv = case["q_heads"], case["kv_heads"]
    if case["family"] == "kv4_attention":
        B, T = case["B"], case["T"]
        pos0 = [max(0, case["ctx"] - 7 * b) for b in range(B)]
        seen = sum(p + T for p in pos0)
        pairs = sum(p + t + 1 for p in pos0 for t in range(T))
        return {"bytes": 2.0 * 68 * Hkv * seen + 4.0 * B * T * Hq * D, "flops": 4.0 * D * Hq * pairs}
    lens, pos0 = _lengths(case)
    N = sum(lens)
    if case["family"] == "kv4_append":
        # keys and values read, 68 bytes of each written, and read back to fp16
        return {"bytes": 2.0 * N * Hkv * (2 * D + 2 * 68 + 2 * D), "flops": 2.0 * N * Hkv * D * 6}
    pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(lens, pos0))
    seen = sum(p for p in pos0)
    return {"bytes": 2.0 * N * (Hq + 2 * Hkv) * D + 2.0 * N * Hq * D + 4.0 * (N + seen) * Hkv * D,
            "flops": 4.0 * D * Hq * pairs}


# ---- inputs --------------------------------------------------------------------

def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _normal(seed, shape, std=1.0, dtype=torch.float16):
    g = torch.Generator(device=_device())
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=_device()).normal_(0.0, std, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=_device())


def _packed(case):
    lens, pos0 = _lengths(case)
    offsets = [sum(lens[:b]) for b in range(len(lens) + 1)]
    return lens, pos0, offsets, offsets[-1] + case.get("pad", 0)


def _empty_kv4(case):
    B, Hkv, C = case["B"], case["kv_heads"], case["max_ctx"]
    u8 = dict(dtype=torch.uint8, device=_device())
    f16 = dict(dtype=torch.float16, device=_device())
    return [torch.zeros((B, Hkv, C, D // 2), **u8), torch.zeros((B, Hkv, C, 2), **f16),
            torch.zeros((B, Hkv, C, D // 2), **u8), torch.zeros((B, Hkv, C, 2), **f16)]


def prepare(case, seed):
    if case["family"] == "logprobs":
        R, V = case["R"], case["vocab"]
        z = _normal(seed, (R, V), 2.0)
        # every third row is sure of its token, as a trained model's often are
        g = torch.Generator(device=_device())
        g.manual_seed(seed + 1)
        tokens = torch.randint(0, V, (R,), device=_device(), generator=g, dtype=torch.int32)
        rows = torch.arange(0, R, 3, device=_device())
        z[rows, tokens[rows].long()] = 24.0
        f32 = dict(dtype=torch.float32, device=_device())
        top = case["top"]
        return {"case": case, "z": z, "tokens": tokens, "logprob": torch.zeros(R, **f32),
                "entropy": torch.zeros(R, **f32),
                "top_tokens": torch.zeros((R, top), dtype=torch.int32, device=_device()),
                "top_logprobs": torch.zeros((R, top), **f32)}
    Hq, Hkv, C, B = case["q_heads"], case["kv_heads"], case["max_ctx"], case["B"]
    if case["family"] == "kv4_attention":
        T = case["T"]
        pos0 = [max(0, case["ctx"] - 7 * b) for b in range(B)]
        cache = _empty_kv4(case)
        # (the caches hold what an append of normal keys and values leaves)
        for i, pack in ((0, _pack_k), (2, _pack_v)):
            codes, params = _quantize(_normal(seed + 1 + i, (B, Hkv, C, D)))
            cache[i], cache[i + 1] = pack(codes), params
        return {"case": case, "qkv": _normal(seed, (B * T, (Hq + 2 * Hkv) * D)), "cache": cache,
                "pos0": _ints(pos0), "last": max(pos0) + T,
                "out": torch.zeros((B * T, Hq * D), dtype=torch.float16, device=_device()),
                "ws": torch.empty(1 << 20, dtype=torch.uint8, device=_device())}
    lens, pos0, offsets, N = _packed(case)
    state = {"case": case, "qkv": _normal(seed, (N, (Hq + 2 * Hkv) * D)), "offsets": _ints(offsets),
             "pos0": _ints(pos0), "end": _ints([p + n for p, n in zip(pos0, lens)]), "rows": offsets[-1],
             "last": max(p + n for p, n in zip(pos0, lens))}
    if case["family"] == "prompt":
        state["k"], state["v"] = _normal(seed + 1, (B, Hkv, C, D)), _normal(seed + 2, (B, Hkv, C, D))
        state["out"] = torch.zeros((N, Hq * D), dtype=torch.float16, device=_device())
        state["ws"] = torch.empty(1 << 20, dtype=torch.uint8, device=_device())
    else:
        state["cache"] = _empty_kv4(case)
        state["k"] = torch.zeros((B, Hkv, C, D), dtype=torch.float16, device=_device())
        state["v"] = torch.zeros_like(state["k"])
    return state


# ---- a pass --------------------------------------------------------------------

def _workspace(state, need):
    """The state's workspace, grown on the first pass as a program would."""
    if state["ws"].numel() < need:
        state["ws"] = torch.empty(need, dtype=torch.uint8, device=_device())
    return state["ws"]


def _run_own(state):
    import paper_2609_21704_gb300 as sq

    case = state["case"]
    if case["family"] == "logprobs":
        sq.sq_logprobs(state["z"], case["temperature"], state["tokens"], state["logprob"], state["entropy"],
                       state["top_tokens"], state["top_logprobs"])
        return [state["logprob"], state["entropy"], state["top_tokens"], state["top_logprobs"]]
    Hq, Hkv, B = case["q_heads"], case["kv_heads"], case["B"]
    if case["family"] == "kv4_attention":
        T = case["T"]
        ws = _workspace(state, sq.sq_attention_kv4_workspace_bytes(B, T, Hq, Hkv, case["max_ctx"]))
        sq.sq_attention_kv4(state["qkv"], B, T, Hq, Hkv, state["pos0"], THETA, *state["cache"], state["out"], ws)
        return [state["out"]]
    if case["family"] == "prompt":
        ws = _workspace(state, sq.sq_attention_prompt_workspace_bytes(B, state["qkv"].shape[0], Hq, Hkv,
                                                                      case["max_ctx"]))
        sq.sq_attention_prompt(state["qkv"], state["offsets"], Hq, Hkv, state["pos0"], THETA, state["k"],
                               state["v"], state["out"], ws)
        return [state["out"], state["k"], state["v"]]
    sq.sq_kv4_append(state["qkv"], Hq, Hkv, state["pos0"], THETA, *state["cache"], offsets=state["offsets"])
    sq.sq_kv4_unpack(*state["cache"], state["pos0"], state["end"], state["k"], state["v"])
    return [state["k"], state["v"]]


def run(state):
    if own:
        return _run_own(state)
    return {"logprobs": _plain_logprobs, "prompt": _plain_prompt, "kv4_append": _plain_kv4_append,
            "kv4_attention": _plain_kv4_attention}[state["case"]["family"]](state)


# ---- plain forms ---------------------------------------------------------------

def _cos_sin(pos):
    """cos and sin of the rotation at positions pos, [..., 64], in 64 bits
    (angles of far positions lose their turn in 32)."""
    f = THETA ** (-torch.arange(D // 2, dtype=torch.float64, device=pos.device) / (D // 2))
    a = pos.double()[..., None] * f
    return a.cos(), a.sin()


def _rotate(x, cs):
    """Rows x [N, heads, D] with the pairs (d, d + 64) turned; cs [N, 64] each."""
    c, s = (t[:, None].to(x.dtype) for t in cs)
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _nearest_f16(x):
    """64-bit values to the nearest fp16 in one rounding (a cast goes by way of 32 bits)."""
    e = (torch.frexp(x)[1] - 1).clamp(min=-14)
    step = torch.ldexp(torch.ones_like(x), e - 10)
    return (torch.round(x / step) * step).half()


def _places(state):
    """Sequence and position of every packed row."""
    off = state["offsets"].long()
    row = torch.arange(state["rows"], device=off.device)
    seq = torch.searchsorted(off[1:].contiguous(), row, right=True)
    return seq, state["pos0"].long()[seq] + row - off[seq]


def _softmax_values(s, seen, v):
    """softmax over the keys that `seen` leaves, times the values."""
    s = s.masked_fill(~seen, -math.inf)
    s = torch.exp(s - s.amax(-1, keepdim=True))
    return torch.matmul(s, v) / s.sum(-1, keepdim=True)


def _plain_prompt(state):
    case = state["case"]
    Hq, Hkv, B, L = case["q_heads"], case["kv_heads"], case["B"], case["longest"]
    G, n = Hq // Hkv, state["rows"]
    seq, pos = _places(state)
    x = state["qkv"][:n].float().view(n, Hq + 2 * Hkv, D)
    qk = _rotate(x[:, :Hq + Hkv], _cos_sin(pos)).half()
    state["k"][seq, :, pos] = qk[:, Hq:]
    state["v"][seq, :, pos] = x[:, Hq + Hkv:].half()
    k, v = (state[c][:, :, :state["last"]].float() for c in ("k", "v"))
    # queries padded to [B, longest]: [B, Hkv, G * L, D]
    off = state["offsets"].long()
    rows = (off[:-1, None] + torch.arange(L, device=off.device)).clamp(max=n - 1)
    q = qk[:, :Hq].float()[rows].view(B, L, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * L, D)
    at = state["pos0"].long()[:, None] + torch.arange(L, device=off.device)
    seen = torch.arange(state["last"], device=off.device) <= at[..., None]
    s = torch.matmul(q, k.transpose(2, 3)) * D ** -0.5
    s = s.view(B, Hkv, G, L, -1)
    o = _softmax_values(s, seen[:, None, None], v[:, :, None]).permute(0, 3, 1, 2, 4).reshape(B, L, Hq * D)
    state["out"][:n] = o[seq, pos - state["pos0"].long()[seq]].half()
    return [state["out"], state["k"], state["v"]]


def _quantize(x):
    """Codes (0..15) and (scale, lowest) of rows x [..., 128] of fp16 values."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = ((hi - lo) / 15.0).half().float()
    s = torch.where((s == 0) & (hi > lo), torch.full_like(s, 2.0 ** -24), s)
    c = torch.round((x - lo) / torch.where(s == 0, torch.ones_like(s), s)).clamp(0, 15)
    return c.to(torch.uint8), torch.cat([s, lo], -1).half()


def _pack_k(c):
    """Codes [..., 128] to bytes [..., 64], the even one in the low half."""
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _pack_v(c):
    """Value codes [..., C, 128]: two bytes (four codes) of an even position,
    then those of the odd one after it."""
    b = _pack_k(c)
    C = b.shape[-2]
    return b.view(*b.shape[:-2], C // 2, 2, D // 4, 2).transpose(-3, -2).reshape(b.shape)


def _codes_k(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _codes_v(b):
    C = b.shape[-2]
    return _codes_k(b.view(*b.shape[:-2], C // 2, D // 4, 2, 2).transpose(-3, -2).reshape(b.shape))


def _values(codes, params):
    p = params.float()
    return codes.float() * p[..., :1] + p[..., 1:]


def _plain_kv4_append(state):
    case = state["case"]
    Hq, Hkv, n = case["q_heads"], case["kv_heads"], state["rows"]
    kc, kp, vc, vp = state["cache"]
    seq, pos = _places(state)
    x = state["qkv"][:n].view(n, Hq + 2 * Hkv, D)[:, Hq:]
    k = _nearest_f16(_rotate(x[:, :Hkv].double(), _cos_sin(pos)))
    (ck, pk), (cv, pv) = _quantize(k), _quantize(x[:, Hkv:])
    kc[seq, :, pos], kp[seq, :, pos], vp[seq, :, pos] = _pack_k(ck), pk, pv
    # a value's bytes lie in pairs between those of its neighbour
    pairs = vc.view(case["B"], Hkv, -1, D // 4, 2, 2)
    pairs[seq, :, pos // 2, :, pos % 2] = _pack_k(cv).view(n, Hkv, D // 4, 2)
    state["k"][seq, :, pos] = _values(_codes_k(kc[seq, :, pos]), pk).half()
    state["v"][seq, :, pos] = _values(_codes_k(pairs[seq, :, pos // 2, :, pos % 2].flatten(-2)), pv).half()
    return [state["k"], state["v"]]


def _plain_kv4_attention(state):
    case = state["case"]
    Hq, Hkv, B, T = case["q_heads"], case["kv_heads"], case["B"], case["T"]
    n = (state["last"] + 1) // 2 * 2
    kc, kp, vc, vp = (t[:, :, :n] for t in state["cache"])
    k, v = _values(_codes_k(kc), kp), _values(_codes_v(vc), vp)
    at = state["pos0"].long()[:, None] + torch.arange(T, device=kc.device)
    x = state["qkv"].float().view(B * T, Hq + 2 * Hkv, D)[:, :Hq]
    q = _rotate(x, _cos_sin(at.view(-1))).view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q, k[:, :, None].transpose(3, 4)) * D ** -0.5
    seen = torch.arange(n, device=kc.device) <= at[..., None]
    o = _softmax_values(s, seen[:, None, None], v[:, :, None])
    return [o.permute(0, 3, 1, 2, 4).reshape(B * T, Hq * D).half()]


def _plain_logprobs(state):
    z, k = state["z"], state["case"]["top"]
    x = z.float()
    x = (x - x.amax(-1, keepdim=True)) / state["case"]["temperature"]
    e = x.exp()
    S = e.sum(-1, dtype=torch.float64)
    lse = S.log()
    entropy = lse + (e * -x).sum(-1, dtype=torch.float64) / S
    logprob = x.gather(1, state["tokens"].long()[:, None])[:, 0].double() - lse
    # order: largest value first, lowest index among equals
    key = (z.float() * 2.0 ** 24).long() * (1 << 20) - torch.arange(z.shape[1], device=z.device)
    at = key.topk(k, dim=1)[1]
    return [logprob.float(), entropy.float(), at.to(torch.int32), (x.gather(1, at).double() - lse[:, None]).float()]


# ---- the definitions in 64 bits ------------------------------------------------

def _exact_turn(row, p):
    """One head's rows [n, 128] in 64 bits turned to positions p [n]."""
    h = row.shape[1] // 2
    w = torch.exp(torch.arange(h, device=row.device, dtype=torch.float64) * (-math.log(THETA) / h))
    z = torch.complex(row[:, :h], row[:, h:]) * torch.polar(torch.ones_like(row[:, :h]), p.double()[:, None] * w)
    return torch.cat([z.real, z.imag], 1)


def _exact_half(x):
    """The nearest fp16 of 64-bit values, as 64-bit values."""
    a = x.abs()
    u = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -14))) - 10.0)
    r = torch.round(a / u) * u
    return torch.copysign(r, x)


def _exact_attend(q, p, k, v):
    """Rows q [n, 128] at positions p over keys k, v [L, 128], all in 64 bits."""
    out = torch.empty_like(q)
    for i in range(0, q.shape[0], 4096):
        w = q[i:i + 4096] @ k.t() / math.sqrt(q.shape[1])
        w[torch.arange(k.shape[0], device=q.device)[None] > p[i:i + 4096, None]] = -math.inf
        out[i:i + 4096] = torch.softmax(w, 1) @ v
    return out


def _exact_store(x):
    """What 4 bits keep of rows x [n, 128] (fp16 values in 64 bits)."""
    x32 = x.float()
    low, high = x32.min(1).values, x32.max(1).values
    scale = ((high - low) / 15).to(torch.float16).float()
    scale[(scale == 0) & (high > low)] = 2.0 ** -24
    div = torch.where(scale == 0, torch.ones_like(scale), scale)
    code = ((x32 - low[:, None]) / div[:, None]).round().clamp(0, 15)
    return code.double() * scale.double()[:, None] + low.double()[:, None]


def exact(case, seed):
    state = prepare(case, seed)
    if case["family"] == "logprobs":
        z, T = state["z"], case["temperature"]
        lp, ent, tt, tl = [], [], [], []
        for r in range(case["R"]):
            d = z[r].double() / T
            row = d - torch.logsumexp(d, 0)
            lp.append(row[int(state["tokens"][r])])
            ent.append(-(row.exp() * row).sum())
            order = torch.sort(z[r], descending=True, stable=True).indices[:case["top"]]
            tt.append(order.to(torch.int32))
            tl.append(row[order])
        return [torch.stack(lp), torch.stack(ent), torch.stack(tt), torch.stack(tl)]
    Hq, Hkv, B = case["q_heads"], case["kv_heads"], case["B"]
    G = Hq // Hkv
    qkv = state["qkv"].double()

    def head(rows, h):
        return qkv[rows, h * D:(h + 1) * D]

    if case["family"] == "kv4_attention":
        T = case["T"]
        out = torch.zeros((B * T, Hq * D), dtype=torch.float64, device=qkv.device)
        kc, kp, vc, vp = state["cache"]
        for b in range(B):
            p0 = max(0, case["ctx"] - 7 * b)
            p = p0 + torch.arange(T, device=qkv.device)
            n = p0 + T
            for h in range(Hkv):
                kn, vn = kc[b, h].long(), vc[b, h].long()
                k = torch.zeros((case["max_ctx"], D), dtype=torch.float64, device=qkv.device)
                v = torch.zeros_like(k)
                k[:, 0::2], k[:, 1::2] = (kn % 16).double(), (kn // 16).double()
                w = vn.reshape(-1, D // 4, 4)  # a pair of positions: bytes e0 e1 o0 o1
                for odd in (0, 1):
                    for byte in (0, 1):
                        v[odd::2, 2 * byte::4] = (w[:, :, 2 * odd + byte] % 16).double()
                        v[odd::2, 2 * byte + 1::4] = (w[:, :, 2 * odd + byte] // 16).double()
                k = k * kp[b, h, :, :1].double() + kp[b, h, :, 1:].double()
                v = v * vp[b, h, :, :1].double() + vp[b, h, :, 1:].double()
                for g in range(G):
                    j = h * G + g
                    rows = slice(b * T, (b + 1) * T)
                    out[rows, j * D:(j + 1) * D] = _exact_attend(_exact_turn(head(rows, j), p), p, k[:n], v[:n])
        return [out]
    lens, pos0, offsets, N = _packed(case)
    # (fp16 where values are copied; the caches are too large for 64 bits of everything)
    K, V = state["k"].double(), state["v"].double()
    out = torch.zeros((N, Hq * D), dtype=torch.float64, device=qkv.device)
    for b in range(B):
        rows = slice(offsets[b], offsets[b + 1])
        p = pos0[b] + torch.arange(lens[b], device=qkv.device)
        e = pos0[b] + lens[b]
        for h in range(Hkv):
            k = _exact_half(_exact_turn(head(rows, Hq + h), p))
            v = head(rows, Hq + Hkv + h)
            if case["family"] == "kv4_append":
                K[b, h, pos0[b]:e], V[b, h, pos0[b]:e] = _exact_store(k), _exact_store(v)
                continue
            K[b, h, pos0[b]:e], V[b, h, pos0[b]:e] = k, v
            for g in range(G):
                j = h * G + g
                q = _exact_half(_exact_turn(head(rows, j), p))
                out[rows, j * D:(j + 1) * D] = _exact_attend(q, p, K[b, h, :e], V[b, h, :e])
    return [K, V] if case["family"] == "kv4_append" else [out, K, V]
