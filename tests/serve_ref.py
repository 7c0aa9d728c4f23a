"""Plain 64-bit references of prompt attention, the 4-bit cache and token log
probabilities, and the bounds that their kernels are held to."""
import numpy as np

import oracle

D = 128
THETA = 1e6


def f16(x):
    """Nearest fp16 (numpy casts 64-bit values in one rounding), in 64 bits."""
    with np.errstate(over="ignore"):
        return np.asarray(x, np.float64).astype(np.float16).astype(np.float64)


def rotated(x, pos, heads):
    """Rows [n, heads * D] turned to positions pos and rounded to fp16: [n, heads, D]."""
    n = len(pos)
    return f16(oracle.rope(np.asarray(x, np.float64), np.asarray(pos), heads, D, THETA)).reshape(n, heads, D)


def attend(q, k, v, pos):
    """(out, bound) of attention in 64 bits.  The bound of an element, with A
    the same weighted mean of |v|:
      2^-11 |out|    the output's rounding to fp16
      2^-11 A        a probability's rounding to fp16
      2^-13 A        scores: 128 fp32 sums of |q_d k_d| / sqrt(128) (about 7 for
                     normal values) of half a step each, in a weight and in its sum
      2^-18 max |v|  probabilities below fp16's normal range."""
    out = oracle.attention(q, k, v, pos)
    a = oracle.attention(q, k, np.abs(v), pos)
    return out, 2.0 ** -11 * np.abs(out) + (2.0 ** -11 + 2.0 ** -13) * a + 2.0 ** -18 * np.abs(v).max(initial=0.0)


def prompt(qkv, lens, pos0, offsets, Hq, Hkv, kc, vc):
    """Reference of sq_attention_prompt on host arrays (fp16 caches [B, Hkv, C, D]):
    (out, bound, kc, vc) with rows of no sequence NaN in `out`."""
    kc, vc = kc.copy(), vc.copy()
    out = np.full((qkv.shape[0], Hq * D), np.nan)
    bound = np.zeros_like(out)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        rows = qkv[offsets[b]:offsets[b] + n].astype(np.float64)
        pos = pos0[b] + np.arange(n)
        q = rotated(rows[:, :Hq * D], pos, Hq)
        kc[b, :, pos] = rotated(rows[:, Hq * D:(Hq + Hkv) * D], pos, Hkv).astype(np.float16)
        vc[b, :, pos] = rows[:, (Hq + Hkv) * D:].reshape(n, Hkv, D).astype(np.float16)
        L = pos0[b] + n
        o, t = attend(q, kc[b, :, :L].transpose(1, 0, 2).astype(np.float64),
                      vc[b, :, :L].transpose(1, 0, 2).astype(np.float64), pos)
        out[offsets[b]:offsets[b] + n] = o.reshape(n, Hq * D)
        bound[offsets[b]:offsets[b] + n] = t.reshape(n, Hq * D)
    return out, bound, kc, vc


def kv4_encode(x):
    """Codes [..., 128] and (scale, lowest) fp16 [..., 2] of fp16 rows x."""
    x = np.asarray(x, np.float16).astype(np.float32)
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    lo = lo + np.float32(0)
    s = ((hi - lo) / np.float32(15)).astype(np.float16).astype(np.float32)
    s = np.where((s == 0) & (hi > lo), np.float32(2.0 ** -24), s)
    c = np.clip(np.rint((x - lo) / np.where(s == 0, np.float32(1), s)), 0, 15)
    return c.astype(np.uint8), np.concatenate([s, lo], -1).astype(np.float16)


def kv4_value(codes, params):
    p = params.astype(np.float64)
    return codes.astype(np.float64) * p[..., :1] + p[..., 1:]


def kv4_pack_k(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def kv4_pack_v(c):
    """Codes [..., C, 128] to the paired bytes, [..., C / 2, 128]."""
    b = kv4_pack_k(c)
    out = np.empty(b.shape[:-2] + (b.shape[-2] // 2, 128), np.uint8)
    for odd in (0, 1):
        for byte in (0, 1):
            out[..., 2 * odd + byte::4] = b[..., odd::2, byte::2]
    return out


def logprobs(z, T, tokens, top):
    """(logprob, entropy, top tokens, top logprobs) of fp16 rows z in 64 bits."""
    R, V = z.shape
    x = z.astype(np.float64)
    x = (x - x.max(-1, keepdims=True)) / T
    e = np.exp(x)
    lse = np.log(e.sum(-1))
    ent = lse - np.where(e > 0, e * np.where(e > 0, x, 0), 0).sum(-1) / e.sum(-1)
    order = np.argsort(-z.astype(np.float64), axis=-1, kind="stable")[:, :top]
    lp = x - lse[:, None]
    return lp[np.arange(R), tokens], ent, order, np.take_along_axis(lp, order, -1)
