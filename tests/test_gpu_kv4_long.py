"""Attention of many queries over long 4-bit caches (more than sixteen queries a
key/value head, where there is work for the tcgen05 kernel), against the 64-bit
reference.  The capacity of the cache counts, so short sequences in large caches
take this path as well."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_21704_gb300 as sq
from gpu_util import dev
from serve_ref import D, THETA, attend, kv4_encode, kv4_pack_k, kv4_pack_v, kv4_value
from test_gpu_kv4 import _attention, _random_cache, _t

pytestmark = pytest.mark.gpu


def _check(got, qkv, vals, cache, B, T, Hq, Hkv, pos0, times=1.0):
    """Within `times` the bound of `attend`, and what a weight's rounding adds: a
    value is w (c - 8) + (8 w + lo), and the rounded weight multiplies the first
    part, which is at most |v| + |8 w + lo|; `attend` has 2^-11 of the mean |v|, so
    2^-11 of the largest |8 w + lo| comes on top.  (With few keys nothing of it
    averages out.)"""
    par = cache[3].astype(np.float64)
    got = got.float().cpu().numpy().astype(np.float64)
    for b in range(B):
        pos = pos0[b] + np.arange(T)
        q = oracle.rope(qkv[b * T:(b + 1) * T, :Hq * D].astype(np.float64), pos, Hq, D, THETA).reshape(T, Hq, D)
        L = pos0[b] + T
        ref, bound = attend(q, vals[0][b, :, :L].transpose(1, 0, 2), vals[1][b, :, :L].transpose(1, 0, 2), pos)
        err = np.abs(got[b * T:(b + 1) * T] - ref.reshape(T, -1))
        more = 2.0 ** -11 * np.abs(8 * par[b, :, :L, 0] + par[b, :, :L, 1]).max()
        over = err - times * (bound.reshape(T, -1) + more)
        assert (over <= 0).all(), (b, pos[0], err.max(), over.max())


CASES = [
    # B, T, Hq, Hkv, pos0, C
    (1, 17, 1, 1, [0], 65536),                   # 17 queries, one tile
    (2, 5, 14, 2, [37, 300], 16384),             # 35
    (1, 32, 6, 1, [130], 16384),                 # 192: four groups
    (3, 7, 7, 1, [0, 121, 8000], 16384),         # 49: two groups of 32
    (1, 25, 8, 1, [16384 - 25], 16384),          # 200, the cache full
    (4, 9, 28, 4, [64, 127, 128, 2055], 2064),   # the cache ends in a tile
    (1, 5, 5, 1, [60000], 65536),                # many shares
    (1, 24, 2, 1, [126], 65536),                 # 48, across a tile's end
    (40, 4, 8, 1, [25 * i for i in range(40)], 1280),  # one CTA a sequence
]


@pytest.mark.parametrize("B,T,Hq,Hkv,pos0,C", CASES)
def test_matches_reference(B, T, Hq, Hkv, pos0, C):
    rng = np.random.default_rng(B * 100 + T + C)
    cache, vals = _random_cache(rng, B, Hkv, C, pos0, T)
    qkv = rng.normal(0, 1, (B * T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    dc = [_t(c) for c in cache]
    out = torch.full((B * T, Hq * D), 7.0, dtype=torch.float16, device=dev())
    _attention(qkv, B, T, Hq, Hkv, pos0, dc, out)
    assert sq.sq_check() == 0
    _check(out, qkv, vals, cache, B, T, Hq, Hkv, pos0)
    again = torch.empty_like(out)
    _attention(qkv, B, T, Hq, Hkv, pos0, dc, again)
    assert torch.equal(out, again)  # bit for bit: sums have one order


@pytest.mark.parametrize("grow", ["scores", "values", "both"])
def test_growing_maxima_rescale(grow):
    """Keys up to four times as long towards the end, values a thousand times as
    large: the running maxima and the values' power of two change in many tiles.
    (Scores four times as large lose four times as much in fp32 sums.)"""
    B, T, Hq, Hkv, C = 1, 5, 7, 1, 40000
    L = 3000
    rng = np.random.default_rng(len(grow))
    size = np.ones((2, C, 1))
    if grow != "values":
        size[0, :L] = np.linspace(0.05, 4.0, L)[:, None]
    if grow != "scores":
        size[1, :L] = 10.0 ** np.linspace(-2, 1, L)[:, None]
    vals, par, codes = [], [], []
    for i in range(2):
        c, p = kv4_encode((rng.normal(0, 1, (B, Hkv, C, D)) * size[i]).astype(np.float16))
        vals.append(kv4_value(c, p))
        codes.append(c)
        par.append(p)
    cache = [kv4_pack_k(codes[0]), par[0], kv4_pack_v(codes[1]).reshape(B, Hkv, C, 64), par[1]]
    qkv = rng.normal(0, 1, (B * T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    out = torch.empty(B * T, Hq * D, dtype=torch.float16, device=dev())
    _attention(qkv, B, T, Hq, Hkv, [L - T], [_t(c) for c in cache], out)
    assert sq.sq_check() == 0
    _check(out, qkv, vals, cache, B, T, Hq, Hkv, [L - T], 1.0 if grow == "values" else 4.0)


@pytest.mark.parametrize("B,C", [(8, 13312), (1, 131072)])
def test_sums_over_many_tiles_keep_their_precision(B, C):
    """About a hundred tiles a CTA, and the longest cache: as a whole within the root
    of the sum of the output's rounding and a weight's (2^-11 / sqrt(3) at most of a
    uniform mantissa, 2.8e-4 each at the worst, 2.0e-4 on average), and a fifth for
    what the sums lose."""
    T, Hq, Hkv = 5, 56, 8
    if B == 1:
        Hq, Hkv = 7, 1
    rng = np.random.default_rng(B)
    pos0 = [C - T] * B
    cache, vals = _random_cache(rng, 1, Hkv, C, pos0[:1], T)
    qkv = rng.normal(0, 1, (T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    dc = [_t(c).repeat(B, 1, 1, 1) for c in cache]
    out = torch.empty(B * T, Hq * D, dtype=torch.float16, device=dev())
    _attention(np.tile(qkv, (B, 1)), B, T, Hq, Hkv, pos0, dc, out)
    assert sq.sq_check() == 0
    pos = C - T + np.arange(T)
    q = oracle.rope(qkv[:, :Hq * D].astype(np.float64), pos, Hq, D, THETA).reshape(T, Hq, D)
    ref = oracle.attention(q, vals[0][0].transpose(1, 0, 2), vals[1][0].transpose(1, 0, 2), pos).reshape(T, -1)
    got = out.float().cpu().numpy().astype(np.float64).reshape(B, T, -1)
    assert (got == got[:1]).all()
    rel = np.linalg.norm(got[0] - ref) / np.linalg.norm(ref)
    assert rel <= 2.8e-4 * 1.2, rel


def test_heads_of_very_different_size():
    """One power of two serves the queries of a CTA: those of a head a ten
    thousandth as large keep their bits."""
    B, T, Hq, Hkv, C, pos0 = 1, 9, 3, 1, 65536, [777]
    rng = np.random.default_rng(12)
    cache, vals = _random_cache(rng, B, Hkv, C, pos0, T)
    x = rng.normal(0, 1, (B * T, (Hq + 2 * Hkv), D))
    x[:, 1] *= 1e-4
    x[:, 2] *= 3.0
    qkv = x.reshape(B * T, -1).astype(np.float16)
    out = torch.empty(B * T, Hq * D, dtype=torch.float16, device=dev())
    _attention(qkv, B, T, Hq, Hkv, pos0, [_t(c) for c in cache], out)
    assert sq.sq_check() == 0
    _check(out, qkv, vals, cache, B, T, Hq, Hkv, pos0, 3.0)


def test_rows_that_are_not_finite_reach_only_those_that_see_them():
    """NaN in the key of token 3, then in a value of token 5, of 24 new ones; and
    queries that are not finite."""
    B, T, Hq, Hkv, C, p = 1, 24, 2, 1, 65536, 200
    rng = np.random.default_rng(5)
    cache, vals = _random_cache(rng, B, Hkv, C, [p], T)
    base = [_t(c) for c in cache]
    qkv = rng.normal(0, 1, (T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    for which, t in ((1, 3), (3, 5)):
        dc = [c.clone() for c in base]
        dc[which][0, 0, p + t] = float("nan")
        out = torch.empty(T, Hq * D, dtype=torch.float16, device=dev())
        _attention(qkv, B, T, Hq, Hkv, [p], dc, out)
        assert sq.sq_check() == 0
        o = out.float().cpu().numpy()
        assert np.isfinite(o[:t]).all() and np.isnan(o[t:]).all()
    odd = qkv.copy()
    odd[7, 5] = np.inf
    odd[9, D + 100] = np.nan
    out = torch.empty(T, Hq * D, dtype=torch.float16, device=dev())
    _attention(odd, B, T, Hq, Hkv, [p], base, out)
    o = out.float().cpu().numpy().reshape(T, Hq, D)
    assert np.isnan(o[7, 0]).all() and np.isnan(o[9, 1]).all()
    o[7, 0] = o[9, 1] = 0.0
    assert np.isfinite(o).all()
    clean = torch.empty_like(out)
    _attention(qkv, B, T, Hq, Hkv, [p], base, clean)
    c = clean.float().cpu().numpy().reshape(T, Hq, D)
    c[7, 0] = c[9, 1] = 0.0
    assert np.abs(o - c).max() <= 2.0 ** -9 * max(1.0, np.abs(c).max())


@pytest.mark.parametrize("T,Hq,C", [(1, 2, 64), (1, 12, 64), (1, 20, 65536), (1, 2, 4096)])
def test_a_row_that_sees_nothing_but_nan_is_nan(T, Hq, C):
    """The only key there is, in each of the three kernels and where shares meet."""
    rng = np.random.default_rng(Hq)
    cache, _ = _random_cache(rng, 1, 1, C, [0], T)
    cache[1][0, 0, 0] = np.nan
    qkv = rng.normal(0, 1, (T, (Hq + 2) * D)).astype(np.float16)
    out = torch.zeros(T, Hq * D, dtype=torch.float16, device=dev())
    _attention(qkv, 1, T, Hq, 1, [0], [_t(c) for c in cache], out)
    assert sq.sq_check() == 0
    assert bool(torch.isnan(out).all())


def test_positions_outside_the_cache():
    B, T, Hq, Hkv, C = 3, 9, 8, 2, 16384
    rng = np.random.default_rng(6)
    cache, _ = _random_cache(rng, B, Hkv, C, [10, 10, 10], T)
    qkv = rng.normal(0, 1, (B * T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    out = torch.full((B * T, Hq * D), 7.0, dtype=torch.float16, device=dev())
    _attention(qkv, B, T, Hq, Hkv, [10, C - T + 1, -1], [_t(c) for c in cache], out)
    assert sq.sq_check() == sq.SQ_DEV_BAD_POSITION
    assert bool((out[:T] != 7.0).any()) and not bool(out[T:].any())


def test_two_streams_and_a_graph_as_positions_advance():
    """A captured step replayed at other lengths, another one beside it on its own
    stream and workspace, with passes of the prompt kernel (which takes all of
    an SM's tensor memory) between them."""
    B, T, Hq, Hkv, C = 2, 5, 14, 2, 16384
    rng = np.random.default_rng(8)
    cache, vals = _random_cache(rng, B, Hkv, C, [900, 900], T)
    dc = [_t(c) for c in cache]
    qkv = rng.normal(0, 1, (B * T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    x, need = _t(qkv), sq.sq_attention_kv4_workspace_bytes(B, T, Hq, Hkv, C)
    pn = 300
    pq = _t(rng.normal(0, 1, (pn, (Hq + 2 * Hkv) * D)).astype(np.float16))
    poff, pp = _t(np.array([0, pn], np.int32)), _t(np.zeros(1, np.int32))
    pk = torch.zeros(1, Hkv, 512, D, dtype=torch.float16, device=dev())
    pv, po = torch.zeros_like(pk), torch.zeros(pn, Hq * D, dtype=torch.float16, device=dev())
    pw = torch.empty(sq.sq_attention_prompt_workspace_bytes(1, pn, Hq, Hkv, 512), dtype=torch.uint8, device=dev())
    sides = []
    torch.cuda.synchronize()
    for i in range(2):
        s, pos = torch.cuda.Stream(), torch.zeros(B, dtype=torch.int32, device=dev())
        out = torch.zeros(B * T, Hq * D, dtype=torch.float16, device=dev())
        ws = torch.empty(need, dtype=torch.uint8, device=dev())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            if i == 0:
                sq.sq_attention_prompt(pq, poff, Hq, Hkv, pp, THETA, pk, pv, po, pw)
            sq.sq_attention_kv4(x, B, T, Hq, Hkv, pos, THETA, *dc, out, ws)
        sides.append((s, pos, out, ws, g))
    starts = [[0, 5], [123, 130], [250, 900], [899, 1]]
    got = [[], []]
    for k in range(4):
        for i, (s, pos, out, _, g) in enumerate(sides):
            with torch.cuda.stream(s):
                pos.copy_(_t(np.array(starts[(k + i) % 4], np.int32)))
                g.replay()
                got[i].append(out.clone())
    torch.cuda.synchronize()
    assert sq.sq_check() == 0
    for k in range(4):
        for i in range(2):
            _check(got[i][k], qkv, vals, cache, B, T, Hq, Hkv, starts[(k + i) % 4])
