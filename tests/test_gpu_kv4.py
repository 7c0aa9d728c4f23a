"""The 4-bit key/value cache: codes and parameters bit for bit, what is read
back, and attention over it against a 64-bit reference."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_21704_gb300 as sq
from gpu_util import dev
from serve_ref import (D, THETA, attend, kv4_encode, kv4_pack_k, kv4_pack_v, kv4_value, rotated)

pytestmark = pytest.mark.gpu


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev())


def _filled(B, Hkv, C, seed):
    """Random bytes and NaN parameters: what an uninitialised cache may hold."""
    rng = np.random.default_rng(seed)
    codes = [rng.integers(0, 256, (B, Hkv, C, 64), dtype=np.uint8) for _ in range(2)]
    return [codes[0], np.full((B, Hkv, C, 2), np.nan, np.float16), codes[1],
            np.full((B, Hkv, C, 2), np.nan, np.float16)]


def _expect(cache, qkv, lens, off, pos0, Hq, Hkv):
    """The caches after the append, from the definition."""
    kc, kp, vc, vp = (c.copy() for c in cache)
    pairs = vc.reshape(vc.shape[0], Hkv, -1, 128)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        rows = qkv[off[b]:off[b] + n].astype(np.float64)
        pos = pos0[b] + np.arange(n)
        k = rotated(rows[:, Hq * D:(Hq + Hkv) * D], pos, Hkv)
        ck, pk = kv4_encode(k)
        cv, pv = kv4_encode(rows[:, (Hq + Hkv) * D:].reshape(n, Hkv, D))
        kc[b, :, pos], kp[b, :, pos], vp[b, :, pos] = kv4_pack_k(ck), pk, pv
        by = kv4_pack_k(cv)
        for t, p in enumerate(pos):
            for byte in (0, 1):
                pairs[b, :, p // 2, 2 * (p % 2) + byte::4] = by[t, :, byte::2]
    return [kc, kp, vc, vp]


CASES = [
    ([1], [0], 12, 2, 16, True),
    ([7, 0, 33, 1], [3, 5, 31, 63], 12, 2, 64, True),
    ([5, 5, 5], [0, 17, 40], 40, 8, 48, False),
    ([1] * 16, list(range(0, 160, 10)), 28, 4, 160, False),
    ([300, 111], [0, 700], 14, 2, 1008, True),
    ([2], [131070], 8, 1, 131072, True),
]


@pytest.mark.parametrize("lens,pos0,Hq,Hkv,C,packed", CASES)
def test_append_and_unpack(lens, pos0, Hq, Hkv, C, packed):
    B = len(lens)
    rng = np.random.default_rng(B + C)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    qkv = rng.normal(0, 1, (off[-1], (Hq + 2 * Hkv) * D)).astype(np.float16)
    cache = _filled(B, Hkv, C, 1)
    dev_cache = [_t(c) for c in cache]
    sq.sq_kv4_append(_t(qkv), Hq, Hkv, _t(np.array(pos0, np.int32)), THETA, *dev_cache,
                     offsets=_t(off) if packed else None)
    assert sq.sq_check() == 0
    want = _expect(cache, qkv, lens, off, pos0, Hq, Hkv)
    for name, g, w in zip(("k codes", "k params", "v codes", "v params"), dev_cache, want):
        g = g.cpu().numpy()
        assert np.array_equal(g.view(np.uint8), w.view(np.uint8)), name
    k = torch.full((B, Hkv, C, D), 7.0, dtype=torch.float16, device=dev())
    v = torch.full_like(k, 7.0)
    end = np.array([p + n for p, n in zip(pos0, lens)], np.int32)
    sq.sq_kv4_unpack(*dev_cache, _t(np.array(pos0, np.int32)), _t(end), k, v)
    assert sq.sq_check() == 0
    k, v = k.cpu().numpy(), v.cpu().numpy()
    for b, n in enumerate(lens):
        inside = np.zeros(C, bool)
        inside[pos0[b]:end[b]] = True
        assert (k[b][:, ~inside] == 7.0).all() and (v[b][:, ~inside] == 7.0).all()
        if n == 0:
            continue
        rows = qkv[off[b]:off[b] + n].astype(np.float64)
        ref_k = rotated(rows[:, Hq * D:(Hq + Hkv) * D], np.arange(pos0[b], end[b]), Hkv).transpose(1, 0, 2)
        ref_v = rows[:, (Hq + Hkv) * D:].reshape(n, Hkv, D).transpose(1, 0, 2)
        for got, x in ((k[b][:, inside], ref_k), (v[b][:, inside], ref_v)):
            c, p = kv4_encode(x)
            val = kv4_value(c, p)
            # one fp32 sum and one rounding to fp16
            assert (np.abs(got - val) <= 2.0 ** -11 * np.abs(val) + 2.0 ** -24 * 32 + 2.0 ** -25).all()


def test_extreme_rows():
    """Constant rows, subnormal steps, fp16's whole range, zeros of both signs, ties between codes."""
    Hq, Hkv, C = 1, 1, 16
    x = np.zeros((9, 3, D), np.float16)
    x[1] = 3.5
    x[2, :, 0] = 6e-8                       # the range rounds to a scale of zero
    x[3, :, 0], x[3, :, 1] = 65504, -65504  # (keys at position 0 only: not rotated beyond the range)
    x[4] = -0.0
    x[4, :, 5] = 0.0
    x[5] = np.arange(D) % 16                # exact codes
    x[6] = (np.arange(D) % 31) / 2.0        # halves: ties to even
    x[7] = np.linspace(-1, 1, D)
    x[8, :, 3] = -1e-3
    for row in range(9):
        qkv = x[row].reshape(1, 3 * D)
        cache = _filled(1, Hkv, C, 2)
        dc = [_t(c) for c in cache]
        sq.sq_kv4_append(_t(qkv), Hq, Hkv, _t(np.zeros(1, np.int32)), THETA, *dc)
        assert sq.sq_check() == 0
        for g, w in zip(dc, _expect(cache, qkv, [1], [0], [0], Hq, Hkv)):
            assert np.array_equal(g.cpu().numpy().view(np.uint8), w.view(np.uint8)), row


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_rows_that_are_not_finite(value):
    Hq, Hkv, C = 4, 2, 32
    rng = np.random.default_rng(4)
    qkv = rng.normal(0, 1, (3, (Hq + 2 * Hkv) * D)).astype(np.float16)
    qkv[1, Hq * D + 5] = value              # key of head 0, token 1
    qkv[2, (Hq + Hkv + 1) * D + 77] = value  # value of head 1, token 2
    dc = [_t(c) for c in _filled(1, Hkv, C, 3)]
    p0 = _t(np.zeros(1, np.int32))
    sq.sq_kv4_append(_t(qkv), Hq, Hkv, p0, THETA, *dc)
    assert sq.sq_check() == sq.SQ_DEV_NONFINITE_KV
    kp, vp = dc[1].cpu().numpy(), dc[3].cpu().numpy()
    assert np.isnan(kp[0, 0, 1]).all() and np.isfinite(kp[0, 0, [0, 2]]).all() and np.isfinite(kp[0, 1, :3]).all()
    assert np.isnan(vp[0, 1, 2]).all() and np.isfinite(vp[0, 1, :2]).all() and np.isfinite(vp[0, 0, :3]).all()
    out = torch.empty(3, Hq * D, dtype=torch.float16, device=dev())
    _attention(qkv, 1, 3, Hq, Hkv, [0], dc, out)
    o = out.float().cpu().numpy().reshape(3, Hq, D)
    # token 0 sees neither; head 0's rows see the key from token 1 on, head 1's the value at token 2
    assert np.isfinite(o[0]).all() and np.isnan(o[1:, :2]).all()
    assert np.isfinite(o[1, 2:]).all() and np.isnan(o[2, 2:]).all()


def _attention(qkv, B, T, Hq, Hkv, pos0, dc, out):
    ws = torch.full((sq.sq_attention_kv4_workspace_bytes(B, T, Hq, Hkv, dc[0].shape[2]),), 255, dtype=torch.uint8,
                    device=dev())
    sq.sq_attention_kv4(_t(qkv), B, T, Hq, Hkv, _t(np.array(pos0, np.int32)), THETA, *dc, out, ws)


def _random_cache(rng, B, Hkv, C, pos0, T, scale=1.0):
    """Codes of normal rows up to pos0 + T; behind that random bytes and NaN parameters."""
    cache = _filled(B, Hkv, C, 5)
    vals = np.zeros((2, B, Hkv, C, D))
    ck, pk = kv4_encode(rng.normal(0, scale, (B, Hkv, C, D)).astype(np.float16))
    cv, pv = kv4_encode(rng.normal(0, 1, (B, Hkv, C, D)).astype(np.float16))
    vals[0], vals[1] = kv4_value(ck, pk), kv4_value(cv, pv)
    for b in range(B):
        L = pos0[b] + T
        pk[b, :, L:] = np.nan
        pv[b, :, L:] = np.nan
    cache[0], cache[1], cache[3] = kv4_pack_k(ck), pk, pv
    cache[2] = kv4_pack_v(cv).reshape(B, Hkv, C, 64)
    return cache, vals


ATT = [
    # B, T, Hq, Hkv, pos0, C
    (1, 1, 12, 2, [0], 16),
    (2, 5, 12, 2, [37, 300], 512),
    (1, 1, 12, 2, [1023], 1024),
    (3, 9, 28, 4, [64, 127, 700], 1024),
    (1, 17, 12, 2, [0], 64),
    (1, 1, 40, 8, [3000], 4096),
    (2, 3, 12, 2, [5, 0], 128),
    (1, 32, 4, 2, [100], 256),
    (4, 1, 8, 8, [0, 15, 16, 17], 32),
    (1, 1, 200, 1, [90], 128),
    (2, 25, 8, 1, [500, 3], 528),
    (16, 1, 5, 1, [60 * i for i in range(16)], 1024),
    (1, 2, 7, 1, [9000], 16384),
]


@pytest.mark.parametrize("B,T,Hq,Hkv,pos0,C", ATT)
def test_attention_matches_reference(B, T, Hq, Hkv, pos0, C):
    rng = np.random.default_rng(B * 100 + T + C)
    cache, vals = _random_cache(rng, B, Hkv, C, pos0, T)
    qkv = rng.normal(0, 1, (B * T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    out = torch.full((B * T, Hq * D), 7.0, dtype=torch.float16, device=dev())
    _attention(qkv, B, T, Hq, Hkv, pos0, [_t(c) for c in cache], out)
    assert sq.sq_check() == 0
    got = out.float().cpu().numpy().astype(np.float64)
    for b in range(B):
        pos = pos0[b] + np.arange(T)
        q = oracle.rope(qkv[b * T:(b + 1) * T, :Hq * D].astype(np.float64), pos, Hq, D, THETA).reshape(T, Hq, D)
        L = pos0[b] + T
        ref, bound = attend(q, vals[0][b, :, :L].transpose(1, 0, 2), vals[1][b, :, :L].transpose(1, 0, 2), pos)
        err = np.abs(got[b * T:(b + 1) * T] - ref.reshape(T, -1))
        assert (err <= bound.reshape(T, -1)).all(), (b, err.max())


def test_attention_positions_outside_the_cache():
    B, T, Hq, Hkv, C = 3, 2, 12, 2, 64
    rng = np.random.default_rng(6)
    cache, _ = _random_cache(rng, B, Hkv, C, [10, 10, 10], T)
    qkv = rng.normal(0, 1, (B * T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    dc = [_t(c) for c in cache]
    out = torch.full((B * T, Hq * D), 7.0, dtype=torch.float16, device=dev())
    _attention(qkv, B, T, Hq, Hkv, [10, 63, -1], dc, out)
    assert sq.sq_check() == sq.SQ_DEV_BAD_POSITION
    assert bool((out[:T] != 7.0).any()) and not bool(out[T:].any())
    before = [c.clone() for c in dc]
    sq.sq_kv4_append(_t(qkv), Hq, Hkv, _t(np.array([63, -1, 63], np.int32)), THETA, *dc)
    assert sq.sq_check() == sq.SQ_DEV_BAD_POSITION
    for x, y in zip(before, dc):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("off", [[0, 4, 2, 6], [-1, 2, 4, 6], [0, 2, 4, 7]])
def test_bad_offsets_write_nothing(off):
    Hq, Hkv, C = 4, 2, 32
    dc = [_t(c) for c in _filled(3, Hkv, C, 8)]
    before = [c.clone() for c in dc]
    qkv = _t(np.ones((6, (Hq + 2 * Hkv) * D), np.float16))
    sq.sq_kv4_append(qkv, Hq, Hkv, _t(np.zeros(3, np.int32)), THETA, *dc, offsets=_t(np.array(off, np.int32)))
    assert sq.sq_check() == sq.SQ_DEV_BAD_POSITION
    for x, y in zip(before, dc):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_unpack_ranges():
    Hkv, C = 2, 32
    dc = [_t(c) for c in _random_cache(np.random.default_rng(1), 4, Hkv, C, [31] * 4, 1)[0]]
    k = torch.full((4, Hkv, C, D), 7.0, dtype=torch.float16, device=dev())
    v = torch.full_like(k, 7.0)
    sq.sq_kv4_unpack(*dc, _t(np.array([5, -1, 3, 0], np.int32)), _t(np.array([5, 4, 33, 32], np.int32)), k, v)
    assert sq.sq_check() == sq.SQ_DEV_BAD_POSITION
    assert bool((k[:3] == 7.0).all()) and bool((v[:3] == 7.0).all()) and not bool((k[3] == 7.0).all())


def test_decode_in_a_graph_and_two_streams():
    """A captured append + attention step replayed as positions advance."""
    B, T, Hq, Hkv, C, n = 2, 1, 10, 2, 64, 40
    rng = np.random.default_rng(17)
    qkv = rng.normal(0, 1, (n, B, (Hq + 2 * Hkv) * D)).astype(np.float16)
    dc = [_t(c) for c in _filled(B, Hkv, C, 6)]
    x = torch.zeros(B, (Hq + 2 * Hkv) * D, dtype=torch.float16, device=dev())
    pos0 = torch.zeros(B, dtype=torch.int32, device=dev())
    out = torch.zeros(B, Hq * D, dtype=torch.float16, device=dev())
    ws = torch.empty(sq.sq_attention_kv4_workspace_bytes(B, T, Hq, Hkv, C), dtype=torch.uint8, device=dev())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sq.sq_kv4_append(x, Hq, Hkv, pos0, THETA, *dc)
        sq.sq_attention_kv4(x, B, T, Hq, Hkv, pos0, THETA, *dc, out, ws)
    got = []
    start = np.array([0, 9], np.int32)
    for i in range(n):
        with torch.cuda.stream(s):
            x.copy_(_t(qkv[i]))
            pos0.copy_(_t(start + i))
            g.replay()
            got.append(out.clone())
    s.synchronize()
    assert sq.sq_check() == 0
    # b = 0 from position 0: the whole history is known
    rows = qkv[:, 0].astype(np.float64)
    pos = np.arange(n)
    k = kv4_value(*kv4_encode(rotated(rows[:, Hq * D:(Hq + Hkv) * D], pos, Hkv)))
    v = kv4_value(*kv4_encode(rows[:, (Hq + Hkv) * D:].reshape(n, Hkv, D)))
    q = oracle.rope(rows[:, :Hq * D], pos, Hq, D, THETA).reshape(n, Hq, D)
    ref, bound = attend(q, k, v, pos)
    o = torch.stack([t[0] for t in got]).float().cpu().numpy().astype(np.float64)
    assert (np.abs(o - ref.reshape(n, -1)) <= bound.reshape(n, -1)).all()


def test_offsets_beyond_32_bits():
    """A code cache of more than 2^31 bytes."""
    B, Hkv, Hq, C, T = 130, 2, 10, 1 << 17, 3
    if torch.cuda.mem_get_info()[0] < 4 * B * Hkv * C * 68:
        pytest.skip("not enough memory")
    rng = np.random.default_rng(3)
    u8, f = dict(dtype=torch.uint8, device=dev()), dict(dtype=torch.float16, device=dev())
    dc = [torch.zeros(B, Hkv, C, 64, **u8), torch.zeros(B, Hkv, C, 2, **f), torch.zeros(B, Hkv, C, 64, **u8),
          torch.zeros(B, Hkv, C, 2, **f)]
    pos0 = np.full(B, C - T, np.int32)
    qkv = rng.normal(0, 3, (B * T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    sq.sq_kv4_append(_t(qkv), Hq, Hkv, _t(pos0), THETA, *dc)
    out = torch.empty(B * T, Hq * D, dtype=torch.float16, device=dev())
    _attention(qkv, B, T, Hq, Hkv, pos0, dc, out)
    assert sq.sq_check() == 0
    for b in (0, B - 1):
        rows = qkv[b * T:(b + 1) * T].astype(np.float64)
        pos = C - T + np.arange(T)
        k = np.zeros((C, Hkv, D))
        v = np.zeros((C, Hkv, D))
        k[-T:] = kv4_value(*kv4_encode(rotated(rows[:, Hq * D:(Hq + Hkv) * D], pos, Hkv)))
        v[-T:] = kv4_value(*kv4_encode(rows[:, (Hq + Hkv) * D:].reshape(T, Hkv, D)))
        q = oracle.rope(rows[:, :Hq * D], pos, Hq, D, THETA).reshape(T, Hq, D)
        ref, bound = attend(q, k, v, pos)
        got = out[b * T:(b + 1) * T].float().cpu().numpy().astype(np.float64)
        # nine times the scores of normal queries and keys
        assert (np.abs(got - ref.reshape(T, -1)) <= 9 * bound.reshape(T, -1)).all()


@pytest.mark.parametrize("T,Hq,Hkv,ctx", [(1, 5, 1, 30000), (5, 7, 1, 30000), (1, 8, 2, 120000), (3, 16, 2, 9000)])
def test_long_caches_keep_their_precision(T, Hq, Hkv, ctx):
    """Over a long cache values cancel to a hundredth of one, and what is left has
    to be right: as a whole within the root of the sum of the output's rounding
    and a weight's (each 2^-11 / sqrt(3) at most of a uniform mantissa, 2.8e-4)
    and half as much for fp32 sums of queries and scores."""
    rng = np.random.default_rng(ctx + T)
    C = (ctx + T + 15) // 16 * 16
    cache, vals = _random_cache(rng, 1, Hkv, C, [ctx], T)
    qkv = rng.normal(0, 1, (T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    out = torch.empty(T, Hq * D, dtype=torch.float16, device=dev())
    _attention(qkv, 1, T, Hq, Hkv, [ctx], [_t(c) for c in cache], out)
    assert sq.sq_check() == 0
    pos = ctx + np.arange(T)
    q = oracle.rope(qkv[:, :Hq * D].astype(np.float64), pos, Hq, D, THETA).reshape(T, Hq, D)
    L = ctx + T
    ref = oracle.attention(q, vals[0][0, :, :L].transpose(1, 0, 2), vals[1][0, :, :L].transpose(1, 0, 2), pos)
    got = out.float().cpu().numpy().astype(np.float64)
    rel = np.linalg.norm(got - ref.reshape(T, -1)) / np.linalg.norm(ref)
    assert rel <= 2.8e-4 * (2 ** 0.5 + 0.5), rel


@pytest.mark.parametrize("T,B,C", [(1, 160, 1 << 17), (3, 160, 1 << 17), (1, 300, 1 << 14), (2, 300, 1 << 14)])
def test_many_long_caches_keep_their_precision(T, B, C):
    """As many sequences as leave a (sequence, head) one CTA (and, of 16384 keys,
    fewer than the clusters that would share one): what sums over their keys lose
    is a fifth of the outputs' and the weights' rounding (as a whole 2.8e-4, see
    test_sums_over_many_tiles_keep_their_precision) at most."""
    Hq, Hkv = 10, 2
    if torch.cuda.mem_get_info()[0] < 2 * B * Hkv * C * 136:
        pytest.skip("not enough memory")
    rng = np.random.default_rng(T)
    cache, vals = _random_cache(rng, 1, Hkv, C, [C - T], T)
    qkv = rng.normal(0, 1, (T, (Hq + 2 * Hkv) * D)).astype(np.float16)
    dc = [_t(c).repeat(B, 1, 1, 1) for c in cache]
    out = torch.empty(B * T, Hq * D, dtype=torch.float16, device=dev())
    _attention(np.tile(qkv, (B, 1)), B, T, Hq, Hkv, [C - T] * B, dc, out)
    assert sq.sq_check() == 0
    pos = C - T + np.arange(T)
    q = oracle.rope(qkv[:, :Hq * D].astype(np.float64), pos, Hq, D, THETA).reshape(T, Hq, D)
    ref = oracle.attention(q, vals[0][0].transpose(1, 0, 2), vals[1][0].transpose(1, 0, 2), pos).reshape(T, -1)
    got = out.float().cpu().numpy().astype(np.float64).reshape(B, T, -1)
    assert (got == got[:1]).all()
    rel = np.linalg.norm(got[0] - ref) / np.linalg.norm(ref)
    assert rel <= 2.8e-4 * 1.2, rel


@pytest.mark.parametrize("T,G,C,p", [(5, 1, 64, 20), (5, 7, 64, 20), (9, 1, 64, 20), (5, 7, 65536, 20),
                                     (24, 2, 65536, 115), (32, 4, 65536, 100)])
def test_a_value_that_a_query_does_not_see_has_no_part_in_its_precision(T, G, C, p):
    """The last token's value is of fp16's whole range, 6e7 times the others' size
    (in each of the three kernels, and where new tokens lie in two tiles).  The
    queries before it: as a whole within the bound of long caches above."""
    rng = np.random.default_rng(T + G)
    cache, vals = _random_cache(rng, 1, 1, C, [p], T)
    v = rng.normal(0, 1e-3, (1, 1, C, D))
    v[:, :, p + T - 1] = np.where(np.arange(D) % 2, 6e4, -6e4)
    cv, pv = kv4_encode(v.astype(np.float16))
    vals[1] = kv4_value(cv, pv)
    pv[:, :, p + T:] = np.nan
    cache[2:] = [kv4_pack_v(cv).reshape(1, 1, C, 64), pv]
    qkv = rng.normal(0, 1, (T, (G + 2) * D)).astype(np.float16)
    out = torch.empty(T, G * D, dtype=torch.float16, device=dev())
    _attention(qkv, 1, T, G, 1, [p], [_t(c) for c in cache], out)
    assert sq.sq_check() == 0
    pos, L = p + np.arange(T), p + T
    q = oracle.rope(qkv[:, :G * D].astype(np.float64), pos, G, D, THETA).reshape(T, G, D)
    ref = oracle.attention(q, vals[0][0, :, :L].transpose(1, 0, 2), vals[1][0, :, :L].transpose(1, 0, 2), pos)
    got = out.float().cpu().numpy().astype(np.float64).reshape(T, G, D)
    rel = np.linalg.norm(got - ref, axis=(1, 2)) / np.linalg.norm(ref, axis=(1, 2))
    assert rel[:-1].max() <= 2.8e-4 * (2 ** 0.5 + 0.5), rel
    # the last one's result is one weight times that value: its rounding to fp16 is no mean
    # over mantissas but 2^-11 at most, alike in every element, and the output's adds as much
    assert rel[-1] <= 2 * 2.0 ** -11, rel
