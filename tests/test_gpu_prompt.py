"""sq_attention_prompt against a 64-bit reference: packed sequences of
different lengths, prefixes, head layouts, empty sequences, rows behind the
last, and what lies in the caches behind a token."""
import numpy as np
import pytest
import torch

import paper_2609_21704_gb300 as sq
from gpu_util import dev
from serve_ref import D, THETA, attend, prompt, rotated

pytestmark = pytest.mark.gpu


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev())


def _workspace(B, N, Hq, Hkv, C):
    # whatever it holds before the call
    return torch.full((sq.sq_attention_prompt_workspace_bytes(B, N, Hq, Hkv, C),), 255, dtype=torch.uint8,
                      device=dev())


def _case(seed, lens, pos0, Hq, Hkv, C, pad=0, lead=0, scale=1.0):
    rng = np.random.default_rng(seed)
    off = lead + np.concatenate([[0], np.cumsum(lens)])
    N = int(off[-1]) + pad
    qkv = rng.normal(0, scale, (N, (Hq + 2 * Hkv) * D)).astype(np.float16)
    kc = rng.normal(0, 1, (len(lens), Hkv, C, D)).astype(np.float16)
    vc = rng.normal(0, 1, (len(lens), Hkv, C, D)).astype(np.float16)
    return qkv, off.astype(np.int32), np.array(pos0, np.int32), kc, vc


def _run(qkv, off, pos0, kc, vc, Hq, Hkv, stream=None):
    B, N, C = len(pos0), qkv.shape[0], kc.shape[2]
    k, v = _t(kc), _t(vc)
    out = torch.full((N, Hq * D), 7.0, dtype=torch.float16, device=dev())
    sq.sq_attention_prompt(_t(qkv), _t(off), Hq, Hkv, _t(pos0), THETA, k, v, out, _workspace(B, N, Hq, Hkv, C),
                           stream)
    torch.cuda.synchronize()
    return out.cpu().numpy(), k.cpu().numpy(), v.cpu().numpy()


def _assert(got, ref, bound, what=""):
    mine = ~np.isnan(ref)
    err = np.abs(got.astype(np.float64) - ref)[mine]
    assert np.isfinite(got.astype(np.float64)[mine]).all(), what
    over = err - bound[mine]
    assert (over <= 0).all(), f"{what}: {over.max():.3e} over the bound, error {err.max():.3e}"
    assert (got[~mine] == 7.0).all(), "rows of no sequence were written"


CASES = [
    # lens, pos0, Hq, Hkv, C, pad
    ([1], [0], 12, 2, 16, 0),
    ([20], [0], 12, 2, 64, 0),
    ([5, 0, 1, 130], [0, 3, 7, 0], 12, 2, 200, 3),
    ([0, 0], [0, 0], 4, 2, 16, 5),
    ([300], [0], 28, 4, 512, 0),
    ([37, 256, 51, 52, 128], [0, 100, 511, 1, 128], 40, 8, 640, 1),
    ([129, 127, 1], [127, 129, 255], 8, 8, 256, 0),
    ([64, 3], [960, 0], 5, 1, 1024, 0),
    ([33] * 9, [5 * i for i in range(9)], 14, 2, 128, 0),
    ([40, 17], [0, 9], 16, 1, 64, 2),
    ([9], [4087], 40, 8, 4096, 0),
    ([70], [0], 130, 2, 70, 0),
]


@pytest.mark.parametrize("lens,pos0,Hq,Hkv,C,pad", CASES)
def test_matches_reference(lens, pos0, Hq, Hkv, C, pad):
    args = _case(sum(lens) + Hq, lens, pos0, Hq, Hkv, C, pad)
    got, k, v = _run(*args, Hq, Hkv)
    assert sq.sq_check() == 0
    qkv, off, p0, kc, vc = args
    ref, bound, rk, rv = prompt(qkv, lens, pos0, off, Hq, Hkv, kc, vc)
    assert np.array_equal(k.view(np.uint16), rk.view(np.uint16))
    assert np.array_equal(v.view(np.uint16), rv.view(np.uint16))
    _assert(got, ref, bound)


def test_rows_before_the_first_sequence_are_left():
    lens, pos0 = [40, 30], [0, 8]
    args = _case(3, lens, pos0, 12, 2, 64, pad=6, lead=5)
    got, _, _ = _run(*args, 12, 2)
    assert sq.sq_check() == 0
    ref, bound, _, _ = prompt(args[0], lens, pos0, args[1], 12, 2, args[3], args[4])
    _assert(got, ref, bound)


@pytest.mark.parametrize("scale", [0.05, 6.0, 30.0])
def test_flat_and_sharp_softmax(scale):
    lens, pos0 = [200, 77], [0, 300]
    args = _case(11, lens, pos0, 12, 2, 400, scale=scale)
    args[3][:] = (args[3].astype(np.float32) * scale).astype(np.float16)
    got, _, _ = _run(*args, 12, 2)
    ref, bound, _, _ = prompt(args[0], lens, pos0, args[1], 12, 2, args[3], args[4])
    # scores are scale^2 as large, and so is what their fp32 sums lose (the
    # part of 2^-13 in the bound), as a share of at most one of the values
    vmax = max(np.abs(args[4].astype(np.float64)).max(), np.abs(args[0].astype(np.float64)).max())
    extra = min(1.0, max(0.0, scale ** 2 - 1) * 2.0 ** -13) * vmax
    _assert(got, ref, bound + extra)


def test_growing_maxima_rescale():
    """Keys that grow along the sequence raise the running maximum block after block."""
    lens, pos0 = [700], [0]
    args = _case(12, lens, pos0, 6, 1, 704)
    ramp = np.linspace(0.1, 9.0, 700)[:, None]
    args[0][:, :7 * D] = np.abs(args[0][:, :7 * D])
    args[0][:, 6 * D:7 * D] = (args[0][:, 6 * D:7 * D].astype(np.float64) * ramp).astype(np.float16)
    got, _, _ = _run(*args, 6, 1)
    ref, bound, _, _ = prompt(args[0], lens, pos0, args[1], 6, 1, args[3], args[4])
    _assert(got, ref, bound + 81 * 2.0 ** -13)


def test_what_lies_behind_a_token_has_no_effect():
    """NaN and infinities in the unused cache, and in the keys and values of later tokens."""
    lens, pos0, Hq, Hkv = [150, 60], [10, 0], 10, 2
    args = _case(5, lens, pos0, Hq, Hkv, 256)
    qkv, off, p0, kc, vc = args
    for b, n in enumerate(lens):
        kc[b, :, pos0[b] + n:] = np.nan
        vc[b, :, pos0[b] + n:] = np.inf
        vc[b, :, pos0[b] + n::3] = np.nan
    clean = _run(*args, Hq, Hkv)[0]
    ref, bound, _, _ = prompt(qkv, lens, pos0, off, Hq, Hkv, np.nan_to_num(kc), np.nan_to_num(vc, posinf=0))
    _assert(clean, ref, bound)
    # token 100 of the first sequence: values of head 0 infinite, of head 1 NaN
    w = (Hq + Hkv) * D
    qkv2 = qkv.copy()
    qkv2[100, w + 3] = np.inf
    qkv2[100, w + 7] = -np.inf
    qkv2[140, w + 7] = np.inf
    qkv2[100, w + D + 9] = np.nan
    got = _run(qkv2, off, p0, kc, vc, Hq, Hkv)[0]
    heads = got.reshape(-1, Hq, D)
    G = Hq // Hkv
    assert np.array_equal(got[:100], clean[:100]) and np.array_equal(got[150:], clean[150:])
    assert np.isposinf(heads[100:150, :G, 3]).all() and np.isneginf(heads[100:140, :G, 7]).all()
    assert np.isnan(heads[140:150, :G, 7]).all() and np.isnan(heads[100:150, G:, 9]).all()
    rest = np.ones(D, bool)
    rest[[3, 7]] = False
    _assert(got.reshape(-1, Hq, D)[:, :G, rest].reshape(len(got), -1),
            ref.reshape(-1, Hq, D)[:, :G, rest].reshape(len(got), -1),
            bound.reshape(-1, Hq, D)[:, :G, rest].reshape(len(got), -1))
    # a NaN key: rows that see it are NaN, rows before it are as they were
    qkv3 = qkv.copy()
    qkv3[100, Hq * D:Hq * D + 5] = np.nan
    got = _run(qkv3, off, p0, kc, vc, Hq, Hkv)[0].reshape(-1, Hq, D)
    assert np.array_equal(got[:100].reshape(100, -1), clean[:100])
    assert np.isnan(got[100:150, :G]).all() and np.isfinite(got[100:150, G:].astype(np.float32)).all()
    sq.sq_check()


@pytest.mark.parametrize("lens,Hkv", [([1], 3), ([2, 3], 3), ([1], 1), ([4], 17), ([600, 500], 5)])
def test_odd_numbers_of_key_value_heads(lens, Hkv):
    """Rows of values that end in the middle of a warp, with one that is not
    finite in the last head of the first token."""
    Hq, C = 2 * Hkv, 608
    args = _case(Hkv, lens, [0] * len(lens), Hq, Hkv, C)
    ref, bound, rk, rv = prompt(args[0], lens, [0] * len(lens), args[1], Hq, Hkv, args[3], args[4])
    args[0][0, -3] = np.inf
    rv[0, -1, 0, -3] = np.inf
    got, k, v = _run(*args, Hq, Hkv)
    assert sq.sq_check() == 0
    assert np.array_equal(k.view(np.uint16), rk.view(np.uint16))
    assert np.array_equal(v.view(np.uint16), rv.view(np.uint16))
    sees = got[:lens[0]].reshape(lens[0], Hq, D)[:, -2:, -3]
    assert np.isposinf(sees).all()
    sees[:] = ref[:lens[0]].reshape(lens[0], Hq, D)[:, -2:, -3]
    _assert(got, ref, bound)


def test_a_prompt_in_chunks_equals_the_whole():
    """Chunks behind their own prefix leave the caches of the whole prompt, bit for bit."""
    Hq, Hkv, C, n = 28, 4, 512, 400
    qkv, off, p0, kc, vc = _case(8, [n], [0], Hq, Hkv, C)
    out, k, v = _run(qkv, off, p0, kc, vc, Hq, Hkv)
    ref, bound, _, _ = prompt(qkv, [n], [0], off, Hq, Hkv, kc, vc)
    kk, vv = kc, vc
    for s, e in ((0, 130), (130, 131), (131, 400)):
        o, kk, vv = _run(qkv[s:e], np.array([0, e - s], np.int32), np.array([s], np.int32), kk, vv, Hq, Hkv)
        _assert(o, ref[s:e], bound[s:e])
    assert np.array_equal(k.view(np.uint16), kk.view(np.uint16))
    assert np.array_equal(v.view(np.uint16), vv.view(np.uint16))


def test_agrees_with_decode_attention():
    """The last tokens through sq_attention over the same caches."""
    Hq, Hkv, C, n, T = 12, 2, 320, 300, 5
    qkv, off, p0, kc, vc = _case(9, [n], [0], Hq, Hkv, C)
    out, k, v = _run(qkv, off, p0, kc, vc, Hq, Hkv)
    o = torch.empty(T, Hq * D, dtype=torch.float16, device=dev())
    ws = torch.empty(sq.sq_attention_workspace_bytes(1, T, Hq, Hkv, C), dtype=torch.uint8, device=dev())
    sq.sq_attention(_t(qkv[n - T:]), 1, T, Hq, Hkv, _t(np.array([n - T], np.int32)), THETA, _t(k), _t(v), o, ws)
    _, bound, _, _ = prompt(qkv, [n], [0], off, Hq, Hkv, kc, vc)
    # sq_attention does not round its queries: 2^-11 of a score of up to 5 more
    diff = np.abs(o.float().cpu().numpy().astype(np.float64) - out[n - T:].astype(np.float64))
    assert (diff <= 2 * bound[n - T:] + 5 * 2.0 ** -11).all()


def test_sequences_that_do_not_fit():
    lens, pos0, Hq, Hkv, C = [20, 30, 10, 7], [0, 40, -1, 57], 12, 2, 64
    args = _case(6, lens, pos0, Hq, Hkv, C)
    got, k, v = _run(*args, Hq, Hkv)
    assert sq.sq_check() == sq.SQ_DEV_BAD_POSITION
    ref, bound, rk, rv = prompt(args[0], [20, 0, 0, 7], [0, 0, 0, 57], args[1], Hq, Hkv, args[3], args[4])
    ref[20:60] = 0.0
    _assert(got, ref, bound)
    assert np.array_equal(k.view(np.uint16), rk.view(np.uint16))
    assert np.array_equal(v.view(np.uint16), rv.view(np.uint16))


@pytest.mark.parametrize("off", [[0, 20, 10, 30], [-1, 5, 10, 30], [0, 10, 20, 31], [30, 20, 10, 0]])
def test_bad_offsets_write_nothing(off):
    Hq, Hkv, C = 12, 2, 64
    qkv, _, _, kc, vc = _case(7, [10, 10, 10], [0, 0, 0], Hq, Hkv, C)
    got, k, v = _run(qkv, np.array(off, np.int32), np.zeros(3, np.int32), kc, vc, Hq, Hkv)
    assert sq.sq_check() == sq.SQ_DEV_BAD_POSITION
    assert (got == 7.0).all()
    assert np.array_equal(k, kc) and np.array_equal(v, vc)


def test_no_rows_and_no_sequences():
    Hq, Hkv, C = 12, 2, 64
    z = torch.zeros
    kw = dict(device=dev())
    kc = z(1, Hkv, C, D, dtype=torch.float16, **kw)
    out = z(0, Hq * D, dtype=torch.float16, **kw)
    sq.sq_attention_prompt(z(0, (Hq + 2 * Hkv) * D, dtype=torch.float16, **kw), z(2, dtype=torch.int32, **kw), Hq,
                           Hkv, z(1, dtype=torch.int32, **kw), THETA, kc, kc.clone(), out, _workspace(1, 1, Hq, Hkv, C))
    assert sq.sq_check() == 0


def test_positions_and_offsets_beyond_32_bits():
    """A cache of 2^31 values: the last sequence's rows lie beyond 32-bit offsets."""
    Hq, Hkv, C, B = 10, 2, 1 << 17, 65
    if torch.cuda.mem_get_info()[0] < 3 * B * Hkv * C * D * 2:
        pytest.skip("not enough memory")
    n, p = 40, C - 40
    rng = np.random.default_rng(2)
    qkv = rng.normal(0, 1, (n, (Hq + 2 * Hkv) * D)).astype(np.float16)
    k = torch.zeros(B, Hkv, C, D, dtype=torch.float16, device=dev())
    v = torch.zeros_like(k)
    old = 500  # the cached tokens that differ from zero
    ko = rng.normal(0, 2, (Hkv, old, D)).astype(np.float16)
    vo = rng.normal(0, 1, (Hkv, old, D)).astype(np.float16)
    k[-1, :, p - old:p], v[-1, :, p - old:p] = _t(ko), _t(vo)
    off = np.array([0] * B + [n], np.int32)
    pos0 = np.array([0] * (B - 1) + [p], np.int32)
    out = torch.full((n, Hq * D), 7.0, dtype=torch.float16, device=dev())
    sq.sq_attention_prompt(_t(qkv), _t(off), Hq, Hkv, _t(pos0), THETA, k, v, out, _workspace(B, n, Hq, Hkv, C))
    assert sq.sq_check() == 0
    kc = np.zeros((1, Hkv, C, D), np.float16)
    vc = np.zeros((1, Hkv, C, D), np.float16)
    kc[0, :, p - old:p], vc[0, :, p - old:p] = ko, vo
    ref, bound, rk, _ = prompt(qkv, [n], [p], [0], Hq, Hkv, kc, vc)
    assert np.array_equal(k[-1, :, p:].cpu().numpy().view(np.uint16), rk[0, :, p:].view(np.uint16))
    assert not bool(k[:-1].any()) and not bool(v[:-1].any())
    _assert(out.cpu().numpy(), ref, bound)


def test_streams_graphs_and_shared_workspace():
    """Two captured calls that share a workspace, replayed in turn on another
    stream, with lengths and positions that change between replays."""
    Hq, Hkv, C, N = 28, 4, 256, 200
    a, b = (_case(s, [N], [0], Hq, Hkv, C) for s in (21, 22))
    ws = _workspace(2, N, Hq, Hkv, C)
    stream = torch.cuda.Stream()
    graphs, bufs = [], []
    for args in (a, b):
        qkv, k, v = _t(args[0]), _t(args[3]).repeat(2, 1, 1, 1), _t(args[4]).repeat(2, 1, 1, 1)
        off, pos0 = _t(np.array([0, 0, 0], np.int32)), _t(np.array([0, 0], np.int32))
        out = torch.full((N, Hq * D), 7.0, dtype=torch.float16, device=dev())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            sq.sq_attention_prompt(qkv, off, Hq, Hkv, pos0, THETA, k, v, out, ws)
        graphs.append(g)
        bufs.append((qkv, k, v, off, pos0, out))
    for lens, pos0 in (([120, 80], [0, 3]), ([1, 150], [200, 9]), ([0, 0], [0, 0])):
        for args, (qkv, k, v, off, p, out) in zip((a, b), bufs):
            k.copy_(_t(args[3]).repeat(2, 1, 1, 1))
            v.copy_(_t(args[4]).repeat(2, 1, 1, 1))
            off.copy_(_t(np.array([0, lens[0], sum(lens)], np.int32)))
            p.copy_(_t(np.array(pos0, np.int32)))
            out.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(3):
                for g in graphs:
                    g.replay()
        stream.synchronize()
        for args, (qkv, k, v, off, p, out) in zip((a, b), bufs):
            ref, bound, _, _ = prompt(args[0], lens, pos0, [0, lens[0]], Hq, Hkv, np.repeat(args[3], 2, 0),
                                      np.repeat(args[4], 2, 0))
            _assert(out.cpu().numpy(), ref, bound)
    assert sq.sq_check() == 0


def test_same_call_same_bits():
    lens, pos0 = [300, 5, 64], [0, 1000, 400]
    args = _case(31, lens, pos0, 40, 8, 1024)
    one = _run(*args, 40, 8)[0]
    for _ in range(3):
        assert np.array_equal(one.view(np.uint16), _run(*args, 40, 8)[0].view(np.uint16))


def test_long_prefix_keeps_its_precision():
    """As a whole within the root of the sum of the output's rounding and a
    weight's (each at most 2.8e-4, 2^-11 / sqrt(3)), and half as much for fp32 sums."""
    lens, pos0, Hq, Hkv = [9], [30000], 10, 2
    args = _case(13, lens, pos0, Hq, Hkv, 30016)
    got, _, _ = _run(*args, Hq, Hkv)
    ref, _, _, _ = prompt(args[0], lens, pos0, args[1], Hq, Hkv, args[3], args[4])
    rel = np.linalg.norm(got.astype(np.float64) - ref) / np.linalg.norm(ref)
    assert rel <= 2.8e-4 * (2 ** 0.5 + 0.5), rel


@pytest.mark.parametrize("B,n,G,Hkv", [(600, 3, 5, 1), (400, 20, 16, 1), (513, 1, 2, 2)])
def test_many_sequences(B, n, G, Hkv):
    """More sequences, and more tiles, than the plan keeps in shared memory."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, n + 1, B).tolist()
    if B == 400:
        lens = [n] * B
    pos0 = rng.integers(0, 40, B).tolist()
    args = _case(B, lens, pos0, G * Hkv, Hkv, 64, pad=2)
    got, k, v = _run(*args, G * Hkv, Hkv)
    assert sq.sq_check() == 0
    ref, bound, rk, rv = prompt(args[0], lens, pos0, args[1], G * Hkv, Hkv, args[3], args[4])
    assert np.array_equal(k.view(np.uint16), rk.view(np.uint16))
    assert np.array_equal(v.view(np.uint16), rv.view(np.uint16))
    _assert(got, ref, bound)


def _some_rows(args, lens, pos0, Hq, Hkv, rows):
    """The reference of `prompt` for some rows of a large batch: (out, bound, kc, vc)."""
    qkv, off, _, kc, vc = args
    kc, vc = kc.copy(), vc.copy()
    out, bound = np.empty((len(rows), Hq * D)), np.empty((len(rows), Hq * D))
    for b, n in enumerate(lens):
        new = qkv[off[b]:off[b] + n].astype(np.float64)
        pos = pos0[b] + np.arange(n)
        kc[b, :, pos] = rotated(new[:, Hq * D:(Hq + Hkv) * D], pos, Hkv).astype(np.float16)
        vc[b, :, pos] = new[:, (Hq + Hkv) * D:].reshape(n, Hkv, D).astype(np.float16)
        at = [i for i, r in enumerate(rows) if off[b] <= r < off[b] + n]
        t = np.array([rows[i] - off[b] for i in at], int)
        if not at:
            continue
        L = pos0[b] + n
        o, e = attend(rotated(new[t, :Hq * D], pos[t], Hq), kc[b, :, :L].transpose(1, 0, 2).astype(np.float64),
                      vc[b, :, :L].transpose(1, 0, 2).astype(np.float64), pos[t])
        out[at], bound[at] = o.reshape(len(at), -1), e.reshape(len(at), -1)
    return out, bound, kc, vc


@pytest.mark.parametrize("lens,pos0,C", [([3000], [0], 3008), ([700, 1, 1500, 333], [0, 900, 257, 2000], 2400),
                                         ([1300, 1201], [3000, 17], 4304)])
def test_ctas_that_take_several_items_of_many_blocks(lens, pos0, C):
    """More tiles than pieces that the plan would cut (40 / 8 heads), three and
    more of many blocks for each CTA in turn: some rows of every sequence, its
    first and last among them."""
    Hq, Hkv = 40, 8
    args = _case(len(lens), lens, pos0, Hq, Hkv, C)
    got, k, v = _run(*args, Hq, Hkv)
    assert sq.sq_check() == 0
    rng = np.random.default_rng(1)
    rows = sorted(set(rng.integers(0, sum(lens), 40)) | set(args[1][:-1]) | set(args[1][1:] - 1))
    ref, bound, rk, rv = _some_rows(args, lens, pos0, Hq, Hkv, rows)
    assert np.array_equal(k.view(np.uint16), rk.view(np.uint16))
    assert np.array_equal(v.view(np.uint16), rv.view(np.uint16))
    _assert(got[rows], ref, bound)
    assert np.array_equal(got.view(np.uint16), _run(*args, Hq, Hkv)[0].view(np.uint16))


def test_uncut_sums_over_the_longest_cache():
    """Tiles that are not cut along 131072 keys, of values with a mean: nothing of
    what the sums lose cancels.  A product of sixteen keys may cut 2^-23 off its
    sum, and a sum has 64 blocks' 512 of them, so 2^-14 of the result at most,
    systematically; the outputs' roundings, of 128 means, add three times
    2^-11 / sqrt(3 x 128) to the mean error."""
    Hq, Hkv, C, n = 64, 1, 1 << 17, 1300
    rng = np.random.default_rng(4)
    mean = rng.uniform(0.5, 2.0, D)
    p = C - n
    kc = rng.normal(0, 1, (1, Hkv, C, D)).astype(np.float16)
    vc = (mean + rng.normal(0, 0.1, (1, Hkv, C, D))).astype(np.float16)
    qkv = rng.normal(0, 1, (n, (Hq + 2) * D))
    qkv[:, :Hq * D] *= 0.3
    qkv[:, -D:] = mean + 0.1 * qkv[:, -D:]
    args = qkv.astype(np.float16), np.array([0, n], np.int32), np.array([p], np.int32), kc, vc
    got, _, _ = _run(*args, Hq, Hkv)
    assert sq.sq_check() == 0
    rows = [0, n - 1]
    ref, bound, _, _ = _some_rows(args, [n], [p], Hq, Hkv, rows)
    _assert(got[rows], ref, bound + 2.0 ** -14 * np.abs(ref))
    bias = ((got[rows].astype(np.float64) - ref) / ref).mean()
    assert abs(bias) <= 2.0 ** -14 + 3 * 2.0 ** -11 / (3 * 128) ** 0.5, bias


@pytest.mark.parametrize("n,p,Hq,Hkv", [(1300, 11000, 64, 1), (1200, 58000, 10, 2)])
def test_sums_put_aside_and_what_changes_between_them(n, p, Hq, Hkv):
    """Tiles of 75 to 100 blocks, uncut and as pieces of a cut tile, whose running
    maxima grow along the keys (up to six times as long as normal ones: scores'
    fp32 sums lose six times as much, a share of at most one of the values), with
    a value of a new token infinite and one of another NaN."""
    C = (p + n + 15) // 16 * 16
    rng = np.random.default_rng(p)
    kc, vc = (rng.standard_normal((1, Hkv, C, D), np.float32) for _ in range(2))
    kc *= np.linspace(0.1, 6.0, C, dtype=np.float32)[:, None]
    qkv = rng.normal(0, 1, (n, (Hq + 2 * Hkv) * D)).astype(np.float16)
    args = qkv, np.array([0, n], np.int32), np.array([p], np.int32), kc.astype(np.float16), vc.astype(np.float16)
    rows = [0, 257, 700, n - 1]
    ref, bound, _, _ = _some_rows(args, [n], [p], Hq, Hkv, rows)
    bound += 5 * 2.0 ** -13 * np.abs(args[4].astype(np.float32)).max()
    got, _, _ = _run(*args, Hq, Hkv)
    assert sq.sq_check() == 0
    _assert(got[rows], ref, bound)
    w = (Hq + Hkv) * D
    qkv[200, w + 3] = np.inf
    qkv[600, w + 9] = np.nan
    odd, _, _ = _run(*args, Hq, Hkv)
    odd, got = (x.reshape(n, Hkv, Hq // Hkv, D) for x in (odd, got))
    assert np.isposinf(odd[200:, 0, :, 3]).all() and np.isnan(odd[600:, 0, :, 9]).all()
    odd[200:, 0, :, 3], odd[600:, 0, :, 9] = got[200:, 0, :, 3], got[600:, 0, :, 9]
    assert np.array_equal(odd, got)
