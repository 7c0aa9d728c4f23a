"""sq_logprobs against a 64-bit reference: vocabularies that do not divide,
ties, banned entries, sure rows, refusals of rows and tokens."""
import numpy as np
import pytest
import torch

import paper_2609_21704_gb300 as sq
from gpu_util import dev
from serve_ref import logprobs

pytestmark = pytest.mark.gpu


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev())


def _run(z, T, tokens, top, skew=0, stream=None):
    R, V = z.shape
    if skew:  # rows that start anywhere: z 2-byte aligned
        buf = torch.zeros(R * V + 8, dtype=torch.float16, device=dev())
        zt = buf[skew:skew + R * V].view(R, V)
        zt.copy_(_t(z))
    else:
        zt = _t(z)
    f = dict(dtype=torch.float32, device=dev())
    lp, ent, tl = torch.zeros(R, **f), torch.zeros(R, **f), torch.zeros(R, top, **f)
    tt = torch.zeros(R, top, dtype=torch.int32, device=dev())
    torch.cuda.synchronize()
    sq.sq_logprobs(zt, T, _t(tokens.astype(np.int32)), lp, ent, tt, tl, stream)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (lp, ent, tt, tl)]


def _close(got, ref, x, V, what):
    """fp32 throughout: a value's own rounding, its distance x from the row's
    largest logit over T (a difference and a product), and the logarithm of a
    sum of V terms, which loses at most half a step for each of a thread's
    V / 256 additions, 32 more to join threads, and 2^-21 in an exponential."""
    bound = 2.0 ** -24 * (np.abs(ref) + 3 * np.abs(x) + V / 256 + 32 + 16)
    err = np.abs(got.astype(np.float64) - ref)
    assert (err <= bound).all(), f"{what}: {(err - bound).max():.2e} over the bound"


def _check(z, T, tokens, top, skew=0):
    got = _run(z, T, tokens, top, skew)
    assert sq.sq_check() == 0
    lp, ent, tt, tl = logprobs(z, T, tokens, top)
    V = z.shape[1]
    assert np.array_equal(got[2], tt)
    with np.errstate(invalid="ignore"):
        _close(got[0], lp, lp, V, "logprob")
        _close(got[3], tl, tl, V, "top")
        # a mean of distances: each as far off as the logarithm, and weights that are
        far = np.abs(z.astype(np.float64) - z.max(-1, keepdims=True)).max(-1) / T
        _close(got[1], ent, np.minimum(far, 40), V * 2, "entropy")


@pytest.mark.parametrize("R,V,top,T,skew", [
    (1, 151936, 20, 1.0, 0), (3, 152064, 32, 0.7, 0), (5, 50021, 5, 1.3, 1), (2, 1, 1, 1.0, 0), (3, 2, 2, 1.0, 0),
    (7, 33, 32, 0.5, 3), (4, 1000, 0, 1.0, 0), (9, 4097, 7, 2.0, 5), (130, 257, 3, 1.0, 0), (2, (1 << 20) - 1, 32, 1.0, 0),
    (3, 300001, 20, 1.0, 7), (400, 32000, 5, 1.0, 0), (1, 40, 32, 1.0, 0)])
def test_matches_reference(R, V, top, T, skew):
    rng = np.random.default_rng(R + V)
    z = rng.normal(0, 2, (R, V)).astype(np.float16)
    _check(z, T, rng.integers(0, V, R), top, skew)


def test_ties_and_signed_zeros_go_to_the_lowest_index():
    V = 5000
    z = np.full((6, V), -3.0, np.float16)
    z[1] = 0.0
    z[1, ::2] = -0.0
    z[2, [4999, 17, 2500]] = 4.0
    z[3] = (np.arange(V) % 7).astype(np.float16)      # 714 equal maxima
    z[4] = np.arange(V).astype(np.float16) / 1000      # runs of equal values
    z[5] = -65504.0
    _check(z, 1.0, np.array([0, 1, 17, 6, 4999, 3]), 32)


@pytest.mark.parametrize("order", ["rising", "falling", "peak", "one_thread"])
def test_adversarial_orders(order):
    """Candidates that arrive in the worst order, or all in one place."""
    V = 60000
    x = np.sort(np.random.default_rng(3).normal(0, 3, V)).astype(np.float16)
    if order == "falling":
        x = x[::-1]
    elif order == "peak":
        x = np.roll(x, 777)
    elif order == "one_thread":
        y = np.random.default_rng(4).permutation(x[:-40])
        x = np.concatenate([y[:30000], x[-40:], y[30000:]])
    z = np.stack([x, x])
    _check(z, 1.0, np.array([0, V - 1]), 32)


def test_banned_entries_and_sure_rows():
    rng = np.random.default_rng(8)
    V = 9000
    z = rng.normal(0, 2, (5, V)).astype(np.float16)
    z[0, ::2] = -np.inf
    z[1] = -np.inf
    z[1, 4321] = 1.0                        # one entry left
    z[2] = -np.inf
    z[2, [5, 8000, 17]] = [1.0, 1.0, 2.0]   # fewer than `top`
    z[3] = -30.0
    z[3, 100] = 20.0                        # sure of one token
    tokens = np.array([2, 4321, 17, 100, 3])
    got = _run(z, 1.0, tokens, 6)
    assert sq.sq_check() == 0
    with np.errstate(invalid="ignore"):
        lp, ent, tt, tl = logprobs(z, 1.0, tokens, 6)
    lp[0] = -np.inf
    assert np.array_equal(got[2], tt)
    assert np.isneginf(got[0][0]) and got[0][1] == 0.0 and got[1][1] == 0.0
    assert np.array_equal(np.isneginf(got[3]), np.isneginf(tl))
    fin = np.isfinite(tl)
    _close(got[3][fin], tl[fin], tl[fin], V, "top")
    # 9000 e^-50: what is left beside a sure token is kept, to fp32's precision
    rest = (V - 1) * np.exp(-50.0)
    assert abs(got[0][3] + rest) <= 1e-4 * rest and abs(got[1][3] - 51 * rest) <= 1e-3 * 51 * rest


def test_rows_and_tokens_that_are_refused():
    rng = np.random.default_rng(9)
    V = 3000
    z = rng.normal(0, 1, (5, V)).astype(np.float16)
    z[1, 2999] = np.nan
    z[2, 0] = np.inf
    z[3] = -np.inf
    tokens = np.array([5, 5, 5, 5, 5])
    got = _run(z, 1.0, tokens, 4)
    assert sq.sq_check() == sq.SQ_DEV_NONFINITE_LOGIT | sq.SQ_DEV_NO_MASS
    for i in (1, 2, 3):
        assert np.isnan(got[0][i]) and np.isnan(got[1][i]) and (got[2][i] == -1).all() and np.isnan(got[3][i]).all()
    ref = logprobs(z[[0, 4]], 1.0, tokens[[0, 4]], 4)
    assert np.array_equal(got[2][[0, 4]], ref[2])
    for bad in (-1, V, 1 << 30):
        got = _run(z[[0, 4]], 1.0, np.array([bad, 7]), 4)
        assert sq.sq_check() == sq.SQ_DEV_BAD_TOKEN_ID
        assert np.isnan(got[0][0]) and np.isfinite(got[0][1]) and np.array_equal(got[2], ref[2])


def test_parts_on_their_own_and_in_a_graph():
    R, V = 6, 7777
    z = np.random.default_rng(10).normal(0, 2, (R, V)).astype(np.float16)
    tokens = np.arange(R) * 1000
    full = _run(z, 1.0, tokens, 5)
    zt, tk = _t(z), _t(tokens.astype(np.int32))
    f = dict(dtype=torch.float32, device=dev())
    lp, ent, tl = torch.zeros(R, **f), torch.zeros(R, **f), torch.zeros(R, 5, **f)
    tt = torch.zeros(R, 5, dtype=torch.int32, device=dev())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sq.sq_logprobs(zt, 1.0, tk, lp)
        sq.sq_logprobs(zt, 1.0, None, None, ent)
        sq.sq_logprobs(zt, 1.0, None, None, None, tt, tl)
    with torch.cuda.stream(s):
        for _ in range(3):
            g.replay()
    s.synchronize()
    for a, b in zip((lp, ent, tt, tl), full):
        assert np.array_equal(a.cpu().numpy(), b)


def test_rows_beyond_32_bit_offsets():
    R, V = 5000, 500000  # 2.5e9 logits
    if torch.cuda.mem_get_info()[0] < 3 * R * V:
        pytest.skip("not enough memory")
    z = torch.zeros(R, V, dtype=torch.float16, device=dev())
    z[-1, 123] = 5.0
    z[-1, 400001] = 6.0
    f = dict(dtype=torch.float32, device=dev())
    ent, tl = torch.zeros(R, **f), torch.zeros(R, 3, **f)
    tt = torch.zeros(R, 3, dtype=torch.int32, device=dev())
    sq.sq_logprobs(z, 1.0, None, None, ent, tt, tl)
    assert sq.sq_check() == 0
    assert tt[-1].tolist() == [400001, 123, 0] and tt[0].tolist() == [0, 1, 2]
    assert abs(float(ent[0]) - np.log(V)) < 1e-4


@pytest.mark.parametrize("T", [1e-4, 1e-6, 1e-9, 1e-30])
@pytest.mark.parametrize("R,V", [(8, 151936), (8, 90), (800, 4099)])
def test_small_temperatures(R, V, T):
    """Down to the smallest temperature only the largest entries have any weight:
    log probability 0 of one, -log n of n equal ones, far ones down to -1e35."""
    T = float(np.float32(T))
    rng = np.random.default_rng(V)
    z = rng.normal(0, 2, (R, V)).astype(np.float16)
    z[1] += np.float16(20)
    z[2, [3, V // 2, V - 1]] = 17.25                     # three equal ones
    z[3] = -np.abs(z[3]) - np.float16(30)                # all below zero
    z[4, V - 3] = 65504.0
    z[5] = -65504.0
    z[6, ::2] = -np.inf                                  # banned entries
    z[7] = 12.3
    best = z.argmax(-1)
    tokens = np.where(np.arange(R) % 3 == 2, rng.integers(0, V // 2, R) * 2 + 1, best)
    _check(z, T, tokens, 5)
