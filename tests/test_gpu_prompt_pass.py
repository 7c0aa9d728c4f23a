"""Prompt attention, the 4-bit cache and log probabilities together, as the
package's own paths run them: packed prompts through a whole decoder, their
scores, and generation behind them, against the oracle's cache-free decoder.

Logits of this decoder lie within 4e-3 of the oracle's (see
test_gpu_generate.py: about a dozen roundings to fp16 on the way).  With every
logit off by at most d a log probability is off by at most 2 d, an entropy by
4 d H, and greedy tokens agree up to the first step where the two largest
logits are within d."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_21704_gb300 as sq
from paper_2609_21704_gb300 import synth
from paper_2609_21704_gb300.generate import Generator, score_prompts
from paper_2609_21704_gb300.stack import DecoderState, LinearStack, PromptState, decoder_pass, prompt_pass
from test_gpu_generate import GAP_TOL, TINY, _oracle_params, dev

pytestmark = pytest.mark.gpu
SEED, LENS, N_NEW = 3, [9, 1, 14, 5], 12


@pytest.fixture(scope="module")
def stack():
    return LinearStack(TINY, dev(), seed=SEED, variants=("int4", "fp8"), host_weights=True)


@pytest.fixture(scope="module")
def params():
    return _oracle_params(TINY, SEED, 5)


def _prompts(lens=LENS, seed=7):
    return [synth.prompt_tokens(seed + i, 1, n, TINY.vocab)[0].tolist() for i, n in enumerate(lens)]


def test_scores_of_packed_prompts(stack, params):
    prompts = _prompts()
    got = score_prompts(stack, prompts, top=3)
    assert sq.sq_check() == 0
    for p, (lp, ent, tt, tl) in zip(prompts, got):
        assert lp.shape == ent.shape == (len(p) - 1,) and tt.shape == tl.shape == (len(p) - 1, 3)
        if len(p) == 1:
            continue
        z = O.decoder_logits(params, p)[:-1]
        ref = z - np.log(np.exp(z - z.max(-1, keepdims=True)).sum(-1, keepdims=True)) - z.max(-1, keepdims=True)
        h = -(np.exp(ref) * ref).sum(-1)
        n = np.arange(len(p) - 1)
        assert np.abs(lp.cpu().numpy() - ref[n, p[1:]]).max() <= 2 * GAP_TOL
        assert (np.abs(ent.cpu().numpy() - h) <= 4 * GAP_TOL * h).all()
        order = np.sort(ref, -1)[:, ::-1]
        clear = (order[:, :3] - order[:, 1:4]).min(-1) > 2 * GAP_TOL  # the three largest in no doubt
        assert np.array_equal(tt.cpu().numpy()[clear], np.argsort(-ref, -1, kind="stable")[clear, :3])
        assert np.abs(tl.cpu().numpy() - order[:, :3]).max() <= 2 * GAP_TOL


def _compare(tokens, params, prompts, n_new):
    """Tokens behind each prompt equal the oracle's greedy ones while those are clear."""
    sure = 0
    for got, p in zip(tokens, prompts):
        assert got[:len(p)] == list(p)
        ref, gaps = O.generate_greedy(params, p, min(n_new, len(got) - len(p)))
        new = got[len(p):]
        for i, (t, g) in enumerate(zip(ref, gaps)):
            if g <= GAP_TOL:
                break
            assert new[i] == t, (p, i)
            sure += 1
    return sure


@pytest.mark.parametrize("K,draft_kv,verifier_kv", [(0, "fp16", "fp16"), (3, "fp16", "fp16"), (3, "int4", "fp16")])
def test_generation_behind_packed_prompts(stack, params, K, draft_kv, verifier_kv):
    """Prompts of different lengths, one pass; the draft's cache may be of 4
    bits: what is generated is the parent's either way."""
    prompts = _prompts()
    s = torch.cuda.Stream()
    g = Generator(stack, len(prompts), K, max(LENS), 160, mode=sq.SQ_ACCEPT_GREEDY, draft_kv=draft_kv,
                  verifier_kv=verifier_kv)
    g.prefill_packed(prompts, s)
    g.run(N_NEW, s)
    assert g.status() == 0
    assert _compare(g.tokens(), params, prompts, N_NEW) >= 20
    # the same generator again, with other lengths
    other = _prompts([2, 14, 3, 7], seed=31)
    g.prefill_packed(other, s)
    g.run(N_NEW, s)
    assert g.status() == 0
    assert _compare(g.tokens(), params, other, N_NEW) >= 20


def test_packed_prefill_equals_prefill(stack, params):
    prompts = np.array(_prompts([10, 10], seed=50), np.int32)
    s = torch.cuda.Stream()
    tokens = []
    for packed in (False, True):
        g = Generator(stack, 2, 2, 10, 96)
        g.prefill_packed(list(prompts), s) if packed else g.prefill(prompts, s)
        g.run(8, s)
        assert g.status() == 0
        tokens.append(g.tokens())
        assert _compare(tokens[-1], params, prompts.tolist(), 8) > 0


def test_decoding_over_a_4_bit_cache_of_the_parent(stack, params):
    """K = 0 with the parent's cache in 4 bits: the prompt's attention is over
    fp16, so the first token is the oracle's; later ones read the cache that the
    prompt left, and are what the oracle's logits allow within the cache's error."""
    prompts = _prompts()
    s = torch.cuda.Stream()
    g = Generator(stack, len(prompts), 0, max(LENS), 96, verifier_kv="int4")
    g.prefill_packed(prompts, s)
    g.run(10, s)
    assert g.status() == 0
    assert _compare(g.tokens(), params, prompts, 1) > 0
    for t, p in zip(g.tokens(), prompts):
        assert len(t) == len(p) + 11


def test_a_pass_over_a_4_bit_cache_is_near_the_fp16_one(stack):
    """The same tokens after a prompt of 30: logits over the 4-bit cache differ
    from those over fp16 by the cache's rounding only.  A value of a row is off
    by at most half a step of its range / 15, here (normal rows of 128, range
    about 5.2) some 0.17 of its standard deviation; attention averages that, and
    the two layers pass it on: half of the logits' own spread is a wide margin,
    and a wrong position, head or half byte is far outside."""
    B, T, C, n = 2, 3, 64, 30
    prompts = _prompts([n, n], seed=70)
    ids = torch.tensor(sum(prompts, []), dtype=torch.int32, device=dev())
    logits = []
    for kv in ("fp16", "int4"):
        cache = DecoderState(stack, B, T, C, context=n, kv=kv, seed=5)
        st = PromptState(stack, B * n, B, C)
        st.offsets.copy_(torch.tensor([0, n, 2 * n], dtype=torch.int32))
        scratch = tuple(torch.zeros((B, TINY.kv_heads, C, 128), dtype=torch.float16, device=dev()) for _ in range(2))
        sq.sq_embed(ids, stack.embedding(), st.x)
        prompt_pass(stack, "fp16", st, cache, scratch=scratch)
        new = torch.arange(B * T, dtype=torch.int32, device=dev()) * 7 + 3
        sq.sq_embed(new, stack.embedding(), cache.x)
        decoder_pass(stack, "fp16", cache)
        assert sq.sq_check() == 0
        logits.append(cache.logits.float().cpu().numpy())
    diff = np.abs(logits[0] - logits[1])
    assert 0 < diff.max() < 0.5 * logits[0].std()


def test_prompts_behind_a_4_bit_prefix(stack):
    """The next part of each text behind what the 4-bit caches hold: bit for bit
    the pass over fp16 caches that hold the same rows read back.  What the
    scratch holds besides, here NaN, has no part in it."""
    B, C, heads = 4, 70, (TINY.q_heads, TINY.kv_heads)
    parts = [LENS, [3, 8, 1, 6]]
    cache = DecoderState(stack, B, 1, C, kv="int4")
    ref = DecoderState(stack, B, 1, C, share_gains=cache)
    shape = (B, heads[1], 80, 128)
    scratch = tuple(torch.full(shape, float("nan"), dtype=torch.float16, device=dev()) for _ in range(2))

    def run(into, lens, pos):
        st = PromptState(stack, sum(lens), B, C)
        st.offsets.copy_(torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32))
        st.pos0.copy_(torch.tensor(pos, dtype=torch.int32))
        ids = torch.tensor(sum(_prompts(lens, seed=90), []), dtype=torch.int32, device=dev())
        sq.sq_embed(ids, stack.embedding(), st.x)
        prompt_pass(stack, "fp16", st, into, scratch=scratch if into.kv4 is not None else None)
        return st.x

    run(cache, parts[0], [0] * B)
    first, last = torch.zeros(B, dtype=torch.int32, device=dev()), torch.tensor(parts[0], dtype=torch.int32, device=dev())
    for li in range(len(stack.layers)):
        back = tuple(torch.zeros(shape, dtype=torch.float16, device=dev()) for _ in range(2))
        sq.sq_kv4_unpack(*cache.kv4[li], first, last, *back)
        ref.k[li].copy_(back[0][:, :, :C])
        ref.v[li].copy_(back[1][:, :, :C])
    for t in scratch:
        t.fill_(float("nan"))
    got, want = run(cache, parts[1], parts[0]), run(ref, parts[1], parts[0])
    assert sq.sq_check() == 0
    assert torch.isfinite(want).all() and torch.equal(got, want)


def test_4_bit_caches_of_any_length(stack, params):
    """max_ctx that is no multiple of 16: the caches hold whole groups."""
    prompts, s = _prompts(), torch.cuda.Stream()
    g = Generator(stack, len(prompts), 0, max(LENS), 70, verifier_kv="int4")
    g.prefill_packed(prompts, s)
    g.run(5, s)
    assert g.status() == 0
    assert _compare(g.tokens(), params, prompts, 1) > 0


def _rows_of(cache, li, b, n):
    """(keys, values, half a step of each) of the first n positions that a 4-bit cache holds."""
    kc, kp, vc, vp = (c[b].cpu().numpy() for c in cache.kv4[li])
    pairs = vc.reshape(vc.shape[0], -1, 128)
    by = np.empty((pairs.shape[0], 2 * pairs.shape[1], 64), np.uint8)
    for odd in (0, 1):
        for byte in (0, 1):
            by[:, odd::2, byte::2] = pairs[..., 2 * odd + byte::4]
    out = []
    for codes, par in ((kc, kp), (by, vp)):
        c = np.empty(codes.shape[:2] + (128,))
        c[..., 0::2], c[..., 1::2] = codes & 15, codes >> 4
        par = par.astype(np.float64)
        out += [(c * par[..., :1] + par[..., 1:])[:, :n].transpose(1, 0, 2), par[:, :n, :1].transpose(1, 0, 2) / 2]
    return out[0], out[2], out[1], out[3]


def _step_over(params, cache, b, token, p):
    """The decoder of the oracle for one token at position p over the rows of a
    4-bit cache, its own among them: its logits; every layer's row of the cache
    has to be this token's key and value within half a step, and as much for a
    dozen roundings to fp16 on the way as 12 x 2^-11 of the row's largest value."""
    Hq, Hkv, D = params["q_heads"], params["kv_heads"], params["head_dim"]
    x = np.asarray(params["embed"], np.float64)[[token]]
    pos = np.array([p])
    for li, (w_qkv, w_o, w_gu, w_dn) in enumerate(params["layers"]):
        qkv = O.linear(O.rmsnorm(x, params["gamma"][2 * li], params["eps"]), w_qkv)
        q = O.rope(qkv[:, :Hq * D], pos, Hq, D, params["theta"])
        k = O.rope(qkv[:, Hq * D:(Hq + Hkv) * D], pos, Hkv, D, params["theta"]).reshape(Hkv, D)
        v = qkv[:, (Hq + Hkv) * D:].reshape(Hkv, D)
        ks, vs, dk, dv = _rows_of(cache, li, b, p + 1)
        for got, want, half in ((ks[p], k, dk[p]), (vs[p], v, dv[p])):
            assert (np.abs(got - want) <= half + 12 * 2.0 ** -11 * np.abs(want).max()).all(), (b, p, li)
        a = O.attention(q.reshape(1, Hq, D), ks, vs, pos)
        x = x + O.linear(a.reshape(1, Hq * D), w_o)
        h = O.rmsnorm(x, params["gamma"][2 * li + 1], params["eps"])
        x = x + O.linear(O.silu_gate_rows(O.linear(h, w_gu), params["intermediate"]), w_dn)
    return O.linear(O.rmsnorm(x, params["gamma"][-1], params["eps"]), params["lm_head"])[0]


@pytest.mark.parametrize("K,max_ctx", [(0, 96), (0, 70), (3, 120)])
def test_each_step_over_the_parents_4_bit_cache(stack, params, K, max_ctx):
    """Steps of one token and verify passes of four, the first eager, the others
    replayed: every token's row in every layer, and the tokens that follow from
    attention over these rows, where the two largest logits are clear."""
    prompts, s, steps = _prompts(), torch.cuda.Stream(), 12 if K == 0 else 5
    g = Generator(stack, len(prompts), K, max(LENS), max_ctx, verifier_kv="int4")
    g.prefill_packed(prompts, s)
    g.run(steps, s)
    s.synchronize()
    assert g.status() == 0
    logits = g.tv.logits.float().cpu().numpy()
    sure = checked = 0
    for b, (t, prompt) in enumerate(zip(g.tokens(), prompts)):
        assert t[:len(prompt)] == prompt and len(t) >= len(prompt) + 1 + steps
        for p in range(len(prompt), len(t) - 1):
            z = _step_over(params, g.tv, b, t[p], p)
            order = np.argsort(-z, kind="stable")
            if z[order[0]] - z[order[1]] > GAP_TOL:
                assert t[p + 1] == order[0], (b, p)
                sure += 1
            checked += 1
        if K == 0:
            assert np.abs(logits[b] - z).max() <= GAP_TOL
    assert checked >= len(prompts) * steps and sure >= checked * 3 // 4


def test_drafts_over_a_4_bit_cache_are_accepted(stack):
    """What is generated is the parent's whatever the draft's cache holds; its
    drafts are accepted about as often as those over an fp16 cache (from a wrong
    cache they agree with the parent's by chance, one in a thousand)."""
    prompts, s, got = _prompts([9, 14, 5, 11], seed=21), torch.cuda.Stream(), []
    for kv in ("fp16", "int4"):
        g = Generator(stack, len(prompts), 3, 14, 160, draft_kv=kv)
        g.prefill_packed(prompts, s)
        g.run(10, s)
        assert g.status() == 0
        got.append(sum(len(t) - len(p) - 1 - 10 for t, p in zip(g.tokens(), prompts)))
    assert got[0] > 20 and got[1] >= got[0] / 2, got


def test_a_4_bit_pass_without_scratch_is_refused(stack):
    cache, st = DecoderState(stack, 1, 1, 16, kv="int4"), PromptState(stack, 4, 1, 16)
    with pytest.raises(ValueError):
        prompt_pass(stack, "fp16", st, cache)


def test_refusals(stack):
    s = torch.cuda.Stream()
    g = Generator(stack, 2, 1, 8, 64)
    for bad in ([[1, 2]], [[1], []], [[1] * 9, [2]]):
        with pytest.raises(ValueError):
            g.prefill_packed(bad, s)
    with pytest.raises(ValueError):
        score_prompts(stack, [])
    with pytest.raises(ValueError):
        DecoderState(stack, 1, 1, 16, kv="fp8")
