"""Refusals of prompt attention, the 4-bit cache and token log probabilities:
argument checks of the C ABI and of the Python binding, without a GPU.  No
call here reaches a kernel."""
import ctypes

import pytest
import torch

import paper_2609_21704_gb300 as sq

P = ctypes.c_void_p
FAKE, OTHER, ODD = P(4096), P(8192), P(4098)
INVALID, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    sq.build()
    return sq.load()


def _prompt(lib, **kw):
    a = dict(qkv=FAKE, N=10, offsets=FAKE, B=2, Hq=12, Hkv=2, D=128, pos0=FAKE, theta=1e6, k=FAKE, v=OTHER, C=64,
             out=OTHER, ws=FAKE, ws_bytes=1 << 40) | kw
    return lib.sq_attention_prompt(a["qkv"], a["N"], a["offsets"], a["B"], a["Hq"], a["Hkv"], a["D"], a["pos0"],
                                   a["theta"], a["k"], a["v"], a["C"], a["out"], a["ws"], a["ws_bytes"], None)


HEADS = [(dict(Hq=13), SHAPE), (dict(Hq=0), SHAPE), (dict(Hkv=0), SHAPE), (dict(B=-1), SHAPE), (dict(B=70000), SHAPE),
         (dict(Hq=514, Hkv=2), SHAPE), (dict(D=64), UNSUPPORTED), (dict(C=0), SHAPE), (dict(C=(1 << 17) + 16), SHAPE),
         (dict(theta=1.0), INVALID), (dict(theta=float("inf")), INVALID), (dict(theta=float("nan")), INVALID)]


@pytest.mark.parametrize("kw,status", HEADS + [
    (dict(N=-1), SHAPE), (dict(N=(1 << 22) + 1, Hq=2), SHAPE), (dict(N=1 << 22, Hq=512), SHAPE),
    (dict(qkv=None), INVALID), (dict(offsets=None), INVALID), (dict(pos0=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(out=None), INVALID), (dict(out=FAKE), INVALID), (dict(v=FAKE), INVALID),
    (dict(qkv=P(4104)), ALIGN), (dict(out=P(8200)), ALIGN), (dict(k=P(4104)), ALIGN), (dict(offsets=ODD), ALIGN),
    (dict(pos0=ODD), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE), (dict(ws=P(4104)), ALIGN),
    (dict(B=0), 0), (dict(N=0), 0), (dict(B=0, qkv=None, ws=None), 0)])
def test_prompt_arguments(lib, kw, status):
    assert _prompt(lib, **kw) == status
    if status:
        assert b"sq_attention_prompt" in lib.sq_last_error()


def _append(lib, **kw):
    a = dict(qkv=FAKE, N=10, offsets=FAKE, B=2, Hq=12, Hkv=2, D=128, pos0=FAKE, theta=1e6, kc=FAKE, kp=FAKE, vc=OTHER,
             vp=OTHER, C=64) | kw
    return lib.sq_kv4_append(a["qkv"], a["N"], a["offsets"], a["B"], a["Hq"], a["Hkv"], a["D"], a["pos0"], a["theta"],
                             a["kc"], a["kp"], a["vc"], a["vp"], a["C"], None)


CACHE = [(dict(C=72), SHAPE), (dict(kc=None), INVALID), (dict(kp=None), INVALID), (dict(vc=None), INVALID),
         (dict(vp=None), INVALID), (dict(kc=P(4104)), ALIGN), (dict(vp=P(8200)), ALIGN), (dict(vc=FAKE), INVALID),
         (dict(vp=FAKE), INVALID)]


@pytest.mark.parametrize("kw,status", HEADS + CACHE + [
    (dict(N=-1), SHAPE), (dict(offsets=None, N=11), SHAPE), (dict(qkv=None), INVALID), (dict(pos0=None), INVALID),
    (dict(qkv=P(4104)), ALIGN), (dict(offsets=ODD), ALIGN), (dict(B=0), 0), (dict(N=0), 0)])
def test_append_arguments(lib, kw, status):
    assert _append(lib, **kw) == status


def _kv4(lib, **kw):
    a = dict(qkv=FAKE, B=2, T=5, Hq=12, Hkv=2, D=128, pos0=FAKE, theta=1e6, kc=FAKE, kp=FAKE, vc=OTHER, vp=OTHER,
             C=64, out=OTHER, ws=FAKE, ws_bytes=1 << 40) | kw
    return lib.sq_attention_kv4(a["qkv"], a["B"], a["T"], a["Hq"], a["Hkv"], a["D"], a["pos0"], a["theta"], a["kc"],
                                a["kp"], a["vc"], a["vp"], a["C"], a["out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", HEADS + CACHE + [
    (dict(T=-1), SHAPE), (dict(T=33), SHAPE), (dict(T=21, Hq=20), SHAPE), (dict(qkv=None), INVALID),
    (dict(out=None), INVALID), (dict(out=FAKE), INVALID), (dict(out=P(8200)), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(ws_bytes=0), WORKSPACE), (dict(ws=P(4104)), ALIGN), (dict(B=0), 0), (dict(T=0), 0)])
def test_kv4_attention_arguments(lib, kw, status):
    assert _kv4(lib, **kw) == status


def _unpack(lib, **kw):
    a = dict(kc=FAKE, kp=FAKE, vc=OTHER, vp=OTHER, B=2, Hkv=2, D=128, C=64, first=FAKE, last=FAKE, k=FAKE, v=OTHER) | kw
    return lib.sq_kv4_unpack(a["kc"], a["kp"], a["vc"], a["vp"], a["B"], a["Hkv"], a["D"], a["C"], a["first"],
                             a["last"], a["k"], a["v"], None)


@pytest.mark.parametrize("kw,status", CACHE + [
    (dict(Hkv=0), SHAPE), (dict(D=64), UNSUPPORTED), (dict(first=None), INVALID), (dict(last=ODD), ALIGN),
    (dict(k=None), INVALID), (dict(k=P(4104)), ALIGN), (dict(v=FAKE), INVALID), (dict(B=0), 0)])
def test_unpack_arguments(lib, kw, status):
    assert _unpack(lib, **kw) == status


def _logprobs(lib, **kw):
    a = dict(z=FAKE, R=3, V=100, T=1.0, tokens=FAKE, lp=FAKE, ent=FAKE, top=5, tt=FAKE, tl=FAKE) | kw
    return lib.sq_logprobs(a["z"], a["R"], a["V"], a["T"], a["tokens"], a["lp"], a["ent"], a["top"], a["tt"], a["tl"],
                           None)


@pytest.mark.parametrize("kw,status", [
    (dict(R=-1), SHAPE), (dict(R=(1 << 24) + 1), SHAPE), (dict(V=0), SHAPE), (dict(V=1 << 20), SHAPE),
    (dict(top=-1), SHAPE), (dict(top=33), SHAPE), (dict(V=4), SHAPE), (dict(T=0.0), INVALID), (dict(T=-1.0), INVALID),
    (dict(T=float("inf")), INVALID), (dict(T=float("nan")), INVALID), (dict(T=1e-39), INVALID), (dict(z=None), INVALID),
    (dict(tokens=None), INVALID), (dict(lp=None), INVALID), (dict(tt=None), INVALID), (dict(tl=None), INVALID),
    (dict(tokens=None, lp=None, ent=None, top=0), INVALID), (dict(z=P(4097)), ALIGN), (dict(tt=ODD), ALIGN),
    (dict(ent=ODD), ALIGN), (dict(R=0), 0)])
def test_logprobs_arguments(lib, kw, status):
    assert _logprobs(lib, **kw) == status


def test_workspace_sizes(lib):
    # rotated queries of every row and head at least
    assert sq.sq_attention_prompt_workspace_bytes(2, 100, 12, 2, 256) >= 100 * 12 * 128 * 2
    assert sq.sq_attention_prompt_workspace_bytes(2, 100, 13, 2, 256) == 0
    assert sq.sq_attention_prompt_workspace_bytes(2, 100, 12, 2, 0) == 0
    assert sq.sq_attention_kv4_workspace_bytes(2, 5, 12, 2, 256) > 0
    assert sq.sq_attention_kv4_workspace_bytes(2, 40, 12, 2, 256) == 0


@pytest.mark.parametrize("name", ["sq_attention_prompt_workspace_bytes", "sq_attention_kv4_workspace_bytes"])
def test_workspace_sizes_are_the_current_device_s(monkeypatch, name):
    """Sizes go by the SMs of the device: another one's answer is not given again."""
    device = [0]

    class Lib:
        def __getattr__(self, _):
            return lambda *args: 1000 + device[0]

    monkeypatch.setattr(sq, "load", Lib)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device[0])
    args = (7, 11, 12, 2, 4242 * 16)  # (asked nowhere else: a remembered size would outlive the test)
    for device[0] in (0, 1, 0):
        assert getattr(sq, name)(*args) == 1000 + device[0]


def _cpu(*shape, dtype=torch.float16):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_refuses_types_shapes_and_host_tensors():
    i32, u8, f32 = torch.int32, torch.uint8, torch.float32
    qkv, off, pos0 = _cpu(10, 16 * 128), _cpu(3, dtype=i32), _cpu(2, dtype=i32)
    k, out, ws = _cpu(2, 2, 64, 128), _cpu(10, 12 * 128), _cpu(16, dtype=u8)

    def prompt(qkv=qkv, off=off, Hq=12, Hkv=2, pos0=pos0, k=k, v=k, out=out):
        sq.sq_attention_prompt(qkv, off, Hq, Hkv, pos0, 1e6, k, v, out, ws)

    with pytest.raises(ValueError, match="CUDA device"):
        prompt()
    for bad in (dict(qkv=qkv.float()), dict(off=off.long()), dict(pos0=pos0.long()), dict(k=k.bfloat16()),
                dict(out=out.float()), dict(qkv=None)):
        with pytest.raises(TypeError):
            prompt(**bad)
    for bad in (dict(Hkv=5), dict(Hq=11), dict(off=off[:2]), dict(k=k[:1]), dict(v=k[:, :, :32]), dict(out=out[:9]),
                dict(k=k[..., :64]), dict(qkv=qkv[:, :128])):
        with pytest.raises(ValueError):
            prompt(**bad)

    cache = [_cpu(2, 2, 64, 64, dtype=u8), _cpu(2, 2, 64, 2), _cpu(2, 2, 64, 64, dtype=u8), _cpu(2, 2, 64, 2)]
    with pytest.raises(ValueError, match="CUDA device"):
        sq.sq_kv4_append(qkv, 12, 2, pos0, 1e6, *cache, offsets=off)
    with pytest.raises(ValueError):
        sq.sq_kv4_append(qkv, 12, 2, pos0, 1e6, *cache, offsets=off[:2])
    with pytest.raises(ValueError):
        sq.sq_kv4_append(qkv, 12, 2, pos0, 1e6, cache[0], cache[1][:, :, :32], *cache[2:])
    with pytest.raises(ValueError):
        sq.sq_kv4_append(qkv, 12, 2, pos0, 1e6, *cache[:2], cache[2][:1], cache[3])
    with pytest.raises(TypeError):
        sq.sq_kv4_append(qkv, 12, 2, pos0, 1e6, cache[0].float(), *cache[1:])
    with pytest.raises(ValueError):
        sq.sq_attention_kv4(qkv, 2, 4, 12, 2, pos0, 1e6, *cache, out, ws)     # 10 rows are not 2 x 4
    with pytest.raises(ValueError):
        sq.sq_kv4_unpack(*cache, pos0, pos0, k, k[:, :, :32])
    with pytest.raises(ValueError, match="CUDA device"):
        sq.sq_kv4_unpack(*cache, pos0, pos0, k, k)

    z, tok, f = _cpu(4, 50), _cpu(4, dtype=i32), _cpu(4, dtype=f32)
    with pytest.raises(ValueError, match="CUDA device"):
        sq.sq_logprobs(z, 1.0, tok, f)
    with pytest.raises(TypeError):
        sq.sq_logprobs(z.float(), 1.0, tok, f)
    with pytest.raises(TypeError):
        sq.sq_logprobs(z, 1.0, tok.long(), f)
    with pytest.raises(ValueError):
        sq.sq_logprobs(z, 1.0, tok[:3], f)
    with pytest.raises(ValueError):
        sq.sq_logprobs(z, 1.0, tok, f, None, _cpu(4, 3, dtype=i32), _cpu(4, 2, dtype=f32))
    with pytest.raises(TypeError):
        sq.sq_logprobs(z, 1.0, tok, f, None, _cpu(4, 3, dtype=i32), None)
