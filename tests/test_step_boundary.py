"""The calls around attention and the gradients, without a GPU: what the C entry points refuse before any launch, the sizes of
workspaces, the table of a set of gradients, and what reaches the C functions through the native part of the binding."""
import ctypes as C
import math

import pytest
import torch

import step_reference as ref

P = 0x1000      # non-null, 16-byte aligned, never dereferenced on these paths
STREAM = 0x7A0


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


# --- refusals ---------------------------------------------------------------------------------

def test_rope_table_refuses(lx):
    def call(rot=64, n=16, base=1e4, table=P, **kw):
        s = dict(kind=0, factor=1.0, trained_length=0.0, low_turns=1.0, high_turns=32.0, gain=1.0)
        s.update(kw)
        s = lx.lx_rope_scaling(*[s[k] for k in ("kind", "factor", "trained_length", "low_turns", "high_turns", "gain")])
        return lx._lib.lx_rope_table(rot, n, base, C.byref(s), table, None)
    for bad in (dict(table=None), dict(rot=0), dict(rot=63), dict(rot=-2), dict(n=0), dict(base=0.0), dict(base=math.inf), dict(base=math.nan),
                dict(gain=math.nan), dict(kind=1, factor=0.0), dict(kind=1, factor=math.inf), dict(kind=2, rot=2, factor=2.0),
                dict(kind=3, factor=2.0), dict(kind=3, factor=2.0, trained_length=64.0, low_turns=4.0, high_turns=4.0)):
        assert call(**bad) == lx.LX_ERR_INVALID_ARG, bad
    assert call(kind=4) == call(kind=-1) == call(n=1 << 27) == lx.LX_ERR_UNSUPPORTED


def rope_tensor(lx, heads=4, S=8, D=64, **kw):
    t = dict(i=P, o=0x9000, heads=heads, si=(heads * S * D, S * D, D), so=(heads * S * D, S * D, D))
    t.update(kw)
    return lx.lx_rope_tensor(t["i"], t["o"], t["heads"], (C.c_int64 * 3)(*t["si"]), (C.c_int64 * 3)(*t["so"]))


def test_rope_refuses(lx):
    def call(dt=None, B=2, S=8, D=64, rot=64, layout=0, table=P, n_pos=8, positions=None, n=1, **kw):
        arr = (lx.lx_rope_tensor * 2)(rope_tensor(lx, **kw), rope_tensor(lx))
        return lx._lib.lx_rope(lx.LX_BF16 if dt is None else dt, B, S, D, rot, layout, 0, table, n_pos, positions, arr if n else None, n or 1, None)
    for bad in (dict(B=0), dict(S=0), dict(D=0), dict(rot=0), dict(rot=31), dict(rot=66), dict(table=None), dict(table=P + 2), dict(n_pos=0),
                dict(n_pos=7), dict(positions=P + 1), dict(n=0), dict(n=3), dict(i=None), dict(o=None), dict(i=P + 1), dict(o=P + 1),
                dict(heads=0), dict(si=(0, -1, 64)), dict(so=(2048, 0, 64)), dict(so=(2048, 512, 63)), dict(i=0x9000, si=(0, 512, 64))):
        assert call(**bad) == lx.LX_ERR_INVALID_ARG, bad
    assert call(dt=7) == call(layout=2) == call(heads=65536) == lx.LX_ERR_UNSUPPORTED
    assert call(B=1 << 20, S=1 << 12, n_pos=1 << 12) == call(B=1 << 14, S=1 << 12, n_pos=1 << 12) == lx.LX_ERR_UNSUPPORTED


def test_key_ranges_refuse(lx):
    f = lx._lib.lx_attn_key_ranges
    for bad in ((0, 8, P, P, None, 1, 1, P, P), (1, 0, P, P, None, 1, 1, P, P), (1, 8, P, P, None, -1, 1, P, P), (1, 8, None, P, None, 1, 1, P, P),
                (1, 8, P, None, None, 1, 1, P, P), (1, 8, P, P, None, 1, 1, None, P), (1, 8, P, P, None, 1, 1, P, None),
                (1, 8, P + 2, P, None, 1, 1, P, P), (1, 8, P, P, P + 1, 1, 1, P, P), (1, 8, P, P, None, 1, 1, P, P + 2)):
        assert f(*bad, None) == lx.LX_ERR_INVALID_ARG, bad
    assert f(1 << 16, 1 << 16, P, P, None, 1, 1, P, P, None) == lx.LX_ERR_UNSUPPORTED


SIZES = dict(dt=1, B=2, Hq=8, Hkv=2, Sq=16, Sk=48, D=64)
BAD_SIZES = (dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Sq=0), dict(Sk=0), dict(D=0), dict(Hkv=3), dict(Hq=-8))
UNSUPPORTED = (dict(dt=9), dict(D=96), dict(B=65536), dict(Hq=1 << 17), dict(Sq=1 << 30), dict(Sk=(1 << 31) - 1), dict(B=32768, Hq=512, Sq=1),
               dict(B=32768, Hq=512, Hkv=512, Sk=1), dict(B=8, Sk=1 << 30), dict(dt=0, B=1, Sq=(1 << 25) + 1), dict(dt=0, B=1, Sk=(1 << 25) + 1))
BAD_RULES = (dict(scale=math.nan), dict(scale=math.inf), dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf), dict(key_lo=P), dict(key_hi=P),
             dict(slopes=P + 1), dict(q_start=P + 2), dict(key_lo=P + 1, key_hi=P))


def rules_of(lx, kw):
    r = dict(scale=0.125, causal=1, cap=0.0, slopes=None, q_start=None, key_lo=None, key_hi=None)
    r.update({k: v for k, v in kw.items() if k in r})
    return lx.lx_score_rules(*[r[k] for k in ("scale", "causal", "cap", "slopes", "q_start", "key_lo", "key_hi")])


def strides(*s):
    return (C.c_int64 * len(s))(*s)


def score_fwd(lx, **kw):
    c = {**SIZES, **dict(Q=P, K=P, V=P, O=P, LSE=P, ws=P, bytes=1 << 40, null=None)}
    c.update({k: v for k, v in kw.items() if k in c})
    st = {"Q": (8192, 1024, 64), "K": (6144, 3072, 64), "V": (6144, 3072, 64), "O": (8192, 1024, 64)}
    st.update({k[1:]: v for k, v in kw.items() if k in ("sQ", "sK", "sV", "sO")})
    rules = None if c["null"] else C.byref(rules_of(lx, kw))
    return lx._lib.lx_score_attn_fwd(c["dt"], c["B"], c["Hq"], c["Hkv"], c["Sq"], c["Sk"], c["D"], rules, c["Q"], strides(*st["Q"]), c["K"],
                                     strides(*st["K"]), c["V"], strides(*st["V"]), c["O"], strides(*st["O"]), c["LSE"], c["ws"], c["bytes"], None)


def test_attention_refuses(lx):
    for bad in BAD_SIZES + BAD_RULES + (
            dict(null=1), dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(Q=P + 8), dict(K=P + 2), dict(O=P + 8), dict(LSE=P + 2),
            dict(sQ=(8192, 1024, 65)), dict(sK=(6144, 3072, 4)), dict(sV=(-8, 3072, 64)), dict(sO=(0, 1024, 64)), dict(sO=(8192, 1024, 56))):
        assert score_fwd(lx, **bad) == lx.LX_ERR_INVALID_ARG, bad
    for bad in UNSUPPORTED:
        assert score_fwd(lx, **bad) == lx.LX_ERR_UNSUPPORTED, bad
    # few queries over many keys need a workspace
    few = dict(Sq=1, Sk=40000, B=1)
    need = lx.lx_score_attn_fwd_workspace_bytes(lx.LX_BF16, 1, 8, 2, 1, 40000, 64)
    assert need > 0
    assert score_fwd(lx, **few, bytes=need - 1) == score_fwd(lx, **few, ws=None) == lx.LX_ERR_WORKSPACE
    assert score_fwd(lx, **few, ws=P + 8) == lx.LX_ERR_INVALID_ARG


def score_bwd(lx, **kw):
    c = {**SIZES, **dict(Q=P, K=P, V=P, O=P, LSE=P, dO=P, dQ=P, dK=P, dV=P, ws=P, bytes=1 << 40, null=None)}
    c.update({k: v for k, v in kw.items() if k in c})
    q, k = [8192, 1024, 64], [6144, 3072, 64]
    st = q + k + k + q + q + q + k + k
    for at, v in kw.get("st", {}).items():
        st[at] = v
    rules = None if c["null"] else C.byref(rules_of(lx, kw))
    return lx._lib.lx_score_attn_bwd(c["dt"], c["B"], c["Hq"], c["Hkv"], c["Sq"], c["Sk"], c["D"], rules,
                                     *[c[n] for n in ("Q", "K", "V", "O", "LSE", "dO", "dQ", "dK", "dV")], strides(*st), c["ws"], c["bytes"], None)


def test_attention_backward_refuses(lx):
    tensors = ("Q", "K", "V", "O", "LSE", "dO", "dQ", "dK", "dV")
    for bad in BAD_SIZES + BAD_RULES + tuple({n: v} for n in tensors for v in (None, P + 2)) + (
            dict(null=1), dict(ws=P + 8), dict(st={2: 65}), dict(st={13: -8}), dict(st={15: 0}), dict(st={19: 8}), dict(st={23: 56})):
        assert score_bwd(lx, **bad) == lx.LX_ERR_INVALID_ARG, bad
    for bad in UNSUPPORTED:
        assert score_bwd(lx, **bad) == lx.LX_ERR_UNSUPPORTED, bad
    need = lx.lx_score_attn_bwd_workspace_bytes(lx.LX_BF16, 2, 8, 2, 16, 48, 64)
    assert need > 0
    assert score_bwd(lx, bytes=need - 1) == score_bwd(lx, ws=None) == lx.LX_ERR_WORKSPACE


@pytest.mark.parametrize("Sq", [1, 3, 16, 17, 200, 4096])
@pytest.mark.parametrize("Sk", [1, 64, 65, 1000, 32768, 1 << 20])
def test_workspaces_are_small(lx, Sq, Sk):
    """Forward: where keys are split, the partial sums of at most as many workgroups as the chip holds.  Backward: the queries'
    numbers, and sums of the key side where its workgroups are few.  Unsupported sizes need none."""
    for dt in (lx.LX_BF16, lx.LX_F16, lx.LX_F32):
        for B, Hq, Hkv, D in ((1, 1, 1, 64), (4, 32, 8, 128), (64, 16, 16, 64)):
            fwd, bwd = (f(dt, B, Hq, Hkv, Sq, Sk, D) for f in (lx.lx_score_attn_fwd_workspace_bytes, lx.lx_score_attn_bwd_workspace_bytes))
            assert fwd == 0 if dt == lx.LX_F32 or Sq > 16 else fwd <= 1 << 26
            assert 0 < bwd <= 64 * B * Hq * (Sq + 64) + 8 * (Hq // Hkv) * 2 * B * Hkv * Sk * D + (1 << 20)
    assert lx.lx_score_attn_fwd_workspace_bytes(lx.LX_BF16, 1, 1, 1, Sq, Sk, 80) == lx.lx_score_attn_bwd_workspace_bytes(9, 1, 1, 1, Sq, Sk, 64) == 0


# --- a set of gradients -----------------------------------------------------------------------

def grads(lx, *entries):
    return (lx.lx_grad_tensor * max(len(entries), 1))(*[lx.lx_grad_tensor(*e) for e in entries]), len(entries)


def test_grad_table(lx):
    piece = 16384
    arr, n = grads(lx, (P, P, 2 * piece + 1, lx.LX_F32), (None, None, 0, lx.LX_BF16), (P, P, 1, lx.LX_F16), (P, P, piece, lx.LX_BF16))
    size = lx._lib.lx_grad_table_bytes(arr, n)
    host, pieces = torch.zeros(size, dtype=torch.uint8), C.c_int32(-1)
    assert lx._lib.lx_grad_table_build(arr, n, host.data_ptr(), size, C.byref(pieces)) == lx.LX_OK
    assert pieces.value == 5
    entries = host[:n * 32].view(torch.int64).view(n, 4)
    of = host[n * 32:n * 32 + 4 * 5].view(torch.int32)
    assert entries[:, 2].tolist() == [2 * piece + 1, 0, 1, piece] and of.tolist() == [0, 0, 0, 2, 3]
    assert lx._lib.lx_grad_table_build(arr, n, host.data_ptr(), size - 1, C.byref(pieces)) == lx.LX_ERR_INVALID_ARG
    assert lx._lib.lx_grad_table_build(arr, n, host.data_ptr() + 4, size, C.byref(pieces)) == lx.LX_ERR_INVALID_ARG
    assert lx._lib.lx_grad_table_build(arr, n, None, size, C.byref(pieces)) == lx.LX_ERR_INVALID_ARG
    assert lx._lib.lx_grad_table_build(arr, n, host.data_ptr(), size, None) == lx.LX_ERR_INVALID_ARG
    arr, _ = grads(lx)
    assert lx._lib.lx_grad_table_build(arr, 0, host.data_ptr(), size, C.byref(pieces)) == lx.LX_OK and pieces.value == 0


def test_grad_set_refuses(lx):
    host, pieces = torch.zeros(4096, dtype=torch.uint8), C.c_int32()

    def build(*entries):
        arr, n = grads(lx, *entries)
        s = lx._lib.lx_grad_table_build(arr, n, host.data_ptr(), 4096, C.byref(pieces))
        assert (lx._lib.lx_grad_table_bytes(arr, n) == 0) == (s != lx.LX_OK)
        return s
    ok = (P, P, 8, lx.LX_F32)
    assert build(ok) == lx.LX_OK
    for bad in ((P, P, -1, lx.LX_F32), (None, P, 8, lx.LX_F32), (P + 2, P, 8, lx.LX_F32), (P, P + 1, 8, lx.LX_BF16), (P, None, 8, lx.LX_F32)):
        assert build(ok, bad) == lx.LX_ERR_INVALID_ARG, bad
        assert build((None, None, 0, lx.LX_F32), ok, bad) == lx.LX_ERR_INVALID_ARG, bad
    assert build((P, P, 8, 5)) == build((P, P, 1 << 46, lx.LX_F32)) == lx.LX_ERR_UNSUPPORTED


def test_clip_refuses(lx):
    f, room = lx._lib.lx_grad_norm_clip, lx._lib.lx_grad_norm_clip_workspace_bytes(3)
    assert 0 < room <= lx._lib.lx_grad_norm_clip_workspace_bytes(1 << 30) <= 1 << 15
    for bad in ((None, 2, 3, 1.0, P, P, room), (P, -1, 3, 1.0, P, P, room), (P, 2, -1, 1.0, P, P, room), (P, 2, 3, -1.0, P, P, room),
                (P, 2, 3, math.nan, P, P, room), (P, 2, 3, 1.0, None, P, room), (P, 2, 3, 1.0, P + 2, P, room), (P + 4, 2, 3, 1.0, P, P, room),
                (P, 2, 3, 1.0, P, P + 4, room)):
        assert f(*bad, None) == lx.LX_ERR_INVALID_ARG, bad
    assert f(P, 2, 3, 1.0, P, None, room, None) == f(P, 2, 3, 1.0, P, P, room - 1, None) == lx.LX_ERR_WORKSPACE


# --- the native part of the binding -----------------------------------------------------------

@pytest.fixture
def calls(lx):
    """(lx, calls made, status to return): every argument, HOST structures opened."""
    names = ("lx_rope", "lx_attn_key_ranges", "lx_score_attn_fwd", "lx_score_attn_bwd", "lx_grad_norm_clip")
    seen, status, keep, addr = [], [0], [], {}

    def opened(v, t):
        if t is C.POINTER(lx.lx_score_rules):
            r = C.cast(v, t).contents
            return (r.scale, r.causal, r.cap, r.slopes, r.q_start, r.key_lo, r.key_hi)
        if t is C.POINTER(lx.lx_rope_tensor):
            return [(x.in_, x.out, x.heads, list(x.in_strides),
                     list(x.out_strides)) for x in (C.cast(v, t)[i] for i in range(2))]
        return v
    for n in names:
        types = getattr(lx._lib, n).argtypes
        plain = [t if t in (C.c_int, C.c_int32, C.c_float, C.c_size_t) else C.c_void_p for t in types]

        def record(*args, _n=n, _t=types):
            out = []
            for i, (v, t) in enumerate(zip(args, _t)):
                if t is C.POINTER(C.c_int64):
                    out.append([C.cast(v, t)[k] for k in range(24 if _n == "lx_score_attn_bwd" else 3)])
                else:
                    out.append(opened(v, t))
            seen.append((_n, out))
            return status[0]
        f = C.CFUNCTYPE(C.c_int, *plain)(record)
        keep.append(f)
        addr[n] = C.cast(f, C.c_void_p).value
    real = {n: C.cast(getattr(lx._lib, n), C.c_void_p).value for n in lx.EXPORTS}

    def room(n, beside):
        return torch.empty(n, dtype=torch.uint8, device=beside.device)

    def bind(a, stream):
        lx._call.bind(real, lx._DTYPES, lx.LxError, stream, torch.uint8, torch.float32, torch.int32)
        lx._call.bind_step({**real, **a}, room)
    bind(addr, lambda: STREAM)
    yield lx, seen, status
    bind({}, lx._stream)


def p(t):
    return t.data_ptr()


def test_rope_arguments(calls):
    lx, seen, _ = calls
    Q, K = torch.zeros(2, 5, 4, 64, dtype=torch.float16).transpose(1, 2), torch.zeros(2, 2, 5, 64, dtype=torch.float16)
    Qo, table, pos = torch.zeros(2, 4, 5, 64, dtype=torch.float16), torch.zeros(9, 32), torch.zeros(2, 5, dtype=torch.int32)
    lx.lx_rope(Q, K, table, pos, Qo, K, interleaved=True)
    lx.lx_rope(Q, None, table, None, Q, None, inverse=True)
    head = [lx.LX_F16, 2, 5, 64, 32]
    q_in, q_out, k = [1280, 64, 256], [1280, 320, 64], [640, 320, 64]
    a, b = (s[1] for s in seen)
    assert a[:10] == head + [1, 0, p(table), 9, p(pos)] and a[11:] == [2, STREAM]
    assert a[10] == [(p(Q), p(Qo), 4, q_in, q_out), (p(K), p(K), 2, k, k)]
    assert b[:10] == head + [0, 1, p(table), 9, None] and b[11:] == [1, STREAM]
    assert b[10][0] == (p(Q), p(Q), 4, q_in, q_in)
    for bad in ((Q, K.float(), table, pos, Qo, K), (Q, K, table.double(), pos, Qo, K), (Q, K, table, pos.long(), Qo, K),
                (Q, K, table, pos[:1], Qo, K), (Q, K[:1], table, pos, Qo, K[:1]), (Q, K, table, pos, Qo[:, :2], K), (Q, K, table, pos, Qo[..., :32], K)):
        with pytest.raises(AssertionError):
            lx.lx_rope(*bad)
    assert len(seen) == 2


def test_key_range_arguments(calls):
    lx, seen, status = calls
    d = [torch.zeros(3, dtype=torch.int32) for _ in range(3)]
    lo, hi = (torch.zeros(2, 7, dtype=torch.int32) for _ in range(2))
    lx.lx_attn_key_ranges(d[0], d[1], None, True, lo, hi)
    lx.lx_attn_key_ranges(*d, False, lo, hi)
    assert [s[1] for s in seen] == [[2, 7, p(d[0]), p(d[1]), None, 3, 1, p(lo), p(hi), STREAM], [2, 7, *map(p, d), 3, 0, p(lo), p(hi), STREAM]]
    with pytest.raises(AssertionError):
        lx.lx_attn_key_ranges(d[0], d[1][:2], None, True, lo, hi)
    with pytest.raises(AssertionError):
        lx.lx_attn_key_ranges(d[0], d[1], None, True, lo, hi.long())
    status[0] = lx.LX_ERR_UNSUPPORTED
    with pytest.raises(lx.LxError) as e:
        lx.lx_attn_key_ranges(*d, False, lo, hi)
    assert e.value.status == lx.LX_ERR_UNSUPPORTED


def test_attention_arguments(calls):
    lx, seen, status = calls

    def t(*s):
        return torch.zeros(s, dtype=torch.bfloat16)
    Q, K, V, O = t(2, 6, 4, 64).transpose(1, 2), t(2, 2, 9, 64), t(2, 2, 9, 128)[..., :64], t(2, 4, 6, 64)
    LSE, slopes, start = torch.zeros(2, 4, 6), torch.zeros(4), torch.zeros(2, dtype=torch.int32)
    lo, hi = (torch.zeros(2, 6, dtype=torch.int32) for _ in range(2))
    ws = torch.zeros(64, dtype=torch.uint8)
    sq, sk, sv, so = [1536, 64, 256], [1152, 576, 64], [2304, 1152, 128], [1536, 384, 64]
    size = [lx.LX_BF16, 2, 4, 2, 6, 9, 64]
    assert lx.lx_score_attn_fwd(Q, K, V, 0.125, True, O, LSE, cap=2.0, slopes=slopes, key_lo=lo, key_hi=hi, q_start=start, workspace=ws) == (O, LSE)
    lx.lx_score_attn_fwd(Q, K, V, 0.5, False, O, None, workspace=ws)
    assert seen.pop(0)[1] == size + [(0.125, 1, 2.0, p(slopes), p(start), p(lo), p(hi)), p(Q), sq, p(K), sk, p(V), sv, p(O), so, p(LSE), p(ws), 64, STREAM]
    assert seen.pop(0)[1] == size + [(0.5, 0, 0.0, None, None, None, None), p(Q), sq, p(K), sk, p(V), sv, p(O), so, None, p(ws), 64, STREAM]
    dQ, dK, dV = t(2, 4, 6, 64), t(2, 2, 9, 64), t(2, 9, 2, 64).transpose(1, 2)
    lx.lx_score_attn_bwd(Q, K, V, O, LSE, Q, 0.125, True, dQ, dK, dV, slopes=slopes, q_start=start, workspace=ws)
    assert seen.pop(0)[1] == size + [(0.125, 1, 0.0, p(slopes), p(start), None, None), p(Q), p(K), p(V), p(O), p(LSE), p(Q), p(dQ), p(dK), p(dV),
                                     sq + sk + sv + so + sq + so + sk + [1152, 64, 128], p(ws), 64, STREAM]
    # without a workspace one is made, of the size that the call needs
    lx.lx_score_attn_bwd(Q, K, V, O, LSE, Q, 0.125, True, dQ, dK, dV)
    assert seen.pop(0)[1][-2] == lx.lx_score_attn_bwd_workspace_bytes(*size)
    # every refusal by the shapes, types and layouts, before the call
    good = dict(Q=Q, K=K, V=V, scale=0.125, causal=True, O=O, LSE=LSE, slopes=slopes, key_lo=lo, key_hi=hi, q_start=start)
    for bad in (dict(K=K.half()), dict(V=V[:, :, :8]), dict(K=K[:1], V=V[:1]), dict(O=O[:, :, :5]), dict(O=O.float()), dict(LSE=LSE[:1]),
                dict(LSE=LSE.double()), dict(slopes=slopes[:3]), dict(slopes=slopes.half()), dict(key_lo=lo.long()), dict(key_hi=hi[:, :5]),
                dict(q_start=start[:1]), dict(K=K.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises(AssertionError):
            lx.lx_score_attn_fwd(**{**good, **bad})
    with pytest.raises(ValueError):         # as unpacking a shape does
        lx.lx_score_attn_fwd(**{**good, "Q": Q[0]})
    assert not seen
    status[0] = lx.LX_ERR_WORKSPACE
    with pytest.raises(lx.LxError) as e:
        lx.lx_score_attn_fwd(**good)
    assert e.value.status == lx.LX_ERR_WORKSPACE


def test_clip_arguments(calls):
    lx, seen, _ = calls

    class Set:
        table, n, pieces, workspace = torch.zeros(40, dtype=torch.uint8), 3, 7, torch.zeros(256, dtype=torch.uint8)
    norm, other = torch.zeros(1), torch.zeros(512, dtype=torch.uint8)
    assert lx.lx_grad_norm_clip(Set, 0.5, norm) is norm
    lx.lx_grad_norm_clip(Set, 0.5, norm, workspace=other)
    assert seen[0][1] == [p(Set.table), 3, 7, 0.5, p(norm), p(Set.workspace), 256, STREAM]
    assert seen[1][1][5:7] == [p(other), 512]
    with pytest.raises(AssertionError):
        lx.lx_grad_norm_clip(Set, 0.5, norm.double())
    with pytest.raises(AssertionError):
        lx.lx_grad_norm_clip(Set, 0.5, torch.zeros(2))


# --- the definitions themselves ---------------------------------------------------------------

@pytest.mark.parametrize("cap,slopes", [(0.0, False), (1.5, False), (0.0, True), (0.8, True)])
def test_reference_gradients_against_differences(cap, slopes):
    """The formula's gradients and central differences of the definition: error of the latter h^2 (third derivative) + 2^-52 / h."""
    g = torch.Generator().manual_seed(5)
    Q, K, V = (torch.randn(1, h, s, 8, generator=g, dtype=torch.float64) for h, s in ((4, 5), (2, 7), (2, 7)))
    dO = torch.randn(1, 4, 5, 8, generator=g, dtype=torch.float64)
    lo = torch.tensor([[0, 1, 2, 3, 3]])
    hi = torch.tensor([[4, 7, 2, 6, 4]])
    kw = dict(cap=cap, slopes=torch.rand(4, generator=g) if slopes else None, key_lo=lo, key_hi=hi)
    grads_ = ref.attention(Q, K, V, dO, 0.4, False, **kw)[2:]
    h = 1e-5
    for t, got in zip((Q, K, V), grads_):
        for _ in range(12):
            at = tuple(int(torch.randint(n, (1,), generator=g)) for n in t.shape)
            v, f = t[at].item(), []
            for x in (v + h, v - h):
                t[at] = x
                f.append((ref.attention(Q, K, V, dO, 0.4, False, **kw)[0] * dO).sum().item())
            t[at] = v
            assert abs((f[0] - f[1]) / (2 * h) - got[at].item()) < 1e-7


def test_reference_rotation_turns_back():
    g = torch.Generator().manual_seed(6)
    x, pos = torch.randn(2, 3, 5, 16, generator=g, dtype=torch.float64), torch.randint(0, 9, (2, 5), generator=g)
    f = torch.tensor(ref.rope_frequencies(12, 1e4, 0, 1.0, 0.0, 1.0, 32.0), dtype=torch.float64)
    a = torch.arange(9, dtype=torch.float64)[:, None] * f
    table = torch.cat([a.cos(), a.sin()], 1)
    for inter in (False, True):
        y = ref.rope(x, table, pos, inter, False)
        assert (ref.rope(y, table, pos, inter, True) - x).abs().max() < 1e-14 and torch.equal(y[..., 12:], x[..., 12:])
        # scores of turned rows depend on the distance of their positions alone
        q, k = torch.randn(1, 1, 1, 16, generator=g, dtype=torch.float64), torch.randn(1, 1, 1, 16, generator=g, dtype=torch.float64)

        def score(i, j):
            r = [ref.rope(t, table, torch.tensor([[n]]), inter, False) for t, n in ((q, i), (k, j))]
            return float((r[0] * r[1]).sum())
        assert abs(score(7, 4) - score(3, 0)) < 1e-13
