"""The softmax attention's checks of its arguments (no GPU needed), its buckets, and the 64-bit reference the GPU tests
use, against differences."""
import ctypes
import math

import pytest
import torch

from paper_2509_24006_amd import binding as sla
from tests import attention_reference as ref


def _params(**kw):
    base = dict(B=2, H=4, Hkv=2, Nq=10, Nk=20, Np=0, d=64, dtype=1, causal=0, q_pos=0, q_from_end=0, table_dtype=0, scale=0.1)
    base.update(kw)
    return sla.sla_attn_params(*[base[n] for n, _ in sla.sla_attn_params._fields_[:-1]])


def _sizes(p):
    a, b = ctypes.c_uint64(), ctypes.c_uint64()
    return sla.lib().sla_attn_sizes(ctypes.byref(p), ctypes.byref(a), ctypes.byref(b))


def test_struct_layout_matches_header():
    assert ctypes.sizeof(sla.sla_buckets) == 65 * 4
    assert ctypes.sizeof(sla.sla_attn_params) == 13 * 4 + 65 * 4
    assert ctypes.sizeof(sla.sla_tensor) == 32


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(B=0), -1), (dict(H=0), -1), (dict(Hkv=0), -1), (dict(Hkv=3), -1), (dict(Nq=0), -1), (dict(Nk=-1), -1),
    (dict(Nk=0), 0), (dict(Np=-1), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1),
    (dict(scale=math.inf), -1), (dict(d=96), -2), (dict(d=256), -2), (dict(dtype=2), -2), (dict(table_dtype=5), -2),
    (dict(B=40000), -2), (dict(Nq=1 << 29), -2), (dict(Nk=1 << 29), -2), (dict(q_pos=1 << 29), -2), (dict(q_pos=-(1 << 29)), -2),
    (dict(B=60000, H=1, Hkv=1, Nq=1 << 20), -2)])
def test_params(kw, code):
    assert _sizes(_params(**kw)) == code


@pytest.mark.parametrize("n,two,borders,code", [
    (0, 0, [], 0), (1, 0, [], 0), (2, 1, [], 0), (3, 1, [1], -1), (-1, 0, [], -1), (65, 0, [1] * 63, -1), (64, 0, list(range(1, 64)), 0),
    (128, 1, list(range(1, 64)), 0), (3, 0, [0, 4], -1), (3, 0, [5, 4], -1), (3, 0, [4, 4], 0), (3, 0, [1, 1025], -1),
    (3, 0, [1, 1024], 0)])
def test_buckets_of_the_c_call(n, two, borders, code):
    p = _params()
    p.buckets.n_buckets, p.buckets.two_sided = n, two
    for i, b in enumerate(borders):
        p.buckets.borders[i] = b
    assert _sizes(p) == code


def _call(p, fwd=True, **kw):
    """the C call with made-up addresses: refused before anything is read"""
    t = lambda sb=64 * 2048, sh=64 * 256, sn=64, data=4096: sla.sla_tensor(data, sb, sh, sn)
    a = dict(Q=t(), K=t(), V=t(), Kp=None, Vp=None, O=t(), dO=t(), L=4096, table=None, q_len=None, k_len=None, dQ=t(), dK=t(),
             dV=t(), dtable=None, ws=4096, bytes=0)
    for k, v in kw.items():
        a[k] = t(**v) if isinstance(v, dict) else v
    r = lambda k: None if a[k] is None else ctypes.byref(a[k])
    if fwd:
        return sla.lib().sla_attn_forward(ctypes.byref(p), r("Q"), r("K"), r("V"), r("Kp"), r("Vp"), a["table"], a["q_len"],
                                          a["k_len"], r("O"), a["L"], a["ws"], a["bytes"], None)
    return sla.lib().sla_attn_backward(ctypes.byref(p), r("Q"), r("K"), r("V"), r("O"), r("dO"), a["L"], a["table"], a["q_len"],
                                       a["k_len"], r("dQ"), r("dK"), r("dV"), a["dtable"], a["ws"], a["bytes"], None)


BIG = 1 << 40


@pytest.mark.parametrize("kw,code", [
    (dict(Q=None), -1), (dict(O=None), -1), (dict(Q=dict(data=None)), -1), (dict(K=dict(data=4104)), -1), (dict(V=dict(sn=60)), -1),
    (dict(V=dict(sn=68)), -1), (dict(Q=dict(sh=4)), -1), (dict(Q=dict(sb=-64)), -1), (dict(O=dict(sn=0)), -1),
    (dict(K=dict(sn=1 << 24)), -2), (dict(table=4096), -1), (dict(q_len=4098), -1), (dict(k_len=4097), -1), (dict(L=4098), -1)])
def test_forward_refuses(kw, code):
    assert _call(_params(), bytes=BIG, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dO=None), -1), (dict(L=None), -1), (dict(dQ=None), -1), (dict(dK=dict(data=8)), -1), (dict(dV=dict(sn=32)), -1),
    (dict(dtable=4096), -1), (dict(ws=None), -1), (dict(ws=4100), -1), (dict(bytes=16), -3), (dict(k_len=4097), -1)])
def test_backward_refuses(kw, code):
    assert _call(_params(), fwd=False, **{"bytes": BIG, **kw}) == code


def test_bias_and_prefix_refusals():
    p = _params(Np=5)
    assert _call(p, bytes=BIG) == -1                                                  # no prefix given
    assert _call(p, bytes=BIG, Kp=dict(), Vp=dict(sn=8)) == -1
    assert _call(p, fwd=False, bytes=BIG) == -2                                       # no backward pass behind a prefix
    p = _params()
    p.buckets.n_buckets = 1
    assert _call(p, bytes=BIG) == -1                                                  # no table
    assert _call(p, bytes=BIG, table=4097) == -1
    long = _params(B=1, H=1, Hkv=1, Nk=1 << 20)
    far = dict(sn=1 << 12)
    assert _call(long, fwd=False, bytes=BIG, K=far) == -2                             # a head of 2^33 bytes


def test_offsets_past_32_bits_are_refused():
    far = dict(sn=1 << 12)                                                            # rows 8 KB apart
    assert _call(_params(B=1, H=8, Hkv=8, Nq=1 << 15, Nk=1 << 19), bytes=BIG, K=far) == -2   # a head of 4 GB through one workgroup
    assert _call(_params(B=1 << 12, H=1, Hkv=1, Nq=1, Nk=1, Np=5), bytes=BIG, Kp=dict(), Vp=dict(), Q=dict(sb=1 << 19)) == -2
    assert _call(_params(B=1 << 10, H=32, Hkv=1, Nq=1 << 17, Nk=1, Np=5), bytes=BIG, Kp=dict(), Vp=dict(), Q=dict(sb=0, sh=0), O=dict(sb=0, sh=0)) == -2


def test_binding_refuses_wrong_tensors():
    from paper_2509_24006_amd import autograd as attn
    q = torch.zeros(1, 2, 3, 64)
    with pytest.raises(sla.SLAError, match="device"):
        attn.dense_attention(q, q, q)
    with pytest.raises(sla.SLAError, match="float32 or bfloat16"):
        attn.dense_attention(q.half(), q.half(), q.half())
    with pytest.raises(sla.SLAError, match="four dimensions"):
        attn.dense_attention(q[0], q[0], q[0])
    with pytest.raises(sla.SLAError, match="table"):
        attn.dense_attention(q, q, q, table=torch.zeros(4, 2))
    with pytest.raises(sla.SLAError):
        attn.dense_attention(q, q[..., :32], q)
    with pytest.raises(sla.SLAError):
        attn.cached_attention(q, q, q, prefix=(q[0], q[0]))


@pytest.mark.parametrize("args", [(1, 10, False), (3, 10, True), (2, 10, True), (65, 100, False), (130, 200, True), (32, 8, True),
                                  (32, 1025, True)])
def test_position_buckets_refuses(args):
    with pytest.raises(sla.SLAError):
        sla.position_buckets(*args)


@pytest.mark.parametrize("n,far,two", [(32, 128, True), (32, 128, False), (16, 64, False), (4, 3, True), (64, 1024, False), (128, 1024, True)])
def test_position_buckets_follow_their_definition(n, far, two):
    b = sla.position_buckets(n, far, two)
    side = n // 2 if two else n
    e, m = side // 2, side - side // 2
    borders = list(b.borders)[:side - 1]
    for dist in range(far + 50):
        k = 0
        while dist >= e and k < m - 1 and dist ** m * e ** (k + 1) >= far ** (k + 1) * e ** m:
            k += 1
        assert sum(x <= dist for x in borders) == (dist if dist < e else e + k), dist


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    Q, K, V, dO, table = r(2, 4, 5, 3), r(2, 2, 7, 3), r(2, 2, 7, 3), r(2, 4, 5, 3), r(6, 4)
    kw = dict(causal=True, q_len=[5, 3], k_len=[6, 0], pos=[1, 2], borders=(1, 3), two_sided=True, result=torch.float32)
    f = lambda Q, K, V, T: float((ref.attention(Q, K, V, 0.7, table=T, **kw)["O"][0] * dO).sum())
    ref.U[torch.float64] = 2.0 ** -53
    want = ref.attention(Q, K, V, 0.7, table=table, dO=dO, **kw)
    at = [Q, K, V, table]
    for i, name in enumerate(("dQ", "dK", "dV", "dtable")):
        for _ in range(12):
            step = r(*at[i].shape)
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + 1e-5 * step, at[i] - 1e-5 * step
            diff = (f(*up) - f(*down)) / 2e-5
            assert abs(diff - float((want[name][0] * step).sum())) < 1e-7 * (1 + abs(diff)), name
    assert float(want["O"][0][0, :, :].abs().max()) > 0 and float(want["O"][0][1].abs().max()) == 0


@pytest.mark.parametrize("scale,code", [(1e-20, 0), (1e20, 0), (9e-21, -2), (1e-38, -2), (1.1e20, -2), (3e38, -2)])
def test_scales_beyond_what_the_backward_pass_can_divide_by(scale, code):
    assert _sizes(_params(scale=scale)) == code


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape,token", [((2, 3, 5, 64), False), ((2, 5, 3, 64), True), ((3, 5, 64), False)])
def test_laid_out_moves_what_begins_at_an_odd_address(dt, shape, token):
    from paper_2509_24006_amd import autograd as attn
    n = math.prod(shape)
    room = torch.arange(n + 16, dtype=torch.float32).to(dt)
    room = room[(-room.data_ptr() // room.element_size()) % (16 // room.element_size()):]   # at a multiple of 16 bytes
    fits, odd = room[:n].view(shape), room[1:n + 1].view(shape)
    assert attn._laid_out(fits, token) is fits
    leaf = odd.detach().requires_grad_(True)
    got = attn._laid_out(leaf, token)
    assert got.data_ptr() % 16 == 0 and got.is_contiguous() and torch.equal(got, odd)
    assert torch.equal(torch.autograd.grad(got, leaf, fits)[0], fits)


def test_forward_mode_is_refused():
    import torch.autograd.forward_ad as fwd
    from paper_2509_24006_amd import autograd as attn
    q, p, t, bk = torch.zeros(1, 2, 3, 64), torch.zeros(2, 3, 64), torch.zeros(8, 2), sla.position_buckets(8, 20)
    with fwd.dual_level():
        for i in range(4):
            a = [q, q, q, t]
            a[i] = fwd.make_dual(a[i].clone(), torch.ones_like(a[i]))
            with pytest.raises(sla.SLAError, match="forward-mode"):
                attn.dense_attention(*a[:3], table=a[3], buckets=bk)
            with pytest.raises(sla.SLAError, match="forward-mode"):
                attn.cached_attention(*a[:3], table=a[3], buckets=bk)
        d = fwd.make_dual(p, torch.ones_like(p))
        for prefix in ((d, p), (p, d)):
            with pytest.raises(sla.SLAError, match="forward-mode"):
                attn.cached_attention(q, q, q, prefix=prefix)


def test_a_traced_call_is_refused():
    from paper_2509_24006_amd import autograd as attn
    q = torch.zeros(1, 2, 3, 64)
    for f in (attn.dense_attention, attn.cached_attention):
        with pytest.raises(sla.SLAError, match="traced"):
            torch.jit.trace(lambda x: f(x, x, x), (q,), check_trace=False)
