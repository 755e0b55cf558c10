"""Norm, rotation and append of new tokens' heads against float64.

A value passes, in fp32: the head's mean square (at most 20 additions deep), its root and reciprocal, two products for
the norm, and two products and a sum for the rotation: together fewer than 32 roundings of 2^-24, so at most 2^-19 of
the rotated pair's magnitude.  Then one rounding to bf16: 2^-8 of the value.  Value heads only move, bit for bit.
"""
import ctypes

import pytest
import torch

import paper_2609_39334_amd as tkv


def _close(got, ref, scale):
    bound = 2.0 ** -8 * ref.abs() + 1.01 * 2.0 ** -19 * scale + 2.0 ** -130
    assert torch.all((got.double() - ref).abs() <= bound), ((got.double() - ref).abs() / bound).max()


def _inputs(n, hq, hkv, d, rot, seed=0, extra=0, nb=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    nb = nb or n // 16 + 3
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    ang = torch.rand((n, rot // 2), generator=g, device="cuda") * 1000
    wide = rand(n, (hq + 2 * hkv) * d + extra).bfloat16()
    return dict(qkv=wide[:, extra // 2:extra // 2 + (hq + 2 * hkv) * d], q_weight=rand(d), k_weight=rand(d), eps=1e-6,
                cos=torch.cos(ang), sin=torch.sin(ang), hq=hq,
                dst=torch.randperm(nb * 16, generator=g, device="cuda")[:n].to(torch.int32),
                k=rand(nb, hkv, 16, d).bfloat16(), v=rand(nb, hkv, 16, d).bfloat16())


def _ref(a):
    """(rotated heads, their pairs' magnitude, value heads), float64."""
    hkv, d = a["k"].shape[1], a["k"].shape[3]
    n, hq, half = a["qkv"].shape[0], a["hq"], a["cos"].shape[1]
    x = a["qkv"].reshape(n, hq + 2 * hkv, d).double()
    w = torch.cat((a["q_weight"].double().expand(hq, d), a["k_weight"].double().expand(hkv, d)))
    y = x[:, :hq + hkv] / torch.sqrt((x[:, :hq + hkv] ** 2).mean(-1, keepdim=True) + a["eps"]) * w
    c, s = a["cos"].double()[:, None], a["sin"].double()[:, None]
    p, q, rest = y[..., :half], y[..., half:2 * half], y[..., 2 * half:]
    return (torch.cat((p * c - q * s, q * c + p * s, rest), -1), torch.cat((p.abs() + q.abs(),) * 2 + (rest.abs(),), -1),
            a["qkv"].reshape(n, hq + 2 * hkv, d)[:, hq + hkv:])


def _check(a, q, k0, v0):
    k, v, hq = a["k"], a["v"], a["hq"]
    nb = k.shape[0]
    ref, scale, vals = _ref(a)
    _close(q, ref[:, :hq], scale[:, :hq])
    keep = torch.ones((nb, 16), dtype=torch.bool, device=k.device)
    ok = ((a["dst"] >= 0) & (a["dst"] < nb * 16)).nonzero()[:, 0]
    at = a["dst"][ok].long()
    _close(k[at // 16, :, at % 16], ref[ok, hq:], scale[ok, hq:])
    assert torch.equal(v[at // 16, :, at % 16], vals[ok])
    keep[at // 16, at % 16] = False
    keep = keep[:, None, :, None].expand_as(k)
    assert torch.equal(k[keep], k0[keep]) and torch.equal(v[keep], v0[keep])


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (28, 4, 128), (1, 1, 128), (15, 5, 64), (16, 1, 64), (40, 8, 128)])
@pytest.mark.parametrize("n,rot", [(1, 64), (5, 64), (33, 16), (257, 32), (1030, 64), (3, 0), (7, 48)])
def test_norm_rope_append(n, hq, hkv, d, rot):
    a = _inputs(n, hq, hkv, d, rot if d == 64 else 2 * rot, seed=n * hq)
    if n > 4:
        a["dst"][1], a["dst"][2], a["dst"][3] = -1, a["k"].shape[0] * 16, -7
    k0, v0 = a["k"].clone(), a["v"].clone()
    _check(a, tkv.tkv_norm_rope_append(**a), k0, v0)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [4, 700])
def test_rows_of_a_wider_product(n):
    a = _inputs(n, 12, 2, 128, 128, extra=48)
    assert a["qkv"].stride(0) > a["qkv"].shape[1]
    k0, v0 = a["k"].clone(), a["v"].clone()
    got = tkv.tkv_norm_rope_append(**a)
    _check(a, got, k0, v0)
    dense = dict(a, qkv=a["qkv"].contiguous(), k=k0, v=v0)
    assert torch.equal(got, tkv.tkv_norm_rope_append(**dense)) and torch.equal(a["k"], dense["k"])


@pytest.mark.gpu
def test_zero_heads_and_extreme_values():
    # a head of zeros stays zero, the smallest and largest bf16 magnitudes that fp32 squares hold keep their precision
    a = _inputs(3, 2, 1, 64, 64)
    a["qkv"][0].zero_()
    a["qkv"][1] *= 2.0 ** -60
    a["qkv"][2] *= 2.0 ** 55
    a["eps"] = 0.0
    k0, v0 = a["k"].clone(), a["v"].clone()
    b = dict(a, eps=1e-30)
    q = tkv.tkv_norm_rope_append(**b)
    assert torch.all(q[0] == 0)
    _check(b, q, k0, v0)
    q = tkv.tkv_norm_rope_append(**a)          # 0 / 0 as the tensor operations give it
    assert torch.all(q[0].isnan())


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_heads():
    inf, nan = float("inf"), float("nan")
    a = _inputs(4, 2, 1, 64, 32)
    for r, bad in enumerate((inf, -inf, nan)):
        a["qkv"][r, 3] = a["qkv"][r, 2 * 64 + 40] = a["qkv"][r, 3 * 64 + 1] = bad
    q = tkv.tkv_norm_rope_append(**a)
    ref, scale, vals = _ref(a)
    at = a["dst"].long()
    got = torch.cat((q, a["k"][at // 16, :, at % 16]), 1)
    assert torch.equal(got.isnan(), ref.isnan())
    ok = ref.isfinite()
    _close(got[ok], ref[ok], scale[ok])
    assert torch.equal(a["v"][at // 16, :, at % 16].nan_to_num(7), vals.nan_to_num(7))


@pytest.mark.gpu
def test_no_tokens():
    a = _inputs(0, 4, 2, 64, 64, nb=2)
    k0 = a["k"].clone()
    assert tkv.tkv_norm_rope_append(**a).shape == (0, 4, 64) and torch.equal(a["k"], k0)


@pytest.mark.gpu
def test_other_streams_and_replays():
    # the same values on another stream, given as a torch stream or a raw handle, and in a replayed graph
    a = _inputs(300, 12, 2, 128, 128)
    k0, v0 = a["k"].clone(), a["v"].clone()
    want = tkv.tkv_norm_rope_append(**a)
    kw, vw = a["k"].clone(), a["v"].clone()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, 0):
        a["k"].copy_(k0), a["v"].copy_(v0)
        torch.cuda.synchronize()
        got = tkv.tkv_norm_rope_append(**a, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(a["k"], kw) and torch.equal(a["v"], vw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = tkv.tkv_norm_rope_append(**a)
    for seed in range(3):
        b = _inputs(300, 12, 2, 128, 128, seed=seed)
        for name in ("qkv", "cos", "sin", "dst", "k", "v", "q_weight", "k_weight"):
            a[name].copy_(b[name])
        graph.replay()
        want = tkv.tkv_norm_rope_append(**b)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(a["k"], b["k"]) and torch.equal(a["v"], b["v"])


@pytest.mark.gpu
def test_inputs_dropped_after_a_call_on_another_stream():
    # their memory is not handed out again while that stream may still read it
    a, side = _inputs(700, 12, 2, 128, 128), torch.cuda.Stream()
    for name in ("qkv", "cos", "dst", "q_weight", "v"):
        args = dict(a, **{name: a[name].clone()})
        torch.cuda.synchronize()
        at = args[name].data_ptr()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        tkv.tkv_norm_rope_append(**args, stream=side)
        del args
        new = torch.empty_like(a[name])
        busy = not side.query()
        torch.cuda.synchronize()
        assert busy and new.data_ptr() != at, name


@pytest.mark.gpu
@pytest.mark.parametrize("rot,extra", [(128, 0), (32, 48)])
def test_calls_of_more_than_256_mib(rot, extra):
    # heads of 128 are then read and written past the caches
    n, hq, hkv, d = 9500, 40, 8, 128
    assert n * (hq + 2 * hkv) * d * 4 >= 256 << 20
    a = _inputs(n, hq, hkv, d, rot, seed=rot, extra=extra)
    a["dst"][::5], a["dst"][7] = -1, a["k"].shape[0] * 16
    k0, v0 = a["k"].clone(), a["v"].clone()
    _check(a, tkv.tkv_norm_rope_append(**a), k0, v0)


@pytest.mark.gpu
def test_tensors_are_checked():
    a = _inputs(4, 4, 2, 64, 64)
    for name, bad in (("qkv", a["qkv"].float()), ("qkv", a["qkv"].t()), ("qkv", a["qkv"][:, :-64]), ("qkv", a["qkv"][:1].expand(4, -1)),
                      ("q_weight", a["q_weight"].bfloat16()), ("k_weight", a["k_weight"][:32]), ("cos", a["cos"][:, ::2]),
                      ("sin", a["sin"][:3]), ("dst", a["dst"].long()), ("dst", a["dst"].cpu()), ("k", a["k"][0]),
                      ("v", a["v"][:1]), ("cos", a["cos"][0])):
        with pytest.raises(ValueError):
            tkv.tkv_norm_rope_append(**dict(a, **{name: bad}))
    narrow = dict(a, cos=a["cos"][:, :12].contiguous(), sin=a["sin"][:, :12].contiguous())
    with pytest.raises(tkv.TkvError, match="multiple of 16"):
        tkv.tkv_norm_rope_append(**narrow)
    shifted = torch.zeros(4 * 512 + 8, dtype=torch.bfloat16, device="cuda")[4:4 + 4 * 512].view(4, 512)
    with pytest.raises(tkv.TkvError, match="aligned"):
        tkv.tkv_norm_rope_append(**dict(a, qkv=shifted))


def test_bad_arguments_are_refused():
    # refused before any device access (no GPU needed)
    L, one = tkv.lib(), 16

    def call(sh=(8, 2, 64, 16, 4), n=1, stride=768, rot=64, q=one, cos=one, qkv=one):
        return L.tkv_norm_rope_append(ctypes.byref(tkv.tkv_shape(*sh)), n, qkv, stride, one, one, 1e-6, cos, one, rot, one, q,
                                      one, one, None)

    for sh in ((8, 2, 96, 16, 4), (8, 2, 64, 32, 4), (0, 2, 64, 16, 4), (8, 0, 64, 16, 4), (8, 2, 64, 16, 1 << 28),
               (8, 2, 64, 16, 0)):
        assert call(sh) == tkv.TKV_EINVAL, sh
    for rot in (-16, 8, 24, 80, 128):
        assert call(rot=rot) == tkv.TKV_EINVAL, rot
    for stride in (767, 764, 772, 0, -768):
        assert call(stride=stride) == tkv.TKV_EINVAL, stride
    assert call(n=-1) == tkv.TKV_EINVAL and call(q=None) == tkv.TKV_EINVAL and call(cos=None) == tkv.TKV_EINVAL
    assert call(q=one + 8) == tkv.TKV_EINVAL and "aligned" in tkv.tkv_last_error()
    assert call(qkv=one + 2) == tkv.TKV_EINVAL and "aligned" in tkv.tkv_last_error()
    assert call(n=0) == tkv.TKV_OK and call(n=0, qkv=None) == tkv.TKV_OK
    assert L.tkv_norm_rope_append(None, 0, one, 768, one, one, 1e-6, one, one, 64, one, one, one, one, None) == tkv.TKV_EINVAL
