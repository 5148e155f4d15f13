"""Front end of the exact layers (kvm_qk_norm_rope), its way into the 8-bit cache (kvm_cache_ingest) and the way back (kvm_cache_read) against the fp64
definitions in oracle/front.py and oracle/exact_cache.py."""
import ctypes as C
import math
import random

import numpy as np
import pytest
import torch

from oracle import exact_cache as ec
from oracle import front as fo
from tests.test_cache import BAD_CACHE, BAD_CALL, Model, _call, _desc, garbage_cache, rows


@pytest.fixture(scope="module")
def kvm():
    from paper_2605_09877_b200 import build
    build.build()
    from paper_2605_09877_b200 import kvm as mod
    return mod


# ---- pins of the definition, and of the frequencies ------------------------------------------------------------------

def test_definition_in_closed_form():
    x = np.array([[3.0, 4.0, 1.0, -1.0]])
    y, _ = fo.front(x, [0], norm="rms", eps=0.0, rope_dims=4)
    assert np.allclose(y, x / math.sqrt(27 / 4))                                      # position 0 rotates nothing
    y, _ = fo.front(x, [0], norm="layer", eps=0.0)
    assert abs(y.mean()) < 1e-15 and np.allclose((y ** 2).mean(), 1)
    f = fo.frequencies(4)
    assert np.allclose(np.asarray(f, float), [1.0, 0.01])
    y, _ = fo.front(x, [1], norm="none", rope_dims=4, layout="half")
    assert np.allclose(y[0, 0] + 1j * y[0, 2], (3 + 1j) * np.exp(1j)) and np.allclose(y[0, 1] + 1j * y[0, 3], (4 - 1j) * np.exp(0.01j))
    y, _ = fo.front(x, [1], norm="none", rope_dims=2, layout="interleaved", magnitude=2.0)
    assert np.allclose(y[0, 0] + 1j * y[0, 1], 2 * (3 + 4j) * np.exp(1j)) and np.allclose(y[0, 2:], x[0, 2:])
    # products of a query and a key depend on the distance alone
    q, k = np.random.default_rng(0).standard_normal((2, 1, 64))
    dots = [float((fo.front(q, [a], norm="none", rope_dims=24)[0] @ fo.front(k, [b], norm="none", rope_dims=24)[0].T).item()) for a, b in ((5, 2), (1005, 1002))]
    assert abs(dots[0] - dots[1]) < 1e-12


ROPES = [dict(), dict(base=500000.0), dict(scaling="linear", factor=7.5), dict(scaling="parts", factor=16.0, original_len=8192),
         dict(scaling="parts", factor=8.0, original_len=2048, low=1.0, high=4.0, base=500000.0)]


@pytest.mark.parametrize("r", [0, 2, 24, 32, 126, 128])
@pytest.mark.parametrize("rope", ROPES)
def test_frequencies(kvm, r, rope):
    got = kvm.Front(norm="none", rope_dims=r, **rope).frequencies(128)
    want = np.asarray(fo.frequencies(r, **rope), np.float64)
    assert len(got) == r // 2 and np.allclose(got, want, rtol=2.0 ** -49, atol=0)


def test_frequencies_of_ones_own(kvm):
    own = (C.c_double * 16)(*[0.5 ** i for i in range(16)])
    out = (C.c_double * 16)()
    assert kvm.lib.kvm_rope_frequencies(C.byref(_front(kvm, frequencies=C.cast(own, C.POINTER(C.c_double)))), 128, out) == 0 and list(out) == list(own)
    for bad in (math.nan, -0.1, 1.5, math.inf):
        own[15] = bad
        assert kvm.lib.kvm_rope_frequencies(C.byref(_front(kvm, frequencies=C.cast(own, C.POINTER(C.c_double)))), 128, out) == 1
    own[15] = 7.0                                      # (behind the pairs that there are: not looked at)
    assert kvm.lib.kvm_rope_frequencies(C.byref(_front(kvm, rope_dims=30, frequencies=C.cast(own, C.POINTER(C.c_double)))), 128, out) == 0


def test_frequencies_by_parts_keep_the_fast_pairs_and_interpolate_the_slow_ones(kvm):
    plain = kvm.Front(norm="none", rope_dims=128).frequencies(128)
    parts = kvm.Front(norm="none", rope_dims=128, scaling="parts", factor=16.0, original_len=8192).frequencies(128)
    turns = [8192 * f / (2 * math.pi) for f in plain]
    for f, g, n in zip(plain, parts, turns):
        assert abs(g - f) < 1e-15 if n > 32 else abs(g - f / 16) < 1e-15 if n < 1 else f / 16 < g < f


# ---- refusals: before anything is launched ---------------------------------------------------------------------------

def _front(kvm, **kw):
    c = dict(norm=1, layout=0, scaling=0, rope_dims=32, base=1e4, factor=1.0, low=1.0, high=32.0, magnitude=1.0, original_len=0, eps=1e-5, frequencies=None,
             q_weight=None, q_bias=None, k_weight=None, k_bias=None)
    c.update(kw)
    return kvm.FrontDesc(*[c[f[0]] for f in kvm.FrontDesc._fields_])


BAD_FRONT = [dict(norm=-1), dict(norm=3), dict(layout=2), dict(layout=-1), dict(scaling=3), dict(scaling=-1), dict(rope_dims=-2), dict(rope_dims=31), dict(rope_dims=130),
             dict(base=0.5), dict(base=math.nan), dict(base=math.inf), dict(magnitude=0.0), dict(magnitude=-1.0), dict(magnitude=math.nan), dict(eps=-1e-5), dict(eps=math.nan),
             dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan), dict(scaling=2, factor=4.0), dict(scaling=2, factor=4.0, original_len=-1),
             dict(scaling=2, factor=4.0, original_len=64, low=4.0, high=4.0), dict(scaling=2, factor=4.0, original_len=64, low=-1.0),
             dict(scaling=2, factor=4.0, original_len=64, high=math.nan), dict(scaling=2, factor=0.0, original_len=64), dict(norm=0, q_weight=1 << 20),
             dict(norm=0, k_bias=1 << 20), dict(q_weight=(1 << 20) + 2), dict(k_bias=(1 << 20) + 1)]


@pytest.mark.parametrize("bad", BAD_FRONT)
def test_refusals_of_the_front(kvm, bad):
    f, d, c, x = C.byref(_front(kvm, **bad)), C.byref(_desc(kvm)), C.byref(_call(kvm)), 1 << 26
    assert kvm.lib.kvm_qk_norm_rope(f, x, 2 * x, None, None, 1, 4, 2, 3, 128, 3 * x, 4 * x, None, None, None, None, None, None) == 1
    assert kvm.lib.kvm_cache_ingest(d, c, f, x, 4, 2 * x, 3 * x, 4 * x, None, None, None, None, None, None) == 1
    assert kvm.lib.kvm_rope_frequencies(f, 128, (C.c_double * 64)()) == 1
    # without rotation what describes it is not looked at
    if set(bad) & {"base", "magnitude", "factor", "original_len", "low", "high"} and "scaling" not in bad:
        assert kvm.lib.kvm_rope_frequencies(C.byref(_front(kvm, **{**bad, "rope_dims": 0})), 128, None) == 0


def test_refusals_of_the_other_arguments(kvm):
    f, x = C.byref(_front(kvm)), 1 << 26
    st = lambda *a: (C.c_int64 * 3)(*a)  # noqa: E731
    ok = dict(f=f, q=x, k=2 * x, start=None, count=None, B=2, Hq=4, Hk=2, T=3, d=128, qo=3 * x, ko=4 * x, qs=None, ks=None, qos=None, kos=None, status=None)
    for kw, code in ((dict(f=None), 1), (dict(q=None, k=None), 1), (dict(qo=None), 1), (dict(ko=None), 1), (dict(q=x + 1), 1), (dict(ko=4 * x + 1), 1), (dict(B=0), 1), (dict(T=0), 1),
                     (dict(Hq=0), 1), (dict(Hk=-1), 1), (dict(d=96), 2), (dict(d=256), 2), (dict(B=65536), 2), (dict(T=(1 << 30) + 1), 2), (dict(Hq=16385), 2),
                     (dict(start=x + 2), 1), (dict(count=x + 1), 1), (dict(status=x + 3), 1), (dict(qs=st(1, -1, 1)), 1), (dict(qos=st(1536, 384, 64)), 1),
                     (dict(kos=st(768, 0, 128)), 1), (dict(qo=x, qs=st(1536, 128, 512), qos=st(1536, 384, 128)), 1)):
        a = dict(ok, **kw)
        assert kvm.lib.kvm_qk_norm_rope(*[a[n] for n in ("f", "q", "k", "start", "count", "B", "Hq", "Hk", "T", "d", "qo", "ko", "qs", "ks", "qos", "kos", "status")], None) == code, kw
    d, c = C.byref(_desc(kvm)), C.byref(_call(kvm))
    ok = dict(c=c, f=f, q=x, hq=4, k=2 * x, v=3 * x, qo=4 * x, qs=None, ks=None, vs=None, qos=None, status=None)
    for kw, code in ((dict(f=None), 1), (dict(c=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(qo=None), 1), (dict(hq=0), 1), (dict(hq=16385), 2), (dict(q=x + 1), 1),
                     (dict(k=x + 1), 1), (dict(v=x + 1), 1), (dict(qs=st(-1, 1, 1)), 1), (dict(ks=st(1, 1, -1)), 1), (dict(vs=st(1, -1, 1)), 1), (dict(qos=st(2048, 512, 64)), 1),
                     (dict(status=x + 2), 1)):
        a = dict(ok, **kw)
        assert kvm.lib.kvm_cache_ingest(d, *[a[n] for n in ("c", "f", "q", "hq", "k", "v", "qo", "qs", "ks", "vs", "qos", "status")], None) == code, kw
    for args in ((None, x, None, None, None), (x, None, None, None, None), (x + 1, x, None, None, None), (x, 2 * x, st(-1, 512, 128), None, None), (x, 2 * x, None, st(1024, 512, 64), None),
                 (x, 2 * x, None, None, x + 1)):
        assert kvm.lib.kvm_cache_read(d, c, *args, None) == 1
    assert kvm.lib.kvm_rope_frequencies(f, 96, (C.c_double * 64)()) == 2 and kvm.lib.kvm_rope_frequencies(f, 128, None) == 1


@pytest.mark.parametrize("cache,call,code", [(c, {}, e) for c, e in BAD_CACHE] + [({}, c, e) for c, e in BAD_CALL])
def test_refusals_of_the_cache_and_the_call(kvm, cache, call, code):
    d, c, f, x = C.byref(_desc(kvm, **cache)), C.byref(_call(kvm, **call)), C.byref(_front(kvm)), 1 << 26
    assert kvm.lib.kvm_cache_ingest(d, c, f, x, 4, 2 * x, 3 * x, 4 * x, None, None, None, None, None, None) == code
    assert kvm.lib.kvm_cache_read(d, c, x, 2 * x, None, None, None, None) == code


def test_binding_refuses_what_it_can_see(kvm):
    for kw in (dict(norm="batch"), dict(layout="quarter"), dict(scaling="log"), dict(q_weight=torch.ones(4, 64)), dict(rope_dims=1 << 32)):
        with pytest.raises(ValueError):
            kvm.Front(**kw)
    f = kvm.Front(norm="none")
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    for args in ((x, None), (None, None), (x.float(), x)):
        with pytest.raises(ValueError):
            kvm.qk_norm_rope(*args, f)                           # not on a GPU, nothing at all, other types


# ---- kernels ---------------------------------------------------------------------------------------------------------

HALF_BF16 = 2.0 ** -8


def params(H, d, norm, seed):
    g = torch.Generator().manual_seed(seed)
    if norm == "none":
        return None, None
    return 1.0 + 0.3 * torch.randn((H, d), generator=g), 0.2 * torch.randn((H, d), generator=g)


def reference(x, start, counts, weight, bias, kw):
    """(result, bound of fp32) [B, H, T, d]; rows behind the counts are NaN."""
    xn = x.float().cpu().double().numpy()
    B, H, T, d = xn.shape
    y, e = np.full(xn.shape, np.nan), np.full(xn.shape, np.nan)
    for b in range(B):
        n = counts[b]
        for h in range(H if n else 0):
            y[b, h, :n], e[b, h, :n] = fo.front(xn[b, h, :n], start[b] + np.arange(n), weight=None if weight is None else weight[h].numpy(),
                                                bias=None if bias is None else bias[h].numpy(), **kw)
    return y, e


def check_rows(out, y, e, counts):
    on = out.float().cpu().double().numpy()
    for b, n in enumerate(counts):
        assert (on[b, :, n:] == 7.0).all()                       # rows behind the count are left as they were
        off = np.abs(on[b, :, :n] - y[b, :, :n])
        bound = HALF_BF16 * np.abs(y[b, :, :n]) + 2 * e[b, :, :n] + 2.0 ** -133
        assert (off <= bound).all(), (b, float((off / bound).max()))


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


FRONTS = [
    (1, 4, 1, 128, 1, [131071], None, dict(norm="rms", layout="interleaved", rope_dims=128, scaling="parts", factor=16.0, original_len=8192, magnitude=1.2772588722239782)),
    (1, 1, 1, 64, 1, [0], None, dict(norm="layer", rope_dims=64)),
    (3, 5, 2, 128, 7, [0, 1000, 2 ** 30], [7, 0, 3], dict(norm="layer", rope_dims=32)),
    (2, 3, 1, 64, 300, [5, 70000], [300, 131], dict(norm="none", rope_dims=24, scaling="linear", factor=7.5)),
    (2, 9, 3, 128, 1000, [0, 12345], [1000, 999], dict(norm="layer", rope_dims=32)),
    (1, 8, 8, 128, 600, [100], None, dict(norm="rms", rope_dims=128, eps=1e-6)),
    (1, 20, 3, 64, 999, [2 ** 20], None, dict(norm="layer", rope_dims=64, layout="interleaved", base=500000.0)),
    (1, 20, 20, 64, 500, [0], None, dict(norm="rms", rope_dims=62, layout="half")),
    (1, 17, 16, 128, 600, [0], None, dict(norm="layer", rope_dims=2, layout="half")),
    (1, 17, 16, 128, 600, [3], None, dict(norm="none", rope_dims=126, layout="interleaved")),
    (300, 40, 2, 64, 2, list(range(300)), [1 + i % 2 for i in range(300)], dict(norm="rms", rope_dims=16)),
    (2, 2, 2, 128, 33, [9, 9], [33, 32], dict(norm="layer")),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hk,d,T,start,counts,kw", FRONTS)
def test_norm_rope_against_the_definition(kvm, B, Hq, Hk, d, T, start, counts, kw):
    q, k = rows((B, Hq, T, d), 1), rows((B, Hk, T, d), 2)
    k[..., d // 3] += 40.0                                       # (a mean far from zero)
    qp, kp = params(Hq, d, kw["norm"], 3), params(Hk, d, kw["norm"], 4)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    f = kvm.Front(q_weight=dev(qp[0]), q_bias=dev(qp[1]), k_weight=dev(kp[0]), k_bias=dev(kp[1]), **kw)
    qo, ko = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), torch.full(k.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    status = i32([0])
    got = kvm.qk_norm_rope(q.cuda(), k.cuda(), f, i32(start), None if counts is None else i32(counts), q_out=qo, k_out=ko, status=status)
    torch.cuda.synchronize()
    assert got[0] is qo and got[1] is ko and status.item() == 0
    n = counts or [T] * B
    check_rows(qo, *reference(q, start, n, *qp, kw), n)
    check_rows(ko, *reference(k, start, n, *kp, kw), n)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,kw", [(1, 128, dict(norm="layer", rope_dims=32)), (900, 128, dict(norm="rms", rope_dims=128)), (900, 64, dict(norm="none", rope_dims=20)),
                                    (700, 64, dict(norm="layer", rope_dims=64, layout="interleaved"))])
def test_norm_rope_takes_any_strides_places_and_streams(kvm, T, d, kw):
    """Rows out of one projection, rows that are not aligned, in place, q or k alone, another stream: all give the same bits."""
    B, Hq, Hk = 2, 9, 4
    x = rows((B, T, Hq + Hk, d), 5).cuda()
    qp, kp = params(Hq, d, kw["norm"], 3), params(Hk, d, kw["norm"], 4)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    f = kvm.Front(q_weight=dev(qp[0]), q_bias=dev(qp[1]), k_weight=dev(kp[0]), k_bias=dev(kp[1]), **kw)
    start = i32([3, 77])
    split = x.transpose(1, 2)
    q, k = split[:, :Hq], split[:, Hq:]
    want = kvm.qk_norm_rope(q.contiguous(), k.contiguous(), f, start)
    for got in (kvm.qk_norm_rope(q, k, f, start), (kvm.qk_norm_rope(q, None, f, start)[0], kvm.qk_norm_rope(None, k, f, start)[1])):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    odd = torch.empty(B * Hq * T * (d + 3) + 1, dtype=torch.bfloat16, device="cuda")[1:].view(B, Hq, T, d + 3)[..., :d]
    odd.copy_(q)
    out = torch.full((B, Hq, T, d + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    kvm.qk_norm_rope(odd, None, f, start, q_out=out[..., 1:d + 1])
    assert torch.equal(out[..., 1:d + 1], want[0]) and (out[..., 0] == 7.0).all() and (out[..., d + 1:] == 7.0).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = kvm.qk_norm_rope(q, k, f, start, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    again = kvm.qk_norm_rope(q, k, f, start, q_out=q, k_out=k)   # (x is changed)
    assert again[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    if T > 1:                                                    # as many calls as tokens give the same rows
        t = T // 2
        one = kvm.qk_norm_rope(odd[:, :, t:t + 1], None, f, start + t)[0]
        assert torch.equal(one, want[0][:, :, t:t + 1])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 900])
def test_norm_rope_reports_lengths_and_leaves_those_rows(kvm, T):
    q, k = rows((4, 8, T, 64), 1).cuda(), rows((4, 3, T, 64), 2).cuda()
    f = kvm.Front(norm="layer", rope_dims=32)
    good = kvm.qk_norm_rope(q, k, f, i32([5] * 4), i32([1] * 4))
    for start, count in (([5, -1, 5, 5], [1] * 4), ([5] * 4, [1, -1, 1, 1]), ([5] * 4, [1, T + 1, 1, 1]), ([5, -2 ** 31, 5, 5], [1] * 4)):
        qo, ko, status = torch.full_like(q, 7.0), torch.full_like(k, 7.0), i32([0])
        kvm.qk_norm_rope(q, k, f, i32(start), i32(count), q_out=qo, k_out=ko, status=status)
        assert status.item() == 1 and (qo[1] == 7.0).all() and (ko[1] == 7.0).all() and (qo[:, :, 1:] == 7.0).all()
        for b in (0, 2, 3):
            assert torch.equal(qo[b, :, 0], good[0][b, :, 0]) and torch.equal(ko[b, :, 0], good[1][b, :, 0])
        status.zero_()
        kvm.qk_norm_rope(None, k, f, i32(start), i32(count), k_out=ko, status=status)
        assert status.item() == 1


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T", [1, 600])
def test_an_infinity_reaches_its_pair_and_no_other_channel(kvm, layout, T):
    """Without a norm: the rotated partner only; beside the rotated channels nothing; with one: its row only."""
    x = rows((1, 30, T, 64), 1)
    x[0, 0, 0, 3] = math.inf                                     # rotated (r = 16)
    x[0, 1, 0, 17] = -math.inf                                   # not rotated
    x[0, 2, 0, 5] = math.nan
    f = kvm.Front(norm="none", rope_dims=16, layout=layout)
    out = kvm.qk_norm_rope(x.cuda(), None, f, i32([7]))[0].float().cpu()
    partner = 11 if layout == "half" else 2
    bad = ~torch.isfinite(out[0, 0, 0])
    assert bad[3] and set(bad.nonzero().flatten().tolist()) == {3, partner}
    assert out[0, 1, 0, 17] == -math.inf and torch.isfinite(out[0, 1, 0]).sum() == 63
    assert torch.isnan(out[0, 2, 0]).sum() == 2 and torch.isfinite(out[0, 3:]).all() and torch.isfinite(out[0, :, 1:]).all()
    out = kvm.qk_norm_rope(x.cuda(), None, kvm.Front(norm="rms", rope_dims=16, layout=layout), i32([7]))[0].float().cpu()
    assert torch.isfinite(out[0, 3:]).all() and torch.isfinite(out[0, :, 1:]).all() and not torch.isfinite(out[0, 0, 0]).all()


@pytest.mark.gpu
def test_norm_rope_of_rows_of_zeros_and_of_the_ends_of_the_range(kvm):
    x = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16)
    x[0, 1] = 2.0 ** 60
    x[0, 2] = 2.0 ** -60
    x[0, 3, :, ::2] = 2.0 ** 60
    for norm in ("layer", "rms"):
        kw = dict(norm=norm, rope_dims=32)
        out = torch.full(x.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        kvm.qk_norm_rope(x.cuda(), None, kvm.Front(**kw), i32([9]), q_out=out)
        check_rows(out, *reference(x, [9], [2], None, None, kw), [2])


# ---- into the cache --------------------------------------------------------------------------------------------------

CALLS = [(1, 1, 64, 16, [[1]] * 20), (2, 3, 128, 64, [[70, 1], [1, 0], [58, 64], [1, 1], [0, 300]]), (3, 2, 64, 128, [[129, 5, 0], [1, 127, 128], [255, 1, 1]]),
         (2, 2, 128, 32, [[31, 33], [1, 1], [1, 1], [100, 95]]), (1, 5, 128, 128, [[1000], [1], [24], [1]]), (2, 1, 128, 16, [[15, 16], [2, 1], [1, 47]]),
         (40, 16, 64, 64, [[63] * 40, [1] * 40, [130] * 40])]


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,d,P,calls", CALLS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_ingest_of_plain_rows_is_append(kvm, B, H, d, P, calls, layout):
    """Without norm and rotation codes and scales are the definition's, call by call, held rows that are rounded again among them."""
    m = Model(kvm, B, H, d, P, 20)
    f = kvm.Front(norm="none", layout=layout)
    for i, counts in enumerate(calls):
        T = max(max(counts), 1) + (i % 2) * (max(counts) > 1)
        grow = 2.0 ** random.Random(i).uniform(-6, 6)
        k, v, q = rows((B, H, T, d), 100 + i) * grow, rows((B, H, T, d), 200 + i) * (1 / grow), rows((B, 2 * H, T, d), 300 + i)
        start = list(m.len)
        out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
        m.cache.ingest(q.cuda(), k.cuda(), v.cuda(), f, m.table, i32(start), i32(counts), q_out=out, status=status)
        assert status.item() == 0
        append = m.cache.append
        m.cache.append = lambda *a, **kw: None                   # (the model's part alone)
        m.append(k, v, counts)
        m.cache.append = append
        for b, n in enumerate(counts):
            assert torch.equal(out[b, :, :n].cpu(), q[b, :, :n]) and (out[b, :, n:] == 7.0).all()
    torch.cuda.synchronize()
    m.check_codes()


def check_keys(cache, table, start, counts, y, e, old=None):
    """Codes and scales of freshly begun blocks against y [B, H, T, d] with its bound e: the scale is that of some maximum within the bound, and what a
    code stands for is within half a step of e4m3 (2^-4 of the value, 2^-10 of the scale) of the value."""
    P, H = cache.page_tokens, cache.n_kv_heads
    kn, sn, tn = cache.k8.float().cpu().double().numpy(), cache.k_scale.cpu().double().numpy(), table.cpu().numpy()
    for b, n in enumerate(counts):
        at = 0
        while at < n:
            block, r0 = divmod(start[b] + at, P)
            m = min(P - r0, n - at)
            page = tn[b, block]
            for h in range(H):
                yy, ee = y[b, h, at:at + m], e[b, h, at:at + m]
                s = sn[page, h]
                i = np.abs(yy).argmax()
                if r0 == 0:
                    lo, hi = np.maximum(np.abs(yy) - ee, 0).max(), (np.abs(yy) + ee).max()
                    assert ec.least_exp(lo) <= math.log2(s) <= ec.least_exp(hi), (b, h, block, i)
                else:
                    assert np.abs(yy).max() <= 448 * s * (1 + 2.0 ** -20)
                off = np.abs(kn[page, h, r0:r0 + m] * s - yy)
                bound = np.maximum(2.0 ** -4 * np.abs(yy), 2.0 ** -10 * s) + 2 * ee
                assert (off <= bound).all(), (b, h, block, float((off / bound).max()))
            at += m


INGESTS = [
    (1, 4, 2, 128, 64, [[1000], [1], [1]], dict(norm="layer", rope_dims=32)),
    (3, 8, 4, 64, 16, [[50, 1, 333], [1, 0, 1], [7, 8, 9]], dict(norm="rms", rope_dims=64, layout="interleaved", scaling="parts", factor=4.0, original_len=64, magnitude=1.1386294361119891)),
    (2, 3, 3, 128, 128, [[129, 600], [300, 1], [1, 1]], dict(norm="none", rope_dims=20)),
    (2, 6, 1, 64, 32, [[100, 31], [1, 1], [5, 40]], dict(norm="layer", rope_dims=62)),
    (5, 16, 8, 128, 32, [[64, 65, 1, 0, 200], [1] * 5], dict(norm="rms", rope_dims=128)),
    (1, 40, 17, 64, 128, [[700], [1]], dict(norm="layer", rope_dims=16, scaling="linear", factor=2.0)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,d,P,calls,kw", INGESTS)
def test_ingest_against_the_definition(kvm, B, Hq, Hkv, d, P, calls, kw):
    blocks = sum(max(c) for c in calls) // P + 2
    cache = garbage_cache(kvm, B * blocks + 3, Hkv, d, P)
    table = torch.randperm(B * blocks + 3, generator=torch.Generator().manual_seed(1))[:B * blocks].to(torch.int32).view(B, blocks).cuda()
    twin = garbage_cache(kvm, B * blocks + 3, Hkv, d, P)        # its values by append
    qp, kp = params(Hq, d, kw["norm"], 3), params(Hkv, d, kw["norm"], 4)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    f = kvm.Front(q_weight=dev(qp[0]), q_bias=dev(qp[1]), k_weight=dev(kp[0]), k_bias=dev(kp[1]), **kw)
    start = [0] * B
    for i, counts in enumerate(calls):
        T = max(counts)
        x = rows((B, T, Hq + 2 * Hkv, d), 10 + i).transpose(1, 2)
        xd = x.cuda()                                            # (strides as they are)
        q, k, v = (x[:, a:b] for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        qd, kd, vd = (xd[:, a:b] for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
        out, status = torch.full((B, Hq, T, d), 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
        assert cache.ingest(qd, kd, vd, f, table, i32(start), i32(counts), q_out=out, status=status) is out
        twin.append(kd, vd, table, i32(start), i32(counts))
        torch.cuda.synchronize()
        assert status.item() == 0
        check_rows(out, *reference(q, start, counts, *qp, kw), counts)
        check_keys(cache, table, start, counts, *reference(k, start, counts, *kp, kw))
        assert torch.equal(cache.v8.view(torch.uint8), twin.v8.view(torch.uint8)) and torch.equal(cache.v_scale.view(torch.int32), twin.v_scale.view(torch.int32))
        one = garbage_cache(kvm, B * blocks + 3, Hkv, d, P)      # keys and values alone: the same codes
        if i == 0:
            assert one.ingest(None, kd, vd, f, table, i32(start), i32(counts)) is None
            assert torch.equal(one.k8.view(torch.uint8), cache.k8.view(torch.uint8)) and torch.equal(one.v8.view(torch.uint8), cache.v8.view(torch.uint8))
        start = [a + n for a, n in zip(start, counts)]


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 130])
def test_ingest_reports_lengths_and_pages_and_touches_nothing_else(kvm, T):
    m = Model(kvm, 4, 2, 64, 16, 20)
    f = kvm.Front(norm="rms", rope_dims=32)
    x = rows((4, 6, T, 64), 1).cuda()
    q, k, v = x[:, :2], x[:, 2:4], x[:, 4:]
    for bad_page, start, count in ((10 ** 6, [32] * 4, [0, 1, 0, 0]), (-1, [32] * 4, [0, 1, 0, 0]), (None, [32, -1, 32, 32], [0, 1, 0, 0]), (None, [32, 320, 32, 32], [0, 1, 0, 0]),
                                   (None, [32] * 4, [0, -1, 0, 0]), (None, [32] * 4, [0, T + 1, 0, 0]), (None, [32, 2 ** 31 - 1, 32, 32], [0, 1, 0, 0])):
        table, status = m.table.clone(), i32([0])
        if bad_page is not None:
            table[1, 2] = bad_page
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        m.cache.ingest(q, k, v, f, table, i32(start), i32(count), q_out=out, status=status)
        assert status.item() == 1
        m.check_codes()
        if bad_page is None:
            assert (out == 7.0).all()
        status.zero_()
        ko, vo = (torch.full((4, 2, T, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        m.cache.read(table, i32(start), T, i32(count), k_out=ko, v_out=vo, status=status)
        assert status.item() == 1
        for o in (ko, vo):
            if bad_page is not None:
                assert torch.isnan(o[1, :, 0].float()).all()
                o[1, :, 0] = 7.0
            assert (o == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 20])
def test_ingest_of_infinities(kvm, T):
    """A row with an infinity or a NaN makes the scale of its block NaN, for that head, and of keys or values alone; the block is sound when it is begun anew."""
    c = kvm.Cache.empty(4, 3, 64, 16)
    k, v = rows((1, 3, T, 64), 1), rows((1, 3, T, 64), 2)
    k[0, 0, 0, 63] = math.inf
    v[0, 1, 0, 5] = math.nan
    table = i32([[2, 1, 3]])
    for f in (kvm.Front(norm="none", rope_dims=16), kvm.Front(norm="layer")):
        c.ingest(None, k.cuda(), v.cuda(), f, table, i32([0]))
        assert torch.isnan(c.k_scale[2]).tolist() == [True, False, False] and torch.isnan(c.v_scale[2]).tolist() == [False, True, False]
        if T == 20:
            assert torch.isfinite(c.k_scale[1]).all() and torch.isfinite(c.v_scale[1]).all()
        ko, vo = c.read(table, i32([0]), T)
        assert torch.isnan(ko[0, 0, :min(T, 16)].float()).all() and torch.isfinite(ko[0, 1:].float()).all()
        assert torch.isnan(vo[0, 1, :min(T, 16)].float()).all() and torch.isfinite(vo[0, 0].float()).all()
        c.ingest(None, rows((1, 3, 1, 64), 4).cuda(), rows((1, 3, 1, 64), 5).cuda(), f, table, i32([0]))
        assert torch.isfinite(c.k_scale[2]).all() and torch.isfinite(c.v_scale[2]).all()


# ---- and back --------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("B,H,d,P,T,starts,counts", [(1, 1, 64, 16, 1, [0], None), (3, 2, 128, 64, 200, [0, 63, 130], [200, 0, 77]), (2, 5, 64, 128, 1000, [1, 255], [1000, 999]),
                                                     (2, 3, 128, 32, 300, [31, 0], None), (40, 8, 128, 16, 1, list(range(40)), None)])
def test_read_against_the_definition(kvm, B, H, d, P, T, starts, counts):
    m = Model(kvm, B, H, d, P, 1300 // P + 1)
    total = [s + n for s, n in zip(starts, counts or [T] * B)]
    m.append(rows((B, H, max(total), d), 1) * 2.0 ** -9, rows((B, H, max(total), d), 2), total)
    n = counts or [T] * B
    wide = torch.full((B, T, H, d + 8), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    odd = torch.full((B, H, T, d + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    for ko, vo in ((torch.full((B, H, T, d), 7.0, dtype=torch.bfloat16, device="cuda"), wide[..., :d]), (odd[..., 1:], torch.full((B, H, T, d), 7.0, dtype=torch.bfloat16, device="cuda"))):
        status = i32([0])
        got = m.cache.read(m.table, i32(starts), T, None if counts is None else i32(counts), k_out=ko, v_out=vo, status=status)
        assert got[0] is ko and got[1] is vo and status.item() == 0
        for o, rws in ((ko, m.k), (vo, m.v)):
            on = o.float().cpu().double().numpy()
            for b in range(B):
                assert (on[b, :, n[b]:] == 7.0).all()
                for h in range(H):
                    assert np.array_equal(on[b, h, :n[b]], rws[b][h].values()[starts[b]:starts[b] + n[b]])
    assert (wide[..., d:] == 7.0).all() and (odd[..., 0] == 7.0).all()


@pytest.mark.gpu
def test_read_of_the_ends_of_the_range(kvm):
    """bf16's largest value is rounded up to 2^128 in 8 bits and comes back as itself; its smallest normal one comes back as nothing."""
    c = kvm.Cache.empty(1, 2, 64, 16)
    x = torch.zeros((1, 2, 2, 64), dtype=torch.bfloat16)
    big = torch.finfo(torch.bfloat16).max
    x[0, 0, 0], x[0, 0, 1], x[0, 1] = big, -big, torch.finfo(torch.bfloat16).tiny
    c.append(x.cuda(), x.cuda(), i32([[0]]), i32([0]))
    ko, vo = c.read(i32([[0]]), i32([0]), 2)
    assert torch.equal(ko.cpu(), torch.where(x.abs() == big, x, torch.zeros(()).bfloat16())) and torch.equal(ko, vo)


@pytest.mark.gpu
def test_read_of_any_code_and_scale(kvm):
    c = kvm.Cache.empty(3, 1, 64, 16)
    codes = torch.arange(256, dtype=torch.uint8).repeat(12)[:3 * 16 * 64].view(3, 1, 16, 64)
    c.k8.view(torch.uint8).copy_(codes)
    c.k_scale.copy_(torch.tensor([[2.0 ** -64], [1.0], [2.0 ** 110]]))
    ko, _ = c.read(i32([[0, 1, 2]]), i32([0]), 48)
    want = c.k8.double().view(48, 64) * c.k_scale.double().repeat_interleave(16, 0).view(48, 1)
    same = (ko[0, 0].double() == want) | (torch.isnan(want) & torch.isnan(ko[0, 0].double()))
    assert same.all()


# ---- together --------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 64])
def test_a_captured_step_of_front_cache_attention_and_read(kvm, T):
    """Ingest, attend and read in one graph that is replayed as the sequences grow, with pages that move; the queries and keys are the front end's, the
    attention is that over what the cache holds, the rows read back are what it holds."""
    B, Hq, Hkv, d, P = 2, 8, 2, 128, 64
    pages, cache = kvm.Pages(64, P), kvm.Cache.empty(64, Hkv, d, P)
    kw = dict(norm="rms", rope_dims=64, scaling="linear", factor=2.0)
    f = kvm.Front(**kw)
    seqs = [pages.open() for _ in range(B)]
    x = torch.zeros((B, T, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    qo, out = (torch.zeros((B, Hq, T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ko, vo = (torch.zeros((B, Hkv, T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, start, status = torch.zeros((B, 20), dtype=torch.int32, device="cuda"), i32([0] * B), i32([0])

    def step():
        cache.ingest(q, k, v, f, table, start, q_out=qo, status=status)
        cache.attend(qo, table, start, out=out, status=status)
        cache.read(table, start, T, k_out=ko, v_out=vo, status=status)

    for s in seqs:
        pages.extend(s, T)
    table[:, :1] = pages.tables(seqs)[0][:, :1]
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        step()
    torch.cuda.current_stream().wait_stream(warm)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    at = [0, 0]
    for i in range(4):
        if i:
            for s in seqs:
                pages.extend(s, T)
        if i == 2:
            extra = pages.fork(seqs[0])                          # the last page of the first sequence is copied before it is written
            pages.extend(extra, 1)
            pages.close(seqs[1])
            src, dst = pages.compact()
            cache.copy_pages(src, dst)
            seqs[1] = pages.open()
            pages.extend(seqs[1], T)
            at[1] = 0
        t, length = pages.tables(seqs, 20)
        table.copy_(t)
        start.copy_(length - T)
        assert (length - T).tolist() == at
        x.copy_(rows((B, Hq + 2 * Hkv, T, d), 50 + i))
        g.replay()
        torch.cuda.synchronize()
        assert status.item() == 0
        yq, eq = reference(q.cpu(), at, [T] * B, None, None, kw)
        check_rows(qo, yq, eq, [T] * B)
        held = cache.read(table, i32([0, 0]), max(at) + T, i32([a + T for a in at]))
        for b in range(B):
            n = at[b] + T
            assert torch.equal(ko[b], held[0][b, :, at[b]:n]) and torch.equal(vo[b], held[1][b, :, at[b]:n])
            for h in range(Hkv):
                K, V = (z[b, h, :n].float().cpu().double().numpy() for z in held)
                qn = qo[b, 4 * h:4 * h + 4].float().cpu().double().numpy().reshape(-1, d)
                ref, bound = ec.attend(qn, K, V, np.tile(np.arange(at[b], n), 4), float(np.float32(d ** -0.5)))
                assert (np.abs(out[b, 4 * h:4 * h + 4].float().cpu().double().numpy().reshape(-1, d) - ref) <= bound).all()
        at = [a + T for a in at]


@pytest.mark.gpu
def test_front_of_the_largest_offsets(kvm):
    """Rows whose offsets pass 32 bits."""
    H, d, T = 4, 128, 2
    big = torch.zeros(((1 << 31) // d + 16 * H * T, d), dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (2, H, T, d), (1 << 31, T * d, d, 1))
    x.copy_(rows((2, H, T, d), 1))
    f = kvm.Front(norm="layer", rope_dims=32)
    want = kvm.qk_norm_rope(x.contiguous(), None, f, i32([4, 5]))[0]
    kvm.qk_norm_rope(x, None, f, i32([4, 5]), q_out=x)
    assert torch.equal(x, want)


def test_without_rotation_frequencies_are_not_looked_at(kvm):
    for at in (1, 4, 1 << 20):                         # (no address that may be read, nor aligned)
        f = _front(kvm, rope_dims=0, frequencies=C.cast(C.c_void_p(at), C.POINTER(C.c_double)))
        assert kvm.lib.kvm_rope_frequencies(C.byref(f), 128, None) == 0
    f = _front(kvm, rope_dims=2, frequencies=C.cast(C.c_void_p(4), C.POINTER(C.c_double)))
    assert kvm.lib.kvm_rope_frequencies(C.byref(f), 128, (C.c_double * 1)()) == 1


# ---- every build over many rows --------------------------------------------------------------------------------------

SIDE, HALVES, MIXED = dict(rope_dims=40, layout="interleaved"), dict(rope_dims=48), dict(rope_dims=60)   # (pairs side by side; two runs; 30 pairs, no whole runs of four)


def placed(x, by):
    """x [..., d] in memory that begins `by` elements behind a border of 16 bytes, its rows 1 element apart if by is odd."""
    if not by:
        return x.cuda().contiguous()
    wide = torch.empty(x.numel() // x.shape[-1] * (x.shape[-1] + by % 2) + by + 16, dtype=x.dtype, device="cuda")
    y = wide[by:by + x.numel() // x.shape[-1] * (x.shape[-1] + by % 2)].view(*x.shape[:-1], x.shape[-1] + by % 2)[..., :x.shape[-1]]
    y.copy_(x)
    return y


def front_of(kvm, Hq, Hk, d, kw, by=0):
    """A front end with weights 8 `by` bytes behind a border of 16; it, and they on the host."""
    qp, kp = params(Hq, d, kw["norm"], 3), params(Hk, d, kw["norm"], 4)
    dev = lambda t: None if t is None else placed(t.reshape(-1), 2 * by).view(t.shape)  # noqa: E731
    return kvm.Front(q_weight=dev(qp[0]), q_bias=dev(qp[1]), k_weight=dev(kp[0]), k_bias=dev(kp[1]), **kw), qp, kp


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw,rows_by,weights_by", [(SIDE, 0, 0), (HALVES, 0, 0), (MIXED, 0, 0), (SIDE, 1, 0), (HALVES, 4, 0), (MIXED, 1, 0), (HALVES, 0, 1), (SIDE, 0, 1)])
def test_norm_rope_of_many_rows_in_every_layout_and_alignment(kvm, d, kw, rows_by, weights_by):
    B, Hq, Hk, T, start, counts = 2, 11, 6, 500, [7, 90000], [500, 333]
    assert B * T * (Hq + Hk) > 16384
    kw = dict(kw, norm="rms" if kw is MIXED else "layer")
    q, k = rows((B, Hq, T, d), 1), rows((B, Hk, T, d), 2)
    f, qp, kp = front_of(kvm, Hq, Hk, d, kw, weights_by)
    qd, kd, status = placed(q, rows_by), placed(k, rows_by), i32([0])
    assert (qd.data_ptr() % 16 == 0) == (rows_by == 0) and (f._desc.q_weight % 16 == 0) == (weights_by == 0)
    qo, ko = torch.full((B, Hq, T, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hk, T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    kvm.qk_norm_rope(qd, kd, f, i32(start), i32(counts), q_out=qo, k_out=ko, status=status)
    assert status.item() == 0
    check_rows(qo, *reference(q, start, counts, *qp, kw), counts)
    check_rows(ko, *reference(k, start, counts, *kp, kw), counts)
    kvm.qk_norm_rope(qd, kd, f, i32(start), i32(counts), q_out=qd, k_out=kd)           # in place
    for b, n in enumerate(counts):
        for got, out, x in ((qd, qo, q), (kd, ko, k)):
            assert torch.equal(got[b, :, :n], out[b, :, :n]) and torch.equal(got[b, :, n:].cpu(), x[b, :, n:])


@pytest.mark.gpu
@pytest.mark.parametrize("d,P", [(64, 16), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("kw,rows_by,weights_by", [(SIDE, 0, 0), (HALVES, 0, 0), (MIXED, 0, 0), (HALVES, 1, 0), (MIXED, 4, 0), (SIDE, 0, 1)])
@pytest.mark.parametrize("Hq", [2, 15])
def test_ingest_of_many_rows_in_every_layout_and_alignment(kvm, d, P, kw, rows_by, weights_by, Hq):
    """Rows of q in the launch of the pages and in one of their own, q_out apart and in place, and the same call once more."""
    B, Hkv, T, counts = 2, 3, 600, [600, 411]
    assert (B * T * Hq > 16384) == (Hq == 15)
    kw = dict(kw, norm="rms" if kw is MIXED else "layer")
    f, qp, kp = front_of(kvm, Hq, Hkv, d, kw, weights_by)
    blocks = (T + 30) // P + 2
    table = torch.randperm(B * blocks + 3, generator=torch.Generator().manual_seed(1))[:B * blocks].to(torch.int32).view(B, blocks).cuda()
    cache, twin, start = garbage_cache(kvm, B * blocks + 3, Hkv, d, P), garbage_cache(kvm, B * blocks + 3, Hkv, d, P), [0, 0]
    bits = lambda c: [c.k8.view(torch.uint8).clone(), c.v8.view(torch.uint8).clone(), c.k_scale.view(torch.int32).clone(), c.v_scale.view(torch.int32).clone()]  # noqa: E731
    for step, n in enumerate(([5, 30], counts)):                  # (the second call begins in the middle of a block)
        q, k, v = (rows((B, H, T, d), 10 * step + i) for i, H in enumerate((Hq, Hkv, Hkv)))
        qd, kd, vd = (placed(x, rows_by) for x in (q, k, v))
        out, status = torch.full((B, Hq, T, d), 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
        cache.ingest(qd, kd, vd, f, table, i32(start), i32(n), q_out=out, status=status)
        twin.append(kd, vd, table, i32(start), i32(n))
        assert status.item() == 0
        check_rows(out, *reference(q, start, n, *qp, kw), n)
        check_keys(cache, table, start, n, *reference(k, start, n, *kp, kw))
        want = bits(cache)
        assert torch.equal(want[1], twin.v8.view(torch.uint8)) and torch.equal(want[3], twin.v_scale.view(torch.int32))
        cache.ingest(qd, kd, vd, f, table, i32(start), i32(n), q_out=qd)
        assert all(torch.equal(x, y) for x, y in zip(bits(cache), want))
        for b in range(B):
            assert torch.equal(qd[b, :, :n[b]], out[b, :, :n[b]]) and torch.equal(qd[b, :, n[b]:].cpu(), q[b, :, n[b]:])
        start = [a + b for a, b in zip(start, n)]


def far(x, at=0):
    """x [2, ...] with its second sequence 2^31 elements behind the first."""
    big = torch.empty((1 << 31) + x[0].numel() + at, dtype=torch.bfloat16, device="cuda")
    y = torch.as_strided(big, x.shape, (1 << 31, *x[0].stride()), at)
    y.copy_(x)
    return y


@pytest.mark.gpu
@pytest.mark.parametrize("at,kw", [(0, dict(rope_dims=32)), (0, dict(rope_dims=20)), (1, dict(rope_dims=32, layout="interleaved"))])
def test_many_rows_of_the_largest_offsets(kvm, at, kw):
    """Rows in front of and behind offsets of 32 bits in the kernel over many rows: 18000 of them."""
    x = rows((2, 9, 1000, 64), 1)
    f, start = kvm.Front(norm="layer", **kw), i32([4, 70000])
    want = kvm.qk_norm_rope(x.cuda(), None, f, start)[0]
    y = far(x, at)
    assert torch.equal(kvm.qk_norm_rope(y, None, f, start, q_out=torch.empty_like(want))[0], want)
    kvm.qk_norm_rope(y, None, f, start, q_out=y)
    assert torch.equal(y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T,Hq", [(1, 4), (300, 4), (300, 40)])
def test_ingest_and_read_of_the_largest_offsets(kvm, T, Hq):
    """A pool of more than 2^31 bytes per tensor and rows 2^31 elements apart, against pages at its front and contiguous rows."""
    H, d, P = 16, 128, 128
    N = (1 << 31) // (H * d * P) + 40
    c, f = kvm.Cache.empty(N, H, d, P), kvm.Front(norm="rms", rope_dims=128)
    q, k, v = rows((2, Hq, T, d), 1), rows((2, H, T, d), 2), rows((2, H, T, d), 3)
    low, start = i32([[0, 1, 2, 3], [4, 5, 6, 7]]), i32([100, 64])
    high = N - 1 - low
    first = rows((2, H, 100, d), 4).cuda()
    for t in (low, high):
        c.append(first, first, t, i32([0, 0]), start)
    want = c.ingest(q.cuda(), k.cuda(), v.cuda(), f, low, start)
    qf = far(q)
    assert c.ingest(qf, far(k), far(v), f, high, start, q_out=qf) is qf
    assert torch.equal(qf, want)
    del qf
    for codes in (c.k8, c.v8):
        x = codes.view(torch.uint8)
        assert torch.equal(x[:8], x[N - 8:].flip(0))
    for s in (c.k_scale, c.v_scale):
        assert torch.equal(s[:8], s[N - 8:].flip(0))
    n = i32([100 + T, 64 + T])
    a = c.read(low, i32([0, 0]), 100 + T, n, *(torch.zeros((2, H, 100 + T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    b = [far(torch.zeros((2, H, 100 + T, d), dtype=torch.bfloat16)) for _ in range(2)]
    c.read(high, i32([0, 0]), 100 + T, n, *b)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[0].float().abs().max() > 0.1


@pytest.mark.gpu
@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("layout,r", [("half", 0), ("interleaved", 0), ("half", 16), ("half", 44), ("interleaved", 22)])
@pytest.mark.parametrize("d", [64, 128])
def test_results_do_not_depend_on_alignment(kvm, norm, layout, r, d):
    """The same bits from rows and weights on 16-byte borders and off them, few rows and many, alone and in ingest."""
    f, odd = (front_of(kvm, 9, 3, d, dict(norm=norm, layout=layout, rope_dims=r), by)[0] for by in (0, 1))
    for T in (1, 100, 2000):
        x, start = rows((1, 9, T, d), T), i32([77])
        want = kvm.qk_norm_rope(x.cuda(), None, f, start)[0]
        for g, by in ((f, 1), (f, 4), (odd, 0)):
            assert torch.equal(kvm.qk_norm_rope(placed(x, by), None, g, start)[0], want)
        c, twin = (garbage_cache(kvm, T // 16 + 8, 3, d, 16) for _ in range(2))
        table = torch.arange(T // 16 + 8, dtype=torch.int32, device="cuda")[None]
        assert torch.equal(c.ingest(x.cuda(), x[:, :3].cuda(), x[:, 3:6].cuda(), f, table, start), want)
        assert torch.equal(twin.ingest(placed(x, 1), placed(x[:, :3], 1), placed(x[:, 3:6], 1), f, table, start), want)
        assert torch.equal(c.k8.view(torch.uint8), twin.k8.view(torch.uint8)) and torch.equal(c.v8.view(torch.uint8), twin.v8.view(torch.uint8))
