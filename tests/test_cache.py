"""Exact attention over the cache in 8 bits (kvm_cache_*, kvm_pages_*) against the fp64 definition in oracle/exact_cache.py."""
import ctypes as C
import math
import random

import numpy as np
import pytest
import torch

from oracle import exact_cache as ec


@pytest.fixture(scope="module")
def kvm():
    from paper_2605_09877_b200 import build
    build.build()
    from paper_2605_09877_b200 import kvm as mod
    return mod


# ---- pins of the definition ------------------------------------------------------------------------------------------

def test_e4m3_rounding_is_that_of_the_type():
    x = np.concatenate([np.linspace(-448, 448, 20001), np.ldexp(np.random.default_rng(0).standard_normal(20000), -6), [0.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0 - 17]])
    ref = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ec.round_e4m3(torch.from_numpy(x).float().double().numpy()), ref)


def test_least_scale_covers_the_maximum_and_no_smaller_one_does():
    for bits in range(0x0080, 0x7f80, 7):
        a = float(torch.tensor([bits], dtype=torch.int16).view(torch.bfloat16))
        e = ec.least_exp(a)
        assert a <= 448.0 * 2.0 ** e and (e == -64 or a > 448.0 * 2.0 ** (e - 1))
    assert ec.least_exp(448.0) == 0 and ec.least_exp(450.0) == 1 and ec.least_exp(0.0) == -64


def test_attention_of_the_definition_in_closed_form():
    v = np.arange(12.0).reshape(6, 2)
    out, _ = ec.attend(np.zeros((6, 2)), np.ones((6, 2)), v, np.arange(6), 1.0)                    # equal weights: running means
    assert np.allclose(out, np.cumsum(v, 0) / np.arange(1, 7)[:, None])
    out, _ = ec.attend(np.zeros((6, 2)), np.ones((6, 2)), v, np.arange(6), 1.0, window=2, sinks=1)
    assert np.allclose(out[5], v[[0, 4, 5]].mean(0)) and np.allclose(out[1], v[:2].mean(0)) and np.allclose(out[0], v[0])
    out, _ = ec.attend(np.zeros((1, 2)), np.ones((6, 2)), v, [5], 1.0, window=1)
    assert np.allclose(out, v[5])


# ---- bookkeeping of pages (host) -------------------------------------------------------------------------------------

def test_pages_share_copy_and_return(kvm):
    p = kvm.Pages(8, 16)
    a = p.open()
    assert p.extend(a, 40) is None and p.table(a) == [0, 1, 2] and p.length(a) == 40
    b = p.fork(a)
    assert p.table(b) == [0, 1, 2] and p.info() == dict(n_free=5, high=3)
    assert p.extend(b, 0) is None                      # nothing is written: nothing is copied
    assert p.extend(b, 1) == (2, 3) and p.table(b) == [0, 1, 3] and p.table(a) == [0, 1, 2]
    assert p.extend(a, 8) is None                      # the parent's page is its own again
    c = p.fork(a)                                      # 48 tokens: the last page is full, so nothing is copied
    assert p.extend(c, 1) is None and p.table(c) == [0, 1, 2, 4]
    with pytest.raises(kvm.KVMError) as e:
        p.extend(c, 16 * 4)                            # three free pages, four wanted
    assert e.value.code == 6 and p.length(c) == 49 and p.info()["n_free"] == 3
    p.close(a)
    assert p.info()["n_free"] == 3                     # b and c still use them
    p.close(c)
    assert p.info()["n_free"] == 5 and p.table(b) == [0, 1, 3]
    p.trim(b, window=8, sinks=4)                       # 41 tokens: the next sees 34.. and 0..3
    assert p.table(b) == [0, -1, 3] and p.length(b) == 41
    src, dst = p.compact()
    assert src.tolist() == [3] and dst.tolist() == [1] and p.table(b) == [0, -1, 1] and p.info() == dict(n_free=6, high=2)
    p.close(b)
    assert p.info() == dict(n_free=8, high=0) and p.open() == 0


@pytest.mark.parametrize("seed", range(6))
def test_pages_against_a_model(kvm, seed):
    """Random calls against a model that holds, per sequence, the contents of every block; pages hold what was copied to them."""
    r, P, N = random.Random(seed), r_choice(seed), 40
    p, seqs, store, stamp = kvm.Pages(N, P), {}, {}, 0

    def check():
        used = set()
        for s, (tokens, blocks) in seqs.items():
            t = p.table(s)
            assert p.length(s) == tokens and len(t) == len(blocks) == -(-tokens // P)
            for page, want in zip(t, blocks):
                if want is None:
                    assert page == -1
                else:
                    used.add(page)
                    assert 0 <= page < N and store[page] == want
        assert p.info()["n_free"] == N - len(used)
        assert p.info()["high"] == (max(used) + 1 if used else 0)

    for _ in range(300):
        what = r.choice(["open", "fork", "close", "extend", "extend", "extend", "trim", "compact"])
        s = r.choice(list(seqs)) if seqs else None
        if what == "open":
            seqs[p.open()] = (0, [])
        elif s is None:
            continue
        elif what == "fork":
            seqs[p.fork(s)] = (seqs[s][0], list(seqs[s][1]))
        elif what == "close":
            p.close(s)
            del seqs[s]
        elif what == "trim":
            W, S = r.randint(1, 4 * P), r.choice([0, 1, P, P + 1])
            p.trim(s, W, S)
            n = seqs[s][0]
            gone = lambda i: not any(j > n - W or j < S for j in range(i * P, (i + 1) * P))  # noqa: E731
            seqs[s] = (n, [None if b is None or gone(i) else b for i, b in enumerate(seqs[s][1])])
        elif what == "compact":
            src, dst = p.compact()
            assert len(set(dst.tolist())) == len(dst) and not set(src.tolist()) & set(dst.tolist())
            new = {d: store[x] for x, d in zip(src.tolist(), dst.tolist())}
            store.update(new)
            assert p.info()["high"] == N - p.info()["n_free"]
        else:
            n = r.randint(0, 3 * P)
            tokens, blocks = seqs[s]
            try:
                copy = p.extend(s, n)
            except kvm.KVMError as e:
                assert e.code == 6
                check()
                continue
            if copy:
                store[copy[1]] = store[copy[0]]
            t = p.table(s)
            blocks = list(blocks) + [None] * (len(t) - len(blocks))
            for i in range(tokens // P, -(-(tokens + n) // P) if n else 0):
                if i < len(seqs[s][1]) and blocks[i] is None:
                    continue                       # (a trimmed block in progress stays without a page)
                stamp += 1
                store[t[i]] = stamp
                blocks[i] = stamp
            seqs[s] = (tokens + n, blocks)
        check()


def r_choice(seed):
    return (16, 32, 64, 128)[seed % 4]


def test_pages_refusals(kvm):
    L, h, n = kvm.lib, C.c_void_p(), C.c_int32()
    assert L.kvm_pages_create(0, 64, C.byref(h)) == 1 and L.kvm_pages_create(8, 48, C.byref(h)) == 2 and L.kvm_pages_create(8, 64, None) == 1
    assert L.kvm_pages_destroy(None) == 0 and L.kvm_pages_open(None, C.byref(n)) == 1
    p = kvm.Pages(4, 16)
    for bad in (lambda: p.close(0), lambda: p.fork(-1), lambda: p.extend(3, 1), lambda: p.table(0), lambda: p.trim(0, 4, 0)):
        with pytest.raises(kvm.KVMError) as e:
            bad()
        assert e.value.code == 1
    s = p.open()
    for bad, code in ((lambda: p.extend(s, -1), 1), (lambda: p.trim(s, 0, 0), 1), (lambda: p.trim(s, 4, -1), 1), (lambda: p.extend(s, 1 << 31), 2),
                      (lambda: p.extend(s, 65), 6)):
        with pytest.raises(kvm.KVMError) as e:
            bad()
        assert e.value.code == code
    p.extend(s, 33)
    b = (C.c_int32 * 4)()
    assert L.kvm_pages_table(p._h, s, b, 2, None, None) == 6 and L.kvm_pages_table(p._h, s, b, 4, None, None) == 0 and list(b) == [0, 1, 2, -1]
    q = p.open()
    p.extend(q, 1)
    p.close(s)
    m = C.c_int64()
    assert L.kvm_pages_compact(p._h, b, b, 0, C.byref(m)) == 6 and p.table(q) == [3]
    assert L.kvm_pages_compact(p._h, None, b, 4, C.byref(m)) == 1


# ---- refusals of the device calls: before anything is launched -------------------------------------------------------

def _desc(kvm, **kw):
    c = dict(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, n_pages=8, n_kv_heads=2, head_dim=128, page_tokens=64)
    c.update(kw)
    return kvm.CacheDesc(*[c[f[0]] for f in kvm.CacheDesc._fields_])


def _call(kvm, **kw):
    c = dict(pages=1 << 24, start=1 << 25, count=None, batch=2, max_pages=4, n_tokens=3 + 1)
    c.update(kw)
    return kvm.CacheCall(*[c[f[0]] for f in kvm.CacheCall._fields_])


BAD_CACHE = [(dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=0), 1), (dict(k=(1 << 20) + 8), 1), (dict(v=(1 << 20) + 1), 1),
             (dict(k_scale=(1 << 20) + 2), 1), (dict(n_pages=0), 1), (dict(n_kv_heads=0), 1), (dict(n_kv_heads=-2), 1), (dict(head_dim=96), 2),
             (dict(head_dim=256), 2), (dict(page_tokens=48), 2), (dict(page_tokens=8), 2), (dict(n_pages=1 << 31), 2), (dict(n_pages=(1 << 31) // 128), 2)]
BAD_CALL = [(dict(pages=None), 1), (dict(start=None), 1), (dict(pages=(1 << 24) + 2), 1), (dict(start=(1 << 24) + 1), 1), (dict(count=(1 << 24) + 2), 1),
            (dict(batch=0), 1), (dict(batch=1025), 2), (dict(max_pages=0), 1), (dict(n_tokens=0), 1), (dict(n_tokens=257), 1), (dict(n_tokens=(1 << 30) + 1, count=1 << 24), 2),
            (dict(max_pages=(1 << 24) + 1), 2)]


@pytest.mark.parametrize("cache,call,code", [(c, {}, e) for c, e in BAD_CACHE] + [({}, c, e) for c, e in BAD_CALL])
def test_refusals_of_the_cache_and_the_call(kvm, cache, call, code):
    d, c, x = _desc(kvm, **cache), _call(kvm, **call), 1 << 26
    assert kvm.lib.kvm_cache_append(C.byref(d), C.byref(c), x, x, None, None, None, None) == code
    assert kvm.lib.kvm_cache_attend(C.byref(d), C.byref(c), x, 4, 1.0, 0, 0, 2 * x, None, None, x, 1 << 30, None, None) == code
    if not call:
        pair = (C.c_int32 * 1)(0), (C.c_int32 * 1)(1)
        assert kvm.lib.kvm_cache_copy_pages(C.byref(d), *pair, 1, None) == code


def test_refusals_of_the_other_arguments(kvm):
    d, c, x = C.byref(_desc(kvm)), C.byref(_call(kvm)), 1 << 26
    L = kvm.lib
    st = lambda *a: (C.c_int64 * 3)(*a)  # noqa: E731
    for args in ((None, c, x, x, None, None, None), (d, None, x, x, None, None, None), (d, c, None, x, None, None, None), (d, c, x, None, None, None, None),
                 (d, c, x + 1, x, None, None, None), (d, c, x, x, st(-128, 128, 128), None, None), (d, c, x, x, None, st(128, 128, -128), None),
                 (d, c, x, x, None, None, x + 2)):
        assert L.kvm_cache_append(*args, None) == 1
    ok = dict(q=x, hq=4, scale=1.0, window=0, sinks=0, out=2 * x, qs=None, os=None, ws=x, n=1 << 30, status=None)
    for kw, code in ((dict(q=None), 1), (dict(out=None), 1), (dict(q=x + 1), 1), (dict(out=2 * x + 1), 1), (dict(hq=0), 1), (dict(hq=5), 1), (dict(window=-1), 1),
                     (dict(sinks=-1), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1),
                     (dict(qs=st(1, 1, -1)), 1), (dict(os=st(4 * 512, 0, 128)), 1), (dict(os=st(2048, 512, 64)), 1), (dict(status=x + 1), 1)):
        a = dict(ok, **kw)
        assert L.kvm_cache_attend(d, c, a["q"], a["hq"], a["scale"], a["window"], a["sinks"], a["out"], a["qs"], a["os"], a["ws"], a["n"],
                                  a["status"], None) == code, kw
    i32 = lambda *a: (C.c_int32 * len(a))(*a)  # noqa: E731
    for src, dst in (((0, 1), (2, 2)), ((0, 1), (1, 2)), ((0,), (8,)), ((-1,), (2,)), ((8,), (2,)), ((0,), (-1,)), ((3,), (3,))):
        assert L.kvm_cache_copy_pages(d, i32(*src), i32(*dst), len(src), None) == 1
    assert L.kvm_cache_copy_pages(d, None, i32(1), 1, None) == 1 and L.kvm_cache_copy_pages(d, i32(1), i32(1), -1, None) == 1
    assert L.kvm_cache_copy_pages(d, None, None, 0, None) == 0
    many = i32(*range(9))
    assert L.kvm_cache_copy_pages(d, many, many, 9, None) == 1
    assert L.kvm_cache_workspace(d, c, 5) == -1 and L.kvm_cache_workspace(d, None, 4) == -1 and L.kvm_cache_workspace(d, c, 4) >= 0


def test_binding_refuses_what_it_can_see(kvm):
    z = torch.zeros((2, 1, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        kvm.Cache(z, z, torch.ones(2, 1), torch.ones(2, 1))      # not on a GPU
    with pytest.raises(ValueError):
        kvm.Cache(z, z[:1], torch.ones(2, 1), torch.ones(2, 1))


# ---- kernels ---------------------------------------------------------------------------------------------------------

NAN_CODE = 0x7f


def garbage_cache(kvm, n_pages, Hkv, d, P):
    """A pool as fresh memory may be: every code a NaN, every scale a NaN."""
    c = kvm.Cache.empty(n_pages, Hkv, d, P)
    c.k8.view(torch.uint8).fill_(NAN_CODE)
    c.v8.view(torch.uint8).fill_(NAN_CODE)
    c.k_scale.fill_(math.nan)
    c.v_scale.fill_(math.nan)
    return c


class Model:
    """The oracle's sequences beside a kvm.Cache."""

    def __init__(self, kvm, B, Hkv, d, P, blocks, extra=3, seed=0):
        self.kvm, self.B, self.Hkv, self.d, self.P = kvm, B, Hkv, d, P
        self.cache = garbage_cache(kvm, B * blocks + extra, Hkv, d, P)
        ids = torch.randperm(B * blocks + extra, generator=torch.Generator().manual_seed(seed))[:B * blocks]
        self.table = ids.to(torch.int32).view(B, blocks).cuda()
        self.k = [[ec.Rows(P, d) for _ in range(Hkv)] for _ in range(B)]
        self.v = [[ec.Rows(P, d) for _ in range(Hkv)] for _ in range(B)]
        self.len = [0] * B

    def append(self, k, v, counts, **kw):
        start = torch.tensor(self.len, dtype=torch.int32).cuda()
        count = torch.tensor(counts, dtype=torch.int32).cuda()
        self.cache.append(k.cuda() if not k.is_cuda else k, v.cuda() if not v.is_cuda else v, self.table, start, count, **kw)
        kn, vn = k.float().cpu().double().numpy(), v.float().cpu().double().numpy()
        for b in range(self.B):
            for h in range(self.Hkv):
                self.k[b][h].add(kn[b, h, :counts[b]])
                self.v[b][h].add(vn[b, h, :counts[b]])
            self.len[b] += counts[b]
        return start, count

    def check_codes(self):
        for codes, scales, rows in ((self.cache.k8, self.cache.k_scale, self.k), (self.cache.v8, self.cache.v_scale, self.v)):
            cn, sn, t = codes.float().cpu().double().numpy(), scales.cpu().double().numpy(), self.table.cpu().numpy()
            written = np.zeros(cn.shape[:3], bool)
            for b in range(self.B):
                for h in range(self.Hkv):
                    for i, blk in enumerate(rows[b][h].blocks):
                        page = t[b, i]
                        written[page, h, :blk.rows] = True
                        if blk.exp is None:
                            assert np.isnan(sn[page, h])
                        else:
                            assert sn[page, h] == 2.0 ** blk.exp, (b, h, i)
                            assert np.array_equal(cn[page, h, :blk.rows], blk.code[:blk.rows]), (b, h, i)
            assert np.isnan(cn[~written]).all()        # nothing else was touched

    def attend(self, q, counts, window=0, sinks=0, scale=None, **kw):
        """The call over tokens that are in the cache already; compares every row."""
        start = torch.tensor([n - c for n, c in zip(self.len, counts)], dtype=torch.int32).cuda()
        count = torch.tensor(counts, dtype=torch.int32).cuda()
        qd = q if q.is_cuda else q.cuda()
        out = kw.pop("out", None)
        if out is None:
            out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = self.cache.attend(qd, kw.pop("table", self.table), start, count, window=window, sinks=sinks, scale=scale, out=out, status=status, **kw)
        torch.cuda.synchronize()
        assert got is out and status.item() == 0
        self.compare(q, out, counts, window, sinks, scale)
        return out

    def compare(self, q, out, counts, window, sinks, scale=None):
        qn, on = q.float().cpu().double().numpy(), out.float().cpu().double().numpy()
        G = q.shape[1] // self.Hkv
        sc = float(np.float32(self.d ** -0.5 if scale is None else scale))
        for b in range(self.B):
            n = counts[b]
            assert (on[b, :, n:] == 7.0).all()         # rows behind the count are left as they were
            pos = np.arange(self.len[b] - n, self.len[b])
            for h in range(self.Hkv if n else 0):
                K, V = self.k[b][h].values(), self.v[b][h].values()
                ref, bound = ec.attend(qn[b, h * G:(h + 1) * G, :n].reshape(-1, self.d), K, V, np.tile(pos, G), sc, window, sinks)
                err = np.abs(on[b, h * G:(h + 1) * G, :n].reshape(-1, self.d) - ref)
                assert (err <= bound).all(), (b, h, float((err / bound).max()))


def rows(shape, seed, outliers=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if outliers:
        x = x * (1.0 + 4.0 * (torch.rand(shape[-1], generator=g) < 0.1))
    return x.to(torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,d,P,calls", [
    (1, 1, 64, 16, [[1]] * 20), (2, 3, 128, 64, [[70, 1], [1, 0], [58, 64], [1, 1], [0, 300]]), (3, 2, 64, 128, [[129, 5, 0], [1, 127, 128], [255, 1, 1]]),
    (2, 2, 128, 32, [[31, 33], [1, 1], [1, 1], [100, 95]]), (1, 5, 128, 128, [[1000], [1], [24], [1]]), (2, 1, 128, 16, [[15, 16], [2, 1], [1, 47]])])
def test_append_against_the_definition(kvm, B, H, d, P, calls):
    """Codes and scales are equal to the definition's, call by call; rows grow from call to call, so that scales rise."""
    m = Model(kvm, B, H, d, P, 20)
    for i, counts in enumerate(calls):
        T = max(max(counts), 1) + (i % 2)          # (padded)
        grow = 2.0 ** random.Random(i).uniform(-6, 6)
        m.append(rows((B, H, T, d), 100 + i) * grow, rows((B, H, T, d), 200 + i) * (1 / grow), counts)
    torch.cuda.synchronize()
    m.check_codes()


@pytest.mark.gpu
def test_append_of_extreme_values(kvm):
    m = Model(kvm, 1, 6, 64, 16, 4)
    x = torch.zeros((1, 6, 20, 64), dtype=torch.bfloat16)
    x[0, 1] = torch.finfo(torch.bfloat16).max
    x[0, 2] = torch.finfo(torch.bfloat16).tiny / 4
    x[0, 3, 3, 7] = math.inf                       # block 0 of head 3 is lost, block 1 is not
    x[0, 4, 17, 0] = math.nan
    x[0, 5] = -rows((20, 64), 3).abs() * 2.0 ** -70
    m.append(x, x.flip(1).contiguous(), [20])
    m.append(x, x.flip(1).contiguous() * 0, [15])
    torch.cuda.synchronize()
    m.check_codes()


@pytest.mark.gpu
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16)])
def test_append_takes_any_strides(kvm, d, P):
    """Rows of a fused projection [B, T, 3, H, d], an odd offset, heads that share rows (stride 0)."""
    B, H, T = 2, 3, 37
    f = rows((B, T, 3, H, d), 5).cuda()
    m = Model(kvm, B, H, d, P, 8)
    m.append(f[:, :, 1].transpose(1, 2), f[:, :, 2].transpose(1, 2), [37, 20])
    flat = torch.zeros(B * H * T * d + 1, dtype=torch.bfloat16, device="cuda")
    odd = flat[1:].view(B, H, T, d)
    odd.copy_(rows((B, H, T, d), 6))
    one = rows((B, 1, T, d), 7).cuda().expand(B, H, T, d)
    m.append(odd, one, [5, 37])
    torch.cuda.synchronize()
    m.check_codes()


ATTEND = [
    # B, Hq, Hkv, d, P, context, tokens, window, sinks
    (1, 1, 1, 64, 16, [0], [1], 0, 0), (1, 1, 1, 128, 64, [0], [1], 1, 0), (2, 4, 4, 128, 64, [130, 63], [1, 1], 0, 0),
    (3, 8, 2, 128, 64, [1000, 0, 127], [1, 1, 1], 0, 0), (2, 16, 1, 64, 32, [300, 511], [1, 1], 0, 0), (2, 32, 1, 128, 16, [300, 17], [1, 1], 0, 0),
    (2, 6, 2, 128, 128, [640, 255], [1, 1], 100, 5), (2, 6, 2, 64, 16, [640, 255], [1, 1], 7, 0), (2, 4, 2, 128, 32, [900, 40], [1, 1], 130, 140),
    (2, 4, 2, 128, 64, [129, 10], [2, 1], 0, 0), (2, 8, 2, 64, 64, [500, 0], [4, 3], 0, 0), (1, 7, 1, 128, 64, [256], [2], 60, 4), (4, 5, 5, 128, 32, [77, 0, 300, 5], [3, 0, 8, 1], 0, 0),
    (1, 2, 2, 128, 64, [0], [200], 0, 0), (2, 4, 2, 64, 16, [0, 300], [129, 77], 0, 0), (2, 8, 2, 128, 128, [130, 0], [100, 128], 0, 0),
    (1, 12, 4, 128, 64, [50], [333], 64, 3), (2, 3, 1, 64, 32, [0, 5], [400, 390], 1, 1), (1, 4, 1, 128, 32, [700], [70], 300, 200), (3, 2, 2, 128, 64, [0, 100, 0], [150, 0, 1], 0, 0),
    (1, 64, 2, 128, 64, [400], [5], 0, 0), (1, 2, 1, 128, 64, [1500], [40], 0, 0), (1, 8, 8, 64, 64, [2100], [1], 0, 0), (1, 2, 2, 64, 128, [0], [700], 100, 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,d,P,ctx,tokens,window,sinks", ATTEND)
def test_attend_against_the_definition(kvm, B, Hq, Hkv, d, P, ctx, tokens, window, sinks):
    blocks = -(-max(c + t for c, t in zip(ctx, tokens)) // P) + 1
    m = Model(kvm, B, Hkv, d, P, blocks, seed=d + P)
    if max(ctx):
        m.append(rows((B, Hkv, max(ctx), d), 1), rows((B, Hkv, max(ctx), d), 2) + 0.5, ctx)
    T = max(tokens) + 1
    m.append(rows((B, Hkv, T, d), 3), rows((B, Hkv, T, d), 4), tokens)
    m.attend(rows((B, Hq, T, d), 5) * 0.7, tokens, window, sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("T,far", [(1, 80), (4, 40), (4, 80), (150, 30), (150, 80)])
def test_a_huge_block_does_not_touch_the_tokens_that_do_not_see_it(kvm, T, far):
    """The values of the call's last block (for a single token: of blocks outside its window) are 2^far times the others: tokens before it get
    what they would get without it, to the same bound."""
    B, H, d, P, n = 1, 2, 64, 16, 318 if T == 4 else 320
    m = Model(kvm, B, H, d, P, 40)
    v = rows((B, H, n, d), 2, False)
    if T == 1:
        v[:, :, 100:180] *= 2.0 ** far
    m.append(rows((B, H, n, d), 1, False), v, [n])
    v = rows((B, H, T, d), 4, False)
    late = 2 if T == 4 else T - 50                 # (of four tokens, the last two lie in a block of their own)
    if T > 1:
        v[:, :, late:] *= 2.0 ** far
    m.append(rows((B, H, T, d), 3, False), v, [T])
    q = rows((B, 2 * H, T, d), 5)
    if T == 1:
        m.attend(q, [T], window=100, sinks=3)
        return
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    m.cache.attend(q.cuda(), m.table, torch.tensor([n], dtype=torch.int32).cuda(), out=out)
    on, qn = out.float().cpu().double().numpy(), q.double().numpy()
    early = late // P * P if T > 4 else 2          # (a block's scale is one: rows that share the block of huge ones lose their codes to it)
    for h in range(H):
        K, V = m.k[0][h].values(), m.v[0][h].values()
        for a, b, L in ((0, early, n + early), (late, T, n + T)):
            ref, bound = ec.attend(qn[0, 2 * h:2 * h + 2, a:b].reshape(-1, d), K[:L], V[:L], np.tile(np.arange(n + a, n + b), 2), float(np.float32(d ** -0.5)))
            assert (np.abs(on[0, 2 * h:2 * h + 2, a:b].reshape(-1, d) - ref) <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 20, 400])
@pytest.mark.parametrize("e", [-120, 120])
def test_values_at_the_ends_of_the_range(kvm, T, e):
    """Values near bf16's largest and smallest: results are in range wherever the definition's are."""
    m = Model(kvm, 1, 2, 128, 64, 40)
    v = rows((1, 2, 1500, 128), 2, False).clamp(-4, 4) * 2.0 ** e
    m.append(rows((1, 2, 1500, 128), 1), v, [1500])
    m.append(rows((1, 2, T, 128), 3), v[:, :, :T], [T])
    m.attend(rows((1, 4, T, 128), 5), [T])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 3, 150])
def test_attend_over_blocks_of_very_different_scales(kvm, T):
    """Neighbouring blocks whose keys and values lie orders of magnitude apart, zero blocks among them; peaked and flat rows."""
    B, H, d, P, n = 1, 3, 128, 16, 400
    k, v = rows((B, H, n, d), 1, False), rows((B, H, n, d), 2, False)
    for i in range(0, n, P):
        k[:, :, i:i + P] *= 2.0 ** ((i // P) % 5 - 3)
        v[:, 0, i:i + P] *= 2.0 ** ((i // P) % 9 * 4 - 16)
        v[:, 1, i:i + P] *= 0.0 if (i // P) % 3 else 2.0 ** -20
        v[:, 2, i:i + P] *= 2.0 ** 100 if i // P == 20 else 1.0
    k[:, :, 64:80] = 0
    m = Model(kvm, B, H, d, P, 40)
    m.append(k, v, [n])
    m.append(k[:, :, :T], v[:, :, 5:5 + T] * 0, [T])
    m.attend(rows((B, 2 * H, T, d), 7) * 2, [T])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 140])
def test_attend_takes_any_strides_scales_and_streams(kvm, T):
    B, Hq, Hkv, d, P = 2, 6, 3, 64, 32
    m = Model(kvm, B, Hkv, d, P, 12)
    m.append(rows((B, Hkv, 200, d), 1), rows((B, Hkv, 200, d), 2), [200, 140])
    q = rows((B, T, Hq, d), 5).cuda().transpose(1, 2)
    out = torch.full((B, T, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    m.attend(q, [T, T], out=out)
    flat, o2 = (torch.full((B * Hq * T * d + 1,), 7.0, dtype=torch.bfloat16, device="cuda")[1:].view(B, Hq, T, d) for _ in range(2))
    flat.copy_(q)
    m.attend(flat, [T, T], window=33, sinks=2, scale=0.3, out=o2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    m.attend(q, [T, T], stream=side)
    m.attend(q[:, :, :, :], [T, max(T - 1, 0)], stream=side)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 130])
def test_freed_and_unwritten_pages_are_not_looked_at(kvm, T):
    """Entries of blocks that no token of the call sees may be anything; rows behind the last token hold NaN codes."""
    m = Model(kvm, 2, 2, 128, 16, 40)
    m.append(rows((2, 2, 400, 128), 1), rows((2, 2, 400, 128), 2), [400, 333])
    m.append(rows((2, 2, T, 128), 3), rows((2, 2, T, 128), 4), [T, T])
    table = m.table.clone()
    for b, n in enumerate(m.len):
        first = n - T
        for i in range(40):
            if (i + 1) * 16 <= first - 50 + 1 and i * 16 >= 5 or i * 16 >= n:
                table[b, i] = (-1, 1 << 30, -(1 << 31), 10 ** 6)[i % 4]
    m.attend(rows((2, 4, T, 128), 5), [T, T], window=50, sinks=5, table=table)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 130])
def test_bad_lengths_and_pages_are_reported_and_nothing_else_is_touched(kvm, T):
    m = Model(kvm, 4, 1, 64, 16, 20)
    m.append(rows((4, 1, 100, 64), 1), rows((4, 1, 100, 64), 2), [100] * 4)
    q = rows((4, 2, T, 64), 5).cuda()
    good = m.cache.attend(q, m.table, torch.full((4,), 90, dtype=torch.int32).cuda(), torch.full((4,), 1, dtype=torch.int32).cuda()).clone()
    for bad_table, start, count in (({1: (2, 10 ** 6)}, [90] * 4, [1] * 4), ({1: (0, -1)}, [90] * 4, [1] * 4), ({}, [90, -1, 90, 90], [1] * 4),
                                    ({}, [90, 321, 90, 90], [1] * 4), ({}, [90] * 4, [1, -1, 1, 1]), ({}, [90] * 4, [1, T + 1, 1, 1]),
                                    ({}, [90, 2 ** 31 - 1, 90, 90], [1] * 4)):
        table = m.table.clone()
        for b, (i, page) in bad_table.items():
            table[b, i] = page
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        s, c = torch.tensor(start, dtype=torch.int32).cuda(), torch.tensor(count, dtype=torch.int32).cuda()
        m.cache.attend(q, table, s, c, out=out, status=status)
        assert status.item() == 1
        if count[1] == 1:
            assert torch.isnan(out[1, :, :1].float()).all() if bad_table else True
        for b in (0, 2, 3):
            assert torch.equal(out[b, :, :1], good[b, :, :1])
        assert (out[:, :, 1:] == 7.0).all()
        if not bad_table or bad_table[1][0] == 2:
            before = [t.clone() for t in (m.cache.k8.view(torch.uint8), m.cache.v8.view(torch.uint8))]
            status.zero_()
            x = rows((4, 1, T, 64), 9).cuda()
            if bad_table:
                s = torch.full((4,), 32, dtype=torch.int32).cuda()
            m.cache.append(x, x, table, s, torch.tensor([0, count[1], 0, 0], dtype=torch.int32).cuda(), status=status)
            assert status.item() == 1
            assert all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(before, (m.cache.k8, m.cache.v8)))


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(2, 128), (8, 64), (130, 128), (130, 64)])
def test_a_page_outside_the_pool_reaches_the_tokens_that_see_it_and_no_others(kvm, T, d):
    """The block of the call's last token is not there: the tokens in front of the block are right, whatever an earlier call left on the chip."""
    held = 32 if T > 2 else 31
    last = (held + T - 1) // 16 * 16                   # the block's first position
    m = Model(kvm, 1, 2, d, 16, 20)
    m.append(rows((1, 2, held + T, d), 1), rows((1, 2, held + T, d), 2), [held + T])
    q = rows((1, 4, T, d), 5)
    table = m.table.clone()
    table[0, last // 16] = 10 ** 6
    nan = garbage_cache(kvm, 64, 8, d, 16)             # codes of NaN
    nan.k_scale.fill_(1.0)
    nan.v_scale.fill_(1.0)
    for rep in range(3):
        nan.attend(rows((64, 16, T, d), 3).cuda(), torch.arange(64, dtype=torch.int32).repeat(64, 1).cuda(), torch.full((64,), 800, dtype=torch.int32).cuda())
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = m.cache.attend(q.cuda(), table, torch.tensor([held], dtype=torch.int32).cuda(), status=status)
        assert status.item() == 1
        ahead = last - held
        assert torch.isnan(out[0, :, ahead:].float()).all()
        on = out[:, :, :ahead].float().cpu().double().numpy()
        for h in range(2):
            K, V = m.k[0][h].values(), m.v[0][h].values()
            ref, bound = ec.attend(q[0, 2 * h:2 * h + 2, :ahead].double().numpy().reshape(-1, d), K, V, np.tile(np.arange(held, last), 2), float(np.float32(d ** -0.5)), 0, 0)
            err = np.abs(on[0, 2 * h:2 * h + 2].reshape(-1, d) - ref)
            assert (err <= bound).all(), (rep, h, float(np.nanmax(err / bound)), np.isnan(err).sum())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 130])
def test_infinities_and_nans_stay_where_they_are_seen(kvm, T):
    """A NaN among the keys or values reaches the queries that see its block and no other; one in q its own row only."""
    m = Model(kvm, 1, 3, 64, 16, 30)
    n = 300
    k, v = rows((1, 3, n, 64), 1), rows((1, 3, n, 64), 2)
    k[0, 0, 20, 3] = math.nan
    v[0, 1, 20, 3] = math.inf
    m.append(k, v, [n])
    m.append(rows((1, 3, T, 64), 3), rows((1, 3, T, 64), 4), [T])
    q = rows((1, 3, T, 64), 5)
    q[0, 2, T // 2, 1] = math.nan
    start = torch.tensor([n], dtype=torch.int32).cuda()
    out = m.cache.attend(q.cuda(), m.table, start)
    assert torch.isnan(out[0, 0].float()).all() and torch.isnan(out[0, 1].float()).all()
    bad = torch.isnan(out[0, 2].float()).all(-1).cpu()
    assert bad[T // 2] and bad.sum() == 1 and not torch.isnan(out[0, 2].float()[~bad.cuda()]).any()
    # the window has left the block (tokens 16..31): finite, and right
    q[0, 2, T // 2, 1] = 0.0
    m.k[0][0].blocks[1].exp = m.v[0][1].blocks[1].exp = 0      # (the definition's rows there are not seen either)
    m.attend(q, [T], window=200, sinks=16)


@pytest.mark.gpu
def test_empty_calls_and_counts_of_zero(kvm):
    m = Model(kvm, 3, 2, 128, 64, 4)
    m.append(rows((3, 2, 70, 128), 1), rows((3, 2, 70, 128), 2), [0, 0, 0])
    m.check_codes()
    m.append(rows((3, 2, 70, 128), 1), rows((3, 2, 70, 128), 2), [0, 70, 1])
    m.check_codes()
    for T in (1, 2, 70):
        out = torch.full((3, 2, T, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        m.attend(rows((3, 2, T, 128), 3), [0, T, 0], out=out)
        m.attend(rows((3, 2, T, 128), 3), [0, 0, 0])
    m.cache.copy_pages([], [])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 200])
def test_results_are_the_same_every_time(kvm, T):
    m = Model(kvm, 3, 2, 128, 64, 40)
    m.append(rows((3, 2, 2000, 128), 1), rows((3, 2, 2000, 128), 2), [2000, 1, 777])
    m.append(rows((3, 2, T, 128), 1), rows((3, 2, T, 128), 2), [T, T, T])
    q = rows((3, 8, T, 128), 3).cuda()
    start = torch.tensor([n - T for n in m.len], dtype=torch.int32).cuda()
    first = m.cache.attend(q, m.table, start)
    for _ in range(5):
        assert torch.equal(first, m.cache.attend(q, m.table, start))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 64])
def test_captured_calls_follow_the_lengths_and_pages_they_are_replayed_with(kvm, T):
    """Append and attend in one graph, replayed as the sequences grow; two graphs do not share their workspaces."""
    B, Hq, Hkv, d, P, n = 2, 8, 2, 128, 64, 700
    m = Model(kvm, B, Hkv, d, P, 30)
    m.append(rows((B, Hkv, n, d), 1), rows((B, Hkv, n, d), 2), [n, n - 100])
    start = torch.tensor(m.len, dtype=torch.int32).cuda()
    k, v, q = (torch.zeros((B, h, T, d), dtype=torch.bfloat16, device="cuda") for h in (Hkv, Hkv, Hq))
    out, out2 = (torch.full((B, Hq, T, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        m.cache.attend(q, m.table, start, out=out)
    torch.cuda.current_stream().wait_stream(warm)
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.cache.append(k, v, m.table, start)
        m.cache.attend(q, m.table, start, out=out)
    with torch.cuda.graph(g2):
        m.cache.attend(q, m.table, start, window=100, sinks=3, out=out2)
    for step in range(4):
        kn, vn, qn = rows((B, Hkv, T, d), 10 + step), rows((B, Hkv, T, d), 20 + step), rows((B, Hq, T, d), 30 + step)
        k.copy_(kn); v.copy_(vn); q.copy_(qn)
        start.copy_(torch.tensor(m.len, dtype=torch.int32))
        if step == 2:                                  # a page moves between two replays
            src, dst = m.table[0, 3].item(), (set(range(63)) - set(m.table.flatten().tolist())).pop()
            m.cache.copy_pages([src], [dst])
            m.table[0, 3] = dst
        g.replay()
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        s1.wait_stream(torch.cuda.current_stream()); s2.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s1):
            g2.replay()
        torch.cuda.synchronize()
        for b in range(B):
            for h in range(Hkv):
                m.k[b][h].add(kn[b, h].double().numpy()); m.v[b][h].add(vn[b, h].double().numpy())
            m.len[b] += T
        m.compare(qn, out, [T, T], 0, 0)
        m.compare(qn, out2, [T, T], 100, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(16))
def test_attend_over_random_shapes(kvm, seed):
    """Shapes, lengths, windows and scales drawn over the range that the calls allow (small enough for the definition on the host)."""
    r = random.Random(1000 + seed)
    d, P, Hkv, G = r.choice([64, 128]), r.choice([16, 32, 64, 128]), r.choice([1, 2, 3]), r.choice([1, 2, 3, 5, 8, 16])
    B, T = r.randint(1, 4), r.choice([1, 1, 2, 5, 17, 60, 200])
    ctx = [r.choice([0, r.randint(1, 20), r.randint(100, 1500)]) for _ in range(B)]
    tokens = [r.randint(0, T) for _ in range(B)]
    tokens[r.randrange(B)] = T
    window, sinks = r.choice([(0, 0), (r.randint(1, 600), r.choice([0, 1, 4, 130, 700]))])
    m = Model(kvm, B, Hkv, d, P, -(-(max(ctx) + T) // P) + r.randint(0, 30), seed=seed)
    if max(ctx):
        m.append(rows((B, Hkv, max(ctx), d), seed), rows((B, Hkv, max(ctx), d), seed + 1) * 2.0 ** r.randint(-20, 20), ctx)
    m.append(rows((B, Hkv, T, d), seed + 2), rows((B, Hkv, T, d), seed + 3), tokens)
    m.attend(rows((B, Hkv * G, T, d), seed + 4) * r.choice([0.1, 1.0, 4.0]), tokens, window, sinks, scale=r.choice([None, 0.02, 0.5]))


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hkv,T", [(1024, 2, 1), (700, 1, 3), (300, 1, 20)])
def test_large_batches_of_short_sequences(kvm, B, Hkv, T):
    """As many sequences as a call may have, most of them a tile or less, some without tokens."""
    r = random.Random(B)
    m = Model(kvm, B, Hkv, 64, 16, 14)
    ctx = [r.choice([0, 1, 15, 16, 17, r.randint(0, 200)]) for _ in range(B)]
    m.append(rows((B, Hkv, 200, 64), 1), rows((B, Hkv, 200, 64), 2), ctx)
    tokens = [r.choice([0, 1, T, T]) for _ in range(B)]
    m.append(rows((B, Hkv, T, 64), 3), rows((B, Hkv, T, 64), 4), tokens)
    m.attend(rows((B, 4 * Hkv, T, 64), 5), tokens)
    m.attend(rows((B, 4 * Hkv, T, 64), 5), tokens, window=40, sinks=2)


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,d,P,counts,window,sinks", [
    (3, 8, 4, 128, 16, [1500, 0, 411], 100, 5), (3, 8, 4, 64, 64, [1500, 1, 130], 300, 0), (2, 9, 9, 64, 128, [1300, 1290], 1, 0),
    (5, 16, 8, 128, 32, [40, 700, 64, 128, 129], 0, 0), (160, 1, 1, 64, 16, [33 + i % 3 for i in range(160)], 0, 0)])
def test_more_row_tiles_than_there_are_multiprocessors(kvm, B, Hq, Hkv, d, P, counts, window, sinks):
    """Short windows and short prompts: what a multiprocessor goes on to has fewer, other or no tiles.  Twice: the same bits."""
    T = max(counts)
    m = Model(kvm, B, Hkv, d, P, (T + 70 + P - 1) // P)
    held = [(7 * b) % 65 for b in range(B)]
    m.append(rows((B, Hkv, 65, d), 1), rows((B, Hkv, 65, d), 2), held)
    k, v = rows((B, Hkv, T, d), 3), rows((B, Hkv, T, d), 4)
    v[:, 0, T // 3] *= 2.0 ** 20                       # (blocks of values that lie far apart, for some of the rows)
    m.append(k, v, counts)
    q = rows((B, T, Hq, d), 5).transpose(1, 2)
    first = m.attend(q, counts, window=window, sinks=sinks)
    odd = torch.full((B, Hq, T, d + 1), 7.0, dtype=torch.bfloat16, device="cuda")[..., :d]     # (rows that are not 16-byte aligned)
    qo = torch.zeros((B, Hq, T, d + 1), dtype=torch.bfloat16, device="cuda")[..., :d]
    qo.copy_(q)
    assert torch.equal(m.attend(qo, counts, window=window, sinks=sinks, out=odd), first)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
def test_calls_side_by_side_on_two_streams(kvm, T):
    """Calls that overlap do not touch one another's workspaces."""
    ms = [Model(kvm, 2, 2, 128, 64, 40, seed=s) for s in range(2)]
    for s, m in enumerate(ms):
        m.append(rows((2, 2, 2000, 128), s), rows((2, 2, 2000, 128), 10 + s), [2000, 1500])
        m.append(rows((2, 2, T, 128), 20 + s), rows((2, 2, T, 128), 30 + s), [T, T])
    qs = [rows((2, 8, T, 128), 40 + s) for s in range(2)]
    outs = [[torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(20)] for q in qs]
    dev, starts = [q.cuda() for q in qs], [torch.tensor([n - T for n in m.len], dtype=torch.int32).cuda() for m in ms]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for s in range(2):
            ms[s].cache.attend(dev[s], ms[s].table, starts[s], out=outs[s][i], stream=streams[s])
    torch.cuda.synchronize()
    for s in range(2):
        ms[s].compare(qs[s], outs[s][0], [T, T], 0, 0)
        assert all(torch.equal(outs[s][0], o) for o in outs[s])


@pytest.mark.gpu
def test_a_call_after_a_split_one_sees_its_results(kvm):
    """What is enqueued behind a call - here a copy of its output - runs after all of it, whether or not anything was left to merge."""
    m = Model(kvm, 1, 2, 128, 64, 40)
    m.append(rows((1, 2, 2300, 128), 1), rows((1, 2, 2300, 128), 2), [2300])
    for T, start in ((1, 2000), (17, 2000), (200, 2000), (300, 0), (20, 100)):
        q, st = rows((1, 8, T, 128), 3).cuda(), torch.tensor([start], dtype=torch.int32).cuda()
        want = m.cache.attend(q, m.table, st)
        torch.cuda.synchronize()
        for _ in range(5):
            out = torch.zeros_like(q)
            m.cache.attend(q, m.table, st, out=out)
            got = out.clone()
            out.fill_(9.0)
            torch.cuda.synchronize()
            assert torch.equal(got, want) and (out == 9.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("H,d,P,n", [(1, 64, 16, 1), (3, 128, 64, 7), (8, 128, 128, 500), (2, 64, 32, 1300)])
def test_copies_of_pages(kvm, H, d, P, n):
    N = 2 * n + 5
    c = kvm.Cache.empty(N, H, d, P)
    g = torch.Generator(device="cuda").manual_seed(n)
    for t in (c.k8, c.v8):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    for t in (c.k_scale, c.v_scale):
        t.copy_(torch.rand(t.shape, generator=g, device="cuda"))
    ids = torch.randperm(N, generator=torch.Generator().manual_seed(n))
    src, dst = ids[:n].clone(), ids[n:2 * n].clone()
    if n > 2:
        src[1] = src[0]                                # one page forked twice
    want = [x.clone() for x in (c.k8.view(torch.uint8), c.v8.view(torch.uint8), c.k_scale, c.v_scale)]
    for x in want:
        x[dst] = x[src]
    c.copy_pages(src.tolist(), dst.to(torch.int32))
    for a, b in zip(want, (c.k8.view(torch.uint8), c.v8.view(torch.uint8), c.k_scale, c.v_scale)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_the_largest_offsets(kvm):
    """A pool of more than 2^31 bytes per tensor: pages behind that border are written, read and copied."""
    H, d, P = 16, 128, 128
    N = (1 << 31) // (H * d * P) + 40
    c = kvm.Cache.empty(N, H, d, P)
    k, v = rows((1, H, 300, d), 1), rows((1, H, 300, d), 2)
    table = torch.tensor([[N - 1, N - 2, N - 3]], dtype=torch.int32).cuda()
    low = torch.tensor([[0, 1, 2]], dtype=torch.int32).cuda()
    zero = torch.zeros(1, dtype=torch.int32).cuda()
    c.append(k.cuda(), v.cuda(), table, zero)
    for T in (1, 300):
        q = rows((1, H, T, d), 3).cuda()
        start = torch.tensor([300 - T], dtype=torch.int32).cuda()
        a = c.attend(q, table, start)
        c.copy_pages([N - 1, N - 2, N - 3], [0, 1, 2])
        b = c.attend(q, low, start)
        assert torch.equal(a, b) and torch.isfinite(a.float()).all() and a.float().abs().max() > 0.1
        c.copy_pages([3, 4, 5], [0, 1, 2])


@pytest.mark.gpu
def test_a_served_run_of_forks_windows_and_compaction(kvm):
    """Prompts, a fork, decode steps on both branches, pages given back behind a window, compaction, more steps: the operators as a
    serving program uses them together, every output against the definition over what each branch has appended."""
    Hq, Hkv, d, P, W, S = 8, 2, 128, 16, 60, 3
    cache, book = garbage_cache(kvm, 64, Hkv, d, P), kvm.Pages(64, P)
    hist = {}

    def step(seqs, n, seed, window):
        T = max(n)
        k, v, q = rows((len(seqs), Hkv, T, d), seed), rows((len(seqs), Hkv, T, d), seed + 1), rows((len(seqs), Hq, T, d), seed + 2)
        start = torch.tensor([book.length(s) for s in seqs], dtype=torch.int32).cuda()
        count = torch.tensor(n, dtype=torch.int32).cuda()
        copies = [c for c in (book.extend(s, m) for s, m in zip(seqs, n)) if c]
        if copies:
            cache.copy_pages([a for a, _ in copies], [b for _, b in copies])
        table, _ = book.tables(seqs)
        cache.append(k.cuda(), v.cuda(), table, start, count)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = cache.attend(q.cuda(), table, start, count, window=window, sinks=S if window else 0, status=status).float().cpu().double().numpy()
        assert status.item() == 0
        for i, s in enumerate(seqs):
            for h in range(Hkv):
                hist[s][0][h].add(k[i, h, :n[i]].double().numpy())
                hist[s][1][h].add(v[i, h, :n[i]].double().numpy())
                L = book.length(s)
                qq = q[i, h * 4:h * 4 + 4, :n[i]].double().numpy().reshape(-1, d)
                ref, bound = ec.attend(qq, hist[s][0][h].values(), hist[s][1][h].values(), np.tile(np.arange(L - n[i], L), 4),
                                       float(np.float32(d ** -0.5)), window, S if window else 0)
                assert (np.abs(out[i, h * 4:h * 4 + 4, :n[i]].reshape(-1, d) - ref) <= bound).all()

    import copy
    a, b = book.open(), book.open()
    for s in (a, b):
        hist[s] = [[ec.Rows(P, d) for _ in range(Hkv)] for _ in range(2)]
    step([a, b], [150, 37], 1, 0)
    c = book.fork(a)
    hist[c] = copy.deepcopy(hist[a])
    for i in range(12):
        step([a, b, c], [1, 1, 1], 10 * i + 20, 0)
    step([c, a], [20, 3], 300, W)
    for s in (a, b, c):
        book.trim(s, W, S)
    for i in range(3):
        step([a, c], [1, 1], 400 + 10 * i, W)
    book.close(b)
    src, dst = book.compact()
    assert len(src) > 0
    cache.copy_pages(src, dst)
    assert book.info()["high"] == 64 - book.info()["n_free"]
    for i in range(20):
        step([c, a], [1, 2], 600 + 10 * i, W)


# ---- mends -----------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("d,P", [(64, 16), (64, 32), (128, 16)])
def test_scales_that_rise_with_every_row_of_many_blocks(kvm, d, P):
    """One row a call, each twice the one before, in many blocks at once: every lane of a page divides what the block holds by the old scale
    over the new one, so all of them have to read the old scale before one of them writes the new one."""
    B, H = 24, 5
    m = Model(kvm, B, H, d, P, 2)
    for i in range(P + 3):
        m.append(rows((B, H, 1, d), 100 + i) * 2.0 ** (i % P), rows((B, H, 1, d), 200 + i) * 2.0 ** (i % P // 2), [1] * B)
    torch.cuda.synchronize()
    m.check_codes()


@pytest.mark.gpu
@pytest.mark.parametrize("T,G", [(1, 8), (4, 4), (75, 512)])
@pytest.mark.parametrize("below", [22.0, 26.0, 28.5])
def test_a_long_flat_tail_below_a_peak_counts_in_the_result(kvm, T, G, below):
    """A million keys, each 2^-below of the first one's weight: together up to a quarter of it, and all of the result, since the first one's value is 0.
    In closed form, to the same bound as everywhere: n w / (1 + n w)."""
    n, d, P = 1 << 20, 64, 128
    c = kvm.Cache.empty(n // P, 1, d, P)
    c.v8.view(torch.uint8).fill_(0x38)                 # 1.0
    c.k8.view(torch.uint8)[0, 0, 0, 0] = 0x38
    c.v8.view(torch.uint8)[0, 0, 0] = 0
    q = torch.zeros((1, G, T, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    table = torch.arange(n // P, dtype=torch.int32, device="cuda")[None]
    out = c.attend(q, table, torch.tensor([n - T], dtype=torch.int32).cuda(), scale=below * math.log(2.0)).double().cpu()
    tail = (torch.arange(n - T, n).double() * math.exp(-float(np.float32(below * math.log(2.0)))))[None, None, :, None]
    ref = tail / (1 + tail)
    bound = (2.0 ** -7 + 2.0 ** -20) * ref + 2.0 ** -11
    assert ((out - ref).abs() <= bound).all(), (float(ref.mean()), float(out.mean()), float(out.min()))


@pytest.mark.parametrize("groups,batch,n_tokens,max_pages", [(256, 4, 1 << 30, 256), (512, 4, 1 << 30, 256), (2, 4, 1 << 30, 256), (64, 1024, 1 << 24, 256), (1, 1024, 1, 1 << 24)])
def test_sizes_that_attention_refuses_have_no_workspace(kvm, groups, batch, n_tokens, max_pages):
    """Query rows, row tiles and key tiles of a call are numbered in 32 bits; both entry points say so before anything is narrowed."""
    d, x = C.byref(_desc(kvm, n_pages=1 << 16, n_kv_heads=128)), 1 << 26
    c = C.byref(_call(kvm, count=1 << 24, batch=batch, n_tokens=n_tokens, max_pages=max_pages))
    assert kvm.lib.kvm_cache_attend(d, c, x, 128 * groups, 1.0, 0, 0, 2 * x, None, None, x, 1 << 62, None, None) == 2
    assert kvm.lib.kvm_cache_workspace(d, c, 128 * groups) == -1


def test_a_book_of_pages_that_outlives_the_module_ends_quietly(kvm):
    """At the interpreter's end the module's names may be gone before the last Pages is."""
    import os
    import subprocess
    import sys
    code = "import sys; from paper_2605_09877_b200 import kvm; p = kvm.Pages(8, 16); sys.kept = kvm.Pages(8, 16); q = kvm.Pages(4, 64); del q"
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stderr == "", r.stderr


def test_binding_takes_no_number_for_another(kvm):
    """Numbers that 32 (or 64) bits do not hold are refused, not cut to those that are left; page numbers are whole."""
    p = kvm.Pages(8, 16)
    s = p.open()
    p.extend(s, 40)
    for bad in (lambda: kvm.Pages(8, (1 << 32) + 16), lambda: kvm.Pages((1 << 64) + 8, 16), lambda: p.fork((1 << 32) + s), lambda: p.close((1 << 32) + s),
                lambda: p.table((1 << 32) + s), lambda: p.length(s - (1 << 32)), lambda: p.tables([(1 << 32) + s], device="cpu"),
                lambda: p.extend(s + (1 << 32), 1), lambda: p.extend(s, (1 << 64) + 1), lambda: p.trim((1 << 32) + s, 8), lambda: p.trim(s, (1 << 32) + 8, 0),
                lambda: p.trim(s, 8, 1 << 32)):
        with pytest.raises(ValueError):
            bad()
    assert p.table(s) == [0, 1, 2] and p.length(s) == 40 and p.info() == dict(n_free=5, high=3)
    for kw in (dict(window=1 << 32), dict(window=(1 << 32) + 512), dict(window=1 << 31), dict(sinks=1 << 32), dict(sinks=-(1 << 32) + 4)):
        with pytest.raises(ValueError):
            kvm.Cache.attend(None, torch.zeros(1, 1, 1, 64), None, None, **kw)
    for src, dst in (([0], torch.tensor([(1 << 32) + 1])), (torch.tensor([1 << 32]), [1]), (np.array([-(1 << 32)]), [1]), ([0.7], [1]), (torch.tensor([0.0]), [1]),
                     ([0], [True]), ([0, 1], [2])):
        with pytest.raises(ValueError):
            kvm.Cache.copy_pages(None, src, dst)


def test_rows_of_the_output_that_lie_on_one_another_are_refused(kvm):
    """Two heads, tokens or sequences that share bytes of `out` would be written in any order."""
    d, c, x = C.byref(_desc(kvm)), C.byref(_call(kvm)), 1 << 26     # 2 sequences, 4 heads, 4 tokens, 128 channels
    for st in ((128, 128, 128), (2048, 128, 128), (512, 512, 128), (1024, 512, 128), (2048, 256, 128), (2048, 512, 510), (128, 512, 128), (1 << 62, 1 << 62, 1 << 61),
               (2047, 512, 128)):
        assert kvm.lib.kvm_cache_attend(d, c, x, 4, 1.0, 0, 0, 2 * x, None, (C.c_int64 * 3)(*st), x, 1 << 30, None, None) == 1, st


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
def test_the_output_may_have_its_dimensions_in_any_order(kvm, T):
    import itertools
    B, Hq, Hkv, d = 2, 4, 2, 64
    m = Model(kvm, B, Hkv, d, 16, 10)
    m.append(rows((B, Hkv, 100, d), 1), rows((B, Hkv, 100, d), 2), [100, 70])
    q = rows((B, Hq, T, d), 3)
    for order in itertools.permutations(range(3)):
        shape = [(B, Hq, T)[i] for i in order]
        for pad in (0, 8):
            wide = torch.full((*shape, d + pad), 7.0, dtype=torch.bfloat16, device="cuda")
            m.attend(q, [T, T], out=wide[..., :d].permute(*[order.index(i) for i in range(3)], 3))
            assert (wide[..., d:] == 7.0).all()


@pytest.mark.gpu
def test_calls_after_an_expired_wait(kvm):
    """The self test lets both forms of the bounded wait run out, the one that the cache's kernels use among them; it is reported once, ends
    in bounded time, and calls over a cache are as before."""
    from paper_2605_09877_b200 import synth
    from tests import parity_util as pu
    wl = synth.Workload("expire", 1, 2, 2, 64, 64 * 3, 64, "sqrt", sqrt_coeff=6, r=16, seed=3)
    st, _ = pu.gpu_layer(wl, synth.make_layer_params(wl))
    m = Model(kvm, 2, 2, 64, 16, 20)
    m.append(rows((2, 2, 200, 64), 1), rows((2, 2, 200, 64), 2), [200, 150])
    for spins in (1, 10000):
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        st.debug_expire_wait(spins)
        t1.record()
        assert st.check() == 7 and st.check() == 0
        assert t0.elapsed_time(t1) < 2000
        for T in (1, 30):
            m.attend(rows((2, 4, T, 64), 3), [T, T])
    st.free()


@pytest.mark.gpu
@pytest.mark.parametrize("H,d,P,n", [(1, 64, 16, 2041), (1, 64, 16, 2042), (1, 64, 16, 2043), (2, 64, 32, 9001), (1, 64, 16, 1)])
def test_copies_of_more_pages_than_one_launch_takes(kvm, H, d, P, n):
    N = 2 * n + 3
    c = kvm.Cache.empty(N, H, d, P)
    g = torch.Generator(device="cuda").manual_seed(n)
    parts = [c.k8.view(torch.uint8), c.v8.view(torch.uint8), c.k_scale, c.v_scale]
    for t in parts[:2]:
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    for t in parts[2:]:
        t.copy_(torch.rand(t.shape, generator=g, device="cuda"))
    ids = torch.randperm(N, generator=torch.Generator().manual_seed(n))
    src, dst = ids[:n], ids[n:2 * n]
    want = [x.clone() for x in parts]
    for x in want:
        x[dst.cuda()] = x[src.cuda()]
    c.copy_pages(src, dst)
    assert all(torch.equal(a, b) for a, b in zip(want, parts))


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d,P,ctx,T,window,sinks,split", [
    (32, 8, 128, 64, 9000, 300, 512, 4, False), (16, 4, 64, 16, 9000, 300, 200, 0, False), (4, 2, 128, 32, 9000, 60, 6000, 3, True), (4, 2, 128, 32, 9000, 60, 0, 0, True)])
def test_a_window_is_planned_as_the_tiles_it_sees(kvm, Hq, Hkv, d, P, ctx, T, window, sinks, split):
    """Behind a long context a window layer's table is as wide as a full one's, with -1 for the pages given back; key tiles that no row sees are no
    reason for key splits, their partial results in the workspace, and a merge."""
    lengths = [ctx + T]
    m = Model(kvm, 1, Hkv, d, P, -(-lengths[0] // P))
    m.append(rows((1, Hkv, ctx + T, d), 1), rows((1, Hkv, ctx + T, d), 2), lengths)
    q = rows((1, Hq, T, d), 3)
    table = m.table.clone()
    if window:
        gone = [i for i in range(table.shape[1]) if (i + 1) * P <= ctx - window + 1 and i * P >= sinks]
        table[0, gone] = -1
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    start = torch.tensor([ctx], dtype=torch.int32).cuda()
    call = kvm.CacheCall(table.data_ptr(), start.data_ptr(), None, 1, table.shape[1], T)
    n = kvm.lib.kvm_cache_workspace(m.cache._ref, C.byref(call), Hq)
    ws = torch.full((max(n, 16),), 0xAB, dtype=torch.uint8, device="cuda")
    qd = q.cuda()
    assert kvm.lib.kvm_cache_attend(m.cache._ref, C.byref(call), qd.data_ptr(), Hq, d ** -0.5, window, sinks, out.data_ptr(), None, None, ws.data_ptr(), n, None,
                                    torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    m.compare(q, out, [T], window, sinks)
    assert (ws != 0xAB).any().item() == split


@pytest.mark.gpu
@pytest.mark.parametrize("d,P,far", [(128, 64, 0), (128, 64, 20), (64, 16, 20), (128, 128, 100)])
def test_a_long_flat_tail_counts_over_values_of_any_scale(kvm, d, P, far):
    """As above, with one block of values 2^far below the others (from 2^14 on the scales go through the weights' exponents)."""
    n, T, G, below = 1 << 19, 80, 512, 25.0
    c = kvm.Cache.empty(n // P, 1, d, P)
    c.v8.view(torch.uint8).fill_(0x38)                 # 1.0
    c.k8.view(torch.uint8)[0, 0, 0, 0] = 0x38
    c.v8.view(torch.uint8)[0, 0, 0] = 0
    c.v_scale[7] = 2.0 ** -far
    q = torch.zeros((1, G, T, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    table = torch.arange(n // P, dtype=torch.int32, device="cuda")[None]
    out = c.attend(q, table, torch.tensor([n - T], dtype=torch.int32).cuda(), scale=below * math.log(2.0)).double().cpu()
    keys, w = torch.arange(n - T, n).double(), math.exp(-float(np.float32(below * math.log(2.0))))
    ref = ((keys - P * (1 - 2.0 ** -far)) * w / (1 + keys * w))[None, None, :, None]
    bound = (2.0 ** -7 + 2.0 ** -20) * ref + 2.0 ** -11
    err = (out - ref).abs()
    assert (err <= bound).all(), (float(ref.mean()), float(out.mean()), float(out.min()))
