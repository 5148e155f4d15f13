"""Attention of groups of sequences that share their first blocks (kvm_cache_attend_shared, kvm_pages_shared) against the fp64 definition in oracle/exact_cache.py."""
import copy
import ctypes as C
import math
import random

import numpy as np
import pytest
import torch

from oracle import exact_cache as ec
from tests.test_cache import BAD_CACHE, BAD_CALL, Model, _call, _desc, garbage_cache, rows


@pytest.fixture(scope="module")
def kvm():
    from paper_2605_09877_b200 import build
    build.build()
    from paper_2605_09877_b200 import kvm as mod
    return mod


# ---- host ------------------------------------------------------------------------------------------------------------

def test_shared_blocks_of_forks(kvm):
    p = kvm.Pages(64, 16)
    a = p.open()
    p.extend(a, 70)                                    # four full blocks and one in progress
    b, c = p.fork(a), p.fork(a)
    assert p.shared([a]) == 4 and p.shared([a], 6) == 4 and p.shared([a], 7) == 3 and p.shared([a], 0) == 4 and p.shared([a], 1000) == 0
    assert p.shared([a, b, c], 0) == 4
    for s in (a, b, c):
        p.extend(s, 30)
    assert p.shared([a, b, c], 30) == 4 and p.shared([c, a]) == 4
    d = p.fork(b)
    p.extend(d, 1)
    p.extend(b, 1)
    assert p.shared([b, d]) == 6 and p.shared([a, b, d]) == 4      # (100 tokens: six full blocks)
    p.trim(b, 20, 16)
    assert p.shared([b, d]) == 1 and p.shared([d, a]) == 4
    e = p.open()
    assert p.shared([e]) == 0 and p.shared([a, e]) == 0
    for bad in (lambda: p.shared([]), lambda: p.shared([a, 99]), lambda: p.shared([99]), lambda: p.shared([a], -1)):
        with pytest.raises(kvm.KVMError) as x:
            bad()
        assert x.value.code == 1
    n = C.c_int32()
    assert kvm.lib.kvm_pages_shared(None, (C.c_int32 * 1)(0), 1, 0, C.byref(n)) == 1 and kvm.lib.kvm_pages_shared(p._h, None, 1, 0, C.byref(n)) == 1
    with pytest.raises(ValueError):
        p.shared([1 << 32])


@pytest.mark.parametrize("cache,call,code", [(c, {}, e) for c, e in BAD_CACHE] + [({}, c, e) for c, e in BAD_CALL])
def test_refusals_of_the_cache_and_the_call(kvm, cache, call, code):
    d, c, x = _desc(kvm, **cache), _call(kvm, **call), 1 << 26
    assert kvm.lib.kvm_cache_attend_shared(C.byref(d), C.byref(c), x, x, 1, x, 4, 1.0, 2 * x, None, None, x, 1 << 40, None, None) == code


def test_refusals_of_the_other_arguments(kvm):
    L, d, c, x = kvm.lib, C.byref(_desc(kvm)), C.byref(_call(kvm)), 1 << 26
    st = lambda *a: (C.c_int64 * 3)(*a)  # noqa: E731
    need = L.kvm_cache_shared_workspace(d, c, 2, 4)
    assert need > 0 and L.kvm_cache_shared_workspace(d, c, 0, 4) == -1 and L.kvm_cache_shared_workspace(d, c, 3, 4) == -1 and L.kvm_cache_shared_workspace(d, c, 2, 5) == -1
    assert L.kvm_cache_shared_workspace(d, None, 2, 4) == -1 and L.kvm_cache_shared_workspace(None, c, 2, 4) == -1
    ok = dict(groups=x, shared=x, n=2, q=x, hq=4, scale=1.0, out=2 * x, qs=None, os=None, ws=x, bytes=need, status=None)
    for kw, code in ((dict(groups=None), 1), (dict(shared=None), 1), (dict(groups=x + 2), 1), (dict(shared=x + 1), 1), (dict(n=0), 1), (dict(n=-1), 1), (dict(n=3), 1),
                     (dict(q=None), 1), (dict(out=None), 1), (dict(q=x + 1), 1), (dict(out=2 * x + 1), 1), (dict(hq=0), 1), (dict(hq=5), 1), (dict(scale=0.0), 1),
                     (dict(scale=-1.0), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1), (dict(qs=st(1, 1, -1)), 1), (dict(os=st(4 * 512, 0, 128)), 1),
                     (dict(os=st(2048, 512, 64)), 1), (dict(status=x + 1), 1), (dict(ws=None), 1), (dict(ws=x + 8), 1), (dict(bytes=need - 1), 6), (dict(bytes=0), 6)):
        a = dict(ok, **kw)
        assert L.kvm_cache_attend_shared(d, c, a["groups"], a["shared"], a["n"], a["q"], a["hq"], a["scale"], a["out"], a["qs"], a["os"], a["ws"], a["bytes"], a["status"], None) == code, kw


# ---- kernel ----------------------------------------------------------------------------------------------------------

def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Shared(Model):
    """Groups of sequences behind lead[g] shared blocks, with own[b] tokens of their own in front of the call to come."""

    def __init__(self, kvm, sizes, lead, own, Hkv, d, P, room=200, seed=0, grow=1.0):
        B = sum(sizes)
        self.sizes, self.lead = sizes, lead
        super().__init__(kvm, B, Hkv, d, P, max(lead) + (max(own) + room) // P + 2, seed=seed)
        self.first = [sum(sizes[:g]) for g in range(len(sizes))]
        self.groups, self.shared = i32(self.first + [B]), i32(lead)
        counts = [0] * B
        for g, n in enumerate(sizes):
            if n:
                counts[self.first[g]] = lead[g] * P
        if max(counts):
            self.append(rows((B, Hkv, max(counts), d), 100 + seed) * grow, rows((B, Hkv, max(counts), d), 101 + seed) / grow, counts)
        for g, n in enumerate(sizes):
            for b in range(self.first[g] + 1, self.first[g] + n):
                f = self.first[g]
                self.table[b, :lead[g]] = self.table[f, :lead[g]]
                self.k[b], self.v[b], self.len[b] = copy.deepcopy(self.k[f]), copy.deepcopy(self.v[f]), self.len[f]
        if max(own):
            self.append(rows((B, Hkv, max(own), d), 102 + seed), rows((B, Hkv, max(own), d), 103 + seed), own)

    def hidden(self):
        """The table with what may be anything as it may be."""
        t = self.table.clone()
        for g, n in enumerate(self.sizes):
            for b in range(self.first[g] + 1, self.first[g] + n):
                t[b, :self.lead[g]] = -7
        return t

    def step(self, T, Hq, counts, seed, status=None, scale=None, check=True, **kw):
        """New tokens and their attention; every row is compared."""
        self.append(rows((self.B, self.Hkv, T, self.d), 200 + seed), rows((self.B, self.Hkv, T, self.d), 201 + seed), counts)
        q = rows((self.B, Hq, T, self.d), 202 + seed)
        start = i32([n - c for n, c in zip(self.len, counts)])
        out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
        got = self.cache.attend_shared(q.cuda(), self.hidden(), start, self.groups, self.shared, None if counts == [T] * self.B else i32(counts), scale=scale, out=out, status=status, **kw)
        torch.cuda.synchronize()
        assert got is out and status.item() == 0
        if check:
            self.compare(q, out, counts, 0, 0, scale)
        return q, start, out


CASES = [   # sizes, lead, own, Hq, Hkv, d, P, T
    ([2], [15], [60, 31], 8, 2, 128, 64, 1),
    ([1], [3], [0], 1, 1, 64, 16, 1),
    ([3], [1], [0, 5, 200], 6, 3, 128, 128, 1),
    ([5], [9], [0, 1, 15, 16, 17], 10, 2, 64, 16, 2),
    ([4, 3], [40, 7], [0, 10, 20, 30, 40, 50, 60], 8, 1, 128, 32, 1),
    ([33], [20], list(range(33)), 4, 1, 128, 64, 1),                         # 132 rows
    ([64], [33], [3 * i for i in range(64)], 8, 2, 128, 64, 1),              # 256 rows
    ([70], [31], [i % 7 for i in range(70)], 8, 2, 64, 16, 1),               # 280 rows
    ([40], [5], [i for i in range(40)], 16, 1, 128, 128, 1),                 # 640 rows, 16 to a sequence
    ([8, 0, 1, 50, 0], [12, 3, 0, 2, 5], [i % 40 for i in range(59)], 14, 2, 128, 64, 2),
    ([6] * 20, [4] * 20, [i % 5 for i in range(120)], 4, 4, 64, 32, 3),
    ([2, 2, 2], [0, 0, 0], [5, 300, 17, 0, 1, 90], 8, 2, 128, 64, 1),        # nothing shared at all
    ([10], [130], [0] * 10, 8, 8, 128, 16, 1),
    ([3], [8], [2, 3, 4], 6, 1, 128, 64, 5),                                 # 30 (token, head) pairs per sequence
    ([3, 2], [10, 4], [300, 0, 77, 5, 1000], 8, 2, 64, 16, 70),              # 280, long parts of their own
    ([9, 1], [40, 0], [17 * i for i in range(10)], 8, 1, 128, 32, 3),
]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,lead,own,Hq,Hkv,d,P,T", CASES)
def test_shared_against_the_definition(kvm, sizes, lead, own, Hq, Hkv, d, P, T):
    m = Shared(kvm, sizes, lead, own, Hkv, d, P)
    r = random.Random(1)
    m.step(T, Hq, [T] * m.B, 0)
    m.step(T, Hq, [r.randint(0, T) for _ in range(m.B)], 1)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(12))
def test_shared_over_random_shapes(kvm, seed):
    r = random.Random(seed)
    Hkv, G, d, P = r.choice([1, 2, 3]), r.choice([1, 2, 3, 4, 7, 8]), r.choice([64, 128]), r.choice([16, 32, 64, 128])
    sizes = [r.choice([0, 1, 2, 5, 20, 40]) for _ in range(r.choice([1, 2, 4]))] + [2]
    lead = [r.choice([0, 1, 2, r.randint(1, 1500 // P)]) for _ in sizes]
    own = [r.randint(0, r.choice([0, 40, 400])) for _ in range(sum(sizes))]
    T = r.choice([1, 1, 2, 16 // G, 7])
    m = Shared(kvm, sizes, lead, own, Hkv, d, P, seed=seed)
    m.step(T, Hkv * G, [r.randint(0, T) if r.random() < 0.3 else T for _ in range(m.B)], seed)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,G,T", [([3], 4, 1), ([50, 9], 4, 1), ([30], 4, 4)])
def test_long_shared_parts_and_more_tiles_than_multiprocessors(kvm, sizes, G, T):
    """Long chains of tiles per unit and CTAs with parts of several units; results are the same every time, and on another stream, and in any strides."""
    B = sum(sizes)
    m = Shared(kvm, sizes, [300] * len(sizes), [37 * b % 300 for b in range(B)], 2, 128, 16, seed=5)
    q, start, out = m.step(T, 2 * G, [T] * B, 0)
    t, s = m.hidden(), torch.cuda.Stream()
    for _ in range(3):
        assert torch.equal(m.cache.attend_shared(q.cuda(), t, start, m.groups, m.shared), out)
    s.wait_stream(torch.cuda.current_stream())
    got = m.cache.attend_shared(q.cuda(), t, start, m.groups, m.shared, stream=s)
    s.synchronize()
    assert torch.equal(got, out)
    odd = torch.empty((B, T, 2 * G, 131), dtype=torch.bfloat16, device="cuda").transpose(1, 2)[..., 1:129]
    odd.copy_(q)
    wide = torch.full((B, T, 2 * G, 130), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    m.cache.attend_shared(odd, t, start, m.groups, m.shared, out=wide[..., :128])
    assert torch.equal(wide[..., :128], out) and (wide[..., 128:] == 7.0).all()
    m.compare(q, m.cache.attend_shared(q.cuda(), t, start, m.groups, m.shared, scale=0.3), [T] * B, 0, 0, 0.3)


@pytest.mark.gpu
@pytest.mark.parametrize("n,d", [(2, 128), (40, 64), (40, 128)])
def test_blocks_of_very_different_scales(kvm, n, d):
    """Shared and own blocks whose values lie up to 2^100 apart, keys of one block that decide everything."""
    m = Shared(kvm, [n], [0], [0] * n, 1, d, 16, room=500)
    L, P = 400, 16
    k, v = rows((n, 1, L, d), 1), rows((n, 1, L, d), 2)
    for i, e in enumerate((0, -60, 30, -14, -15, 3, 40, -59, 0, -100)):
        v[:, :, 40 * i:40 * i + 40] *= 2.0 ** e
    k[:, :, 200:216] *= 16.0
    m.append(k[:1].expand(n, -1, -1, -1).contiguous(), v[:1].expand(n, -1, -1, -1).contiguous(), [L] + [0] * (n - 1))
    for b in range(1, n):
        m.table[b, :L // P] = m.table[0, :L // P]
        m.k[b], m.v[b], m.len[b] = copy.deepcopy(m.k[0]), copy.deepcopy(m.v[0]), L
    m.append(rows((n, 1, 33, d), 5), rows((n, 1, 33, d), 6) * 2.0 ** 20, [33] * n)
    m.lead, m.shared = [L // P], i32([L // P])
    m.step(1, 4, [1] * n, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("n,below", [(2, 22.0), (2, 28.5), (60, 26.0)])
def test_a_long_flat_shared_tail_below_a_peak_counts(kvm, n, below):
    """The first shared key has logit `below` * ln 2 above all others, whose values are 1 where its own is 0: they weigh L 2^-below together."""
    L, d, P = 1 << 18, 64, 128
    c = kvm.Cache.empty(L // P + n + 1, 1, d, P)
    c.k_scale.fill_(1.0)
    c.v8.view(torch.uint8)[:L // P] = 0x38                         # 1.0
    c.v8.view(torch.uint8)[0, 0, 0] = 0
    k = torch.zeros(d)
    k[0] = 64.0
    c.k8.view(torch.uint8)[0, 0, 0] = k.to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    table = torch.full((n, L // P + 1), -1, dtype=torch.int32)
    table[0, :L // P] = torch.arange(L // P)
    table[:, L // P] = L // P + torch.arange(n)
    q = torch.zeros((n, 4, 1, d), dtype=torch.bfloat16)
    q[..., 0] = 1.0
    scale = below * math.log(2) / 64.0
    zero = torch.zeros((n, 1, 1, d), dtype=torch.bfloat16, device="cuda")
    c.append(zero, zero, table.cuda(), i32([L] * n))               # (its own: value 0)
    out = c.attend_shared(q.cuda(), table.cuda(), i32([L] * n), i32([0, n]), i32([L // P]), scale=scale).double().cpu()
    w = math.exp(-64.0 * float(np.float32(scale)))
    want = (L - 1) * w / (1 + L * w)
    # bf16 2^-8; a weight 2^-11 of itself, or half a step of fp16's least number, 2^-25 in units of 2^-6 of the reference: 2^-31 each; the logit 2^-21 of itself
    assert (abs(out - want) <= want * (2.0 ** -8 + 2.0 ** -11 + below * 2.0 ** -21) + L * 2.0 ** -31).all(), (float(out.min()), want)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[2, 2, 1], [40, 40, 3]])
def test_nans_stay_where_they_are_seen(kvm, sizes):
    """A NaN among the shared keys or values reaches the rows of its group and head, one in q its own row, one in a sequence's own block its rows."""
    B = sum(sizes)
    m = Shared(kvm, sizes, [20, 9, 4], [20] * B, 3, 64, 16)
    m.cache.k_scale[m.table[0, 7], 0] = math.nan
    m.cache.v_scale[m.table[sizes[0], 3], 1] = math.nan
    m.cache.v_scale[m.table[B - 1, 4], 2] = math.nan
    q, start, out = m.step(1, 12, [1] * B, 0, check=False)
    bad = torch.isnan(out.float())
    want = torch.zeros((B, 12), dtype=torch.bool)
    want[:sizes[0], :4] = True
    want[sizes[0]:sizes[0] + sizes[1], 4:8] = True
    want[B - 1, 8:] = True
    assert torch.equal(bad.all(-1)[:, :, 0].cpu(), want) and torch.equal(bad.any(-1)[:, :, 0].cpu(), want)
    qn = q.clone()
    qn[1, 11, 0, 5] = math.nan
    qn[B - 2, 9, 0, 0] = -math.inf
    got = m.cache.attend_shared(qn.cuda(), m.hidden(), start, m.groups, m.shared)
    want2 = want.clone()
    want2[1, 11] = want2[B - 2, 9] = True
    assert torch.equal(torch.isnan(got.float()).all(-1)[:, :, 0].cpu(), want2)
    assert torch.equal(got[~want2], out[~want2])


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[2, 2, 1], [40, 40, 3]])
def test_bad_groups_lengths_and_pages_are_reported(kvm, sizes):
    B = sum(sizes)
    m = Shared(kvm, sizes, [20, 9, 4], [20] * B, 2, 64, 16)
    q, start, out = m.step(1, 8, [1] * B, 0)
    q, t = q.cuda(), m.hidden()
    n0, n1 = sizes[0], sizes[0] + sizes[1]

    def run(table=t, start=start, groups=m.groups, shared=m.shared, count=None):
        got, status = torch.full(out.shape, 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
        m.cache.attend_shared(q, table, start, groups, shared, count, out=got, status=status)
        assert status.item() == 1
        return got

    # offsets that do not ascend from 0 to the batch: nothing is written
    for g in ([0, n1, n0, B], [1, n0, n1, B], [0, n0, n1, B - 1], [0, n0, n1, B + 1], [0, -5, n1, B], [-1, n0, n1, B], [0, 2 ** 31 - 1, n1, B]):
        assert (run(groups=i32(g)) == 7.0).all()
    # numbers of blocks that are not allowed: that group gets no rows
    for s in (-1, 10, 2 ** 31 - 1, -2 ** 31, m.table.shape[1] + 1, m.table.shape[1]):
        if s == 10:
            got = run(shared=i32([20, 9 + 2, 4]), start=start)             # (start = 9 * 16 + 20: the eleventh block is not in front of it)
        else:
            got = run(shared=i32([20, s, 4]))
        assert (got[n0:n1] == 7.0).all() and torch.equal(got[:n0], out[:n0]) and torch.equal(got[n1:], out[n1:])
    # lengths
    for b, x in ((n0, -1), (n0 + 1, 2 ** 31 - 1), (n0 + 1, 9 * 16 - 1)):
        s2 = start.clone()
        s2[b] = x
        got = run(start=s2)
        keep = [i for i in range(B) if i != b]
        assert (got[b] == 7.0).all() and torch.equal(got[keep], out[keep])
    # a page outside the pool among the shared ones: the group's rows are NaN
    for x in (-1, 10 ** 6):
        t2 = t.clone()
        t2[n0, 5] = x
        got = run(table=t2)
        assert torch.isnan(got[n0:n1].float()).all() and torch.equal(got[:n0], out[:n0]) and torch.equal(got[n1:], out[n1:])
    # among a sequence's own
    t2 = t.clone()
    t2[0, 20] = -1
    got = run(table=t2)
    assert torch.isnan(got[0].float()).all() and torch.equal(got[1:], out[1:])


@pytest.mark.gpu
def test_captured_calls_follow_groups_lengths_and_pages(kvm):
    """Two graphs of the same call do not share their workspaces; a replay follows the arrays."""
    m = Shared(kvm, [3, 5], [10, 20], [5 * b for b in range(8)], 2, 128, 32)
    q0, start0, want0 = m.step(1, 8, [1] * 8, 0)
    q, start, table = q0.cuda(), start0.clone(), m.hidden()
    groups, shared = m.groups.clone(), m.shared.clone()
    out, out2 = torch.zeros_like(q), torch.zeros_like(q)
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        m.cache.attend_shared(q, table, start, groups, shared, out=out)
    torch.cuda.current_stream().wait_stream(warm)
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.cache.attend_shared(q, table, start, groups, shared, out=out)
    with torch.cuda.graph(g2):
        m.cache.attend_shared(q, table, start, groups, shared, out=out2)
    s = torch.cuda.Stream()
    for step in range(3):
        if step == 1:                                              # sequences go on
            qn, sn, _ = m.step(1, 8, [1] * 8, 4)
            q.copy_(qn); start.copy_(sn); table.copy_(m.hidden())
        if step == 2:                                              # other groups, fewer shared blocks: the tables as they are
            groups.copy_(i32([0, 2, 8])); shared.copy_(i32([10, 0])); table.copy_(m.table)
        g.replay()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g2.replay()
        g.replay()
        torch.cuda.synchronize()
        qc = q.cpu()
        m.compare(qc, out, [1] * 8, 0, 0)
        m.compare(qc, out2, [1] * 8, 0, 0)


@pytest.mark.gpu
def test_samples_of_prompts_served_behind_their_shared_blocks(kvm):
    """Prompts, forks into samples, steps with ingest and shared attention, samples that end and fork again, compaction: each step against what the cache holds."""
    P, d, Hq, Hkv = 16, 64, 8, 2
    pages, cache = kvm.Pages(400, P), kvm.Cache.empty(400, Hkv, d, P)
    f = kvm.Front(norm="rms", rope_dims=32)
    r = random.Random(3)
    prompts = []
    for i, n in enumerate((300, 37)):
        s = pages.open()
        pages.extend(s, n)
        t, length = pages.tables([s])
        x = rows((1, 2 * Hkv, n, d), 10 + i).cuda()
        cache.ingest(None, x[:, :Hkv], x[:, Hkv:], f, t, length - n)
        prompts.append([s] + [pages.fork(s) for _ in range(4)])
    for step in range(12):
        if step == 5:
            pages.close(prompts[0].pop(0))
            prompts[0].append(pages.fork(prompts[0][1]))
        if step == 8:
            src, dst = pages.compact()
            cache.copy_pages(src, dst)
        seqs = [s for p in prompts for s in p]
        T, B = r.choice([1, 1, 2]), len(seqs)
        copies = [c for c in (pages.extend(s, T) for s in seqs) if c]
        if copies:
            cache.copy_pages(*[list(x) for x in zip(*copies)])
        t, length = pages.tables(seqs)
        x = rows((B, Hq + 2 * Hkv, T, d), 50 + step).cuda()
        status = i32([0])
        q = cache.ingest(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], f, t, length - T, status=status)
        groups = i32([0, len(prompts[0]), B])
        shared = i32([pages.shared(p, T) for p in prompts])
        assert shared.tolist()[0] >= 300 // P and shared.tolist()[1] >= 37 // P
        out = cache.attend_shared(q, t, length - T, groups, shared, status=status)
        assert status.item() == 0
        n = length.tolist()
        held = cache.read(t, i32([0] * B), max(n), length)
        for b in range(B):
            for h in range(Hkv):
                K, V = (z[b, h, :n[b]].float().cpu().double().numpy() for z in held)
                qn = q[b, 4 * h:4 * h + 4].float().cpu().double().numpy().reshape(-1, d)
                ref, bound = ec.attend(qn, K, V, np.tile(np.arange(n[b] - T, n[b]), 4), float(np.float32(d ** -0.5)))
                assert (np.abs(out[b, 4 * h:4 * h + 4].float().cpu().double().numpy().reshape(-1, d) - ref) <= bound).all()


@pytest.mark.gpu
def test_many_groups(kvm):
    """As many groups as a call may have sequences, and one group of all of them."""
    B, d, P = 1024, 64, 16
    c = kvm.Cache.empty(3 * B, 1, d, P)
    x = torch.randn((B, 2, 40, d), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    table = torch.arange(3 * B, dtype=torch.int32, device="cuda").view(B, 3)
    c.append(x[:, :1], x[:, 1:], table, i32([0] * B))
    q = rows((B, 2, 1, d), 3).cuda()
    start = i32([39] * B)
    want = c.attend(q, table, start).float()
    got = c.attend_shared(q, table, start, torch.arange(B + 1, dtype=torch.int32, device="cuda"), i32([2] * B)).float()
    assert (got - want).abs().max() <= 2.0 ** -7 * want.abs().max()
    table[:, :2] = table[0, :2].clone()
    want = c.attend(q, table, start).float()
    got = c.attend_shared(q, table, start, i32([0, B]), i32([2])).float()
    assert (got - want).abs().max() <= 2.0 ** -7 * want.abs().max()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2, 40, 70])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_far_from_zero_and_far_apart(kvm, n, d):
    """Heads whose logits are tiny, large, all far below zero or far above, and rows whose maximum grows by a hundred and more from tile to tile."""
    H, P, L = 5, 64, 640
    m = Shared(kvm, [n], [0], [0] * n, H, d, P, room=L + 200)
    k, v = rows((n, H, L, d), 1), rows((n, H, L, d), 2)
    u = torch.ones(d) / math.sqrt(d)
    k[:, 1] = k[:, 1] * 0.05 + 8 * u                               # logits near q . u * 8
    k[:, 2] = k[:, 2] * 0.05 - 8 * u
    k[:, 3] = (k[:, 3].float() * 0.05 + 2.0 * (torch.arange(L) // 100)[:, None] * u).bfloat16()     # grows along the keys
    k[:, 4, 400:410] *= 8.0                                        # a few keys that decide everything
    one = [L] + [0] * (n - 1)
    m.append(k[:1].expand(n, -1, -1, -1).contiguous(), v[:1].expand(n, -1, -1, -1).contiguous(), one)
    for b in range(1, n):
        m.table[b, :L // P] = m.table[0, :L // P]
        m.k[b], m.v[b], m.len[b] = copy.deepcopy(m.k[0]), copy.deepcopy(m.v[0]), L
    m.lead, m.shared = [L // P], i32([L // P])
    m.append(rows((n, H, 3, d), 5), rows((n, H, 3, d), 6), [b % 4 for b in range(n)])
    T, G = 1, 4
    m.append(rows((n, H, T, d), 7), rows((n, H, T, d), 8), [T] * n)
    q = rows((n, H * G, T, d), 9)
    q[:, G:4 * G] = (q[:, G:4 * G].float() * 0.05 + 60.0 * u).bfloat16()
    start = i32([x - T for x in m.len])
    for scale in (1e-4, 0.1, 1.0):                                 # heads 1 and 2: logits of +- 480 and less
        out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
        m.cache.attend_shared(q.cuda(), m.hidden(), start, m.groups, m.shared, scale=scale, out=out, status=status)
        assert status.item() == 0
        m.compare(q, out, [T] * n, 0, 0, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("n,d", [(2, 64), (50, 64), (50, 128)])
def test_values_far_below_the_largest_of_their_block(kvm, n, d):
    """The row that sets the blocks' scale has no weight; what is left are the least codes, 1 to 7 times 2^-9: each counts in full."""
    P, L = 64, 512
    c = kvm.Cache.empty(L // P + n, 1, d, P)
    codes = torch.randint(1, 8, (L, d), generator=torch.Generator().manual_seed(1)) | (torch.randint(0, 2, (L, d), generator=torch.Generator().manual_seed(2)) << 7)
    codes[::P] = 0x7e                                              # 448
    c.v8.view(torch.uint8)[:L // P] = codes.to(torch.uint8).view(L // P, 1, P, d).cuda()
    c.v_scale.fill_(2.0 ** -3)
    k = torch.zeros((L, d))
    k[::P, 0] = -256.0
    c.k8.view(torch.uint8)[:L // P] = k.to(torch.float8_e4m3fn).view(torch.uint8).view(L // P, 1, P, d).cuda()
    table = torch.cat([torch.arange(L // P).repeat(n, 1), L // P + torch.arange(n)[:, None]], 1).to(torch.int32).cuda()
    q = torch.zeros((n, 4, 1, d), dtype=torch.bfloat16)
    q[..., 0] = 2.0
    zero = torch.zeros((n, 1, 1, d), dtype=torch.bfloat16, device="cuda")
    c.append(zero, zero, table, i32([L] * n))
    out = c.attend_shared(q.cuda(), table, i32([L] * n), i32([0, n]), i32([L // P]), scale=1.0).double().cpu()
    v = c.v8.view(torch.uint8)[:L // P].cpu().view(torch.float8_e4m3fn).double().view(L, d) * 2.0 ** -3
    live = torch.ones(L, dtype=torch.bool)
    live[::P] = False
    want = v[live].sum(0) / (live.sum() + 1)                       # (its own key: weight 1, value 0)
    # equal weights: 2^-8 for the output; sums of 2^9 terms in fp32, 2^-24 2^9 of the sum of magnitudes
    assert (abs(out - want) <= 2.0 ** -8 * abs(want) + 2.0 ** -15 * v[live].abs().mean(0)).all(), float(abs(out - want).max())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2, 40, 70])
@pytest.mark.parametrize("d", [64, 128])
def test_references_that_move_by_a_little(kvm, n, d):
    """Rows whose maximum grows by a few powers of two from tile to tile, each at its own rate, in one half of a tile or the other, over blocks of several scales."""
    H, P, L = 3, 32, 128 * 9 + 32
    m = Shared(kvm, [n], [0], [0] * n, H, d, P, room=L + 100)
    k, v = rows((n, H, L, d), 1), rows((n, H, L, d), 2)
    u = torch.ones(d) / math.sqrt(d)
    t = torch.arange(L)
    steps = [t // 128, (t + 58) // 128, 9 - t // 128]              # from the first column, from the 71st, downwards
    for h in range(H):
        k[:, h] = (k[:, h].float() * 0.05 + steps[h][:, None] * u).bfloat16()
    v = (v.float() * torch.exp2(((t // 32) % 5 - 2).float())[:, None]).bfloat16()
    m.append(k[:1].expand(n, -1, -1, -1).contiguous(), v[:1].expand(n, -1, -1, -1).contiguous(), [L] + [0] * (n - 1))
    for b in range(1, n):
        m.table[b, :L // P] = m.table[0, :L // P]
        m.k[b], m.v[b], m.len[b] = copy.deepcopy(m.k[0]), copy.deepcopy(m.v[0]), L
    m.lead, m.shared = [L // P], i32([L // P])
    m.append(rows((n, H, 1, d), 7), rows((n, H, 1, d), 8), [1] * n)
    G = 4
    rate = torch.linspace(-3.0, 10.0, n * H * G).view(n, H * G, 1, 1)   # logits per tile: up to 2^14 from tile to tile
    q = (rows((n, H * G, 1, d), 9).float() * 0.05 + rate * u).bfloat16()
    out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
    m.cache.attend_shared(q.cuda(), m.hidden(), i32([x - 1 for x in m.len]), m.groups, m.shared, scale=1.0, out=out, status=status)
    assert status.item() == 0
    m.compare(q, out, [1] * n, 0, 0, 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("n,d", [(24, 128), (48, 64)])
def test_few_results_are_rounded_otherwise_than_the_definition(kvm, n, d):
    """A weight of fp16 is off by 2^-11 / sqrt(3) of itself (standard deviation) at most, q in two parts and fp32 by less than 2^-16: a result is rounded to the
    neighbour only where the definition's lies that near to the border between them."""
    P, L = 64, 2048
    c = kvm.Cache.empty(L // P + n, 1, d, P)
    k, v = rows((1, 1, L, d), 1), rows((1, 1, L, d), 2)
    head = torch.arange(L // P, dtype=torch.int32)[None]
    c.append(k.cuda(), v.cuda(), head.cuda(), i32([0]))
    table = torch.cat([head.repeat(n, 1), L // P + torch.arange(n, dtype=torch.int32)[:, None]], 1).cuda()
    own = torch.zeros((n, 1, 1, d), dtype=torch.bfloat16, device="cuda")
    q = rows((n, 4, 1, d), 3)
    c.append(own, own, table, i32([L] * n))
    out = c.attend_shared(q.cuda(), table, i32([L] * n), i32([0, n]), i32([L // P])).cpu()
    value = lambda codes, s: (codes[:L // P].float().cpu().double() * s[:L // P].cpu().double()[:, :, None, None]).reshape(L, d)  # noqa: E731
    kk, vv = value(c.k8, c.k_scale), value(c.v8, c.v_scale)
    x = q[:, :, 0].double() @ kk.T * float(np.float32(d ** -0.5))
    p = torch.exp(x)
    p = p / (p.sum(-1, keepdim=True) + 1)                          # (its own key: logit 0, value 0)
    want = p @ vv
    off = torch.sqrt((p * p) @ (vv * vv)) * math.sqrt(2.0 ** -22 / 3 + 2.0 ** -32)
    step = torch.exp2(torch.floor(torch.log2(want.abs())) - 7)
    chance = torch.clamp(off / step, max=1.0)                      # (the mean of |x| is no more than its standard deviation)
    others = (out[:, :, 0].double() != want.bfloat16().double()).sum().item()
    assert others <= chance.sum().item() + 6 * math.sqrt(chance.sum().item()), (others, chance.sum().item())


@pytest.mark.gpu
@pytest.mark.parametrize("n,d", [(8, 64), (70, 128)])
def test_results_are_the_same_every_time(kvm, n, d):
    """Also where references move for some rows in most tiles, alone and beside another call on a second stream."""
    P, L = 64, 4096
    c = kvm.Cache.empty(L // P + n, 2, d, P)
    u = torch.ones(d) / math.sqrt(d)
    k = (rows((1, 2, L, d), 1).float() * 0.3 + (torch.arange(L) // 130)[:, None] * 0.6 * u).bfloat16()
    head = torch.arange(L // P, dtype=torch.int32)[None]
    c.append(k.cuda(), rows((1, 2, L, d), 2).cuda(), head.cuda(), i32([0]))
    table = torch.cat([head.repeat(n, 1), L // P + torch.arange(n, dtype=torch.int32)[:, None]], 1).cuda()
    start = i32([L] * n)
    c.append(rows((n, 2, 1, d), 4).cuda(), rows((n, 2, 1, d), 5).cuda(), table, start)
    q = (rows((n, 8, 1, d), 3).float() + torch.linspace(0.0, 16.0, n * 8).view(n, 8, 1, 1) * u).bfloat16().cuda()
    args = (q, table, start, i32([0, n]), i32([L // P]))
    want = c.attend_shared(*args, scale=1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        with torch.cuda.stream(side):
            other = c.attend_shared(*args, scale=1.0)
        assert torch.equal(c.attend_shared(*args, scale=1.0).view(torch.int16), want.view(torch.int16))
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(other.view(torch.int16), want.view(torch.int16))
    assert not torch.isnan(want.float()).any()


@pytest.mark.gpu
@pytest.mark.parametrize("d,P,T,G,n,aligned", [(128, 64, 4, 4, 20, True), (64, 16, 6, 2, 40, True), (128, 32, 2, 4, 70, False), (64, 64, 70, 4, 6, False)])
def test_rows_behind_the_counts_reach_nothing(kvm, d, P, T, G, n, aligned):
    """Whatever the padding of q holds, every bit of the results in front of it is the same, and the rows of out behind it are left as they were."""
    Hkv, lead = 2, 40
    m = Shared(kvm, [n], [lead], [50 + b % 7 for b in range(n)], Hkv, d, P)
    counts = [b % T + (1 if b % 3 else 0) if b % 5 else 0 for b in range(n)]
    m.append(rows((n, Hkv, T, d), 1), rows((n, Hkv, T, d), 2), counts)
    q, start = rows((n, G * Hkv, T, d), 3).cuda(), i32([x - c for x, c in zip(m.len, counts)])
    live = (torch.arange(T)[None] < torch.tensor(counts)[:, None]).cuda()[:, None, :, None]
    want = None
    for i, fill in enumerate((0.0, 1.0, 50.0, 3e4, 1e38, math.inf, math.nan)):
        x = torch.where(live, q, rows(q.shape, 4).cuda() * 50.0 if i == 2 else torch.full_like(q, fill))
        if not aligned:
            wide = torch.empty((n, G * Hkv, T, d + 1), dtype=torch.bfloat16, device="cuda")
            wide[..., 1:] = x
            x = wide[..., 1:]
        out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
        m.cache.attend_shared(x, m.hidden(), start, m.groups, m.shared, i32(counts), out=out, status=status)
        assert status.item() == 0 and (torch.where(live, 7.0, out.float()) == 7.0).all()
        want = out if want is None else want
        assert torch.equal(out, want), (fill, int((out != want).sum()))
    m.compare(q.cpu(), want, counts, 0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("d,P,T,n", [(64, 16, 1, 1024), (128, 16, 4, 300), (64, 32, 2, 700), (128, 64, 1, 200)])
def test_offsets_of_many_groups_beside_the_first_tiles(kvm, d, P, T, n):
    """As many groups as sequences, each with blocks of its own behind its shared one: what a CTA knows of the groups is not where it loads tiles."""
    m = Shared(kvm, [1] * n, [1] * n, [3 * P + b % 40 for b in range(n)], 1, d, P, room=10)
    m.step(T, 4, [T] * n, 0)
    q, start, out = m.step(T, 4, [b % T + 1 for b in range(n)], 1)
    count = i32([b % T + 1 for b in range(n)])
    for _ in range(3):
        assert torch.equal(m.cache.attend_shared(q.cuda(), m.hidden(), start, m.groups, m.shared, count, out=torch.full_like(out, 7.0)), out)


def dealt(m, q, table, start, groups, shared):
    """How a call deals its key tiles: (those of a CTA, whether a CTA has tiles of one unit only), from the last 32 bytes that it leaves per sequence in the workspace."""
    L, c, B = m.lib, C.byref(m.CacheCall(table.data_ptr(), start.data_ptr(), None, table.shape[0], table.shape[1], q.shape[2])), table.shape[0]

    def run(cache):
        n = L.kvm_cache_shared_workspace(cache._ref, c, shared.numel(), q.shape[1])
        ws, out = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
        assert L.kvm_cache_attend_shared(cache._ref, c, groups.data_ptr(), shared.data_ptr(), shared.numel(), q.data_ptr(), q.shape[1], 1.0, out.data_ptr(), None, None,
                                         ws.data_ptr(), n, None, torch.cuda.current_stream().cuda_stream) == 0
        deal = set(ws[n - 32 * B:].view(torch.int32).view(B, 8)[:, 7].tolist())
        assert len(deal) == 1
        return deal.pop() >> 1, bool(ws[n - 4:].view(torch.int32).item() & 1)
    return run


@pytest.mark.gpu
@pytest.mark.parametrize("short,short_tiles,long,long_tiles,Hkv,share,whole", [
    (12, 2, 1, 256, 8, 43, True),            # (a length of the 32 fits: 96 units and 8 times six CTAs)
    (13, 2, 1, 256, 8, 16, False),           # (none does: the longest unit would be 256 tiles, an equal share is 16)
    (17, 2, 1, 256, 8, 16, False),
    (110, 1, 38, 60, 1, 60, True),           # (none does either, but an equal share of 17 tiles may lie in 17 units of one tile)
    (140, 1, 1, 40, 1, 5, True),             # (180 tiles: shares of 2, or of up to 5, and 140 + 40 / 5 are 148 CTAs)
    (142, 1, 1, 40, 1, 2, False)])           # (two more than there are)
def test_short_prompts_beside_long_documents(kvm, short, short_tiles, long, long_tiles, Hkv, share, whole):
    """No CTA gets a long unit whole where most units are short, and every row is right however the tiles are dealt."""
    d, P, G, per = 64, 128, 2, 2
    lead = [short_tiles] * (short // 2) + [long_tiles] * long + [short_tiles] * (short - short // 2)
    B, width = per * len(lead), max(lead) + 1
    c = kvm.Cache.empty(sum(lead) + B, Hkv, d, P)
    for i, (codes, scale) in enumerate(((c.k8, c.k_scale), (c.v8, c.v_scale))):       # values of +-2^-3 .. 2^1, scales of a few powers of two
        g = torch.Generator().manual_seed(i)
        codes.view(torch.uint8).copy_(torch.randint(0x20, 0x40, codes.shape, generator=g) | (torch.randint(0, 2, codes.shape, generator=g) << 7))
        scale.copy_(torch.exp2(torch.randint(-2, 2, scale.shape, generator=g).float()))
    table, at = torch.full((B, width), -1, dtype=torch.int32), 0
    for i, n in enumerate(lead):
        table[per * i:per * i + per, :n] = torch.arange(at, at + n)
        at += n
    for b in range(B):
        table[b, lead[b // per]] = at + b
    own = [1 + b % 90 for b in range(B)]
    start = i32([lead[b // per] * P + own[b] - 1 for b in range(B)])
    groups, shared, q, t = i32(list(range(0, B + 1, per))), i32(lead), rows((B, G * Hkv, 1, d), 3, outliers=False).cuda(), table.cuda()
    out, status = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), i32([0])
    c.attend_shared(q, t, start, groups, shared, scale=0.2, out=out, status=status)
    assert status.item() == 0
    for _ in range(3):
        assert torch.equal(c.attend_shared(q, t, start, groups, shared, scale=0.2), out)
    K, V = ((x.view(torch.float8_e4m3fn).float() * s[:, :, None, None]).cpu().double().numpy() for x, s in ((c.k8, c.k_scale), (c.v8, c.v_scale)))
    qn, on = q.float().cpu().double().numpy(), out.float().cpu().double().numpy()
    for b in range(B):
        n = lead[b // per] * P + own[b]
        pages = table[b, :lead[b // per] + 1].numpy()
        for h in range(Hkv):
            ref, bound = ec.attend(qn[b, G * h:G * h + G, 0], K[pages, h].reshape(-1, d)[:n], V[pages, h].reshape(-1, d)[:n], np.full(G, n - 1), float(np.float32(0.2)))
            assert (np.abs(on[b, G * h:G * h + G, 0] - ref) <= bound).all(), (b, h)
    assert dealt(kvm, q, t, start, groups, shared)(c) == (share, whole)


@pytest.mark.gpu
@pytest.mark.parametrize("d,P,T,moving", [(64, 16, 2, False), (128, 32, 1, True), (64, 64, 1, True), (128, 16, 3, True)])
def test_runs_of_tiles_through_units_of_all_lengths(kvm, d, P, T, moving):
    """More units than CTAs, of 1 to 20 tiles and 3 to 128 rows, the borders of the CTAs' shares anywhere in them: every row against the definition, with references that move in
    most of the units, the same every time, and with a NaN in one unit alone."""
    r = random.Random(d + P)
    Hkv, G, per = 3, 4, 128 // P
    sizes = [1, 2, 1, 45, 1, 3, 1, 1] + [r.choice([1, 1, 2, 3]) for _ in range(44)]
    lead = [per * (1 + i * 7 % 20) - r.choice([0, 0, per // 2, 1]) * (per > 1) for i in range(len(sizes))]
    lead = [max(1, x) for x in lead]
    n = sum(sizes)
    m = Shared(kvm, sizes, [0] * len(sizes), [0] * n, Hkv, d, P, room=max(lead) * P + 200)
    L = max(lead) * P
    k, v = rows((n, Hkv, L, d), 1), rows((n, Hkv, L, d), 2)
    u = torch.ones(d) / math.sqrt(d)
    if moving:                                                     # logits that grow from tile to tile, from another column on in every head, over blocks of several scales
        for h in range(Hkv):
            k[:, h] = (k[:, h].float() * 0.05 + ((torch.arange(L) + 43 * h) // 128)[:, None] * u).bfloat16()
        v = (v.float() * torch.exp2(((torch.arange(L) // P) % 5 - 2).float())[:, None]).bfloat16()
    counts = [0] * n
    for g in range(len(sizes)):
        counts[m.first[g]] = lead[g] * P
    m.append(k, v, counts)
    for g, size in enumerate(sizes):
        f = m.first[g]
        for b in range(f + 1, f + size):
            m.table[b, :lead[g]] = m.table[f, :lead[g]]
            m.k[b], m.v[b], m.len[b] = copy.deepcopy(m.k[f]), copy.deepcopy(m.v[f]), m.len[f]
    m.lead, m.shared = lead, i32(lead)
    own = [b % 37 for b in range(n)]
    m.append(rows((n, Hkv, 40, d), 5), rows((n, Hkv, 40, d), 6), own)
    m.append(rows((n, Hkv, T, d), 7), rows((n, Hkv, T, d), 8), [T] * n)
    q, scale = rows((n, Hkv * G, T, d), 9), None
    if moving:                                                     # up to 2^14 from tile to tile, for some rows downwards
        q, scale = (q.float() * 0.05 + torch.linspace(-3.0, 10.0, n * Hkv * G).view(n, Hkv * G, 1, 1) * u).bfloat16(), 1.0
    start, t, q = i32([x - T for x in m.len]), m.hidden(), q.cuda()
    tiles = sum(Hkv * -(-size * T * G // 128) * -(-x // per) for size, x in zip(sizes, lead))
    assert dealt(kvm, q, t, start, m.groups, m.shared)(m.cache) == (-(-tiles // 148), False)
    run = lambda: m.cache.attend_shared(q, t, start, m.groups, m.shared, scale=scale, out=torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), status=status)  # noqa: E731
    status = i32([0])
    out = run()
    assert status.item() == 0
    m.compare(q.cpu(), out, [T] * n, 0, 0, scale)
    for _ in range(10):
        assert torch.equal(run(), out)
    g = 20                                                         # (neither a CTA's first unit nor its last, wherever the shares end)
    m.cache.v_scale[m.table[m.first[g], lead[g] - 1], 1] = math.nan
    got, want = run(), torch.zeros((n, Hkv * G), dtype=torch.bool)
    want[m.first[g]:m.first[g] + sizes[g], G:2 * G] = True
    assert torch.equal(torch.isnan(got.float()).all(-1).all(-1).cpu(), want) and torch.equal(got[~want], out[~want])
