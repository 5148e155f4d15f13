"""Exact attention over the 8-bit cache where its loops are long and its borders are sharp: workers that take many tiles, prompts that see many,
and rows in which one key more or less shows at once.  Against the fp64 definition in oracle/exact_cache.py."""
import numpy as np
import pytest
import torch

from oracle import exact_cache as ec
from tests.test_cache import Model, kvm, rows  # noqa: F401  (kvm: a fixture)

SMS = 148


def filled(kvm, B, Hkv, d, P, lengths, seed):
    """A cache with `lengths` tokens per sequence, whose pages lie in any order, and its table.  (Written by the library: what append writes is
    compared with the definition elsewhere, here the rows of a few heads are read back from the codes.)"""
    blocks = -(-max(lengths) // P)
    used = [-(-n // P) for n in lengths]
    ids = torch.randperm(sum(used) + 2, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    cache = kvm.Cache.empty(sum(used) + 2, Hkv, d, P)
    table, at = torch.full((B, blocks), -1, dtype=torch.int32), 0
    for b, n in enumerate(used):
        table[b, :n] = ids[at:at + n]
        at += n
    table = table.cuda()
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda: torch.randn((B, Hkv, max(lengths), d), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    cache.append(draw(), draw() + 0.25, table, torch.zeros(B, dtype=torch.int32, device="cuda"), torch.tensor(lengths, dtype=torch.int32).cuda())
    return cache, table


def held(cache, table, b, h, n):
    """The first n rows of a sequence and head in fp64: code * scale."""
    out = []
    for codes, scale in ((cache.k8, cache.k_scale), (cache.v8, cache.v_scale)):
        ids = table[b, :-(-n // cache.page_tokens)].long()
        x = codes.view(torch.uint8)[ids, h].view(torch.float8_e4m3fn).double() * scale[ids, h].double()[:, None, None]
        out.append(x.reshape(-1, cache.head_dim)[:n].cpu().numpy())
    return out


def attend_and_compare(cache, table, lengths, counts, q, window, sinks, pairs):
    B, Hq, T, d = q.shape
    G = Hq // cache.n_kv_heads
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    start = torch.tensor([n - c for n, c in zip(lengths, counts)], dtype=torch.int32).cuda()
    cache.attend(q, table, start, torch.tensor(counts, dtype=torch.int32).cuda(), window=window, sinks=sinks, out=out, status=status)
    again = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    cache.attend(q, table, start, torch.tensor(counts, dtype=torch.int32).cuda(), window=window, sinks=sinks, out=again)
    assert status.item() == 0 and torch.equal(out, again)
    for b in range(B):
        assert (out[b, :, counts[b]:] == 7.0).all() and torch.isfinite(out[b].float()).all()
    for b, h in pairs:
        n, c = lengths[b], counts[b]
        if c == 0:
            continue
        K, V = held(cache, table, b, h, n)
        qn = q[b, h * G:(h + 1) * G, :c].double().cpu().numpy().reshape(-1, d)
        ref, bound = ec.attend(qn, K, V, np.tile(np.arange(n - c, n), G), float(np.float32(d ** -0.5)), window, sinks)
        err = np.abs(out[b, h * G:(h + 1) * G, :c].double().cpu().numpy().reshape(-1, d) - ref)
        assert (err <= bound).all(), (b, h, float((err / bound).max()))


def tiles_seen(length, count, P, window, sinks):
    """Key tiles of 128 that the call's tokens of a sequence see, made of whole pages."""
    if not count:
        return 0
    first = max(0, length - count - window + 1) // P if window else 0
    pages = min(first, -(-sinks // P)) + -(-length // P) - first
    return -(-pages * P // 128)


# B, Hq, Hkv, d, P, least and most tokens, tokens of the call, window, sinks: calls of at most 8 and of 9 to 16 (token, head) columns
LONG = [
    (24, 32, 8, 128, 16, 1500, 6000, 1, 0, 0), (24, 8, 8, 128, 128, 1500, 6000, 1, 0, 0), (20, 24, 8, 128, 64, 2000, 5000, 2, 0, 0),
    (20, 64, 8, 128, 64, 2000, 6000, 2, 0, 0), (24, 32, 8, 128, 16, 1000, 5000, 4, 0, 0), (16, 80, 5, 128, 32, 3000, 9000, 1, 0, 0),
    (24, 64, 8, 64, 64, 1500, 6000, 1, 0, 0), (24, 8, 8, 64, 16, 1500, 6000, 3, 0, 0), (20, 64, 8, 64, 32, 2000, 6000, 2, 0, 0), (24, 24, 8, 64, 128, 1000, 5000, 5, 0, 0),
    (64, 16, 16, 128, 64, 10, 4000, 1, 700, 5), (64, 32, 16, 128, 16, 10, 4000, 4, 600, 130), (64, 16, 16, 64, 128, 10, 4000, 7, 900, 1), (64, 64, 16, 64, 16, 10, 4000, 4, 700, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,d,P,low,high,T,window,sinks", LONG)
def test_workers_that_take_many_tiles(kvm, B, Hq, Hkv, d, P, low, high, T, window, sinks):  # noqa: F811
    """A worker takes at least six tiles, so its ring turns over several times, results are rescaled from tile to tile, and units end and begin in
    the middle of its share."""
    lengths = [low + (high - low) * ((7 * b + 3) % B) // B for b in range(B)]
    counts = [T if b % 5 or T == 1 else (b // 5) % (T + 1) for b in range(B)]
    lengths = [max(n, c) for n, c in zip(lengths, counts)]
    cols = T * Hq // Hkv
    assert cols <= 16
    total = Hkv * sum(tiles_seen(n, c, P, window, sinks) for n, c in zip(lengths, counts))
    assert -(-total // (SMS * (4 if cols <= 8 else 3))) >= 6
    cache, table = filled(kvm, B, Hkv, d, P, lengths, seed=d + P + T)
    g = torch.Generator(device="cuda").manual_seed(9)
    q = torch.randn((B, Hq, T, d), generator=g, device="cuda").to(torch.bfloat16)
    pairs = [(b, (3 * b) % Hkv) for b in range(B)] + [(b, h) for b in (0, B - 1) for h in range(Hkv)]
    attend_and_compare(cache, table, lengths, counts, q, window, sinks, pairs)


@pytest.mark.gpu
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16), (64, 128)])
def test_references_that_rise_and_fall_along_a_workers_tiles(kvm, d, P):  # noqa: F811
    """One token per sequence over keys whose logits climb by far from tile to tile, then fall, with values of rising and falling scale."""
    B, H, n = 24, 8, 4000
    cache, table = filled(kvm, B, H, d, P, [n] * B, seed=5)
    step = torch.arange(cache.n_pages, device="cuda", dtype=torch.float32)[:, None]
    cache.k_scale.mul_(torch.exp2(torch.floor(3 * torch.sin(step))))
    cache.v_scale.mul_(torch.exp2(torch.floor(12 * torch.sin(1.7 * step))))
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((B, 2 * H, 1, d), generator=g, device="cuda").to(torch.bfloat16)
    attend_and_compare(cache, table, [n] * B, [1] * B, q, 0, 0, [(b, b % H) for b in range(B)])


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,d,P,length,T,window,sinks", [
    (2, 16, 16, 128, 64, 3000, 2600, 0, 0), (3, 16, 4, 64, 16, 4100, 1700, 0, 0), (2, 16, 8, 128, 16, 4500, 2500, 2900, 70), (1, 32, 4, 64, 128, 5000, 1300, 0, 0)])
def test_prompts_that_see_many_tiles(kvm, B, Hq, Hkv, d, P, length, T, window, sinks):  # noqa: F811
    """More row tiles than are split, each with twenty key tiles and more: every ring of the kernel turns over several times."""
    lengths = [length - 131 * b for b in range(B)]
    assert B * Hkv * -(-T * (Hq // Hkv) // 128) > 4 * SMS // 2 and min(tiles_seen(n, 1, P, window, sinks) for n in lengths) >= 20
    cache, table = filled(kvm, B, Hkv, d, P, lengths, seed=T)
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn((B, Hq, T, d), generator=g, device="cuda").to(torch.bfloat16)
    attend_and_compare(cache, table, lengths, [T - 57 * b for b in range(B)], q, window, sinks, [(0, 0), (B - 1, Hkv - 1)])


# ---- borders of what a token sees ------------------------------------------------------------------------------------


def marks(n, T, window, sinks):
    """Positions next to every border of what the last T of n tokens see, for the first and for the last of them."""
    at = {0, n - 1, n - 2}
    for p in (n - T, n - 1):
        at |= {p, p + 1}
        if window:
            at |= {p - window, p - window + 1, sinks - 1, sinks}
    return sorted(x for x in at if 0 <= x < n)


def marked_rows(n, d, at):
    """Keys and values with one heavy key at each marked position, each with a channel of its own."""
    k, v = torch.zeros((1, 1, n, d)), torch.full((1, 1, n, d), 0.0)
    v[..., 0] = 1.0
    for i, x in enumerate(at):
        k[0, 0, x, 0] = 1.0
        v[0, 0, x, 1 + i] = 8.0
    return k.to(torch.bfloat16), v.to(torch.bfloat16)


def marked_query(G, T, d, n):
    """A logit of ln(n) for the heavy keys (scale 1): each weighs as much as all the others together."""
    q = torch.zeros((1, G, T, d))
    q[..., 0] = float(np.log(n))
    return q.to(torch.bfloat16)


BORDERS = [(n, T, G, d, P, window, sinks) for n, P in ((2100, 64), (2101, 16), (900, 128)) for T, G, d in ((1, 1, 128), (1, 8, 64), (1, 16, 128), (3, 4, 64), (40, 2, 128))
           for window, sinks in ((0, 0), (100, 0), (130, 5), (512, 4), (128, 130))]


def test_marked_rows_show_every_border_taken_wrongly():
    """Mistakes planted in the definition: a window or first tokens by one too many or too few, the first or last key lost, exceed the bound by far."""
    for n, T, G, d, P, window, sinks in BORDERS:
        k, v = (x[0, 0].double().numpy() for x in marked_rows(n, d, marks(n, T, window, sinks)))
        q, pos = marked_query(1, T, d, n)[0, 0].double().numpy(), np.arange(n - T, n)
        ref, bound = ec.attend(q, k, v, pos, 1.0, window, sinks)
        wrong = []
        if window:
            wrong += [ec.attend(q, k, v, pos, 1.0, window + e, sinks)[0] for e in (-1, 1)]
            wrong += [ec.attend(q, k, v, pos, 1.0, window, sinks + e)[0] for e in (-1, 1) if sinks + e >= 0]
        lost = k.copy(), v.copy()
        lost[0][0, 0] = -4.0                           # (the first key weighs next to nothing)
        if not window or sinks:
            wrong.append(ec.attend(q, *lost, pos, 1.0, window, sinks)[0])
        if T > 1:
            wrong.append(ec.attend(q, k, v, np.minimum(pos + 1, n - 1), 1.0, window, sinks)[0])
        for w in wrong:
            assert (np.abs(w - ref) / bound).max() > 4, (n, T, window, sinks)


@pytest.mark.gpu
@pytest.mark.parametrize("n,T,G,d,P,window,sinks", BORDERS)
def test_borders_of_what_a_token_sees(kvm, n, T, G, d, P, window, sinks):  # noqa: F811
    m = Model(kvm, 1, 1, d, P, -(-n // P) + 1)
    k, v = marked_rows(n, d, marks(n, T, window, sinks))
    m.append(k, v, [n])
    m.attend(marked_query(G, T, d, n), [T], window, sinks, scale=1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,P", [(1, 128, 64), (3, 64, 16), (300, 128, 128), (300, 64, 16)])
def test_positions_up_to_the_largest(kvm, T, d, P):  # noqa: F811
    """A stream that a window layer has followed to the last position that a call may name: the same bits as the same rows near the front."""
    B, Hq, Hkv, W, S = 1, 8, 2, 500, 5
    width = (1 << 30) // P                             # the widest table
    near = 40 * P
    far = near + ((1 << 30) - T - near) // P * P        # the same place within a page
    blocks = (W + T) // P + 3
    g = torch.Generator().manual_seed(T)
    k, v, q = (torch.randn((B, h, n, d), generator=g).to(torch.bfloat16).cuda() for h, n in ((Hkv, W + T), (Hkv, W + T), (Hq, T)))
    out = []
    for at in (near, far):
        assert at % P == near % P and at + T <= 1 << 30
        cache = kvm.Cache.empty(blocks + 2, Hkv, d, P)
        table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        first = (at - W) // P
        used = -(-(at + T) // P) - first
        table[0, first:first + used] = torch.arange(1, used + 1, dtype=torch.int32, device="cuda")
        table[0, 0] = 0
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        place = lambda x: torch.tensor([x], dtype=torch.int32).cuda()  # noqa: E731
        cache.append(k[:, :, :S], v[:, :, :S], table, place(0), status=status)
        cache.append(k, v, table, place(at - W), status=status)
        out.append(cache.attend(q, table, place(at), window=W, sinks=S, status=status))
        assert status.item() == 0
    assert torch.isfinite(out[0].float()).all() and out[0].float().abs().max() > 0.05 and torch.equal(*out)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    still = torch.full_like(q, 7.0)
    cache.attend(q, table, torch.tensor([(1 << 30) - T + 1], dtype=torch.int32).cuda(), window=W, sinks=S, out=still, status=status)
    assert status.item() == 1 and (still == 7.0).all()
