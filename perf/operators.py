"""Exact attention beside the compressed one: a cache of keys and values in 8 bits, in pages, the attention that reads it
(sliding window, first tokens that stay visible) and the copies of its pages, as cases to measure.

The cache is what the uncompressed layers of a hybrid stack keep: codes k8, v8 of e4m3 [n_pages, Hkv, page_tokens, d] and one
scale, a power of two, for each page ("block of tokens") and head, [n_pages, Hkv]; a page table [batch, max_pages] says where a
sequence's blocks are.  What a code stands for is code * scale.

  append  writes the rows of T new tokens behind the `start` tokens that each sequence has.  A block's scale is the least power
          of two 2^e, e >= -64, with amax <= 448 * 2^e over the rows that were written; where new rows raise it, the codes that
          the block holds are divided by the factor and rounded.
  attend  queries of T tokens at positions start .. start + T - 1 over the cache, which holds their own keys already: position i
          sees j <= i with j > i - window (window 0: all) or j < sinks.
  copy    pages to other pages: forks of sequences (beams, shared prompts), compaction.

T is the padded length of the call; with `ragged` the sequences have contexts and counts of their own, and rows behind a
sequence's count stay as they are.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
LEAST_EXP = -64


def _case(name=None, **kw):
    c = dict(op="attend", B=1, Hq=8, Hkv=8, d=128, P=64, T=1, ctx=0, ragged=False, window=0, sinks=0, pages=0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one token for each of 64 sequences: what every decode step of a served batch writes
        _case("append_decode_64", op="append", B=64, Hkv=8, ctx=4096, ragged=True),
        # prompts of odd lengths, small pages, 64 channels
        _case("append_prompts_ragged_d64", op="append", B=7, Hkv=5, d=64, P=16, T=1777, ctx=300, ragged=True),
        # long prompts of four sequences
        _case("append_prompts_4x8192", op="append", B=4, Hkv=32, T=8192),
        # one token of one sequence with a short context: launches and latency count
        _case("decode_1x1000", Hq=32, Hkv=8, ctx=1000),
        # a served batch with grouped queries and contexts of every length
        _case("decode_64_gqa_ragged", B=64, Hq=32, Hkv=8, ctx=16384, ragged=True),
        # long-context retrieval: one sequence, eight heads, 131072 tokens
        _case("decode_131k", Hq=8, Hkv=8, ctx=131071),
        # a window layer of a hybrid stack: window of two blocks of 256, four first tokens, a head of its own for every query head
        _case("decode_64_window512", B=64, Hq=32, Hkv=32, ctx=4096, ragged=True, window=512, sinks=4),
        # a turn of a conversation: 300 tokens behind 3000
        _case("prompt_turn_300", Hq=32, Hkv=8, T=300, ctx=3000),
        # two prompts of 8192 tokens, 16 heads
        _case("prompt_2x8192", B=2, Hq=16, Hkv=16, T=8192),
        # the same length through a window layer, 64 channels, ragged
        _case("prompt_window512_ragged_d64", B=3, Hq=16, Hkv=4, d=64, P=32, T=8192, ragged=True, window=512, sinks=4),
        # forks of 48 sequences: the last, partly filled page of each is copied
        _case("copy_last_pages_48", op="copy", Hkv=8, pages=48),
        # compaction: many pages move to the front of the pool
        _case("copy_2000_pages", op="copy", Hkv=8, pages=2000),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "copy"])
    d, P = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    Hkv = rng.choice([1, 2, 3, 4, 5, 8, 16])
    if op == "copy":
        return _case(op="copy", Hkv=Hkv, d=d, P=P, pages=_log_int(rng, 1, max(1, (1 << 17) // (Hkv * P))))
    G = rng.choice([1, 1, 2, 3, 4, 7, 8, 16])
    ragged = rng.random() < 0.6
    if op == "append":
        T = rng.choice([1, 1, _log_int(rng, 2, 8192)])
        B = _log_int(rng, 1, max(1, min(96, (1 << 20) // (T * Hkv))))
        return _case(op="append", B=B, Hkv=Hkv, d=d, P=P, T=T, ctx=rng.choice([0, _log_int(rng, 1, 4096)]), ragged=ragged)
    window, sinks = rng.choice([(0, 0), (0, 0), (_log_int(rng, 1, 4096), rng.choice([0, 1, 4, 130]))])
    kind = rng.choice(["token", "token", "few", "prompt"])
    if kind == "prompt":
        T = _log_int(rng, 16, 6000)
        ctx = rng.choice([0, _log_int(rng, 1, 6000)])
        B = _log_int(rng, 1, max(1, min(16, (1 << 29) // (T * (T + ctx) * Hkv * G))))
        while T * (T + ctx) * Hkv * G * B > 1 << 30:
            T, ctx = max(1, T // 2), ctx // 2
    else:
        T = 1 if kind == "token" else rng.choice([2, 3, 4, 5, 8])
        ctx = _log_int(rng, 1, 65536)
        B = _log_int(rng, 1, max(1, min(96, (1 << 22) // ((T + ctx) * Hkv))))
    return _case(B=B, Hq=Hkv * G, Hkv=Hkv, d=d, P=P, T=T, ctx=ctx, ragged=ragged, window=window, sinks=sinks)


def _lengths(c):
    """(tokens before the call, tokens of the call) of each sequence; with `ragged` spread evenly over the range."""
    if not c["ragged"]:
        return [c["ctx"]] * c["B"], [c["T"]] * c["B"]
    frac = [((b + 1) * 0.6180339887498949) % 1.0 for b in range(c["B"])]
    return [int(c["ctx"] * f) for f in frac], [max(1, int(c["T"] * (1.0 - 0.6 * f) + 0.5)) for f in reversed(frac)]


def _visible(c, start, count):
    """(query, key) pairs of one sequence, and the keys that some query of the call sees."""
    W, S = c["window"] or (1 << 40), c["sinks"]
    pairs = 0
    for p in range(start, start + count) if W < (1 << 40) else ():
        first = max(0, p + 1 - W)
        pairs += p + 1 - first + min(S, first)
    if W >= 1 << 40:
        pairs = count * start + count * (count + 1) // 2
    first = max(0, start + 1 - W)
    return pairs, start + count - first + min(S, first) if count else 0


def work(c):
    if c["op"] == "copy":
        return {"bytes": 2 * c["pages"] * c["Hkv"] * (2 * c["P"] * c["d"] + 8), "flops": 0}
    starts, counts = _lengths(c)
    if c["op"] == "append":
        rows = sum(counts) * c["Hkv"]
        return {"bytes": rows * c["d"] * 2 * (2 + 1), "flops": 4 * rows * c["d"]}
    pairs = keys = 0
    for s, n in zip(starts, counts):
        a, b = _visible(c, s, n)
        pairs, keys = pairs + a, keys + b
    return {"bytes": 2 * keys * c["Hkv"] * c["d"] + 4 * sum(counts) * c["Hq"] * c["d"], "flops": 4 * pairs * c["Hq"] * c["d"]}


def _rows(g, *shape):
    """bf16 rows as a projection gives them: normal, some channels larger than the others."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    return x * (1.0 + 2.0 * (torch.rand(shape[-1], generator=g, device="cuda") < 0.05)).to(torch.bfloat16)


def _pool(g, n, c):
    """Codes and scales of n pages that hold tokens already."""
    shape = (n, c["Hkv"], c["P"], c["d"])
    code = lambda: (torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) * 96).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.exp2(torch.randint(-8, -5, shape[:2], generator=g, device="cuda").float())  # noqa: E731
    return {"k8": code(), "v8": code(), "k_scale": scale(), "v_scale": scale()}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "copy":
        n = c["pages"]
        s = _pool(g, 2 * n + 3, c)
        ids = torch.randperm(2 * n + 3, generator=g, device="cuda").to(torch.int32)
        s.update(case=c, src=ids[:n].cpu(), dst=ids[n:2 * n].cpu(), src_dev=ids[:n].long(), dst_dev=ids[n:2 * n].long())
    else:
        starts, counts = _lengths(c)
        blocks = [-(-(s + n) // c["P"]) for s, n in zip(starts, counts)]
        # a window layer has given back the pages that no later token sees: their entries are -1
        W, S = c["window"] or (1 << 40), c["sinks"]
        live = [[i for i in range(m) if c["op"] == "append" or (i + 1) * c["P"] > s + 1 - W or i * c["P"] < S] for m, s in zip(blocks, starts)]
        if c["op"] == "append":   # only the blocks that the call writes need a page here
            live = [[i for i in range(m) if (i + 1) * c["P"] > s] for m, s in zip(blocks, starts)]
        total = sum(len(x) for x in live)
        s = _pool(g, total + 2, c)
        ids = torch.randperm(total + 2, generator=g, device="cuda")[:total].tolist()
        table = torch.full((c["B"], max(blocks)), -1, dtype=torch.int32)
        at = 0
        for b, x in enumerate(live):
            table[b, x] = torch.tensor(ids[at:at + len(x)], dtype=torch.int32)
            at += len(x)
        s.update(case=c, pages=table.cuda(), start=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                 count=torch.tensor(counts, dtype=torch.int32, device="cuda") if c["ragged"] else None)
        if c["op"] == "append":
            s["k"], s["v"] = _rows(g, c["B"], c["Hkv"], c["T"], c["d"]), _rows(g, c["B"], c["Hkv"], c["T"], c["d"])
        else:
            s["q"] = _rows(g, c["B"], c["Hq"], c["T"], c["d"])
            s["out"] = torch.zeros_like(s["q"])
    if own:
        from paper_2605_09877_b200 import kvm
        s["cache"] = kvm.Cache(s["k8"], s["v8"], s["k_scale"], s["v_scale"])
    return s


def run(state):
    s, c = state, state["case"]
    if c["op"] == "copy":
        if own:
            s["cache"].copy_pages(s["src"], s["dst"])
        else:
            for name in ("k8", "v8", "k_scale", "v_scale"):
                x = s[name].view(torch.uint8) if s[name].dtype == torch.float8_e4m3fn else s[name]
                x[s["dst_dev"]] = x[s["src_dev"]]
    elif c["op"] == "append":
        if own:
            s["cache"].append(s["k"], s["v"], s["pages"], s["start"], s["count"])
        else:
            _append(s, s["k"], s["k8"], s["k_scale"])
            _append(s, s["v"], s["v8"], s["v_scale"])
    else:
        if own:
            return s["cache"].attend(s["q"], s["pages"], s["start"], s["count"], window=c["window"], sinks=c["sinks"], out=s["out"])
        return _attend(s)
    return {"k8": s["k8"], "v8": s["v8"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# ---- plain forms ----------------------------------------------------------------------------------------------------------

def _append(s, rows, codes, scales):
    c = s["case"]
    B, Hkv, T, d = rows.shape
    P, dev = c["P"], rows.device
    start, count = s["start"].long(), torch.full_like(s["start"], T).long() if s["count"] is None else s["count"].long()
    npg = (T + P - 1) // P + 1                                       # blocks that T tokens can touch
    i = torch.arange(npg * P, device=dev)[None] - (start % P)[:, None]                   # [B, npg P] token of the call
    new = (i >= 0) & (i < count[:, None])
    at = i.clamp(0, T - 1)[:, None, :, None].expand(B, Hkv, npg * P, d)
    x = torch.where(new[:, None, :, None], rows.gather(2, at).float(), 0.0).view(B, Hkv, npg, P, d)
    block = (start // P)[:, None] + torch.arange(npg, device=dev)[None]                  # [B, npg]
    touched = new.view(B, npg, P).any(-1)
    page = s["pages"].long().gather(1, block.clamp(max=s["pages"].shape[1] - 1))
    b_at, n_at = touched.nonzero(as_tuple=True)
    page = page[b_at, n_at]                                                              # [N] pages written
    x, new = x[b_at, :, n_at], new.view(B, npg, P)[b_at, n_at]                           # [N, Hkv, P, d], [N, P]
    held = (torch.arange(P, device=dev)[None] < (start % P)[b_at][:, None]) & (n_at == 0)[:, None]   # rows of earlier calls
    amax = x.abs().amax((-1, -2))                                                        # [N, Hkv]
    m, e = torch.frexp(amax)                                                             # amax = m 2^e, m in [1/2, 1)
    e = torch.where(amax > 0, e - 9 + (m > 0.875).int(), LEAST_EXP).clamp(min=LEAST_EXP)
    scale = torch.exp2(e.float())
    old = scales[page]
    scale = torch.where(held.any(-1)[:, None], torch.maximum(scale, old), scale)
    c_old = codes.view(torch.uint8)[page].view(torch.float8_e4m3fn).float() * (old / scale)[..., None, None]
    value = torch.where(new[:, None, :, None], x / scale[..., None, None], c_old)
    keep = ~(new | held)[:, None, :, None]
    got = value.to(torch.float8_e4m3fn).view(torch.uint8)
    codes.view(torch.uint8)[page] = torch.where(keep, codes.view(torch.uint8)[page], got)
    scales[page] = scale


def _attend(s):
    c, q, pages = s["case"], s["q"], s["pages"].long().clamp(min=0)
    B, Hq, T, d = q.shape
    P, Hkv = c["P"], c["Hkv"]
    L, G, dev = pages.shape[1] * P, Hq // c["Hkv"], q.device
    start = s["start"].long()[:, None]
    count = torch.full_like(start, T) if s["count"] is None else s["count"].long()[:, None]
    def rows(codes, scale):
        x = codes.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float() * scale[pages][..., None, None]   # [B, blocks, Hkv, P, d]
        return x.transpose(1, 2).reshape(B, Hkv, L, d)
    j = torch.arange(L, device=dev)[None]
    at = start + torch.arange(T, device=dev)[None]                                       # [B, T] positions
    see = j[:, None] <= at[..., None]
    if c["window"]:
        see &= (j[:, None] > at[..., None] - c["window"]) | (j[:, None] < c["sinks"])
    z = q.float().view(B, Hkv, G * T, d) @ rows(s["k8"], s["k_scale"]).transpose(-1, -2)
    z = z.view(B, Hkv, G, T, L).mul_(1.0 / math.sqrt(d)).masked_fill_(~see[:, None, None], -math.inf)
    z = z.sub_(z.amax(-1, keepdim=True)).exp_()
    den = z.sum(-1, keepdim=True)
    v = rows(s["v8"], s["v_scale"]).masked_fill_((j >= start + count)[:, None, :, None], 0.0)
    o = ((z.view(B, Hkv, G * T, L) @ v).view(B, Hkv, G, T, d) / den).view(B, Hq, T, d)
    live = (torch.arange(T, device=dev)[None] < count)[:, None, :, None]
    s["out"].copy_(torch.where(live, o.to(torch.bfloat16), s["out"]))
    return s["out"]


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------

def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "copy":
        r = {n: s[n].double().clone() for n in ("k8", "v8", "k_scale", "v_scale")}
        for x in r.values():
            x[s["dst_dev"]] = x[s["src_dev"]]
        return r
    start = s["start"].tolist()
    count = s["count"].tolist() if s["count"] is not None else [c["T"]] * c["B"]
    table = s["pages"].tolist()
    P, Hkv, d = c["P"], c["Hkv"], c["d"]
    if c["op"] == "append":
        r = {n: s[n].double() for n in ("k8", "v8", "k_scale", "v_scale")}
        for kind in "kv":
            code, scale = r[kind + "8"], r[kind + "_scale"]
            for b in range(c["B"]):
                done = 0
                while done < count[b]:
                    block, r0 = divmod(start[b] + done, P)
                    n, page = min(P - r0, count[b] - done), table[b][block]
                    x = s[kind][b, :, done:done + n].double()                            # [Hkv, n, d]
                    top = x.abs().amax((1, 2))
                    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -200) / E4M3_MAX) - 0.25)    # least power, or one below it
                    e = torch.where(top > E4M3_MAX * 2.0 ** e, e + 1, e)
                    new = 2.0 ** torch.where(top > E4M3_MAX * 2.0 ** e, e + 1, e).clamp(min=LEAST_EXP)
                    if r0:
                        new = torch.maximum(new, scale[page])
                        code[page, :, :r0] = (code[page, :, :r0] * (scale[page] / new)[:, None, None]).to(torch.float8_e4m3fn).double()
                    code[page, :, r0:r0 + n] = (x / new[:, None, None]).to(torch.float8_e4m3fn).double()
                    scale[page] = new
                    done += n
        return r
    out = torch.zeros_like(s["q"], dtype=torch.float64)
    G = c["Hq"] // Hkv
    for b in range(c["B"]):
        end = start[b] + count[b]
        ids = [max(0, p) for p in table[b][:-(-end // P)]]
        ids = torch.tensor(ids, device="cuda")
        k8, v8 = (s[n].view(torch.uint8)[ids].view(torch.float8_e4m3fn) for n in ("k8", "v8"))
        pos = torch.arange(start[b], end, device="cuda")[:, None]
        key = torch.arange(end, device="cuda")[None]
        hidden = key > pos
        if c["window"]:
            hidden |= (pos - key >= c["window"]) & (key >= c["sinks"])
        for h in range(Hkv):
            k = (k8[:, h].double() * s["k_scale"][ids, h].double()[:, None, None]).reshape(-1, d)[:end]
            v = (v8[:, h].double() * s["v_scale"][ids, h].double()[:, None, None]).reshape(-1, d)[:end]
            for g in range(G):
                z = s["q"][b, h * G + g, :count[b]].double() @ k.T / d ** 0.5
                z[hidden] = -math.inf
                w = torch.exp(z - z.max(1, keepdim=True).values)
                out[b, h * G + g, :count[b]] = (w @ v) / w.sum(1, keepdim=True)
    return out
