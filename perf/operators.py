"""Attention over blocks of 64 tokens, as cases that can be timed and compared: the selection of blocks by a cheap score with the
attention that reads only those (prefill and training), a cache of blocks held in 8 bits with the single-token attention
over it, and the eviction of blocks by accumulated attention weight.

A case is one pass as a user's program makes it.  Distributions are those of perf/cases.py: q, k, v ~ N(0,1)/sqrt(d); where
blocks are selected, keys carry a drift that is shared inside a stretch of text, so that neighbouring queries agree in part on
what they select.  Softmax scales are such that the logits spread by about 2, as in trained layers.
"""
import math

import torch

own = False

BLOCK = 64      # tokens per block
TINY = 2.0 ** -100   # a block whose largest value is below this is held as zeros


# ---- the cases -------------------------------------------------------------------------------------------------------------

def _prefill(B, H, Hkv, n, d, top):
    return dict(kind="prefill", B=B, H=H, Hkv=Hkv, n=n, d=d, top=top)


def _train(B, H, Hkv, n, d, top):
    return dict(kind="train", B=B, H=H, Hkv=Hkv, n=n, d=d, top=top)


def _decode(B, H, Hkv, d, longest, format, top=0):
    return dict(kind="decode", B=B, H=H, Hkv=Hkv, d=d, longest=longest, format=format, top=top)


def _fill(B, Hkv, c, d, format):
    return dict(kind="fill", B=B, Hkv=Hkv, c=c, d=d, format=format)


def _evict(B, Hkv, blocks, budget, sink, recent):
    return dict(kind="evict", B=B, Hkv=Hkv, blocks=blocks, budget=budget, sink=sink, recent=recent)


def listed():
    cases = {
        # one short head: the smallest prefill, a unit of development and of tests
        "prefill_one_head": _prefill(1, 1, 1, 1000, 64, 4),
        # a batch of prompts of a length nobody chose, four query heads to a key/value head
        "prefill_ragged": _prefill(2, 16, 4, 5003, 128, 12),
        # a long document, grouped heads, 16 blocks and the query's own: as many keys as k = 1024 selected ones
        "prefill_long": _prefill(1, 32, 8, 32768, 128, 16),
        # training of a mid-size layer at 8 K tokens, a key/value head for every query head
        "train_layer": _train(4, 16, 16, 8192, 128, 8),
        # training of a GPT-2-small-shaped layer, ragged length
        "train_gpt2": _train(4, 12, 12, 2000, 64, 4),
        # one token for each of two short conversations: latency
        "decode_short": _decode(2, 4, 4, 64, 200, "int8"),
        # one token for one user with a long document: the work of a few heads split over the whole chip
        "decode_one": _decode(1, 32, 8, 128, 32768, "int8"),
        # one token for each of 64 users of all lengths: throughput of a serving batch
        "decode_batch": _decode(64, 32, 8, 128, 8192, "e4m3"),
        # one token for each of 16 users with long documents, of which each reads 16 blocks
        "decode_selected": _decode(16, 32, 8, 128, 65536, "e4m3", top=16),
        # the keys and values of four prompts go into the cache
        "fill_prompts": _fill(4, 8, 8192, 128, "int8"),
        # one user's cache is brought back to its budget
        "evict_one": _evict(1, 8, 129, 128, 1, 8),
        # a batch of long prompts is brought to a quarter of its blocks
        "evict_batch": _evict(64, 8, 2048, 512, 1, 16),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    H = rng.choice([4, 8, 12, 16, 25, 32])
    return H, rng.choice([h for h in range(1, H + 1) if H % h == 0])


def draw(rng):
    while True:
        kind = rng.choice(["prefill", "prefill", "train", "train", "decode", "decode", "decode", "fill", "evict"])
        B, (H, Hkv), d, top = rng.choice([1, 1, 2, 3, 4, 8]), _heads(rng), rng.choice([64, 128, 128]), _log(rng, 2, 16)
        format = rng.choice(["int8", "e4m3"])
        if kind in ("prefill", "train"):
            n = _log(rng, 300, 32768 if kind == "prefill" else 8192)
            cost = B * H * n * (top + 1) * d
            if cost <= (32 * 32768 * 17 * 128 if kind == "prefill" else 4 * 16 * 8192 * 9 * 128) and B * Hkv <= 64:
                return (_prefill if kind == "prefill" else _train)(B, H, Hkv, n, d, top)
        elif kind == "decode":
            B, longest = rng.choice([1, 1, 2, 4, 8, 17, 32, 64]), _log(rng, 70, 65536)
            if B * Hkv * longest * d <= 64 * 8 * 8192 * 128:
                return _decode(B, H, Hkv, d, longest, format, top if rng.random() < 0.4 else 0)
        elif kind == "fill":
            c = _log(rng, 100, 32768)
            if B * Hkv * c * d <= 4 * 8 * 8192 * 128:
                return _fill(B, Hkv, c, d, format)
        else:
            blocks, B = _log(rng, 20, 2048), rng.choice([1, 2, 5, 16, 64])
            if B * Hkv <= 512:
                budget = rng.randint(12, blocks)
                return _evict(B, Hkv, blocks, budget, rng.randint(0, 2), rng.randint(1, 10))


def work(c):
    if c["kind"] in ("prefill", "train"):
        B, H, Hkv, n, d, top = (c[x] for x in ("B", "H", "Hkv", "n", "d", "top"))
        past = sum(min(top, i // BLOCK) for i in range(n)) * BLOCK
        pairs = past + sum(i % BLOCK + 1 for i in range(n))            # attended (query, key) pairs of a head
        cheap = 2.0 * B * Hkv * d * sum(i // BLOCK for i in range(n))   # the cheap score
        qs, ks = B * H * n * d * 2.0, B * Hkv * n * d * 2.0
        if c["kind"] == "prefill":
            return {"bytes": 2 * qs + 2 * ks + 4.0 * B * H * n + 4.0 * B * Hkv * (n * top + -(-n // BLOCK)),
                    "flops": 4.0 * B * H * pairs * d + cheap}
        return {"bytes": 5 * qs + 6 * ks + 4.0 * B * H * n + 4.0 * B * Hkv * n * top, "flops": 14.0 * B * H * pairs * d + cheap}
    if c["kind"] == "decode":
        B, H, Hkv, d, top = (c[x] for x in ("B", "H", "Hkv", "d", "top"))
        tokens = blocks = 0
        for n in _lens(c):
            n += 1
            blocks += (n - 1) // BLOCK if top else 0
            tokens += min(top, (n - 1) // BLOCK) * BLOCK + (n - 1) % BLOCK + 1 if top else n
        return {"bytes": 2.0 * Hkv * tokens * d + Hkv * blocks * d + 4.0 * B * H * d + 4.0 * B * Hkv * d, "flops": 4.0 * H * tokens * d}
    if c["kind"] == "fill":
        return {"bytes": 6.0 * c["B"] * c["Hkv"] * c["c"] * c["d"], "flops": 0.0}
    return {"bytes": 16.0 * c["B"] * c["Hkv"] * c["blocks"], "flops": 0.0}


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _drifting(B, H, n, d, g):
    """N(0,1) plus a part that is shared by the heads of a stretch of 512 tokens."""
    x = torch.randn(B, H, n, d, device="cuda", generator=g)
    topic = torch.randn(B, 1, -(-n // 512), d, device="cuda", generator=g)
    return x + 0.5 * topic.repeat_interleave(512, 2)[:, :, :n]


def _lens(c):
    """Tokens of every sequence ahead of the step: all lengths up to the longest, the first one the longest."""
    return [max(1, c["longest"] - 1 - (c["longest"] * b * 5 // (6 * c["B"]))) for b in range(c["B"])]


def _empty_cache(B, Hkv, cap, d, format, g):
    t = torch.int8 if format == "int8" else torch.float8_e4m3fn
    pages = B * Hkv * cap
    byte = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda").view(t)   # noqa: E731
    zero = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    return dict(k8=byte(pages, BLOCK, d), v8=byte(pages, d, BLOCK), ks=zero(pages), vs=zero(pages), km=zero(pages, d, dt=torch.int8),
                kms=zero(pages), kt=zero(B, Hkv, BLOCK, d, dt=torch.bfloat16), vt=zero(B, Hkv, d, BLOCK, dt=torch.bfloat16),
                table=torch.randperm(pages, device="cuda", generator=g).to(torch.int32).view(B, Hkv, cap), mass=zero(B, Hkv, cap))


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    s = dict(case=c)
    if c["kind"] in ("prefill", "train"):
        B, H, Hkv, n, d = (c[x] for x in ("B", "H", "Hkv", "n", "d"))
        s["scale"] = 2.0 * math.sqrt(d)
        s["q"], s["k"], s["v"] = ((x / d ** 0.5).bfloat16() for x in (_drifting(B, H, n, d, g), _drifting(B, Hkv, n, d, g), rnd(B, Hkv, n, d)))
        if c["kind"] == "train":
            s["dO"] = rnd(B, H, n, d).bfloat16()
    elif c["kind"] == "decode":
        B, H, Hkv, d = (c[x] for x in ("B", "H", "Hkv", "d"))
        cap = c["longest"] // BLOCK + 1
        s["scale"] = 2.0 * math.sqrt(d)
        s["cache"] = k = _empty_cache(B, Hkv, cap, d, c["format"], g)
        if c["format"] == "int8":   # what a block's rounding leaves: its largest value is 127
            for x in ("k8", "v8"):
                k[x].copy_((rnd(*k[x].shape) * 30).round_().clamp_(-127, 127))
        else:
            for x in ("k8", "v8"):
                k[x].copy_((rnd(*k[x].shape) * 100).clamp_(-448, 448).to(torch.float8_e4m3fn))
        top = 30.0 if c["format"] == "int8" else 100.0
        for x in ("ks", "vs"):   # the scale gives back N(0,1)/sqrt(d), some blocks louder than others
            k[x].copy_(torch.exp(0.2 * rnd(*k[x].shape)) / (top * d ** 0.5))
        k["km"].copy_((rnd(*k["km"].shape) * 40).round_().clamp_(-127, 127))
        k["kms"].copy_(torch.exp(0.2 * rnd(*k["kms"].shape)) / (40 * 8 * d ** 0.5))
        k["kt"].copy_(rnd(*k["kt"].shape) / d ** 0.5)
        k["vt"].copy_(rnd(*k["vt"].shape) / d ** 0.5)
        k["mass"].copy_(rnd(*k["mass"].shape).abs())
        s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
        s["after"] = s["lens"] + 1
        s["q"] = (rnd(B, H, d) / d ** 0.5).bfloat16()
        s["k"], s["v"] = ((rnd(B, Hkv, 1, d) / d ** 0.5).bfloat16() for _ in range(2))
    elif c["kind"] == "fill":
        B, Hkv, n, d = (c[x] for x in ("B", "Hkv", "c", "d"))
        s["cache"] = _empty_cache(B, Hkv, n // BLOCK + 1, d, c["format"], g)
        s["lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        counts = [n] + [max(1, n - n * b // (2 * B) - 7 * b) for b in range(1, B)]   # prompts of several lengths, padded to the longest
        s["counts"] = torch.tensor(counts, dtype=torch.int32, device="cuda")
        s["k"], s["v"] = (((rnd(B, Hkv, n, d)) / d ** 0.5).bfloat16() for _ in range(2))
    else:
        B, Hkv, n = (c[x] for x in ("B", "Hkv", "blocks"))
        s["cache"] = k = _empty_cache(B, Hkv, n, 64, "int8", g)
        k["mass"].copy_(torch.exp(2.0 * rnd(B, Hkv, n)))
        k["mass"][rnd(B, Hkv, n) < -1.0] = 0.0     # blocks that nobody has looked at: ties
        lens = [n * BLOCK + 17 - (0 if b % 4 else 64 * (b % (n // 2))) for b in range(B)]
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["out"] = dict(table=torch.empty_like(k["table"]), mass=torch.empty_like(k["mass"]), lens=torch.empty_like(s["lens"]))
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------------

def _in8(x):
    """Rounded to whole numbers of at most 127 along the last dimension, and the scale."""
    top = x.abs().amax(-1, keepdim=True)
    some = top >= TINY
    codes = torch.where(some, (x * (127.0 / torch.where(some, top, 1.0))).round_().clamp_(-127, 127), 0.0)
    return codes, torch.where(some, top / 127.0, 0.0).squeeze(-1)


def _means(k):
    """The mean key of every whole block, in 8 bits: [.., blocks, d] whole numbers in fp32 and [.., blocks] scales."""
    B, Hkv, n, d = k.shape
    nb = n // BLOCK
    return _in8((k[:, :, :nb * BLOCK].view(B, Hkv, nb, BLOCK, d).double().sum(3) / BLOCK).float())


def _top_of(score, allowed, top):
    """The positions of the `top` largest allowed scores in ascending order, padded with -1; of equal ones the lowest."""
    N = score.shape[-1]
    score = torch.where(allowed, score, float("-inf"))
    at = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :top]
    at = torch.where(torch.gather(allowed.expand(score.shape), -1, at), at, N).sort(-1).values
    at = torch.where(at < N, at, -1).to(torch.int32)
    return torch.nn.functional.pad(at, (0, top - at.shape[-1]), value=-1)


def _select(q, k, top):
    B, H, n, d = q.shape
    Hkv = k.shape[1]
    pooled = _in8(q.view(B, Hkv, H // Hkv, n, d).double().sum(2).float())[0]
    m, ms = _means(k)
    score = (pooled @ m.transpose(-1, -2).contiguous()) * ms.unsqueeze(-2)
    i, j = torch.arange(n, device=q.device), torch.arange(m.shape[2], device=q.device)
    return _top_of(score, j < (i // BLOCK).unsqueeze(-1), top)


def _gathered(x, idx):
    """[n, (top + 1) * 64, d]: the rows of the selected blocks of every query and of its own, of one head, and which of them are attended."""
    n, d = x.shape
    i = torch.arange(n, device=x.device)
    blocks = torch.cat([idx.long(), (i // BLOCK).unsqueeze(-1)], -1)
    at = (blocks.unsqueeze(-1) * BLOCK + torch.arange(BLOCK, device=x.device)).view(n, -1)
    ok = (at >= 0) & (at <= i.unsqueeze(-1))
    return at.clamp_(0, n - 1), ok


def _attend_head(q, k, v, idx, scale):
    """One key/value head: q [G, n, d]; o, lse, the probabilities [n, G, keys] and what was attended, all in fp32."""
    at, ok = _gathered(k, idx)
    kg = k[at]                                                       # [n, keys, d]
    s = torch.bmm(q.transpose(0, 1), kg.transpose(1, 2)) * scale
    s = torch.where(ok.unsqueeze(1), s, float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    p = p / total
    o = torch.bmm(p, v[at])
    return o.transpose(0, 1), (top + torch.log(total)).squeeze(-1).transpose(0, 1), p, at, ok


def _block_attn(q, k, v, idx, scale):
    B, H, n, d = q.shape
    Hkv = k.shape[1]
    o, lse = torch.empty_like(q), torch.empty(B, H, n, device=q.device)
    nb = -(-n // BLOCK)
    mass = torch.zeros(B, Hkv, nb, device=q.device)
    for b, g in ((b, g) for b in range(B) for g in range(Hkv)):   # (a head at a time: the gathered keys of all would not fit)
        hs = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
        oh, lh, p, at, ok = _attend_head(q[b, hs].float(), k[b, g].float(), v[b, g].float(), idx[b, g], scale)
        o[b, hs], lse[b, hs] = oh.to(q.dtype), lh
        w = torch.where(ok, p.sum(1), 0.0).view(n, -1, BLOCK).double().sum(-1)   # (thousands of weights meet in a block: summed in 64 bits)
        mass[b, g] = torch.zeros(nb, dtype=torch.float64, device=q.device).index_add_(0, (at.view(n, -1, BLOCK)[..., 0] // BLOCK).view(-1), w.view(-1)).float()
    return o, lse, mass


def _block_attn_bwd(q, k, v, idx, o, lse, dO, scale):
    B, H, n, d = q.shape
    Hkv = k.shape[1]
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for b, g in ((b, g) for b in range(B) for g in range(Hkv)):
        hs = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
        qt, dt = q[b, hs].float().transpose(0, 1), dO[b, hs].float().transpose(0, 1)   # [n, G, d]
        kf, vf = k[b, g].float(), v[b, g].float()
        at, ok = _gathered(kf, idx[b, g])
        kg = kf[at]
        p = torch.where(ok.unsqueeze(1), torch.exp(torch.bmm(qt, kg.transpose(1, 2)) * scale - lse[b, hs].transpose(0, 1).unsqueeze(-1)), 0.0)
        delta = (dt * o[b, hs].float().transpose(0, 1)).sum(-1, keepdim=True)
        ds = p * (torch.bmm(dt, vf[at].transpose(1, 2)) - delta) * scale
        dq[b, hs] = torch.bmm(ds, kg).transpose(0, 1).to(q.dtype)
        flat = at.view(-1)
        dv[b, g] = torch.zeros_like(vf).index_add_(0, flat, torch.bmm(p.transpose(1, 2), dt).view(-1, d)).to(v.dtype)
        dk[b, g] = torch.zeros_like(kf).index_add_(0, flat, torch.bmm(ds.transpose(1, 2), qt).view(-1, d)).to(k.dtype)
    return dq, dk, dv


def _in_format(x, like):
    """Blocks [.., 64 * d] in the format of `like`, and their scales."""
    most = 127.0 if like.dtype == torch.int8 else 448.0
    top = x.abs().amax(-1, keepdim=True)
    some = top >= TINY
    y = torch.where(some, x * (most / torch.where(some, top, 1.0)), 0.0).clamp_(-most, most)
    return (y.round_() if like.dtype == torch.int8 else y).to(like.dtype), torch.where(some, top / most, 0.0).squeeze(-1)


def _store(cache, pages, whole, k, v):
    """Blocks k, v [.., 64, d] fp32 go to their pages [..], where `whole` says so; the other pages keep what they hold."""
    def put(name, x):
        t = cache[name].view(torch.uint8) if cache[name].element_size() == 1 else cache[name]   # (codes as bytes: 8-bit floats have no indexing)
        x = x.view(torch.uint8) if x.element_size() == 1 else x
        t[pages] = torch.where(whole.view(whole.shape + (1,) * (x.dim() - whole.dim())), x, t[pages])

    for x, codes, scales in ((k, "k8", "ks"), (v.transpose(-1, -2).contiguous(), "v8", "vs")):
        y, s = _in_format(x.flatten(-2), cache[codes])
        put(codes, y.view(x.shape))
        put(scales, s)
    y, s = _in8((k.double().sum(-2) / BLOCK).float())
    put("km", y.to(torch.int8))
    put("kms", s)


def _append_one(cache, lens, k, v):
    """One token for every sequence."""
    B, Hkv = k.shape[:2]
    b, at = torch.arange(B, device=k.device), (lens % BLOCK).long()
    kt, vt, full = cache["kt"].clone(), cache["vt"].clone(), at == BLOCK - 1
    kt[b, :, at] = k[:, :, 0]
    vt[b, :, :, at] = v[:, :, 0]
    pages = torch.gather(cache["table"].long(), 2, (lens // BLOCK).long().view(B, 1, 1).expand(B, Hkv, 1))[..., 0]
    _store(cache, pages, full.unsqueeze(1).expand(B, Hkv), kt.float(), vt.float().transpose(-1, -2))
    for x, t in ((kt, "kt"), (vt, "vt")):   # (a block that is whole leaves nothing behind here)
        cache[t].copy_(torch.where(full.view(B, 1, 1, 1), cache[t], x))


def _append_prompts(cache, counts, k, v):
    """Prompts of `counts` tokens for empty sequences."""
    B, Hkv, n, d = k.shape
    nb = n // BLOCK
    whole = (torch.arange(nb, device=k.device) < (counts // BLOCK).unsqueeze(-1)).unsqueeze(1).expand(B, Hkv, nb)
    blocks = [x[:, :, :nb * BLOCK].view(B, Hkv, nb, BLOCK, d).float() for x in (k, v)]
    _store(cache, cache["table"][:, :, :nb].long(), whole, *blocks)
    at = (counts // BLOCK * BLOCK).unsqueeze(-1) + torch.arange(BLOCK, device=k.device)   # [B, 64]
    live = (at < counts.unsqueeze(-1)).view(B, 1, BLOCK, 1)
    at = at.clamp(max=n - 1).long().view(B, 1, BLOCK, 1).expand(B, Hkv, BLOCK, d)
    cache["kt"].copy_(torch.where(live, torch.gather(k, 2, at), cache["kt"]))
    cache["vt"].copy_(torch.where(live, torch.gather(v, 2, at), cache["vt"].transpose(-1, -2)).transpose(-1, -2))


def _cache_select(cache, lens, q, top):
    B, H, d = q.shape
    Hkv, cap = cache["table"].shape[1:]
    pooled = _in8(q.view(B, Hkv, H // Hkv, d).double().sum(2).float())[0]
    pages = cache["table"].long()
    score = (cache["km"][pages].float() @ pooled.unsqueeze(-1)).squeeze(-1) * cache["kms"][pages]
    return _top_of(score, torch.arange(cap, device=q.device) < ((lens - 1) // BLOCK).view(B, 1, 1), top)


def _cache_attn(cache, lens, q, scale, idx=None):
    """One query for every sequence; what it gives each block joins the cache's masses."""
    B, H, d = q.shape
    Hkv, cap = cache["table"].shape[1:]
    G = H // Hkv
    nb = (lens // BLOCK).view(B, 1, 1).long()
    if idx is None:
        at = torch.arange(cap, device=q.device).view(1, 1, cap).expand(B, Hkv, cap)
        ok = at < nb
    else:   # (a query that ends a block has that block as its own)
        own_block = ((lens - 1) // BLOCK).view(B, 1, 1).expand(B, Hkv, 1)
        at = torch.cat([idx.long(), torch.where(own_block < nb, own_block.long(), -1)], -1)
        ok = at >= 0
        at = at.clamp(min=0)
    pages = torch.gather(cache["table"].long(), 2, at)
    K = cache["k8"][pages].float() * cache["ks"][pages].view(*pages.shape, 1, 1)                    # [B, Hkv, N, 64, d]
    V = cache["v8"][pages].float().transpose(-1, -2) * cache["vs"][pages].view(*pages.shape, 1, 1)
    N = at.shape[2] + 1
    tails = cache["kt"].float(), cache["vt"].float().transpose(-1, -2)
    K, V = (torch.cat([x, t.unsqueeze(2)], 2).view(B * Hkv, N * BLOCK, d) for x, t in zip((K, V), tails))
    in_tail = (torch.arange(BLOCK, device=q.device) < (lens % BLOCK).view(B, 1, 1)).expand(B, Hkv, BLOCK)
    ok = torch.cat([ok.unsqueeze(-1).expand(B, Hkv, N - 1, BLOCK), in_tail.unsqueeze(2)], 2).reshape(B * Hkv, 1, N * BLOCK)
    s = torch.where(ok, torch.bmm(q.float().view(B * Hkv, G, d), K.transpose(1, 2)) * scale, float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    p = p / total
    o = torch.bmm(p, V).view(B, H, d).to(q.dtype)
    w = p.view(B, Hkv, G, N, BLOCK).sum((2, 4))
    at = torch.cat([at, torch.where(in_tail[:, :, :1], nb.expand(B, Hkv, 1), 0)], -1)
    cache["mass"].scatter_add_(2, at, w)
    return o, (top + torch.log(total)).view(B, H)


def _evict_plain(cache, lens, budget, sink, recent, out):
    B, Hkv, cap = cache["table"].shape
    j, nb = torch.arange(cap, device=lens.device).view(1, 1, cap), (lens // BLOCK).view(B, 1, 1)
    over = nb > budget
    always = (j < sink) | (j >= nb - recent)
    order = torch.where(j >= nb, -1.0, torch.where(always, float("inf"), cache["mass"]))
    rank = torch.sort(order, dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(rank).scatter_(2, rank, j.expand(B, Hkv, cap))
    # kept blocks by age, then those that go, then what lies behind the last block
    new = torch.where(j >= nb, j + 2 * cap, torch.where((place < budget) | ~over, j, j + cap)).sort(-1).indices
    out["table"].copy_(torch.gather(cache["table"], 2, new))
    mass, tail = torch.gather(cache["mass"], 2, new), torch.gather(cache["mass"], 2, nb.clamp(max=cap - 1).long().expand(B, Hkv, 1))
    moved = torch.where(j < budget, mass, torch.where((j == budget) & (nb < cap), tail, 0.0))   # the last, unfinished block keeps its mass
    out["mass"].copy_(torch.where(over, moved, cache["mass"]))
    out["lens"].copy_((lens // BLOCK).clamp(max=budget) * BLOCK + lens % BLOCK)


def _handle(s):
    """The cache as the library's calls take it; a program keeps it beside its tensors."""
    import paper_2406_16747_amd as spk

    if "handle" not in s:
        c = s["case"]
        s["handle"] = spk.Cache8(**s["cache"], H=c.get("H", c["Hkv"]), scale=s.get("scale", 1.0))
    return s["handle"]


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        import paper_2406_16747_amd as spk
    if kind in ("prefill", "train"):
        q, k, v, scale = s["q"], s["k"], s["v"], s["scale"]
        if own:
            idx = spk.sparsek_block_select(q, k, c["top"])
            if kind == "prefill":
                o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, scale, mass=True)
            else:
                o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, scale)
                dq, dk, dv = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, s["dO"], scale)
        else:
            idx = _select(q, k, c["top"])
            o, lse, mass = _block_attn(q, k, v, idx, scale)
            if kind == "train":
                dq, dk, dv = _block_attn_bwd(q, k, v, idx, o, lse, s["dO"], scale)
        return dict(idx=idx, o=o, lse=lse, mass=mass) if kind == "prefill" else dict(o=o, dq=dq, dk=dk, dv=dv)
    cache = s["cache"]
    if kind == "decode":
        idx = None
        if own:
            h = _handle(s)
            spk.sparsek_cache8_append(h, s["lens"], s["k"], s["v"])
            if c["top"]:
                idx = spk.sparsek_cache8_select(h, s["after"], s["q"], c["top"])
            o, lse = spk.sparsek_cache8_attn(h, s["after"], s["q"], idx, accumulate=True)
        else:
            _append_one(cache, s["lens"], s["k"], s["v"])
            if c["top"]:
                idx = _cache_select(cache, s["after"], s["q"], c["top"])
            o, lse = _cache_attn(cache, s["after"], s["q"], s["scale"], idx)
        state = {x: cache[x] for x in ("mass", "kt", "vt", "ks", "vs", "kms")}
        return dict(o=o, lse=lse, **state, **({"idx": idx} if c["top"] else {}))
    if kind == "fill":
        if own:
            spk.sparsek_cache8_append(_handle(s), s["lens"], s["k"], s["v"], counts=s["counts"])
        else:
            _append_prompts(cache, s["counts"], s["k"], s["v"])
        return {x: cache[x] for x in ("k8", "v8", "ks", "vs", "km", "kms", "kt", "vt")}
    if own:
        spk.sparsek_cache8_evict(_handle(s), s["lens"], c["budget"], c["sink"], c["recent"], out=s["out"])
    else:
        _evict_plain(cache, s["lens"], c["budget"], c["sink"], c["recent"], s["out"])
    return dict(s["out"])


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c, kind = s["case"], case["kind"]
    if kind in ("prefill", "train"):
        B, H, n, d = s["q"].shape
        Hkv = s["k"].shape[1]
        idx = _select(s["q"], s["k"], c["top"])     # (whole numbers: the choice itself has one answer)
        f = lambda x: x.double()                    # noqa: E731
        o, lse = torch.empty(B, H, n, d, dtype=torch.float64, device="cuda"), torch.empty(B, H, n, dtype=torch.float64, device="cuda")
        dq, dk, dv = (torch.zeros_like(f(s[x])) for x in "qkv")
        nb = -(-n // BLOCK)
        mass = torch.zeros(B, Hkv, nb, dtype=torch.float64, device="cuda")
        j = torch.arange(n, device="cuda")
        step = 2048
        for b in range(B):
            for h in range(H):
                g = h // (H // Hkv)
                k, v = f(s["k"][b, g]), f(s["v"][b, g])
                for i0 in range(0, n, step):   # dense rows under a mask of what was selected
                    rows = slice(i0, min(n, i0 + step))
                    i, m = j[rows], min(n, i0 + step)
                    has = torch.zeros(len(i), nb + 1, dtype=torch.bool, device="cuda")
                    has.scatter_(1, torch.where(idx[b, g, rows] < 0, nb, idx[b, g, rows]).long(), True)
                    has[:, nb] = False
                    has.scatter_(1, (i // BLOCK).unsqueeze(1), True)
                    see = has[:, :nb].repeat_interleave(BLOCK, 1)[:, :m] & (j[:m] <= i.unsqueeze(1))
                    x = (f(s["q"][b, h, rows]) @ k[:m].T * s["scale"]).masked_fill(~see, -math.inf)
                    lse[b, h, rows] = z = torch.logsumexp(x, 1)
                    p = torch.exp(x - z.unsqueeze(1))
                    o[b, h, rows] = y = p @ v[:m]
                    if kind == "prefill":
                        t = torch.nn.functional.pad(p.sum(0), (0, nb * BLOCK - m))
                        mass[b, g] += t.view(nb, BLOCK).sum(1)
                    else:   # (the program's backward starts from the o that it has, which is rounded)
                        dO = f(s["dO"][b, h, rows])
                        dS = p * (dO @ v[:m].T - (dO * y.to(torch.bfloat16).double()).sum(1, keepdim=True)) * s["scale"]
                        dv[b, g, :m] += p.T @ dO
                        dk[b, g, :m] += dS.T @ f(s["q"][b, h, rows])
                        dq[b, h, rows] = dS @ k[:m]
        return dict(idx=None, o=o, lse=lse, mass=mass) if kind == "prefill" else dict(o=o, dq=dq, dk=dk, dv=dv)
    cache = s["cache"]
    if kind == "decode":
        _append_one(cache, s["lens"], s["k"], s["v"])
        idx = _cache_select(cache, s["after"], s["q"], c["top"]) if c["top"] else None
        B, H, d = s["q"].shape
        Hkv = c["Hkv"]
        o, lse = torch.empty(B, H, d, dtype=torch.float64, device="cuda"), torch.empty(B, H, dtype=torch.float64, device="cuda")
        mass, lens = cache["mass"].double(), s["after"].tolist()
        for b in range(B):
            for g in range(Hkv):
                whole, rest = divmod(lens[b], BLOCK)
                blocks = list(range(whole)) if idx is None else [x for x in idx[b, g].tolist() if x >= 0] + ([whole - 1] if rest == 0 else [])
                at = torch.tensor(blocks, dtype=torch.long, device="cuda")
                pages = cache["table"][b, g][at].long()
                K = (cache["k8"][pages].double() * cache["ks"][pages].double().view(-1, 1, 1)).reshape(-1, d)
                V = (cache["v8"][pages].double() * cache["vs"][pages].double().view(-1, 1, 1)).transpose(1, 2).reshape(-1, d)
                K, V = torch.cat([K, cache["kt"][b, g, :rest].double()]), torch.cat([V, cache["vt"][b, g, :, :rest].T.double()])
                hs = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
                x = s["q"][b, hs].double() @ K.T * s["scale"]
                lse[b, hs] = torch.logsumexp(x, 1)
                p = torch.softmax(x, 1)
                o[b, hs] = p @ V
                w = p.sum(0)
                mass[b, g].index_add_(0, at, w[:len(blocks) * BLOCK].view(-1, BLOCK).sum(1))
                if rest:
                    mass[b, g, whole] += w[len(blocks) * BLOCK:].sum()
        return dict(o=o, lse=lse, mass=mass, kt=None, vt=None, ks=None, vs=None, kms=None, idx=None)
    if kind == "fill":
        B, Hkv, n, d = s["k"].shape
        most = 127.0 if c["format"] == "int8" else 448.0
        ks, vs, kms = (torch.zeros(cache["ks"].shape, dtype=torch.float64, device="cuda") for _ in range(3))
        for b, count in enumerate(s["counts"].tolist()):
            m = count // BLOCK
            pages = cache["table"][b, :, :m].long()
            kb, vb = (s[x][b, :, :m * BLOCK].double().view(Hkv, m, BLOCK, d) for x in "kv")
            ks[pages], vs[pages] = kb.abs().amax((2, 3)) / most, vb.abs().amax((2, 3)) / most
            kms[pages] = kb.mean(2).abs().amax(2) / 127.0
        return dict(k8=None, v8=None, ks=ks, vs=vs, km=None, kms=kms, kt=None, vt=None)
    return None
