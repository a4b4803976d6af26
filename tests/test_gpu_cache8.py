"""The key/value cache in blocks held in 8 bits: what goes in, the single-token attention over it, and eviction, against their
definitions in 64 bits."""
import pytest
import torch

import block_ref as ref
import paper_2406_16747_amd as spk
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu
FORMATS = [torch.int8, torch.float8_e4m3fn]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *s):
    return torch.randn(*s, generator=g).bfloat16().cuda()


def shuffled(cache, seed):
    """The table's pages in an order of no kind."""
    n = cache.table.numel()
    cache.table.copy_(torch.randperm(n, generator=gen(seed)).to(torch.int32).view(cache.table.shape))
    return cache


def filled(seed, lens, H, Hkv, d, fmt, cap=None, scale=None):
    B, c = len(lens), max(max(lens), 1)
    cache = shuffled(spk.Cache8.empty(B, H, Hkv, d, cap or c // 64 + 1, fmt, scale=scale), seed)
    g = gen(seed)
    k, v = rand(g, B, Hkv, c, d), rand(g, B, Hkv, c, d)
    L = torch.tensor(lens, dtype=torch.int32).cuda()
    spk.sparsek_cache8_append(cache, torch.zeros_like(L), k, v, counts=L)
    return cache, L, k, v


def check_contents(cache, lens, k, v):
    """Every token is where it belongs, rounded as the definition says (whole numbers and 8-bit values: equal)."""
    fmt = cache.k8.dtype
    K8, V8 = ref.values(cache.k8), ref.values(cache.v8)
    for b, n in enumerate(lens.tolist()):
        whole, rest = divmod(n, 64)
        for g in range(cache.Hkv):
            for j in range(whole):
                page = int(cache.table[b, g, j])
                kb, vb = k[b, g, 64 * j:64 * j + 64], v[b, g, 64 * j:64 * j + 64]
                for x, codes, scale in ((kb, K8[page], cache.ks[page]), (vb, V8[page].T, cache.vs[page])):
                    y, s = ref.block_codes(x, fmt)
                    assert torch.equal(codes, y) and float(scale) == float(s), (b, g, j)
                y, s = ref.mean_codes(kb)
                assert torch.equal(cache.km[page].cpu().float(), y) and float(cache.kms[page]) == float(s), (b, g, j)
            assert torch.equal(cache.kt[b, g, :rest], k[b, g, 64 * whole:n])
            assert torch.equal(cache.vt[b, g, :, :rest], v[b, g, 64 * whole:n].T)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,pieces", [(64, [1]), (128, [63, 1]), (64, [64, 64]), (128, [40, 100, 1, 1, 300]), (64, [10, 117, 1, 64, 200]), (128, [127, 1])])
def test_append_in_pieces(fmt, d, pieces):
    require_gpu()
    say("cache append", fmt, d, pieces)
    B, Hkv, n = 2, 3, sum(pieces)
    cache = shuffled(spk.Cache8.empty(B, Hkv, Hkv, d, n // 64 + 1, fmt), 3)
    g = gen(1)
    k, v = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d)
    lens = torch.zeros(B, dtype=torch.int32).cuda()
    for c in pieces:
        a = int(lens[0])
        spk.sparsek_cache8_append(cache, lens, k[:, :, a:a + c].contiguous(), v[:, :, a:a + c].contiguous())
        lens += c
    torch.cuda.synchronize()
    check_contents(cache, lens, k, v)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_padded_prompts(fmt):
    """Counts of nothing, of some and of all; what lies behind a sequence's last token stays as it was."""
    require_gpu()
    say("cache append, padded", fmt)
    lens = [0, 1, 64, 200, 131]
    cache, L, k, v = filled(5, lens, 4, 2, 64, fmt)
    torch.cuda.synchronize()
    check_contents(cache, L, k, v)
    for b, n in enumerate(lens):
        assert (cache.kt[b, :, n % 64:] == 0).all() and (cache.vt[b, :, :, n % 64:] == 0).all()
        for g in range(2):
            rest = cache.table[b, g, n // 64:].long()
            assert (cache.ks[rest] == 0).all() and (cache.k8.view(torch.uint8)[rest] == 0).all() and (cache.km[rest] == 0).all()


def test_append_refuses_nothing_but_writes_nothing_beyond():
    """Counts and lengths of any size, pages outside the pool: everything else stays as it was."""
    require_gpu()
    say("cache append, out of range")
    g = gen(9)
    cache = spk.Cache8.empty(4, 2, 2, 64, 2, torch.int8, pages=8)
    cache.table[0, 0, 0], cache.table[0, 1, 0] = -1, 8
    cache.table[0, :, 1] = 2 ** 31 - 1
    cache.table[1:] = torch.arange(12, dtype=torch.int32).view(3, 2, 2).cuda() % 4 + 4
    k, v = rand(g, 4, 2, 300, 64), rand(g, 4, 2, 300, 64)
    lens = torch.tensor([0, 191, 2 ** 31 - 1, -5], dtype=torch.int32).cuda()
    counts = torch.tensor([300, 300, 2 ** 31 - 1, -1], dtype=torch.int32).cuda()
    spk.sparsek_cache8_append(cache, lens, k, v, counts=counts)
    torch.cuda.synchronize()
    assert (cache.k8 == 0).all() and (cache.ks == 0).all()           # 0: bad pages; 1 and 2: full; 3: no tokens
    assert torch.equal(cache.kt[0, :, :63], k[0, :, 128:191])        # 191 of 300 fit
    assert (cache.kt[1:] == 0).all() and (cache.kt[0, :, 63] == 0).all()


@pytest.mark.parametrize("kind", ["zeros", "tiny", "one value", "outlier"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks_of_all_kinds(kind, fmt):
    require_gpu()
    say("cache append,", kind, fmt)
    g = gen(4)
    k, v = rand(g, 1, 1, 128, 64), rand(g, 1, 1, 128, 64)
    for x in (k, v):
        if kind == "zeros":
            x[:, :, :64] = 0
        elif kind == "tiny":
            x[:, :, :64] *= 2.0 ** -110
        elif kind == "one value":
            x[:, :, :64] = -3.0
        else:
            x[:, :, 5, 7] = 3e38
    cache = spk.Cache8.empty(1, 1, 1, 64, 3, fmt)
    L = torch.zeros(1, dtype=torch.int32).cuda()
    spk.sparsek_cache8_append(cache, L, k, v)
    torch.cuda.synchronize()
    check_contents(cache, L + 128, k, v)


ROWS = [[1], [63, 64, 65, 0], [700, 128, 1, 129, 513], [2000]]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,Hkv,d", [(1, 1, 64), (3, 1, 128), (8, 2, 128), (32, 2, 64), (25, 1, 128)])
@pytest.mark.parametrize("lens", ROWS)
def test_attention_of_a_single_token(fmt, H, Hkv, d, lens):
    require_gpu()
    say("cache attention", fmt, H, Hkv, d, lens)
    cache, L, _, _ = filled(21, lens, H, Hkv, d, fmt)
    cache.kt[:, :, 63], cache.vt[:, :, :, 63] = float("nan"), float("inf")   # behind the last token: anything
    q = rand(gen(22), len(lens), H, d)
    before = torch.rand(cache.mass.shape, generator=gen(23)).cuda()
    cache.mass.copy_(before)
    o, lse = spk.sparsek_cache8_attn(cache, L, q, accumulate=True)
    torch.cuda.synchronize()
    ro, rl, rm, ob = ref.cache_attn(cache, lens, q)
    assert ((ref.f64(o) - ro).abs() <= ob).all(), float(((ref.f64(o) - ro).abs() / ob).max())
    empty = torch.tensor([n == 0 for n in lens])
    assert (o[empty] == 0).all() and (lse[empty] == float("-inf")).all()
    assert ((lse.cpu().double() - rl)[~empty].abs() <= 2e-4).all()           # logits to 60: 128 products of 2^-24 each, twice
    want = ref.f64(before) + rm
    assert ((ref.f64(cache.mass) - want).abs() <= 2 ** -12 * rm + 2 ** -23 * want).all()
    o2, lse2 = spk.sparsek_cache8_attn(cache, L, q)                          # without masses: the same, and none move
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,Hkv,d,top", [(4, 4, 64, 1), (8, 2, 128, 5), (20, 1, 128, 7)])
def test_selected_blocks(fmt, H, Hkv, d, top):
    """The selection is the definition's; the attention reads it, and selections of the caller's own: repeated, out of range, none."""
    require_gpu()
    say("cache selection", fmt, H, Hkv, d, top)
    lens = [900, 64, 640, 641, 1, 0, 330]
    cache, L, _, _ = filled(31, lens, H, Hkv, d, fmt)
    B = len(lens)
    q = rand(gen(32), B, H, d)
    idx = spk.sparsek_cache8_select(cache, L, q, top)
    torch.cuda.synchronize()
    p8, _ = ref.codes_i8(ref.f64(q).view(B, Hkv, H // Hkv, d).sum(2).float())
    for b in range(B):
        for g in range(Hkv):
            nb = max(lens[b] - 1, 0) // 64
            pages = cache.table[b, g, :nb].cpu().long()
            score = (cache.km.cpu()[pages].double() @ p8[b, g].double()).float() * cache.kms.cpu()[pages]
            assert idx[b, g].tolist() == ref.top_of(score, [True] * nb, top), (b, g)
    other = torch.randint(-4, 20, idx.shape, generator=gen(33), dtype=torch.int32).cuda()
    other[0, :, top // 2:] = 3
    other[2, :, 0] = 2 ** 31 - 1
    for x in (idx, other, torch.full_like(idx, -1)):
        cache.mass.zero_()
        o, lse = spk.sparsek_cache8_attn(cache, L, q, x, accumulate=True)
        torch.cuda.synchronize()
        ro, rl, rm, ob = ref.cache_attn(cache, lens, q, x.cpu())
        assert ((ref.f64(o) - ro).abs() <= ob).all()
        assert ((ref.f64(cache.mass) - rm).abs() <= 2 ** -12 * rm).all()
        some = torch.tensor([n > 0 for n in lens])
        assert ((lse.cpu().double() - rl)[some].abs() <= 2e-4).all()


def test_pages_outside_the_pool_are_attended_by_nobody():
    require_gpu()
    say("cache attention, bad pages")
    cache, L, _, _ = filled(41, [500, 300], 4, 2, 64, torch.int8)
    cache.table[0, 0, 2], cache.table[0, 1, 0], cache.table[1, 1] = -1, cache.cfg.pages, -7
    q = rand(gen(42), 2, 4, 64)
    o, lse = spk.sparsek_cache8_attn(cache, L, q, accumulate=True)
    idx = spk.sparsek_cache8_select(cache, L, q, 3)
    torch.cuda.synchronize()
    ro, rl, rm, ob = ref.cache_attn(cache, [500, 300], q)
    assert ((ref.f64(o) - ro).abs() <= ob).all()
    assert ((ref.f64(cache.mass) - rm).abs() <= 2 ** -12 * rm).all()
    assert idx.min() >= -1 and 2 not in idx[0, 0].tolist()


@pytest.mark.parametrize("cap,lens,budget,sink,recent", [
    (5, [320 + 17, 5, 256, 0], 3, 1, 1), (40, [2560, 2000, 64 * 40 + 63, 64 * 12], 12, 2, 3), (1100, [70000, 40000, 64 * 1100], 700, 0, 0),
    (9, [9 * 64, 600, 8 * 64 + 1], 8, 8, 0), (9, [9 * 64, 600, 8 * 64 + 1], 0, 0, 0), (7, [448, -3, 2 ** 31 - 1], 6, 0, 6)])
def test_eviction(cap, lens, budget, sink, recent):
    require_gpu()
    say("cache eviction", cap, lens, budget, sink, recent)
    B, Hkv = len(lens), 3
    cache = shuffled(spk.Cache8.empty(B, Hkv, Hkv, 64, cap), 51)
    mass = torch.exp(2 * torch.randn(B, Hkv, cap, generator=gen(52)))
    mass[torch.rand(mass.shape, generator=gen(53)) < 0.4] = 0.0
    mass[:, 1] = 1.0                                        # all equal: the older stay
    cache.mass.copy_(mass)
    L = torch.tensor(lens, dtype=torch.int32).cuda()
    out = spk.sparsek_cache8_evict(cache, L, budget, sink, recent)
    torch.cuda.synchronize()
    for got, want in zip((out["table"], out["mass"], out["lens"]), ref.evict(cache.table, cache.mass, L, budget, sink, recent)):
        assert torch.equal(got.cpu(), want)


def test_the_longest_table():
    """8192 blocks of a row that share 96 pages: selection, attention over all and over a selection longer than a workgroup's share
    with repeated places, eviction."""
    require_gpu()
    say("cache of 8192 blocks")
    B, H, d, cap = 2, 2, 64, 8192
    cache = spk.Cache8.empty(B, H, 1, d, cap, torch.float8_e4m3fn, pages=96)
    g = gen(81)
    lens = torch.full((B,), 0, dtype=torch.int32).cuda()
    spk.sparsek_cache8_append(cache, lens, rand(g, B, 1, 96 * 64, d), rand(g, B, 1, 96 * 64, d))
    cache.table.copy_(torch.randint(0, 96, cache.table.shape, generator=g, dtype=torch.int32))
    cache.kt.copy_(rand(g, *cache.kt.shape))
    cache.vt.copy_(rand(g, *cache.vt.shape))
    L = [cap * 64 + 63, 5000 * 64]
    lens = torch.tensor(L, dtype=torch.int32).cuda()
    q = rand(g, B, H, d)
    idx = spk.sparsek_cache8_select(cache, lens, q, 100)
    torch.cuda.synchronize()
    p8, _ = ref.codes_i8(ref.f64(q).sum(1).float())
    for b in range(B):
        nb = (L[b] - 1) // 64
        pages = cache.table[b, 0, :nb].cpu().long()
        score = (cache.km.cpu()[pages].double() @ p8[b].double()).float() * cache.kms.cpu()[pages]
        assert idx[b, 0].tolist() == ref.top_of(score, [True] * nb, 100)
    many = torch.randint(-5, 5200, (B, 1, 300), generator=g, dtype=torch.int32)
    many[:, :, 200:] = many[:, :, :100]
    for x in (None, idx, many.cuda()):
        cache.mass.zero_()
        o, lse = spk.sparsek_cache8_attn(cache, lens, q, x, accumulate=True)
        torch.cuda.synchronize()
        ro, rl, rm, ob = ref.cache_attn(cache, L, q, None if x is None else x.cpu())
        assert ((ref.f64(o) - ro).abs() <= ob).all()
        assert ((lse.cpu().double() - rl).abs() <= 2e-4).all()
        assert ((ref.f64(cache.mass) - rm).abs() <= 2 ** -12 * rm).all()
    cache.mass.copy_(torch.randint(0, 50, cache.mass.shape, generator=g).float())     # many of one size
    out = spk.sparsek_cache8_evict(cache, lens, 4000, 4, 100)
    torch.cuda.synchronize()
    for got, want in zip((out["table"], out["mass"], out["lens"]), ref.evict(cache.table, cache.mass, lens, 4000, 4, 100)):
        assert torch.equal(got.cpu(), want)


def test_the_handle_keeps_its_tensors():
    require_gpu()
    cache = spk.Cache8.empty(1, 2, 1, 64, 4)
    with pytest.raises(AttributeError):
        cache.mass = torch.zeros_like(cache.mass)
    table, mass = cache.table.clone(), torch.ones_like(cache.mass)
    cache.adopt(table, mass)
    assert cache.mass is mass and cache.table is table


def test_calls_on_streams_of_their_own():
    """Two caches stepped on two streams at once give what they give one after the other."""
    require_gpu()
    say("cache steps on two streams")
    made = [filled(90 + x, [700 + 60 * x, 90], 8, 2, 128, FORMATS[x], cap=14) for x in range(2)]
    q = [rand(gen(95 + x), 2, 8, 128) for x in range(2)]
    torch.cuda.synchronize()
    want = [spk.sparsek_cache8_attn(c, L, y) for (c, L, _, _), y in zip(made, q)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for x in range(2):
            with torch.cuda.stream(streams[x]):
                got[x].append(spk.sparsek_cache8_attn(made[x][0], made[x][1], q[x]))
    torch.cuda.synchronize()
    for x in range(2):
        for o, lse in got[x]:
            assert torch.equal(o, want[x][0]) and torch.equal(lse, want[x][1])


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_conversation(fmt):
    """Prefill over selected blocks, its keys, values and masses into the cache, then tokens one by one with eviction: every step
    against the definition on what the cache then holds, and the first against the prefill's own next row."""
    require_gpu()
    say("a conversation", fmt)
    B, H, Hkv, d, n, top, cap, budget = 2, 4, 2, 64, 500, 3, 10, 6
    g = gen(61)
    scale = d ** -0.5
    k, v, q = rand(g, B, Hkv, n + 200, d), rand(g, B, Hkv, n + 200, d), rand(g, B, H, n + 200, d)
    cut = lambda x: x[:, :, :n].contiguous()  # noqa: E731
    idx = spk.sparsek_block_select(cut(q), cut(k), top)
    o, lse, mass = spk.sparsek_block_attn_fwd(cut(q), cut(k), cut(v), idx, scale, mass=True)
    cache = spk.Cache8.empty(B, H, Hkv, d, cap, fmt, scale=scale)
    lens = torch.zeros(B, dtype=torch.int32).cuda()
    spk.sparsek_cache8_append(cache, lens, cut(k), cut(v))
    lens = lens + n
    cache.mass[:, :, :mass.shape[2]] = mass
    for t in range(n, n + 200):
        if int(lens[0]) // 64 > budget:
            out = spk.sparsek_cache8_evict(cache, lens, budget, 1, 2)
            want = ref.evict(cache.table, cache.mass, lens, budget, 1, 2)
            assert torch.equal(out["table"].cpu(), want[0]) and torch.equal(out["lens"].cpu(), want[2])
            cache.adopt(out["table"], out["mass"])
            lens = out["lens"]
        spk.sparsek_cache8_append(cache, lens, k[:, :, t:t + 1].contiguous(), v[:, :, t:t + 1].contiguous())
        lens = lens + 1
        qt = q[:, :, t].contiguous()
        sel = spk.sparsek_cache8_select(cache, lens, qt, top) if t % 2 else None
        o, lse = spk.sparsek_cache8_attn(cache, lens, qt, sel, accumulate=True)
        if t % 23 == 0 or t < n + 3:
            torch.cuda.synchronize()
            ro, rl, rm, ob = ref.cache_attn(cache, lens.tolist(), qt, None if sel is None else sel.cpu())
            assert ((ref.f64(o) - ro).abs() <= ob).all(), t
            if t == n + 1 and sel is not None:     # no eviction has moved a place by now: the prefill's choice
                all_idx = spk.sparsek_block_select(q[:, :, :t + 1].contiguous(), k[:, :, :t + 1].contiguous(), top)
                if int(lens[0]) == t + 1:
                    assert torch.equal(all_idx[:, :, t], sel)
    assert (cache.mass >= 0).all() and torch.isfinite(cache.mass).all()


def test_decode_step_replays_as_a_graph():
    """One step captured (lengths move on inside the graph), replayed over the end of a block, against eager steps; and two graphs
    with workspaces of their own replayed in turn."""
    require_gpu()
    say("cache step as a graph")
    B, H, Hkv, d, top = 2, 8, 2, 128, 2
    lens0 = [250, 190]

    def fresh():
        return filled(71, lens0, H, Hkv, d, torch.float8_e4m3fn, cap=6)[:2]

    def step(cache, lens, q, k, v):
        spk.sparsek_cache8_append(cache, lens, k, v)
        lens.add_(1)
        idx = spk.sparsek_cache8_select(cache, lens, q, top)
        return spk.sparsek_cache8_attn(cache, lens, q, idx, accumulate=True) + spk.sparsek_cache8_attn(cache, lens, q)

    g = gen(72)
    new = [(rand(g, B, H, d), rand(g, B, Hkv, 1, d), rand(g, B, Hkv, 1, d)) for _ in range(10)]
    ec, el = fresh()
    eager = []
    for x in new:
        eager.append([t.clone() for t in step(ec, el, *x)])
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        cache, lens = fresh()
        q, k, v = (t.clone() for t in new[0])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            wc, wl = fresh()
            step(wc, wl, q, k, v)
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(cache, lens, q, k, v)
        graphs.append((graph, cache, lens, (q, k, v), out))
    for i, x in enumerate(new):
        for graph, cache, lens, args, out in graphs:
            for dst, src in zip(args, x):
                dst.copy_(src)
            graph.replay()
        torch.cuda.synchronize()
        for graph, cache, lens, args, out in graphs:
            for a, b in zip(out, eager[i]):
                assert torch.equal(a, b), i
    for _, cache, lens, _, _ in graphs:
        assert torch.equal(cache.mass, ec.mass) and torch.equal(lens, el)
        assert torch.equal(cache.k8.view(torch.uint8), ec.k8.view(torch.uint8)) and torch.equal(cache.kt, ec.kt)


@pytest.mark.parametrize("cap", [4, 40])   # one workgroup has all of it, or several
@pytest.mark.parametrize("where", ["key", "value", "last token's key", "last token's value"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("fmt", FORMATS)
def test_values_that_are_not_finite_reach_who_attends_them(fmt, bad, where, cap):
    """One value of a head, in its second block of three and a half, or of its last token (in bf16, where a value of infinity is one of the
    result's column): nothing finite for that head's queries unless they leave the block out, and the same bits as ever for everybody else."""
    B, H, Hkv, d, n = 2, 4, 2, 64, 220
    g = gen(5)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    q[1, 2:, 9] = q[1, 2:, 9].abs() + 1   # (a logit of +inf or NaN, or -inf where `bad` is that)
    zero, L = torch.zeros(B, dtype=torch.int32).cuda(), torch.full((B,), n, dtype=torch.int32).cuda()
    last = where.startswith("last")

    def run(k, v):
        cache = shuffled(spk.Cache8.empty(B, H, Hkv, d, cap, fmt), 5)
        spk.sparsek_cache8_append(cache, zero, k, v)
        without = torch.tensor([0, 2], dtype=torch.int32).cuda().expand(B, Hkv, 2).contiguous()
        return spk.sparsek_cache8_attn(cache, L, q, accumulate=True) + spk.sparsek_cache8_attn(cache, L, q, without)

    clean = run(k, v)
    (k if "key" in where else v)[1, 1, n - 1 if last else 100, 9] = bad
    for x, (got, want) in enumerate(zip(run(k, v), clean)):
        mine = got[1, 2:]
        if where == "last token's key" and bad == float("-inf"):   # (a weight of 0)
            assert torch.isfinite(mine).all()
        elif last and "value" in where and x in (0, 2):
            assert not torch.isfinite(mine[:, 9]).any(), x
        elif x == 0 or last and x == 2:
            assert torch.isnan(mine).all(), x
        elif x == 2:   # (without the second block)
            assert torch.equal(mine, want[1, 2:])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1, :2], want[1, :2]), x
