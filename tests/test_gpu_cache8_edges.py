"""The cache in 8 bits at its edges: values of no ordinary size in the unfinished block, queries that are not finite, selections
without a place, pools smaller than the table."""
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


def filled(k, v, H, cap, fmt, scale=None):
    """A cache of its own with all of k, v [B,Hkv,n,d] in it, and its lengths."""
    B, Hkv, n, d = k.shape
    cache = spk.Cache8.empty(B, H, Hkv, d, cap, fmt, scale=scale)
    spk.sparsek_cache8_append(cache, torch.zeros(B, dtype=torch.int32).cuda(), k, v)
    return cache, torch.full((B,), n, dtype=torch.int32).cuda()


@pytest.mark.parametrize("d,cap,n", [(64, 4, 220), (128, 40, 220), (64, 40, 129), (128, 4, 40)])   # one workgroup has all of it, or several
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), 1e30])
def test_a_value_of_the_unfinished_block_stays_in_its_column(bad, d, cap, n):
    """One value of the last token: its column is what the definition says, all other columns, the logarithms and the masses have the bits
    they have without it."""
    require_gpu()
    say("cache attention, unfinished block", bad, d, cap, n)
    B, H, Hkv = 2, 4, 2
    g = gen(5)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    own = torch.full((B, Hkv, 2), -1, dtype=torch.int32).cuda()
    runs = []
    for spoil in (False, True):
        if spoil:
            v[1, 1, n - 1, 9] = bad
        cache, L = filled(k, v, H, cap, torch.int8)
        runs.append([])
        for idx in (None, own):
            cache.mass.zero_()
            runs[-1].append(spk.sparsek_cache8_attn(cache, L, q, idx, accumulate=True) + (cache.mass.clone(),))
    torch.cuda.synchronize()
    for (o, lse, mass), (o1, lse1, mass1), idx in zip(*runs, (None, own)):
        want = ref.cache_attn(cache, [n] * B, q, idx)[0][1, 2:, 9]      # (infinite or NaN, or within 2^-8)
        got = ref.f64(o1[1, 2:, 9])
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
        some = torch.isfinite(want)
        assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
        assert ((got - want)[some].abs() <= (2 ** -8 + 2 ** -13) * want[some].abs()).all()
        o1[1, 2:, 9] = o[1, 2:, 9]
        assert torch.equal(o, o1) and torch.equal(lse, lse1) and torch.equal(mass, mass1)


@pytest.mark.parametrize("cap,n", [(4, 220), (40, 220), (40, 128), (4, 5)])
def test_a_selection_of_no_places_is_the_own_block(cap, n):
    """top = 0 is what a column of -1 is, masses included, and not all tokens."""
    require_gpu()
    say("cache attention, empty selection", cap, n)
    B, H, Hkv, d = 2, 4, 2, 64
    g = gen(15)
    cache, L = filled(rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), H, cap, torch.int8)
    q, none = rand(g, B, H, d), torch.full((B, Hkv, 1), -1, dtype=torch.int32).cuda()
    runs = []
    for idx in (none, none[..., :0], torch.empty(B, Hkv, 0, dtype=torch.int32).cuda()):
        cache.mass.zero_()
        runs.append(spk.sparsek_cache8_attn(cache, L, q, idx, accumulate=True) + (cache.mass.clone(),))
    torch.cuda.synchronize()
    ro, rl, rm, ob = ref.cache_attn(cache, [n] * B, q, none)
    assert ((ref.f64(runs[0][0]) - ro).abs() <= ob).all()
    for run in runs[1:]:
        for a, b in zip(run, runs[0]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", FORMATS)
def test_sequences_of_a_small_pool_keep_apart(fmt):
    """A pool of half the table: what goes in at once lies in pages of its own, codes and scales of one block together; blocks beyond a
    row's share are dropped and attended by nobody."""
    require_gpu()
    say("cache of a small pool", fmt)
    B, H, Hkv, d, cap, n = 3, 4, 2, 64, 8, 6 * 64 + 9
    g = gen(25)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    cache = spk.Cache8.empty(B, H, Hkv, d, cap, fmt, pages=B * Hkv * cap // 2)
    L = torch.full((B,), n, dtype=torch.int32).cuda()
    spk.sparsek_cache8_append(cache, torch.zeros_like(L), k, v)
    o, lse = spk.sparsek_cache8_attn(cache, L, q, accumulate=True)
    torch.cuda.synchronize()
    K8, V8 = ref.values(cache.k8), ref.values(cache.v8)
    for b in range(B):
        for h in range(Hkv):
            for j in range(cap // 2):
                page = int(cache.table[b, h, j])
                for x, codes, scale in ((k, K8[page], cache.ks[page]), (v, V8[page].T, cache.vs[page])):
                    y, s = ref.block_codes(x[b, h, 64 * j:64 * j + 64], fmt)
                    assert torch.equal(codes, y) and float(scale) == float(s), (b, h, j)
    ro, rl, rm, ob = ref.cache_attn(cache, [n] * B, q)
    assert ((ref.f64(o) - ro).abs() <= ob).all()
    assert ((ref.f64(cache.mass) - rm).abs() <= 2 ** -12 * rm).all() and (cache.mass[..., cap // 2:6] == 0).all()


@pytest.mark.parametrize("cap,n", [(4, 220), (40, 220), (40, 128), (4, 30)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("H", [4, 40])
def test_a_query_that_is_not_finite_gets_nan(value, cap, n, H):
    """Whatever the sign of its products: with keys of one sign in its column they are all +inf or all -inf, and the latter are not a
    sequence without tokens.  Other heads have the bits they have without it; a sequence without tokens gives it 0 and -inf."""
    require_gpu()
    say("cache attention, a query of", value, cap, n, H)
    B, Hkv, d = 3, 2, 64
    g = gen(35)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    k[..., 7] = 4.0     # (no code of 0 in the column)
    cache, L = filled(k, v, H, cap, torch.int8)
    L[2] = 0
    own = torch.full((B, Hkv, 1), -1, dtype=torch.int32).cuda()
    for idx in (None, own):
        runs = []
        for x in (q[1, 1, 7].item(), value):
            q[1:, 1, 7] = x
            runs.append(spk.sparsek_cache8_attn(cache, L, q, idx))
        torch.cuda.synchronize()
        (o, lse), (o1, lse1) = runs
        assert torch.isnan(o1[1, 1]).all() and torch.isnan(lse1[1, 1])
        assert (o1[2] == 0).all() and (lse1[2] == float("-inf")).all()
        o1[1, 1], lse1[1, 1] = o[1, 1], lse[1, 1]
        assert torch.equal(o, o1) and torch.equal(lse, lse1)
        q[1:, 1, 7] = 0.5


@pytest.mark.parametrize("cap", [4, 40])
def test_keys_of_minus_infinity_alone_are_not_no_keys(cap):
    """A sequence whose only token has a logit of -inf: 0 / 0, and not what a sequence without tokens has; with others it has weight 0."""
    require_gpu()
    say("cache attention, only logits of -inf", cap)
    g = gen(45)
    k, v, q = rand(g, 2, 1, 3, 64), rand(g, 2, 1, 3, 64), rand(g, 2, 2, 64).abs()
    k[:, :, 2, 9] = float("-inf")
    cache, L = filled(k[:, :, 2:].contiguous(), v[:, :, 2:].contiguous(), 2, cap, torch.int8)
    L[1] = 0
    o, lse = spk.sparsek_cache8_attn(cache, L, q, accumulate=True)
    torch.cuda.synchronize()
    assert torch.isnan(o[0]).all() and torch.isnan(lse[0]).all()
    assert (o[1] == 0).all() and (lse[1] == float("-inf")).all() and (cache.mass[1] == 0).all()
    cache, L = filled(k, v, 2, cap, torch.int8)
    o, lse = spk.sparsek_cache8_attn(cache, L, q)
    cache, L = filled(k[:, :, :2].contiguous(), v[:, :, :2].contiguous(), 2, cap, torch.int8)
    o2, lse2 = spk.sparsek_cache8_attn(cache, L, q)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("cap,n", [(4, 220), (40, 220), (40, 128)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("e", [8, 20, 23, 24, 25, 26, 27, 30, 60])
def test_logits_of_all_sizes(e, sign, cap, n):
    """Logits up to 2^e, each block's and token's apart: the weight is the largest one's alone."""
    require_gpu()
    say("cache attention, logits of 2^%d" % e, sign, cap, n)
    g = gen(55)
    c = (torch.randperm(255, generator=g)[:n].float() + 1) / 256
    k = c.view(1, 1, n, 1).expand(1, 1, n, 64).bfloat16().contiguous().cuda()
    v, q = rand(g, 1, 1, n, 64), torch.full((1, 2, 64), float(sign)).bfloat16().cuda()
    cache, L = filled(k, v, 2, cap, torch.int8, scale=0.7 * 2.0 ** e / 64)
    o, lse = spk.sparsek_cache8_attn(cache, L, q)
    torch.cuda.synchronize()
    ro, rl, rm, ob = ref.cache_attn(cache, [n], q)
    K = ref.row_tokens(cache, [n], 0, 0)[0][:, 0] * sign
    first, second = torch.unique(K).topk(2).values.tolist()
    if e >= 20:   # (codes of equal keys in one block share the weight; the next logit is far behind)
        assert (first - second) * 0.7 * 2.0 ** e > 2.0 ** 10
        assert ((ref.f64(o) - ro).abs() <= ob + 2 ** -11 * ro.abs()).all()
    else:
        assert ((ref.f64(o) - ro).abs() <= ob + 2 ** -22 * 2 ** e * ro.abs().amax()).all()
    assert ((lse.cpu().double() - rl).abs() <= 2 ** -21 * rl.abs() + 2 ** -20).all()


@pytest.mark.parametrize("cap", [6, 40])
@pytest.mark.parametrize("who", ["query", "block"])
def test_weights_that_are_nan_are_the_masses_of_all_that_is_attended(who, cap):
    """A query that is NaN, or a block that makes it so: every block that it attends has a mass of NaN, the spoiled one too, and no other;
    eviction keeps the older of those, whatever the NaN's sign."""
    require_gpu()
    say("cache attention, masses of NaN", who, cap)
    H, n = 2, 300
    g = gen(65)
    k, v, q = rand(g, 2, 1, n, 64), rand(g, 2, 1, n, 64), rand(g, 2, H, 64)
    if who == "block":
        k[0, 0, 70, 3] = float("nan")
    else:
        q[0, 1, 3] = float("nan")
    cache, L = filled(k, v, H, cap, torch.int8)
    idx = torch.tensor([1, 3], dtype=torch.int32).cuda().expand(2, 1, 2).contiguous()
    spk.sparsek_cache8_attn(cache, L, q, idx, accumulate=True)
    torch.cuda.synchronize()
    bad = torch.isnan(cache.mass[0, 0, :5])
    assert bad.tolist() == [False, True, False, True, True] and (cache.mass[0, 0, [0, 2]] == 0).all()
    assert torch.isfinite(cache.mass[1]).all() and float(cache.mass[1].sum()) > H - 1e-3
    cache.mass[0, 0, :4] = torch.tensor([float("inf"), -float("nan"), 7.0, float("nan")])
    cache.mass[0, 0, 1] = -cache.mass[0, 0, 3].abs()
    out = spk.sparsek_cache8_evict(cache, L, 2, 0, 0)
    torch.cuda.synchronize()
    assert out["table"][0, 0, :4].tolist() == [int(cache.table[0, 0, x]) for x in (1, 3, 0, 2)]


@pytest.mark.parametrize("cap", [4, 40])
def test_the_lowest_finite_logits_are_above_minus_infinity(cap):
    """Logits just above the lowest number, beside a last token of -inf: the weights are theirs."""
    require_gpu()
    say("cache attention, the lowest logits", cap)
    g = gen(75)
    k, v = torch.full((1, 1, 129, 64), -1.0).bfloat16().cuda(), rand(g, 1, 1, 129, 64)
    k[:, :, 128, 5] = float("-inf")
    q = torch.ones(1, 2, 64).bfloat16().cuda()
    cache, L = filled(k, v, 2, cap, torch.int8, scale=3.35e38 / (64 * 1.4427))
    o, lse = spk.sparsek_cache8_attn(cache, L, q)
    torch.cuda.synchronize()
    want = ref.row_tokens(cache, [128], 0, 0)[1].mean(0)
    assert ((ref.f64(o[0]) - want).abs() <= 2 ** -8 * want.abs() + 2 ** -11).all()
    assert ((lse.cpu().double() + 3.35e38 / 1.4427).abs() <= 2 ** -20 * 3.35e38).all()
