"""Attention over selected blocks at its edges: queries that are not finite, what lies behind a padded sequence, values and logits of
all sizes, and gradients at the sizes of training."""
import math

import pytest
import torch

import block_ref as ref
import paper_2406_16747_amd as spk
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def draw(seed, B, H, Hkv, n, d, qk=1.5):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q, k, v, dO = r(B, H, n, d) * qk, r(B, Hkv, n, d) + 0.7 * r(B, 1, -(-n // 64), d).repeat_interleave(64, 2)[:, :, :n], r(B, Hkv, n, d), r(B, H, n, d)
    return [x.bfloat16().cuda() for x in (q, k, v, dO)]


def within(got, want, bound, what):
    err = (ref.f64(got) - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), "%s: %d of %d beyond their bound, worst %.3g of it (err %.3g)" % (
        what, int(bad.sum()), bad.numel(), float((err / bound).max()), float(err.max()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 40, 300])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_a_query_that_is_not_finite_gets_nan(value, at, d):
    """Whatever the sign of its products (those of +inf and -inf with one column of keys of one sign are all +inf or all -inf): NaN for
    its o, lse and dq and for the gradients of the keys it attends, and for nobody else."""
    require_gpu()
    say("block attention, a query of", value, at, d)
    n, H, top = 400, 2, 2
    q, k, v, dO = draw(83, 1, H, 1, n, d)
    k[..., 7] = k[..., 7].abs() + 0.1
    idx = spk.sparsek_block_select(q, k, top)
    runs = []
    for spoil in (False, True):
        if spoil:
            q[0, 0, at, 7] = value
        o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125)
        runs.append((o, lse) + spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.125))
    torch.cuda.synchronize()
    (o, lse, dq, dk, dv), (o1, lse1, dq1, dk1, dv1) = runs
    assert torch.isnan(lse1[0, 0, at]) and torch.isnan(o1[0, 0, at]).all() and torch.isnan(dq1[0, 0, at]).all()
    for a, b in ((o, o1), (lse, lse1), (dq, dq1)):
        b[0, 0, at] = a[0, 0, at]
        assert torch.equal(a, b)
    keys = ref.seen(idx[0, 0].cpu().numpy(), n)[at].cuda()
    assert torch.isnan(dk1[0, 0][keys]).all() and torch.isnan(dv1[0, 0][keys]).all()
    assert torch.equal(dk[0, 0][~keys], dk1[0, 0][~keys]) and torch.equal(dv[0, 0][~keys], dv1[0, 0][~keys])


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("e", [8, 20, 23, 24, 25, 26, 27, 30, 60, 100])
def test_logits_of_all_sizes(e, sign):
    """Logits up to 2^e, each of its own: the weight is the largest one's alone.  The products are exact here, so nothing but the size is
    at stake."""
    require_gpu()
    say("block attention, logits of 2^%d" % e, sign)
    n, d, top = 250, 64, 2
    g = torch.Generator().manual_seed(91)
    c = (torch.randperm(255, generator=g)[:n].float() + 1) / 256
    q, k = torch.full((1, 2, n, d), float(sign)).bfloat16().cuda(), c.view(1, 1, n, 1).expand(1, 1, n, d).bfloat16().contiguous().cuda()
    v = torch.randn(1, 1, n, d, generator=g).bfloat16().cuda()
    scale = 0.7 * 2.0 ** e / d
    idx = spk.sparsek_block_select(q, k, top)
    o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, scale, mass=True)
    torch.cuda.synchronize()
    ro, rl, rm, ob, _ = ref.attn(q, k, v, idx, scale)
    if e >= 20:   # (the next logit is 2^-8 * 0.7 * 2^e behind, at least)
        within(o, ro, 2 ** -8 * ro.abs() + 2 ** -11 * ro.abs() + 2 ** -24, "o")
    else:
        within(o, ro, ob + 2 ** -22 * 2 ** e * ro.abs().amax(), "o")     # (a logit of 2^e is off by 2^-23 of it, twice)
    within(lse, rl, 2 ** -21 * rl.abs() + 2 ** -20, "lse")
    if e == 8:    # masses go by the fp32 lse, whose own rounding is a factor of its size beyond that
        within(mass, rm, 2 ** -12 * rm + 1e-9, "mass")


def behind(kind, g, shape):
    """What may lie behind a sequence that is shorter than its batch: finite numbers of any size."""
    if kind == "largest":
        return torch.full(shape, torch.finfo(torch.bfloat16).max)
    if kind == "lowest":
        return torch.full(shape, torch.finfo(torch.bfloat16).min)
    x = torch.randn(shape, generator=g)
    return x * 2.0 ** 45 if kind == "large" else x * torch.exp2(torch.randint(-120, 100, shape, generator=g).float())


PADDED = [(kind, d, real) for kind in ("large", "any", "largest", "lowest") for d in (64, 128)
          for real in (200, 129, 191)]                             # in the middle of a block, one token and all but one of it


def padded(kind, d, real):
    n, H, Hkv, top = 300, 4, 2, 2
    g = torch.Generator().manual_seed(7)
    q, k, v, dO = draw(93, 1, H, Hkv, n, d)
    dO[:, :, real:] = 0                                            # (no gradient comes from behind)
    idx = spk.sparsek_block_select(q, k, top)
    v[:, :, real:] = behind(kind, g, (1, Hkv, n - real, d)).bfloat16().cuda()
    if kind in ("large", "any"):                                   # (products with the largest numbers are infinite, and NaN in a sum)
        k[:, :, real:] = behind("large", g, (1, Hkv, n - real, d)).bfloat16().cuda()
    return q, k, v, dO, idx, lambda x: x[:, :, :real].contiguous()


@pytest.mark.parametrize("kind,d,real", PADDED)
def test_what_lies_behind_a_padded_sequence_reaches_nobody(kind, d, real):
    """Keys and values behind a sequence's end, in its last block and in further ones: what is ahead of them has the results of the
    sequence alone."""
    require_gpu()
    say("block attention, behind a padded sequence", kind, d, real)
    q, k, v, _, idx, cut = padded(kind, d, real)
    o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125)
    torch.cuda.synchronize()
    ro, rl, _, ob, lb = ref.attn(cut(q), cut(k), cut(v), cut(idx), 0.125)
    within(cut(o), ro, ob, "o")
    within(cut(lse), rl, lb, "lse")


@pytest.mark.parametrize("spread", [20, 40, 80])
@pytest.mark.parametrize("d", [64, 128])
def test_tokens_of_all_sizes_in_one_block(spread, d):
    """Values whose tokens differ by up to 2^spread: every row is right relative to what it attends.  The queries look at single tokens,
    so that the small ones' rows are small."""
    require_gpu()
    say("block attention, values of 2^%d" % spread, d)
    n, top = 330, 2
    g = torch.Generator().manual_seed(spread)
    k, v = torch.randn(1, 1, n, d, generator=g), torch.randn(1, 1, n, d, generator=g)
    target = (torch.arange(n) - torch.randint(0, 40, (n,), generator=g)).clamp(min=0)
    target = torch.maximum(target, torch.arange(n) // 64 * 64)      # (in the own block)
    q = (k / k.norm(dim=3, keepdim=True))[:, :, target].expand(1, 2, n, d) * 400
    v = v * torch.exp2(torch.randint(-spread // 2, spread // 2 + 1, (1, 1, n, 1), generator=g).float())
    q, k, v = (x.bfloat16().contiguous().cuda() for x in (q, k, v))
    idx = spk.sparsek_block_select(q, k, top)
    o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.5)
    torch.cuda.synchronize()
    ro, rl, _, _, _ = ref.attn(q, k, v, idx, 0.5)
    see = ref.seen(idx[0, 0].cpu().numpy(), n)
    K, V = ref.f64(k[0, 0]), ref.f64(v[0, 0])
    for h in range(2):
        x = (ref.f64(q[0, h]) @ K.T * 0.5).masked_fill(~see, -math.inf)
        p = torch.softmax(x, 1)
        # outputs and weights rounded, a partial result relative to its row's largest, and logits up to 2^13 off by 2^-23 of their products
        e = 2 ** -23 * 2 * (ref.f64(q[0, h]).abs() @ K.abs().T * 0.5).amax(1, keepdim=True) * 1.5
        bound = (2 ** -8 + 2 ** -11) * ro[0, h].abs() + (2 ** -11 + 2 ** -14 + e) * (p @ V.abs()) + 2 ** -22 * (p @ V.abs()).amax(1, keepdim=True)
        within(o[0, h], ro[0, h], bound, "o")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("exponent", [127, 100, -100, -120])
def test_values_at_both_ends_of_the_range(exponent, d):
    """A weighted mean of numbers is never larger than they are, up to the largest and down to the smallest ones with all their bits."""
    require_gpu()
    say("block attention, values of 2^%d" % exponent, d)
    n, top = 700, 6
    q, k, v, _ = draw(97, 1, 2, 1, n, d, qk=0.5)
    v = (torch.sign(v.float()) * (1 + 0.99 * torch.rand(v.shape, generator=torch.Generator().manual_seed(1)).cuda()) * 2.0 ** exponent).bfloat16()
    v[:, :, :400] = v[:, :, :400].abs()
    idx = spk.sparsek_block_select(q, k, top)
    o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125)
    torch.cuda.synchronize()
    ro, _, _, ob, _ = ref.attn(q, k, v, idx, 0.125)
    within(o, ro, ob, "o")


@pytest.mark.parametrize("kind,d,real", PADDED)
def test_gradients_of_a_padded_sequence(kind, d, real):
    """The gradients of the sequence alone, whatever keys and values lie behind it."""
    require_gpu()
    say("block attention backward, behind a padded sequence", kind, d, real)
    q, k, v, dO, idx, cut = padded(kind, d, real)
    o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125)
    got = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.125)
    torch.cuda.synchronize()
    want, bound = ref.attn_bwd(*[cut(x) for x in (q, k, v, idx, o, lse, dO)], 0.125)
    for name, x, y, z in zip(("dq", "dk", "dv"), got, want, bound):
        # (ds is off by p times what o's rounding and lse's error make of delta: both are the same on both sides, and part of the bound)
        within(cut(x), y, z, name)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("spread", [20, 40, 80])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_tokens_of_all_sizes_in_one_block(spread, d, which):
    """Keys or values whose tokens differ by up to 2^spread, in a block's own rows: a row's dq is right relative to what it attends.  Sizes
    grow along a block, so that its first rows see the small ones only."""
    require_gpu()
    say("block attention backward, %s of 2^%d" % (which, spread), d)
    n = 192
    q, k, v, dO = draw(spread, 1, 2, 1, n, d)
    size = torch.exp2((torch.arange(n) % 64 * spread // 63 - spread).float()).view(1, 1, n, 1).cuda()
    if which == "k":
        k = (k.float() * size).bfloat16()
    else:
        v = (v.float() * size).bfloat16()
    idx = torch.full((1, 1, n, 1), -1, dtype=torch.int32).cuda()
    o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125)
    got = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.125)
    torch.cuda.synchronize()
    want, bound = ref.attn_bwd(q, k, v, idx, o, lse, dO, 0.125)
    for name, x, y, z in zip(("dq", "dk", "dv"), got, want, bound):
        within(x, y, z, name)


@pytest.mark.parametrize("shape", [(1, 4, 2, 700, 64, 3), (1, 6, 2, 500, 128, 2), (2, 2, 2, 333, 128, 1)])
def test_dv_is_rounded_once(shape):
    """dv is off by its own rounding to bf16 (2^-8), weights as two bf16 numbers (2^-16) and fp32 sums and exponentials (2^-14, logits below
    2^5): beyond that rounding by a 16th of what weights in bf16 would leave."""
    require_gpu()
    say("block attention, dv", shape)
    B, H, Hkv, n, d, top = shape
    q, k, v, dO = draw(101, B, H, Hkv, n, d)
    scale = 1 / math.sqrt(d)
    idx = spk.sparsek_block_select(q, k, top)
    ro, rl = ref.attn(q, k, v, idx, scale)[:2]
    o, lse = ro.bfloat16().cuda(), rl.float().cuda()
    dv = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, scale)[2]
    torch.cuda.synchronize()
    (_, _, want), _ = ref.attn_bwd(q, k, v, idx, o, lse, dO, scale)
    size = ref.attn_bwd(q, k, v, idx, o, lse, dO.abs(), scale)[0][2]       # p^T |dO|
    within(dv, want, 2 ** -8 * want.abs() + (2 ** -16 + 2 ** -14) * size, "dv")


def check_blocks(q, k, v, dO, idx, o, lse, dk, dv, scale, g, blocks):
    """dk and dv of single blocks of long input, from all the rows that attend them, for the o and lse that the backward was given."""
    n, G = q.shape[2], q.shape[1] // k.shape[1]
    sel, i = idx[0, g].cpu(), torch.arange(n)
    for j in blocks:
        K, V = ref.f64(k[0, g, 64 * j:64 * j + 64]), ref.f64(v[0, g, 64 * j:64 * j + 64])
        rows = i[((sel == j).any(1) & (i // 64 > j)) | (i // 64 == j)]
        see = (64 * j + torch.arange(len(K))).view(1, -1) <= rows.view(-1, 1)
        wk, wv, bk, bv = (torch.zeros_like(K) for _ in range(4))
        for h in range(g * G, (g + 1) * G):
            Q, D, O = (ref.f64(x[0, h])[rows] for x in (q, dO, o))
            p = torch.exp((Q @ K.T * scale).masked_fill(~see, -math.inf) - ref.f64(lse[0, h])[rows].view(-1, 1))
            ds = p * (D @ V.T - (D * O).sum(1, keepdim=True)) * scale
            e = 2 ** -14 * ds.abs() + 2 ** -17 * p * (D.abs() @ V.abs().T + (D * O).abs().sum(1, keepdim=True)) * scale   # (as ref.attn_bwd)
            wv += p.T @ D
            wk += ds.T @ Q
            bv += (2 ** -16 + 2 ** -14) * p.T @ D.abs()
            bk += (e + 2 ** -16 * ds.abs()).T @ Q.abs()
        at = slice(64 * j, 64 * j + len(K))
        within(dv[0, g, at], wv, 2 ** -8 * wv.abs() + bv + 1e-30, "dv of block %d, %d rows" % (j, G * len(rows)))
        within(dk[0, g, at], wk, 2 ** -8 * wk.abs() + bk + 1e-30, "dk of block %d, %d rows" % (j, G * len(rows)))


@pytest.mark.parametrize("H,Hkv,n,d,top", [(8, 2, 10007, 128, 6), (4, 2, 9001, 64, 8), (6, 2, 5003, 128, 9), (4, 1, 30000, 128, 16)])
def test_gradients_of_keys_at_the_sizes_of_training(H, Hkv, n, d, top):
    """More blocks and pairs than one launch of the lists takes, units of 2048 and 1024 rows, blocks of one unit and of many (one that
    everybody selects), the first, the last and ragged one, and blocks in every stride of the join."""
    require_gpu()
    say("block attention, gradients of keys", H, Hkv, n, d, top)
    q, k, v, dO = draw(111, 1, H, Hkv, n, d)
    scale = 1 / math.sqrt(d)
    idx = spk.sparsek_block_select(q, k, top)
    idx[:, 0, :, 0] = 1                                  # (in any order, perhaps twice: it counts once)
    idx[:, -1, ::3, 1] = 17
    o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, scale)
    dq, dk, dv = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, scale)
    torch.cuda.synchronize()
    nb = -(-n // 64)
    for g in range(Hkv):
        check_blocks(q, k, v, dO, idx, o, lse, dk, dv, scale, g, [0, 1, 2, 15, 16, 17, 18, nb // 3, nb // 2, nb - 17, nb - 2, nb - 1])


def test_gradients_of_keys_of_several_passes_of_the_lists():
    """More than 4096 blocks."""
    require_gpu()
    say("block attention, gradients of keys, 300000 tokens")
    n, d, top = 300000, 64, 2
    g = torch.Generator(device="cuda").manual_seed(9)
    q, k, v, dO = (torch.randn(1, 1, n, d, device="cuda", generator=g).bfloat16() for _ in range(4))
    idx = torch.randint(-1, n // 64, (1, 1, n, top), device="cuda", generator=g, dtype=torch.int32)
    idx[:, :, ::2, 0] = 4200
    o, lse = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125)
    dq, dk, dv = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.125)
    torch.cuda.synchronize()
    check_blocks(q, k, v, dO, idx, o, lse, dk, dv, 0.125, 0, [0, 1, 4095, 4096, 4100, 4199, 4200, 4201, n // 64 - 1, n // 64])
