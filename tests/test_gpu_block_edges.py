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
