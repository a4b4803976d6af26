"""Attention over selected blocks of 64 tokens: selection, forward and backward against their definitions in 64 bits."""
import math

import pytest
import torch

import block_ref as ref
import paper_2406_16747_amd as spk
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

# B, H, Hkv, n, d, top: lengths of one token, around a block's and a chunk's ends and beyond; groups of 1 to 25 heads
SHAPES = [
    (1, 1, 1, 1, 64, 2), (2, 2, 1, 63, 128, 1), (1, 2, 2, 64, 64, 4), (1, 3, 1, 65, 128, 3), (1, 2, 2, 129, 128, 1), (2, 4, 2, 300, 64, 2),
    (1, 8, 1, 517, 128, 3), (1, 25, 1, 200, 64, 64), (1, 16, 1, 385, 128, 0), (1, 3, 3, 1000, 64, 5), (1, 4, 2, 1030, 128, 9),
]


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


def check_all(q, k, v, dO, idx, scale):
    o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, scale, mass=True)
    torch.cuda.synchronize()
    ro, rl, rm, ob, lb = ref.attn(q, k, v, idx, scale)
    within(o, ro, ob, "o")
    within(lse, rl, lb, "lse")
    within(mass, rm, 2 ** -12 * rm + 1e-9, "mass")   # (a logit below 2^5 is off by 128 products of 2^-24 at most)
    o, lse = ro.bfloat16().cuda(), rl.float().cuda()
    got = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, scale)
    torch.cuda.synchronize()
    want, bound = ref.attn_bwd(q, k, v, idx, o, lse, dO, scale)
    for name, x, y, z in zip(("dq", "dk", "dv"), got, want, bound):
        within(x, y, z, name)


@pytest.mark.parametrize("shape", SHAPES)
def test_selection_is_the_definitions(shape):
    require_gpu()
    B, H, Hkv, n, d, top = shape
    say("block select", shape)
    q, k, _, _ = draw(11, B, H, Hkv, n, d)
    idx = spk.sparsek_block_select(q, k, top)
    torch.cuda.synchronize()
    assert torch.equal(idx.cpu(), ref.select(q, k, top))


@pytest.mark.parametrize("n,d,tops", [(9000, 64, (1, 17, 64)), (40000, 128, (5,)), (300000, 64, (3,))])
def test_selection_of_many_blocks(n, d, tops):
    """More blocks than a wave keeps in registers (128 and 512 of them), more than 4096; scores that differ in their last bits only."""
    require_gpu()
    say("block select, many blocks", n, d, tops)
    g = torch.Generator(device="cuda").manual_seed(12)
    q, k = (torch.randn(1, h, n, d, device="cuda", generator=g) for h in (2, 1))
    q, k = q.bfloat16(), (k * 0.001 + torch.randn(d, device="cuda", generator=g)).bfloat16()
    nb = n // 64
    m8, ms = ref.mean_codes(k[0, 0, :nb * 64].view(nb, 64, d))
    for top in tops:
        idx = spk.sparsek_block_select(q, k, top).cpu()
        for i in list(range(0, n, n // 11)) + [n - 1]:
            p8, _ = ref.codes_i8(ref.f64(q[0, :, i]).sum(0).float())
            score = (m8.double() @ p8.double()).float() * ms
            assert idx[0, 0, i].tolist() == ref.top_of(score, [j < i // 64 for j in range(nb)], top), (top, i)


@pytest.mark.parametrize("kind", ["equal keys", "zeros", "tiny", "huge", "one sign"])
def test_selection_of_equal_and_extreme_scores(kind):
    require_gpu()
    say("block select", kind)
    q, k, _, _ = draw(13, 1, 2, 1, 700, 64)
    if kind == "equal keys":
        k[:] = k[:, :, :1]
    elif kind == "zeros":
        q.zero_()
    elif kind == "tiny":
        k.mul_(2.0 ** -120)
    elif kind == "huge":
        k.mul_(2.0 ** 100)
        q.mul_(2.0 ** 100)
    else:
        k.abs_()
        q.copy_(-q.abs())
    assert torch.equal(spk.sparsek_block_select(q, k, 3).cpu(), ref.select(q, k, 3))


@pytest.mark.parametrize("shape", SHAPES)
def test_attention_and_gradients(shape):
    require_gpu()
    B, H, Hkv, n, d, top = shape
    say("block attention", shape)
    q, k, v, dO = draw(21, B, H, Hkv, n, d)
    idx = spk.sparsek_block_select(q, k, top)
    check_all(q, k, v, dO, idx, 1 / math.sqrt(d))


@pytest.mark.parametrize("kind", ["none", "all", "one block", "repeated", "out of range", "any order"])
@pytest.mark.parametrize("d,H,Hkv", [(64, 2, 2), (128, 6, 2)])
def test_selections_of_the_callers_own(kind, d, H, Hkv):
    """Rows that select nothing, everything, the same block all of them, a block twice, blocks that do not exist or are not behind the
    query, in any order."""
    require_gpu()
    say("block attention, selection", kind, d, H, Hkv)
    n, top = 460, 8
    g = torch.Generator().manual_seed(5)
    idx = torch.randint(-3, n // 64 + 3, (1, Hkv, n, top), generator=g, dtype=torch.int32)
    if kind == "none":
        idx.fill_(-1)
    elif kind == "all":
        idx[:] = torch.arange(top, dtype=torch.int32)
    elif kind == "one block":
        idx.fill_(-1)
        idx[..., 3] = 0
    elif kind == "repeated":
        idx[:] = torch.randint(0, 2, idx.shape, generator=g, dtype=torch.int32)
    elif kind == "out of range":
        idx[:] = torch.where(torch.rand(idx.shape, generator=g) < 0.5, idx, torch.tensor(2 ** 31 - 1, dtype=torch.int32))
        idx[:, :, ::3, 0] = -2 ** 31
        idx[:, :, 1::3, 1] = 2 ** 30
    q, k, v, dO = draw(31, 1, H, Hkv, n, d)
    check_all(q, k, v, dO, idx.cuda(), 1 / math.sqrt(d))


@pytest.mark.parametrize("kind", ["v zero", "v large", "v small", "peaked", "flat"])
def test_values_of_all_sizes(kind):
    """Partial results are held relative to their block's largest value: of any size; and softmaxes of one key and of all."""
    require_gpu()
    say("block attention,", kind)
    q, k, v, dO = draw(41, 1, 4, 2, 400, 64, qk={"peaked": 4.0, "flat": 0.0}.get(kind, 1.5))
    if kind == "v zero":
        v[:, :, 64:256] = 0
    elif kind == "v large":
        v.mul_(2.0 ** 40)
        dO.mul_(2.0 ** -40)
    elif kind == "v small":
        v.mul_(2.0 ** -60)
    idx = spk.sparsek_block_select(q, k, 3)
    check_all(q, k, v, dO, idx, 1 / 8)


def test_many_rows_select_one_block():
    """A block that everybody selects: its rows span many units."""
    require_gpu()
    say("block attention, a popular block")
    n, H, Hkv, d = 900, 8, 2, 128
    q, k, v, dO = draw(51, 1, H, Hkv, n, d)
    idx = torch.full((1, Hkv, n, 2), -1, dtype=torch.int32)
    idx[:, 0, :, 0] = 1
    idx[:, 1, :, 1] = 0
    check_all(q, k, v, dO, idx.cuda(), 1 / math.sqrt(d))


def check_rows(q, k, v, dO, idx, o, dq, scale, heads, rows):
    """Single rows of every kind of long input against a definition of their own."""
    G = q.shape[1] // k.shape[1]
    for h in heads:
        K, V = ref.f64(k[0, h // G]), ref.f64(v[0, h // G])
        for i in rows:
            at = torch.cat([torch.arange(64) + 64 * j for j in idx[0, h // G, i].tolist() if j >= 0] + [torch.arange(i // 64 * 64, i + 1)])
            p = torch.softmax(K[at] @ ref.f64(q[0, h, i]) * scale, 0)
            want = p @ V[at]
            within(o[0, h, i], want, 2 ** -8 * want.abs() + (2 ** -11 + 2 ** -11 + 2 ** -14) * (p @ V[at].abs()) + 2 ** -22 * V.abs().max(), "o of row %d" % i)
            if dq is None:
                continue
            g, oo = ref.f64(dO[0, h, i]), ref.f64(o[0, h, i])
            ds = p * (V[at] @ g - (g * oo).sum()) * scale
            e = (2 ** -11 + 2 ** -11 + 2 ** -14) * ds.abs() + 2 ** -17 * p * (V[at].abs() @ g.abs() + (g * oo).abs().sum()) * scale
            want = ds @ K[at]
            within(dq[0, h, i], want, 2 ** -8 * want.abs() + e @ K[at].abs() + 2 ** -22 * (ds.abs() @ K[at].abs()).max(), "dq of row %d" % i)


def test_a_long_document_row_by_row():
    """30000 tokens: rows picked all over it against a definition of their own."""
    require_gpu()
    say("block attention, 30000 tokens")
    n, H, Hkv, d, top = 30000, 4, 1, 128, 16
    q, k, v, dO = draw(61, 1, H, Hkv, n, d)
    scale = 1 / math.sqrt(d)
    idx = spk.sparsek_block_select(q, k, top)
    o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, scale, mass=True)
    dq, dk, dv = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, scale)
    torch.cuda.synchronize()
    assert abs(float(mass.double().sum()) / (n * H) - 1) < 1e-5      # every row hands out a weight of 1
    check_rows(q, k, v, dO, idx, o, dq, scale, range(H), list(range(0, n, 1777)) + [n - 1])
    assert torch.isfinite(dk).all() and torch.isfinite(dv).all()


@pytest.mark.parametrize("H,Hkv,n,top", [(16, 2, 131000, 32), (20, 10, 100000, 16)])
def test_documents_of_several_stretches(H, Hkv, n, top):
    """More than the forward's workspace holds at a time: the queries, or the heads, go through it in parts (17.7 and 8.7 GB of partial
    results); the masses of a block come from all of them."""
    require_gpu()
    say("block attention, several stretches", H, Hkv, n, top)
    d, scale = 128, 1 / math.sqrt(128)
    g = torch.Generator(device="cuda").manual_seed(7)
    q, k, v = (torch.randn(1, h, n, d, device="cuda", generator=g).bfloat16() for h in (H, Hkv, Hkv))
    idx = spk.sparsek_block_select(q, k, top)
    o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, scale, mass=True)
    torch.cuda.synchronize()
    assert ((mass.double().sum(2) / (n * (H // Hkv)) - 1).abs() < 1e-5).all()
    check_rows(q, k, v, None, idx, o, None, scale, (0, H // 2, H - 1), list(range(0, n, n // 9)) + [n - 1])


def test_more_blocks_than_one_pass_of_the_lists():
    """300000 tokens have 4688 blocks; the lists take 4096 at a time."""
    require_gpu()
    say("block attention, 300000 tokens")
    n, d, top = 300000, 64, 3
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v, dO = (torch.randn(1, 1, n, d, device="cuda", generator=g).bfloat16() for _ in range(4))
    idx = torch.randint(-1, n // 64, (1, 1, n, top), device="cuda", generator=g, dtype=torch.int32)
    idx[:, :, :, 2] = idx[:, :, :, 0]       # (and every block twice)
    o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125, mass=True)
    dq, dk, dv = spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.125)
    torch.cuda.synchronize()
    assert abs(float(mass.double().sum()) / n - 1) < 1e-5
    seen = torch.where(idx < (torch.arange(n, device="cuda") // 64).view(1, 1, n, 1), idx, -1)
    seen[..., 2] = -1
    seen[..., 1] = torch.where(seen[..., 1] == seen[..., 0], -1, seen[..., 1])
    check_rows(q, k, v, dO, seen.cpu(), o, dq, 0.125, (0,), list(range(0, n, 23456)) + [n - 1, n - 37856])
    assert torch.isfinite(dk).all() and torch.isfinite(dv).all()


@pytest.mark.parametrize("what", ["q", "k", "v", "dO"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite_reach_who_attends_them(what, value, d):
    """One such value, in a block that some rows attend and others do not, and in front of and behind queries of its own block: the
    rows that do not attend its key (or, for q and dO, the keys that its row does not attend) have the results they have without it."""
    require_gpu()
    say("block attention,", what, value)
    n, H, at, top = 500, 2, 150, 2
    q, k, v, dO = draw(83, 1, H, 1, n, d)
    idx = spk.sparsek_block_select(q, k, top)
    x = dict(q=q, k=k, v=v, dO=dO)
    runs = []
    for spoil in (False, True):
        if spoil:
            x[what][0, 0, at, 7] = value
        o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125, mass=True)
        runs.append((o, lse) + spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.125))
    torch.cuda.synchronize()
    (o, lse, dq, dk, dv), (o1, lse1, dq1, dk1, dv1) = runs
    see = ref.seen(idx[0, 0].cpu().numpy(), n).cuda()          # [queries, keys]
    if what in ("k", "v"):
        rows = see[:, at]                                      # who attends the key
        for h in range(H):
            assert torch.equal(o[0, h][~rows], o1[0, h][~rows]) and torch.equal(dq[0, h][~rows], dq1[0, h][~rows])
            assert torch.equal(lse[0, h][~rows], lse1[0, h][~rows])
            bad = ~torch.isfinite(o1[0, h]).all(1)
            assert torch.equal(bad[rows], torch.ones_like(bad[rows]))
        keys = see[rows].any(0)                                # keys that those rows attend
        assert torch.equal(dk[0, 0][~keys], dk1[0, 0][~keys]) and torch.equal(dv[0, 0][~keys], dv1[0, 0][~keys])
    else:
        rows = torch.arange(n, device="cuda") != at
        assert torch.equal(o[0, 0][rows], o1[0, 0][rows]) and torch.equal(o[0, 1], o1[0, 1])
        assert torch.equal(dq[0, 0][rows], dq1[0, 0][rows]) and torch.equal(dq[0, 1], dq1[0, 1])
        keys = see[at]
        assert torch.equal(dk[0, 0][~keys], dk1[0, 0][~keys]) and torch.equal(dv[0, 0][~keys], dv1[0, 0][~keys])
        assert not torch.isfinite(dk1[0, 0][keys]).all(1).any()


def test_results_do_not_depend_on_timing():
    require_gpu()
    say("block attention, twice")
    q, k, v, dO = draw(71, 2, 8, 2, 2500, 128)
    runs = []
    for _ in range(2):
        idx = spk.sparsek_block_select(q, k, 6)
        o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.1, mass=True)
        runs.append((idx, o, lse, mass) + spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.1))
    torch.cuda.synchronize()
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def test_training_step_replays_as_a_graph():
    """Selection, forward and backward captured once, replayed on new inputs with eager work in between, and on a side stream."""
    require_gpu()
    say("block attention as a graph")
    shape = (1, 4, 2, 700, 64)
    q, k, v, dO = draw(81, *shape)

    def step(q, k, v, dO):
        idx = spk.sparsek_block_select(q, k, 4)
        o, lse, mass = spk.sparsek_block_attn_fwd(q, k, v, idx, 0.125, mass=True)
        return (idx, o, lse, mass) + spk.sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, 0.125)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(q, k, v, dO)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(q, k, v, dO)
    for rep in range(4):
        new = draw(90 + rep, *shape)
        for a, b in zip((q, k, v, dO), new):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step(*new)):
            assert torch.equal(a, b), rep
        torch.cuda.synchronize()
