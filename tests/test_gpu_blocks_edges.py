"""The operators around an encoder's blocks where results depend on how sums,
roundings and rows are arranged: rows of very unequal weight, and the like.
The bounds count the roundings that the formulas of each operator leave."""
import math

import pytest
import torch

import blocks_reference as ref
import paper_2608_03199_gb300 as sieve
from test_gpu_encoder import BF16, DEV, FP16, FP32, gen, randn

pytestmark = pytest.mark.gpu
I32, I64 = torch.int32, torch.int64


# ---------------------------------------------------------------- embedding
@pytest.mark.parametrize("tokens,often,vocab,width", [(600, 0.95, 70, 24), (70_000, 0.5, 1_000, 33), (200_000, 0.99, 65, 8), (3_000, 1.0, 40, 260)])
def test_embed_backward_of_a_frequent_id(tokens, often, vocab, width):
    """One id has most tokens; of those beside it some have a few and some none."""
    g = gen(tokens)
    for frequent in (0, vocab // 2, vocab - 1):
        ids = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
        ids = torch.where((torch.rand(tokens, generator=g, device=DEV) < often) | (ids % 3 == 1), frequent, ids)
        dout = randn(g, tokens, width).to(BF16)
        want, bound = ref.embed_backward(dout, ids, vocab, 1.5, FP32)
        ref.assert_within(sieve.embed_backward(dout, ids, vocab, scale=1.5, out=torch.full((vocab, width), math.nan, device=DEV)), want, bound, "dtable")


def test_embed_backward_does_not_wait_for_a_frequent_id():
    """The blocks that look for rows without a token cost little even where four
    million tokens share one id: the call takes at most twice as long as one that writes no
    zeros (accumulate).  Reading all of that id's keys took 3.6 times as long."""
    ids = torch.full((1 << 22,), 3, device=DEV)
    dout, out, ws = torch.ones(1 << 22, 64, dtype=BF16, device=DEV), torch.zeros(40, 64, device=DEV), sieve.Workspace()

    def best(accumulate):
        times = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            sieve.embed_backward(dout, ids, 40, out=out, accumulate=accumulate, workspace=ws)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    added = best(True)
    assert best(False) < 2 * added
    assert (out[3] == 1 << 22).all() and not out[:3].any() and not out[4:].any()


# ------------------------------------------------------------ cross entropy
@pytest.mark.parametrize("rows", [120, 600, 270_000])
@pytest.mark.parametrize("down", [4, 12, 16, 20])
def test_cross_entropy_a_class_that_only_light_rows_reach(rows, down):
    """Light rows' dloss is 2^-down of the heavy ones', and one class has nothing of
    the heavy ones (its score there is -64).  Scores are zero else, so q is known: a
    light row's q is off by its rounding (2^-11; up to 256 rows hold the remainder too,
    2^-20) and by 2^-18 for exp and log, a sum of m terms by 2 m 2^-24; the weighted
    copy of h in fp16 is exact down to 2^-29 of its largest and off by 2^-40 of it below,
    twice that with the mantissa of dloss."""
    g = gen(down)
    live = min(rows, 600)
    at = torch.randperm(rows, generator=g, device=DEV)[:live].sort().values
    h = (randn(g, live, 256) / 16).to(FP16)
    light = torch.arange(live, device=DEV) % 2 == 0
    h[:, 0] = torch.where(light, 0.0, 1.0)
    h[4::40] = 0                                          # light rows of zeros
    dloss = (1 + torch.rand(live, generator=g, device=DEV)) * torch.where(light, 2.0 ** -down, 1.0)
    dloss[1::40] = 0                                      # heavy rows without a weight
    dloss[2::40] = -dloss[2::40]
    weight = torch.zeros(8, 256, dtype=FP16, device=DEV)
    weight[7, 0] = -64
    t = torch.randint(8, (live,), generator=g, device=DEV)
    t = torch.where(light, t, t % 7)
    h_all = torch.full((rows, 256), math.nan, dtype=FP16, device=DEV)
    d_all = torch.full((rows,), 1e30, device=DEV)
    t_all = torch.full((rows,), -1, device=DEV)
    h_all[at], d_all[at], t_all[at] = h, dloss, t
    loss, lse = sieve.cross_entropy(h_all, weight, t_all, check=True)
    dw = torch.empty(8, 256, device=DEV)
    sieve.cross_entropy_backward(d_all, h_all, weight, t_all, loss, lse, dweight=dw, check=True)
    x, gg = h[light].double(), dloss[light].double()
    q = 1 / 8 - (t[light] == 7).double()
    m = int(light.sum())
    off = (2.0 ** -20 if live <= 256 else 2.0 ** -11) + 2.0 ** -18 + 2 * m * 2.0 ** -24
    largest = float((dloss.abs() * h.abs().amax(1)).max())
    bound = off * (gg * q).abs() @ x.abs() + 2.0 ** -39 * largest * float(q.abs().sum()) + 1e-26
    ref.assert_within(dw[7], (gg * q) @ x, bound, "dweight")


@pytest.mark.parametrize("rows", [90, 700])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("weights", ["same", "differ"])
def test_cross_entropy_gradients_of_hidden_targets_and_tables(rows, dtype, weights):
    """A hidden target: p elsewhere, -1 at it.  Every class hidden: -1 at the
    target alone, in all three gradients."""
    g = gen(rows)
    h, weight, t = randn(g, rows, 72).to(dtype), randn(g, 300, 72).to(dtype), torch.randint(300, (rows,), generator=g, device=DEV)
    dloss = torch.full((rows,), 0.5, device=DEV) if weights == "same" else randn(g, rows)
    for b in (torch.where(torch.arange(300, device=DEV) % 3 == 0, -math.inf, randn(g, 300)), torch.full((300,), -math.inf, device=DEV)):
        loss, lse = sieve.cross_entropy(h, weight, t, bias=b, scale=0.25)
        dw = torch.empty(300, 72, device=DEV)
        got = dict(zip(("dh", "dweight", "dbias"), sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=b, scale=0.25, dweight=dw)))
        want, bound = ref.cross_entropy(h, weight, t, b, 0.25, dloss, FP32)
        for name, x in got.items():
            ref.assert_within(x, want[name], bound[name], name)


@pytest.mark.parametrize("rows,live", [(2_100, 256), (5_000, 200), (300_000, 31)])
@pytest.mark.parametrize("dtype,bias", [(BF16, False), (FP16, True)])
def test_cross_entropy_few_rows_in_a_large_batch(rows, live, dtype, bias):
    """Up to 256 rows with a target are worked out the same way whatever the
    batch that they come in: the bits of a call without the other rows."""
    g = gen(rows)
    weight, b = (randn(g, 900, 320) / 8).to(dtype), randn(g, 900) if bias else None
    at = torch.randperm(rows, generator=g, device=DEV)[:live].sort().values
    h, t, dloss = torch.full((rows, 320), math.nan, dtype=dtype, device=DEV), torch.full((rows,), -7, device=DEV), torch.ones(rows, device=DEV)
    h[at], t[at] = randn(g, live, 320).to(dtype), torch.randint(900, (live,), generator=g, device=DEV)
    for d in (dloss, dloss.index_copy(0, at, randn(g, live))):
        got = sieve.cross_entropy(h, weight, t, bias=b, check=True)
        alone = sieve.cross_entropy(h[at], weight, t[at], bias=b)
        assert torch.equal(got[0][at], alone[0]) and torch.equal(got[1][at], alone[1])
        got = sieve.cross_entropy_backward(d, h, weight, t, *got, bias=b, dweight=torch.empty(900, 320, device=DEV), check=True)
        alone = sieve.cross_entropy_backward(d[at], h[at], weight, t[at], *alone, bias=b, dweight=torch.empty(900, 320, device=DEV))
        assert torch.equal(got[0][at], alone[0]) and torch.equal(got[1], alone[1])
        assert not bias or torch.equal(got[2], alone[2])


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_cross_entropy_of_few_rows_in_pieces_of_the_classes(dtype):
    """More classes than the pool holds at a time for the 512 rows of a panel."""
    g = gen(40)
    h, weight, t = randn(g, 7, 8).to(dtype), randn(g, 1_200_007, 8).to(dtype), torch.tensor([0, 1_200_006, -1, 1_048_576, 5, 1_200_007, 600_000], device=DEV)
    dloss = randn(g, 7)
    loss, lse = sieve.cross_entropy(h, weight, t, check=True)
    dw = torch.full(weight.shape, math.nan, device=DEV)
    dh, dw, _ = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, dweight=dw, check=True)
    want, bound = ref.cross_entropy(h, weight, t, None, 1.0, dloss, FP32)
    for name, got in dict(loss=loss, lse=lse, dh=dh, dweight=dw).items():
        ref.assert_within(got, want[name], bound[name], name)


@pytest.mark.parametrize("rows", [1, 700])
def test_cross_entropy_weighted_rows_without_any_target_or_weight(rows):
    """fp16, dloss of every row another: no target, or weights of zero, both signs."""
    h, weight = torch.ones(rows, 64, dtype=FP16, device=DEV), torch.ones(70, 64, dtype=FP16, device=DEV)
    dloss = torch.arange(rows, device=DEV) - 0.5
    for t, d in ((torch.full((rows,), -1, device=DEV), dloss), (torch.arange(rows, device=DEV) % 70, torch.where(dloss > 9, 0.0, -0.0))):
        loss, lse = sieve.cross_entropy(h, weight, t)
        for dt in (FP16, FP32):
            dh, dw, _ = sieve.cross_entropy_backward(d, h, weight, t, loss, lse, dweight=torch.full((70, 64), math.nan, dtype=dt, device=DEV), check=True)
            assert not dh.any() and not dw.any()


def away(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("dtype,off", [(BF16, 2.0 ** -14), (FP16, 2.0 ** -15)])
def test_cross_entropy_few_rows_keep_what_rounding_q_leaves_off(dtype, off):
    """Two parts of q leave 2^-16 of it off (bf16; fp16 2^-22), the scores of 320
    products 20 steps of 2^-23 of |z|, about 1e-5 of p; one part would leave 1.6e-3 and
    2e-4 of dweight's norm."""
    g = gen(30)
    h, weight, t = randn(g, 200, 320).to(dtype), (randn(g, 900, 320) / 8).to(dtype), torch.randint(900, (200,), generator=g, device=DEV)
    for dloss in (torch.ones(200, device=DEV), randn(g, 200)):
        loss, lse = sieve.cross_entropy(h, weight, t)
        dw = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, dweight=torch.empty(900, 320, device=DEV))[1]
        assert away(dw, ref.cross_entropy(h, weight, t, None, 1.0, dloss)[0]["dweight"]) < off


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("rows", [100, 700])
def test_cross_entropy_dh_among_classes_that_are_much_alike(rows, dtype):
    """Every class is a common row and a fortieth of its own: dh is a difference, in
    which the rounding of a probability counts with its class' distance from the target's.
    Rounding q and the result leave less than two roundings of the type; what a row's
    rounded q add up to, times the common row, would leave over ten."""
    g = gen(31)
    common = randn(g, 128)
    weight = (common + randn(g, 2_000, 128) / 40).to(dtype)
    h, t = randn(g, rows, 128).to(dtype), torch.randint(2_000, (rows,), generator=g, device=DEV)
    dloss = torch.ones(rows, device=DEV)
    loss, lse = sieve.cross_entropy(h, weight, t)
    dh = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse)[0]
    assert away(dh, ref.cross_entropy(h, weight, t, None, 1.0, dloss)[0]["dh"]) < 2 * ref.U[dtype]


@pytest.mark.parametrize("rows,classes,steps", [(64, 40, (8, 8)), (300, 40, (8, 8)), (5_000, 1_000, (24, 16))])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_cross_entropy_scores_of_many_products_of_one_sign(rows, classes, steps, dtype):
    """The tensor cores add 16 products at a step and cut each off at 2^-25 of the
    power of two in the sum so far.  In a chunk of `steps` steps of one sign the sum
    is half of the chunk's on average, so a score is off by less than 17 steps / 2 of
    2^-25 of itself in fp16, and on average, with half of a unit cut off and sums of 1.44
    times their power of two, by 16 steps / 4 / 1.44.  Products of bf16 values from 1/2 to
    3/2 are multiples of 2^-16, sums of 384 of them below 2^10: nothing is cut off.  Each of
    the 128 / steps chunks is added with a rounding of 2^-24 (on average half of it), and the
    rest of lse takes 2^-22 (2^-24).  (In one chunk fp16 is off by 1.0e-5 and bf16 by
    2.1e-6.)  Up to 256 rows, and where every pair of blocks has one tile, chunks have 8
    steps, else 24 in bf16 and 16 in fp16 (1.6e-6 with 24)."""
    g = gen(32)
    h, weight = (0.5 + torch.rand(rows, 2048, generator=g, device=DEV)).to(dtype), (0.5 + torch.rand(classes, 2048, generator=g, device=DEV)).to(dtype)
    t = torch.zeros(rows, dtype=I64, device=DEV)
    lse = sieve.cross_entropy(h, weight, t, scale=40 / 2048)[1]
    want = torch.logsumexp(40 / 2048 * h.double() @ weight.double().T, 1)
    steps = steps[dtype == FP16]
    cut = steps if dtype == FP16 else 0
    assert ((lse.double() / want - 1).abs() < 8.5 * cut * 2.0 ** -25 + 128 / steps * 2.0 ** -24 + 2.0 ** -22).all()
    assert away(lse, want) < 4 / 1.44 * cut * 2.0 ** -25 + 128 / steps * 2.0 ** -25 + 2.0 ** -24


# ------------------------------------------------------------ residual norm
@pytest.mark.parametrize("dtype,wtype", [(FP32, FP32), (BF16, FP32), (FP16, FP16)])
def test_residual_norm_gradients_of_one_column(dtype, wtype):
    """One column less its mean is nothing: neither norm passes a gradient on,
    whatever its factor (316 here), so dh is alpha dstream and dy is zero."""
    g = gen(21)
    h, y, ds, dx = (randn(g, 700, 1).to(dtype) for _ in range(4))
    kw = dict(zip(("weight", "bias", "post_weight", "post_bias", "gate"), (randn(g, 1).to(wtype) for _ in range(5))))
    stats = sieve.residual_norm(h, y, alpha=-0.5, **kw)[2]
    dh, dy, dweight, dbias, dpw, dpb, dgate = sieve.residual_norm_backward(ds, dx, h, y, stats, alpha=-0.5, **kw)
    assert torch.equal(dh, -0.5 * ds) and not dy.any() and not dweight.any() and not dpw.any()
    sums = (700 / 152 + 65) * 2.0 ** -24
    for got, terms, factor in ((dbias, dx, 1), (dpb, ds, kw["gate"]), (dgate, ds, kw["post_bias"])):
        want, mag = float((terms.double() * factor).sum()), float((terms.double() * factor).abs().sum())
        assert abs(float(got) - want) <= (sums + 2.0 ** -22) * mag + ref.U[wtype] * abs(want)


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_residual_norm_means_of_equal_values(dtype):
    """Sums of small whole numbers are exact, so the mean of equal values is
    that value at every width, and what is left of them zero.  In the backward pass
    too; past 128 columns the sum of dstream and r d is rounded before the mean is
    taken off, and r times the mean is: two roundings of r d."""
    g = gen(22)
    for width in [*range(1, 260, 3), 301, 1001, 2100, 4099, 8191]:
        h, y, one = (torch.full((3, width), v, dtype=dtype, device=DEV) for v in (2.0, 3.0, 1.0))
        w, ds = torch.full((width,), 5.0, device=DEV), randn(g, 3, width).to(dtype)
        stream, x, stats = sieve.residual_norm(h, y, w, post_weight=w)
        assert (stats[0] == 3).all() and (stats[2] == 2).all() and torch.equal(stream, h) and not x.any(), width
        dh = sieve.residual_norm_backward(ds, one, h, y, stats, w, post_weight=w)[0]
        off = 0 if width <= 128 else 2 * 2.0 ** -24 * (5 * float(stats[3, 0]) + 6)
        assert ((dh.double() - ds.double()).abs() <= off + (0 if dtype == FP32 or not off else 2.0 ** -8 * ds.double().abs())).all(), width


# ------------------------------------------------------------------- graphs
FIRST_IN_A_GRAPH = """
import torch, sys
import paper_2608_03199_gb300 as sieve
g = torch.Generator("cuda").manual_seed(0)
x = torch.randn(300, 64, generator=g, device="cuda").half()
table = torch.randn(900, 64, generator=g, device="cuda").half()
ids = torch.randint(900, (300,), generator=g, device="cuda")
w = torch.ones(64, device="cuda")
dloss = torch.rand(300, generator=g, device="cuda")
ws = [sieve.Workspace() for _ in range(4)]
for i in ws:
    i.get(1 << 28, x.device)
def step():
    h = sieve.embed(ids, table)
    stream, y, stats = sieve.residual_norm(h, x, w, post_weight=w)
    loss, lse = sieve.cross_entropy(y, table, ids, workspace=ws[0])
    dy, dtable, _ = sieve.cross_entropy_backward(dloss, y, table, ids, loss, lse, dweight=torch.empty(900, 64, device="cuda"), workspace=ws[1])
    dh, dx, dw, *_ = sieve.residual_norm_backward(None, dy, h, x, stats, w, post_weight=w, workspace=ws[2])
    sieve.embed_backward(dh, ids, 900, out=dtable, accumulate=True, workspace=ws[3])
    return loss, lse, dtable, dx, dw, stream
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    got = step()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, step())), "the plain calls give other bits"
print("captured")
"""


def test_first_calls_of_a_process_in_a_graph():
    """No call before the capture: what the library looks up once it can look
    up while a stream is captured."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FIRST_IN_A_GRAPH], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "captured" in run.stdout, run.stdout + run.stderr[-2000:]
