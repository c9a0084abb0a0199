"""Cross entropy from hidden states and its gradient on the GPU, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests import head_ce_reference as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}                     # half a step, relative
ERR_ARG = -1


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding
    binding.lib()
    return binding


def problem(rows, vocab, d, dt, seed, spread=2.5, known=2.0, none=0.2):
    """h knows something of its target, from nothing to nearly everything; some rows have no target."""
    g = torch.Generator("cuda").manual_seed(seed)
    W = (torch.randn(vocab, d, device="cuda", generator=g) * spread / d ** 0.5).to(DT[dt])
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    k = torch.rand(rows, 1, device="cuda", generator=g) * known
    h = (torch.randn(rows, d, device="cuda", generator=g) + k * W[t.long()].float()).to(DT[dt])
    t[torch.rand(rows, device="cuda", generator=g) < none] = -1
    return h, W, t, g


def logit_error(h, W, scale):
    """A logit is the sum of d exact products, 16 at a time: d / 16 + 17 roundings or truncations of at most the largest partial
    sum (2^-23 each), and two roundings (2^-23) of scaling it; per row, of the largest."""
    big = (h.double().abs() @ W.double().abs().T).amax(-1) * scale
    return ((h.shape[1] / 16 + 17) * 2.0 ** -23 + 2.0 ** -22) * big


def check_forward(got, h, W, t, scale):
    loss, lse = ref.forward(h, W, t, scale)
    e = logit_error(h, W, scale)
    # sums of weights: exp2 and differences of logits in base 2 (2^-21 and 2^-23 of their size), at most 512 additions in a row
    # (2^-24 each) with a few joins
    summed = 600 * 2.0 ** -24 + 2.0 ** -20
    assert ((got.lse.double() - lse).abs() <= e + summed + 2.0 ** -21 * lse.abs() + e * 2.0 ** -20).all()
    rel = 2 * e + summed + 2.0 ** -21 * (lse.abs() + 1) + 2.0 ** -21 * loss   # of the others' weight relative to the target's
    # (d loss / d log of that weight is 1 - exp(-loss), and at most 1)
    ok = (got.loss.double() - loss).abs() <= rel * torch.where(rel < 0.01, -torch.expm1(-loss) * 1.01, 1.0) + 2.0 ** -21 * loss + 1e-37
    assert ok.all(), (got.loss[~ok][:4], loss[~ok][:4])
    assert (got.loss[t < 0] == 0).all()


def backward_bounds(h, W, t, lse, a, b, scale, dt):
    """G's relative error is that of p (twice a logit's, exp2's 2^-21 and the rounding of x - lse) and half a step; sums of fp32
    add 2^-23 each along at most d or rows or vocab / 16 steps; fp16's subnormals 2^-25 relative to 2^13 times the row's weight; the result
    half a step."""
    dh, dW, G = ref.backward(h, W, t, lse, a, b, scale)
    hd, Wd, V = h.double(), W.double(), W.shape[0]
    e = logit_error(h, W, scale) + 2.0 ** -21 * lse.double().abs() + 2.0 ** -20
    there = (t >= 0) & (t < V)
    aa = torch.where(there, a.double(), 0.0).abs()
    bb = torch.zeros_like(aa) if b is None else b.double().abs()
    p = torch.exp((hd @ Wd.T) * scale - lse.double()[:, None])
    dG = G.abs() * (HALF[dt] * 1.001) + scale * (aa + bb)[:, None] * p * (2 * e)[:, None]
    if dt == "f16":
        dG += scale * (aa + bb)[:, None] * 2.0 ** -37
    live = ((aa != 0) | (bb != 0))[:, None]
    dG = torch.where(live, dG, 0.0)
    hz = torch.where(live, hd, 0.0)
    steps = 2.0 ** -23 * 1.01
    Ga = G.abs() + dG
    eh = dG @ Wd.abs() + (V / 16 + 40) * steps * (Ga @ Wd.abs())
    eW = dG.T @ hz.abs() + (h.shape[0] / 16 + 40) * steps * (Ga.T @ hz.abs())
    if dt == "f16":
        # rows of h at their weight over the largest one's, the subnormals' half step 2^-25
        top = scale * (aa + bb).max()
        eW += Ga.T @ (live * 2.0 ** -24 * (top / (scale * (aa + bb)[:, None]).clamp(min=1e-300)).clamp(max=1e30)).expand_as(hz)
    tiny = 2.0 ** -25 if dt == "f16" else 1e-38
    return dh, eh + HALF[dt] * (dh.abs() + eh) + tiny, dW, eW + HALF[dt] * (dW.abs() + eW) + tiny


def within(got, want, bound):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], bound[bad][:4])


SHAPES = [(1, 1, 8), (1, 500, 64), (3, 7, 72), (77, 1111, 264), (128, 256, 128), (129, 257, 1024), (300, 9001, 136), (5, 20000, 512), (513, 700, 2056),
          (16, 33000, 64)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,d", SHAPES)
def test_forward(B, dt, rows, vocab, d):
    h, W, t, _ = problem(rows, vocab, d, dt, seed=rows + vocab)
    for scale in (1.0, 0.37):
        check_forward(B.szo_head_ce(h, W, t, scale=scale), h, W, t, scale)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,d", SHAPES)
def test_backward(B, dt, rows, vocab, d):
    h, W, t, g = problem(rows, vocab, d, dt, seed=rows + vocab + 1)
    scale = 0.8
    lse = B.szo_head_ce(h, W, t, scale=scale).lse
    a = torch.randn(rows, device="cuda", generator=g)
    for b in (None, 0.3 * torch.randn(rows, device="cuda", generator=g)):
        dh, dW = B.szo_head_ce_bwd(h, W, t, lse, a, b, scale=scale)
        wh, eh, wW, eW = backward_bounds(h, W, t, lse, a, b, scale, dt)
        within(dh, wh, eh)
        within(dW, wW, eW)
    # one of the two alone: the same numbers
    assert torch.equal(B.szo_head_ce_bwd(h, W, t, lse, a, b, scale=scale, need_dW=False)[0], dh)
    assert torch.equal(B.szo_head_ce_bwd(h, W, t, lse, a, b, scale=scale, need_dh=False)[1], dW)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt,rows,vocab,d", [("bf16", 16, 140001, 64), ("f16", 100, 131073, 72), ("bf16", 140, 140001, 64), ("f16", 4100, 50001, 64),
                                             ("bf16", 2300, 60000, 136)])
def test_vocabularies_of_many_pieces(B, dt, rows, vocab, d):
    """G in several pieces of the vocabulary, its buffers used again; last pieces of a few entries."""
    h, W, t, g = problem(rows, vocab, d, dt, seed=rows)
    lse = B.szo_head_ce(h, W, t).lse
    a, b = torch.randn(rows, device="cuda", generator=g), 0.2 * torch.randn(rows, device="cuda", generator=g)
    check_forward(B.szo_head_ce(h, W, t), h, W, t, 1.0)
    dh, dW = B.szo_head_ce_bwd(h, W, t, lse, a, b)
    wh, eh, wW, eW = backward_bounds(h, W, t, lse, a, b, 1.0, dt)
    within(dh, wh, eh)
    within(dW, wW, eW)
    assert torch.equal(B.szo_head_ce_bwd(h, W, t, lse, a, b, need_dW=False)[0], dh)
    assert torch.equal(B.szo_head_ce_bwd(h, W, t, lse, a, b, need_dh=False)[1], dW)
    assert B.device_status() == 0


def test_two_calls_at_once(B):
    """Two gradients on two streams share the SMs; each hands out its own units."""
    p = [problem(600 + 40 * i, 30000, 256, "bf16", 30 + i) for i in (0, 1)]
    lse = [B.szo_head_ce(h, W, t).lse for h, W, t, _ in p]
    a = [torch.randn(x[0].shape[0], device="cuda") for x in p]
    want = [B.szo_head_ce_bwd(*p[i][:3], lse[i], a[i]) for i in (0, 1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in (0, 1)]
    for _ in range(3):
        got = [None, None]
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = [B.szo_head_ce_bwd(*p[i][:3], lse[i], a[i]) for _ in range(3)]
        torch.cuda.synchronize()
        for i in (0, 1):
            for dh, dW in got[i]:
                assert torch.equal(dh, want[i][0]) and torch.equal(dW, want[i][1])
    assert B.device_status() == 0


def test_confident_rows_keep_their_relative_precision(B):
    d, vocab = 128, 2000
    h, W, t, _ = problem(64, vocab, d, "bf16", 3, known=0.0, none=0.0)
    h = (h.float() + torch.linspace(2, 7, 64, device="cuda")[:, None] * W[t.long()].float()).to(torch.bfloat16)
    got = B.szo_head_ce(h, W, t)
    loss, _ = ref.forward(h, W, t, 1.0)
    assert loss.min() < 1e-9 and loss.max() > 1e-6
    check_forward(got, h, W, t, 1.0)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_slices_of_wider_buffers(B, dt):
    """h and W as slices, a vocabulary smaller than the matrix, results into slices: what lies around stays."""
    rows, vocab, d = 70, 600, 136
    hw, Ww, t, g = problem(rows, vocab + 41, d + 24, dt, 8)
    t = t.clamp(max=vocab - 1)
    h, W = hw[:, 8:8 + d], Ww[:vocab, 16:16 + d]
    got = B.szo_head_ce(h, W, t)
    check_forward(got, h, W, t, 1.0)
    a = torch.randn(rows, device="cuda", generator=g)
    bh, bW = torch.full((rows + 2, d + 16), 7.0, dtype=DT[dt], device="cuda"), torch.full((vocab + 3, d + 8), 7.0, dtype=DT[dt], device="cuda")
    B.szo_head_ce_bwd(h, W, t, got.lse, a, out_dh=bh[1:1 + rows, 8:8 + d], out_dW=bW[1:1 + vocab, :d])
    wh, eh, wW, eW = backward_bounds(h, W, t, got.lse, a, None, 1.0, dt)
    within(bh[1:1 + rows, 8:8 + d], wh, eh)
    within(bW[1:1 + vocab, :d], wW, eW)
    bh[1:1 + rows, 8:8 + d] = 7.0
    bW[1:1 + vocab, :d] = 7.0
    assert (bh == 7).all() and (bW == 7).all()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_rows_that_weigh_nothing(B, dt):
    """Rows without a target may hold anything; nothing of them reaches a gradient."""
    rows, vocab, d = 150, 900, 64
    h, W, t, g = problem(rows, vocab, d, dt, 11)
    a = torch.randn(rows, device="cuda", generator=g)
    a[7], t[7] = 0.0, 5                                   # a target with no weight
    a[t < 0] = float("nan")                               # d_loss of a row without a target is not used
    dead = (t < 0) | (a == 0)
    h[dead] = float("nan")
    got = B.szo_head_ce(h, W, t)
    assert (got.loss[t < 0] == 0).all() or got.loss[t < 0].isnan().any()
    live = ~dead
    check_forward(B.HeadCe(got.loss[live], got.lse[live]), h[live], W, t[live], 1.0)
    dh, dW = B.szo_head_ce_bwd(h, W, t, got.lse, a)
    assert (dh[dead] == 0).all()
    wh, eh, wW, eW = backward_bounds(h[live], W, t[live], got.lse[live], a[live], None, 1.0, dt)
    within(dh[live], wh, eh)
    within(dW, wW, eW)
    # no row weighs anything
    dh, dW = B.szo_head_ce_bwd(h, W, torch.full_like(t, -1), got.lse, a)
    assert (dh == 0).all() and (dW == 0).all()
    # nor does what W holds
    Wn = W.clone()
    Wn[3, 1] = float("inf")
    assert (B.szo_head_ce_bwd(h, Wn, t, got.lse, a, need_dW=False)[0][dead] == 0).all()
    # a row of which lse says that it has no probability anywhere
    l2 = got.lse.clone()
    l2[live] = -float("inf")
    dh, dW = B.szo_head_ce_bwd(h, W, t, l2, torch.nan_to_num(a))
    assert (dh == 0).all() and (dW == 0).all()


def test_nan_and_infinities_stay_in_their_rows(B):
    rows, vocab, d = 200, 700, 128
    h, W, t, _ = problem(rows, vocab, d, "bf16", 12, none=0.0)
    h[3, 5], h[130, 0], h[131, 1] = float("nan"), float("inf"), -float("inf")
    got = B.szo_head_ce(h, W, t)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[3, 130, 131]] = True
    assert got.loss[bad].isnan().all() and got.lse[bad].isnan().all()
    check_forward(B.HeadCe(got.loss[~bad], got.lse[~bad]), h[~bad], W, t[~bad], 1.0)
    dh, dW = B.szo_head_ce_bwd(h, W, t, got.lse, torch.ones(rows, device="cuda"))
    assert dh[bad].isnan().all() and not dh[~bad].isnan().any() and dW.isnan().any()


def test_targets_beyond_the_vocabulary_are_reported(B):
    h, W, t, _ = problem(40, 300, 64, "bf16", 13, none=0.0)
    t[4], t[9] = 300, 2 ** 31 - 1
    got = B.szo_head_ce(h, W, t)
    assert B.device_status() == ERR_ARG
    bad = t >= 300
    assert got.loss[bad].isnan().all() and got.lse.isfinite().all()
    check_forward(B.HeadCe(got.loss[~bad], got.lse[~bad]), h[~bad], W, t[~bad], 1.0)
    a = torch.ones(40, device="cuda")
    dh, dW = B.szo_head_ce_bwd(h, W, t, got.lse, a)
    assert (dh[bad] == 0).all()
    wh, eh, wW, eW = backward_bounds(h, W, t, got.lse, a, None, 1.0, "bf16")
    within(dh, wh, eh)
    within(dW, wW, eW)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_weights_of_very_different_sizes(B, dt):
    """Rows weighed from 2^-12 to 2^12: each row's dh keeps its own precision."""
    rows, vocab, d = 100, 1500, 128
    h, W, t, _ = problem(rows, vocab, d, dt, 14, none=0.0)
    a = 2.0 ** torch.linspace(-12, 12, rows, device="cuda").round() * torch.where(torch.arange(rows, device="cuda") % 2 == 0, 1.0, -1.7)
    lse = B.szo_head_ce(h, W, t).lse
    dh, dW = B.szo_head_ce_bwd(h, W, t, lse, a)
    wh, eh, wW, eW = backward_bounds(h, W, t, lse, a, None, 1.0, dt)
    within(dh, wh, eh)
    within(dW, wW, eW)


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 100.0, 1e30])
def test_extreme_scales(B, scale):
    h, W, t, _ = problem(30, 400, 64, "bf16", 15, none=0.0)
    check_forward(B.szo_head_ce(h, W, t, scale=scale), h, W, t, scale)


def test_logits_beyond_fp32(B):
    """-inf counts nothing, +inf makes its row NaN."""
    h, W, t, _ = problem(12, 400, 64, "bf16", 15, none=0.0)
    W[:, 0] = -1e3
    W[5, 0] = 0.0
    h[:, 0] = 0.0
    h[0, 0], h[1, 0], h[2, 0] = 1e38, -1e38, 1e38
    t[0], t[2] = 5, 6
    got = B.szo_head_ce(h, W, t)
    x5 = (h[[0, 2], 1:].double() @ W[5, 1:].double())
    assert ((got.lse[[0, 2]].double() - x5).abs() <= logit_error(h[:, 1:], W[:, 1:], 1.0)[[0, 2]] + 2.0 ** -20 * (1 + x5.abs())).all()
    assert got.loss[0] == 0 and got.loss[2] == float("inf") and got.loss[1].isnan() and got.lse[1].isnan()
    check_forward(B.HeadCe(got.loss[3:], got.lse[3:]), h[3:], W, t[3:], 1.0)


def test_no_rows_and_empty_gradients(B):
    W = torch.randn(50, 64, device="cuda").bfloat16()
    h, t, e = W[:0], torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    got = B.szo_head_ce(h, W, t)
    assert got.loss.shape == (0,) and got.lse.shape == (0,)
    dW = torch.full((52, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    B.szo_head_ce_bwd(h, W, t, e, e, out_dW=dW[1:51])
    assert (dW[1:51] == 0).all() and (dW[0] == 3).all() and (dW[51] == 3).all()


def test_same_bits_again_on_other_streams_and_in_graphs(B):
    rows, vocab, d = 260, 5000, 192
    h, W, t, g = problem(rows, vocab, d, "bf16", 16)
    a = torch.randn(rows, device="cuda", generator=g)

    def both():
        f = B.szo_head_ce(h, W, t)
        return (f.loss, f.lse) + B.szo_head_ce_bwd(h, W, t, f.lse, a)
    first = [x.clone() for x in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = both()
    graph.replay()
    torch.cuda.synchronize()
    for x, y, z in zip(first, second, third):
        assert torch.equal(x, y) and torch.equal(x, z)
    # the graph serves new contents
    h2, W2, t2, _ = problem(rows, vocab, d, "bf16", 17)
    h.copy_(h2)
    W.copy_(W2)
    t.copy_(t2)
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(third, both()):
        assert torch.equal(x, y)
    assert B.device_status() == 0


def test_workspaces_may_hold_anything(B):
    rows, vocab, d = 130, 3000, 72
    h, W, t, g = problem(rows, vocab, d, "f16", 18)
    a = torch.randn(rows, device="cuda", generator=g)
    L, st = B.lib(), torch.cuda.current_stream().cuda_stream
    want = B.szo_head_ce(h, W, t)
    wh, wW = B.szo_head_ce_bwd(h, W, t, want.lse, a)
    for byte in (0x00, 0xff, 0x7f):
        n = L.szo_head_ce_workspace_bytes(rows, vocab, d)
        ws = torch.full((n + 16,), byte, dtype=torch.uint8, device="cuda")
        loss = torch.empty(rows, device="cuda")
        B._check(L.szo_head_ce(h.data_ptr(), d, W.data_ptr(), d, 2, rows, vocab, d, 1.0, t.data_ptr(), loss.data_ptr(), None, ws.data_ptr(), n, st))
        assert torch.equal(loss, want.loss) and (ws[n:] == byte).all()
        n = L.szo_head_ce_bwd_workspace_bytes(rows, vocab, d, 1, 1)
        ws = torch.full((n + 16,), byte, dtype=torch.uint8, device="cuda")
        dh, dW = torch.empty_like(h), torch.empty_like(W)
        B._check(L.szo_head_ce_bwd(h.data_ptr(), d, W.data_ptr(), d, 2, rows, vocab, d, 1.0, t.data_ptr(), want.lse.data_ptr(), a.data_ptr(), None,
                                   dh.data_ptr(), d, dW.data_ptr(), d, ws.data_ptr(), n, st))
        assert torch.equal(dh, wh) and torch.equal(dW, wW) and (ws[n:] == byte).all()


def test_binding_refuses_what_does_not_fit(B):
    h, W, t, _ = problem(8, 50, 64, "bf16", 19)
    e = torch.zeros(8, device="cuda")
    bad = [(h.float(), W.float(), t), (h, W.half(), t), (h, W[:, :56], t), (h, W, t.long()), (h, W, t[:7]), (h.T, W.T, t), (h.cpu(), W, t), (h, W.T, t),
           (h, W, t.cpu())]
    for args in bad:
        with pytest.raises(ValueError):
            B.szo_head_ce(*args)
        with pytest.raises(ValueError):
            B.szo_head_ce_bwd(*args, e, e)
    for lse, a, b in [(e[:7], e, None), (e, e.double(), None), (e, e, e[:3]), (e.cpu(), e, None)]:
        with pytest.raises(ValueError):
            B.szo_head_ce_bwd(h, W, t, lse, a, b)
    with pytest.raises(ValueError):
        B.szo_head_ce_bwd(h, W, t, e, e, out_dh=h.half())
    with pytest.raises(B.SzoError):                       # a view that does not start on 16 bytes
        B.szo_head_ce(torch.zeros(8 * 64 + 8, dtype=torch.bfloat16, device="cuda")[4:4 + 512].view(8, 64), W, t)


def test_agrees_with_the_log_probabilities_of_logits(B):
    """The same quantity by way of stored logits (szo_token_logprobs)."""
    h, W, t, _ = problem(64, 3000, 256, "bf16", 20)
    got = B.szo_head_ce(h, W, t)
    x = (h.double() @ W.double().T).float()
    r = B.szo_token_logprobs(x, t.view(-1, 1))
    assert torch.allclose(got.lse, r.lse, rtol=0, atol=1e-4) and torch.allclose(got.loss, -r.logp[:, 0], rtol=0, atol=1e-4)


@pytest.mark.parametrize("rows", [12, 200])
def test_rows_whose_logits_are_all_minus_infinity(B, rows):
    """log sum exp is -inf and the loss, a difference of two infinities, NaN; with a vocabulary of the target alone too.  Nothing of
    them reaches a gradient."""
    h, W, t, g = problem(rows, 400, 64, "bf16", 21, none=0.0)
    W[:, 0] = -1e3
    h[:, 0] = 0.0
    dead = torch.zeros(rows, dtype=torch.bool, device="cuda")
    dead[[2, rows - 1]] = True
    h[dead, 0] = 1e38
    got = B.szo_head_ce(h, W, t)
    assert (got.lse[dead] == -float("inf")).all() and got.loss[dead].isnan().all()
    check_forward(B.HeadCe(got.loss[~dead], got.lse[~dead]), h[~dead], W, t[~dead], 1.0)
    a = torch.randn(rows, device="cuda", generator=g)
    dh, dW = B.szo_head_ce_bwd(h, W, t, got.lse, a)
    assert (dh[dead] == 0).all()
    wh, eh, wW, eW = backward_bounds(h[~dead], W, t[~dead], got.lse[~dead], a[~dead], None, 1.0, "bf16")
    within(dh[~dead], wh, eh)
    within(dW, wW, eW)
    one = B.szo_head_ce(h, W[:1], torch.zeros_like(t))
    assert (one.lse[dead] == -float("inf")).all() and one.loss[dead].isnan().all() and (one.loss[~dead] == 0).all()
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [40, 300])
def test_rows_without_a_target_have_no_loss_whatever_they_hold(B, dt, rows):
    """A padding row's NaN or infinity stays in its lse: the losses' sum is that of the other rows."""
    h, W, t, _ = problem(rows, 500, 64, dt, 22)
    t[:4] = -1
    none = t < 0
    h[none, 3] = float("nan")
    h[1], h[2, 5], h[3] = float("inf"), -float("inf"), 0.0
    got = B.szo_head_ce(h, W, t)
    assert (got.loss[none] == 0).all() and got.loss.isfinite().all()
    odd = none.clone()
    odd[3] = False                                        # (log of the vocabulary's size)
    assert got.lse[odd].isnan().all()
    check_forward(B.HeadCe(got.loss[~odd], got.lse[~odd]), h[~odd], W, t[~odd], 1.0)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt,rows,vocab,d", [("bf16", 17000, 12301, 64), ("f16", 9001, 13345, 136), ("bf16", 9000, 700, 72), ("f16", 33000, 12289, 72),
                                             ("bf16", 8193, 16001, 264)])
def test_many_rows(B, dt, rows, vocab, d):
    """Pieces of the vocabulary at their shortest, with their buffers used again; dh alone of some thousand rows at a time (4352 and
    3841 to four times 6656 and 6376), into a slice and with nothing around it touched."""
    h, W, t, g = problem(rows, vocab, d, dt, seed=rows)
    got = B.szo_head_ce(h, W, t)
    check_forward(got, h, W, t, 1.0)
    a, b = torch.randn(rows, device="cuda", generator=g), 0.2 * torch.randn(rows, device="cuda", generator=g)
    dh, dW = B.szo_head_ce_bwd(h, W, t, got.lse, a, b)
    wh, eh, wW, eW = backward_bounds(h, W, t, got.lse, a, b, 1.0, dt)
    within(dh, wh, eh)
    within(dW, wW, eW)
    assert torch.equal(B.szo_head_ce_bwd(h, W, t, got.lse, a, b, need_dh=False)[1], dW)
    wide = torch.full((rows + 2, d + 16), 7.0, dtype=DT[dt], device="cuda")
    alone = B.szo_head_ce_bwd(h, W, t, got.lse, a, b, out_dh=wide[1:-1, 8:-8], need_dW=False)[0].clone()
    within(alone, wh, eh)
    wide[1:-1, 8:-8] = 7.0
    assert (wide == 7).all()
    L, n = B.lib(), B.lib().szo_head_ce_bwd_workspace_bytes(rows, vocab, d, 1, 0)
    ws, out = torch.full((n + 16,), 0x7f, dtype=torch.uint8, device="cuda"), torch.empty_like(h)
    B._check(L.szo_head_ce_bwd(h.data_ptr(), d, W.data_ptr(), d, 1 if dt == "bf16" else 2, rows, vocab, d, 1.0, t.data_ptr(), got.lse.data_ptr(), a.data_ptr(),
                               b.data_ptr(), out.data_ptr(), d, None, 0, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(out, alone) and (ws[n:] == 0x7f).all()
    assert B.device_status() == 0


@pytest.mark.parametrize("dt,rows,vocab,d", [("bf16", 17, 33001, 1032), ("f16", 17, 33001, 1032), ("bf16", 100, 70001, 520), ("bf16", 128, 8300, 4096)])
def test_few_rows_of_a_large_matrix(B, dt, rows, vocab, d):
    """W of more than 64 MB, whose last part the gradient keeps in L2 between its two readings: kept from within a tile on, over one piece of
    G and over two."""
    assert vocab * d * 2 > 64 << 20
    h, W, t, g = problem(rows, vocab, d, dt, seed=rows + d)
    t[0] = vocab - 1
    lse = B.szo_head_ce(h, W, t).lse
    a, b = torch.randn(rows, device="cuda", generator=g), 0.2 * torch.randn(rows, device="cuda", generator=g)
    dh, dW = B.szo_head_ce_bwd(h, W, t, lse, a, b)
    wh, eh, wW, eW = backward_bounds(h, W, t, lse, a, b, 1.0, dt)
    within(dh, wh, eh)
    within(dW, wW, eW)
    assert torch.equal(B.szo_head_ce_bwd(h, W, t, lse, a, b, need_dW=False)[0], dh)
    assert torch.equal(B.szo_head_ce_bwd(h, W, t, lse, a, b, need_dh=False)[1], dW)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt,rows,vocab,d", [("bf16", 3137, 700, 8192), ("f16", 3400, 523, 8192), ("bf16", 3137, 10900, 8192), ("bf16", 1600, 300, 16392)])
def test_rows_taken_in_bands(B, dt, rows, vocab, d):
    """Hidden states of more than 48 MB go by in bands of row tiles (7 and 6 of 13; 7 of 14; the same over two pieces of G; 4 and 3 of 7)."""
    h, W, t, g = problem(rows, vocab, d, dt, seed=rows + d)
    got = B.szo_head_ce(h, W, t)
    check_forward(got, h, W, t, 1.0)
    a = torch.randn(rows, device="cuda", generator=g)
    dh, dW = B.szo_head_ce_bwd(h, W, t, got.lse, a)
    wh, eh, wW, eW = backward_bounds(h, W, t, got.lse, a, None, 1.0, dt)
    within(dh, wh, eh)
    within(dW, wW, eW)
    assert B.device_status() == 0
