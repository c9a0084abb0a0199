"""Token log probabilities, entropy, best alternatives and their gradient on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding
    binding.lib()
    return binding


def sum_error(V):
    """Relative error of a sum of V terms taken by at least 128 threads, then joined: sequential roundings of a part."""
    return (V / 128 + 64) * 2.0 ** -24 + 2.0 ** -21


def check(B, x, targets, n_top, scale, store=None):
    """x: CPU tensor [rows, vocab]; store: CUDA view holding the same values."""
    logits = x.cuda() if store is None else store
    r = B.szo_token_logprobs(logits, None if targets is None else targets.cuda(), n_top=n_top, scale=scale)
    xs = x.double().numpy()
    lp, lse, ent = ref.logprobs(xs, scale)
    rows, V = xs.shape
    with np.errstate(invalid="ignore"):
        size = np.nan_to_num(np.abs(lse), posinf=0, nan=0)
        top = np.nan_to_num(np.max(np.where(np.isfinite(xs), np.abs(xs), 0), 1) * scale)
        tol = sum_error(V) + 2.0 ** -22 * (size + 1)
    bad_row = np.isnan(lse) | np.isposinf(lse)
    good = ~bad_row & np.isfinite(lse)
    g_lse, g_ent = r.lse.double().cpu().numpy(), r.entropy.double().cpu().numpy()
    assert np.isnan(g_lse[bad_row]).all() and np.isnan(g_ent[bad_row]).all()
    assert (np.abs(g_lse[good] - lse[good]) <= tol[good]).all()
    empty = np.isneginf(lse)
    assert np.isneginf(g_lse[empty]).all() and (g_ent[empty] == 0).all()
    # sum p x over sum p, both with their own roundings; |log p| weighted by p is at most log V + 1
    assert (np.abs(g_ent[good] - ent[good]) <= (tol[good] + 2.0 ** -22) * (2 * np.log(V) + 8)).all()

    def compare(got, want, rr):
        fin = np.isfinite(want)
        assert np.array_equal(np.isneginf(got), np.isneginf(want))
        # a scaled logit is rounded once, and so is the difference
        assert (np.abs(got[fin] - want[fin]) <= (tol[rr] + 2.0 ** -23 * (top[rr] + size[rr]))[fin]).all()
    if targets is not None:
        got = r.logp.double().cpu().numpy()
        for i in range(targets.shape[1]):
            t = targets[:, i].numpy()
            inside = (t >= 0) & (t < V)
            assert (got[t < 0, i] == 0).all() and np.isnan(got[t >= V, i]).all()
            use = inside & ~bad_row
            compare(got[use, i], lp[use, t[use]], np.flatnonzero(use))
            assert np.isnan(got[inside & bad_row, i]).all()
    if n_top:
        key = np.where(np.isnan(xs), np.inf, xs) + 0.0
        first = np.isnan(xs)
        order = np.lexsort((np.broadcast_to(np.arange(V), xs.shape), -key, ~first), axis=1)[:, :n_top]
        assert np.array_equal(r.top_ids.cpu().numpy(), order)
        use = np.flatnonzero(~bad_row)
        got = r.top_logp.double().cpu().numpy()
        for i in range(n_top):
            compare(got[use, i], lp[use, order[use, i]], use)
    return r


def values(g, rows, V, dt, spread=3.0):
    return torch.from_numpy(g.normal(0, spread, (rows, V))).to(DT[dt])


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V,pad,nt,top", [(1, 1, 0, 1, 1), (3, 7, 0, 2, 7), (5, 32, 3, 1, 32), (2, 1024, 0, 0, 20), (7, 1001, 1, 3, 5),
                                               (1, 32000, 0, 1, 20), (9, 32000, 8, 2, 32), (160, 5003, 0, 1, 0), (200, 4099, 2, 4, 20),
                                               (2, 50272, 0, 64, 1), (3, 131077, 0, 1, 32), (1, 500009, 0, 2, 32), (300, 33, 0, 1, 3)])
def test_against_64_bits(B, dt, rows, V, pad, nt, top):
    g = np.random.default_rng(V + rows)
    x = values(g, rows, V, dt)
    store = torch.full((rows, V + pad), float("nan"), dtype=DT[dt], device="cuda")     # what lies between the rows is not read
    store[:, :V] = x.cuda()
    t = torch.from_numpy(g.integers(-1, V, (rows, nt)).astype(np.int32)) if nt else None
    for scale in (1.0, 0.6, 2.5):
        check(B, x, t, top, scale, store[:, :V])
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_masks_ties_and_non_finite_rows(B, dt):
    g = np.random.default_rng(2)
    V = 3001
    x = values(g, 14, V, dt)
    low = torch.finfo(DT[dt]).min
    x[0, g.random(V) < 0.9] = float("-inf")
    x[1] = float("-inf")                                 # nothing left
    x[2] = float("-inf")
    x[2, 1234] = 0.5                                     # one token left
    x[3, g.random(V) < 0.9] = low                        # masked by the type's lowest value
    x[4] = low
    x[5] = 1.0                                           # all equal
    x[6] = torch.from_numpy(np.round(g.normal(0, 1, V))).to(DT[dt])        # many ties
    x[7, 17] = float("nan")
    x[8, 18] = float("inf")
    x[9, 100:900] = 0.0
    x[9, 150:800:2] = -0.0
    x[10] = torch.sort(x[10]).values                     # rising
    x[11] = torch.sort(x[11], descending=True).values
    x[12, ::256] += 50                                   # the largest all lie a stride apart
    x[13, 0], x[13, V - 1] = 60, 60.0                    # ends
    t = torch.from_numpy(g.integers(-1, V, (14, 3)).astype(np.int32))
    t[2, 0], t[13, 0], t[13, 1], t[0, 0] = 1234, 0, V - 1, int(np.flatnonzero(np.isneginf(x[0].numpy() if dt != "bf16" else x[0].float().numpy()))[0])
    for top in (1, 5, 32):
        for scale in (1.0, 0.5, 1.7):
            check(B, x, t, top, scale)
    # the same in many rows at once (rows spread over blocks otherwise)
    many = x.repeat(40, 1)
    check(B, many, t.repeat(40, 1), 20, 1.0)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_best_tokens_where_the_largest_logits_crowd(B, dt):
    g = np.random.default_rng(8)
    V = 120001
    x = values(g, 5, V, dt)
    vec = 4 if dt == "f32" else 8
    crowd = (np.arange(V) // vec) % 256 < 31             # all with a few of a block's threads
    x[0, crowd] += 50
    x[1, crowd] = 50.0
    x[2, : V - 700] = float("-inf")                      # a mask that leaves some, all at one end
    x[3] = float("-inf")
    x[3, [5, 70000, V - 1]] = torch.tensor([1.0, 1.0, 2.0]).to(DT[dt])     # fewer than are asked for
    x[4, crowd] = float("nan")
    for top in (1, 31, 32):
        check(B, x, None, top, 1.0)
    check(B, x.repeat(80, 1), None, 32, 1.0)             # (a block per row)


def test_targets_beyond_the_vocabulary_are_reported(B):
    x = torch.randn(2, 100)
    r = B.szo_token_logprobs(x.cuda(), torch.tensor([[100, 5], [-5, 2 ** 31 - 1]], dtype=torch.int32, device="cuda"))
    assert B.device_status() == -1
    got = r.logp.cpu()
    assert got[0, 0].isnan() and got[1, 1].isnan() and got[1, 0] == 0 and got[0, 1].isfinite()
    assert B.device_status() == 0


def grad_bound(want, xs, scale, targets, d_logp, d_entropy, dt):
    """fp32 throughout: p is off by the roundings of its exponent (2^-23 of the logit's size, lse's own error given), the
    formula by a handful of roundings of its terms, then the one rounding of the result."""
    lp, lse, ent = ref.logprobs(xs, scale)
    p = np.exp(lp)
    with np.errstate(invalid="ignore"):
        size = np.nan_to_num(np.abs(lse)) + np.abs(np.where(np.isfinite(xs), xs, 0)).max(1) * scale
    rel = (sum_error(xs.shape[1]) + 2.0 ** -21 * (size + 4))[:, None]
    gsum = np.abs(d_logp).sum(1, keepdims=True)
    term = p * gsum + (0 if d_entropy is None else np.abs(d_entropy)[:, None] * p * (np.abs(np.where(p > 0, lp, 0)) + np.abs(np.nan_to_num(ent))[:, None] + 4))
    return scale * (rel * term + 2.0 ** -21 * gsum * (want != 0)) + HALF[dt] * np.abs(want) + (2.0 ** -25 if dt == "f16" else 1e-38)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V,pad,nt,ent", [(1, 1, 0, 1, True), (3, 7, 0, 2, True), (5, 33, 3, 1, False), (2, 1024, 0, 0, True), (7, 1001, 1, 3, True),
                                               (4, 32000, 0, 1, True), (300, 257, 0, 2, False), (2, 50272, 8, 64, True), (3, 131077, 1, 2, True)])
def test_gradient_against_the_formula(B, dt, rows, V, pad, nt, ent):
    g = np.random.default_rng(V + 5 * rows)
    x = values(g, rows, V, dt)
    if V > 100:
        x[0, g.random(V) < 0.5] = float("-inf")
        x[rows - 1, : V // 2] = torch.finfo(DT[dt]).min
    t = torch.from_numpy(g.integers(-1, V, (rows, nt)).astype(np.int32))
    if nt > 1:
        t[:, 1] = t[:, 0]                                # the same target twice
    dl, de = g.normal(0, 1, (rows, nt)).astype(np.float32), g.normal(0, 0.5, rows).astype(np.float32)
    store = torch.full((rows, V + pad), 7.0, dtype=DT[dt], device="cuda")
    store[:, :V] = x.cuda()
    for scale in (1.0, 0.7):
        r = B.szo_token_logprobs(store[:, :V], t.cuda() if nt else None, scale=scale)
        args = (t.cuda() if nt else None, r.lse, r.entropy, torch.from_numpy(dl).cuda() if nt else None, torch.from_numpy(de).cuda() if ent else None)
        got = B.szo_token_logprobs_bwd(store[:, :V], *args, scale=scale)
        want = ref.logprobs_grad(x.double().numpy(), scale, t.numpy(), dl.astype(np.float64), de.astype(np.float64) if ent else None)
        tol = grad_bound(want, x.double().numpy(), scale, t.numpy(), dl.astype(np.float64), de.astype(np.float64) if ent else None, dt)
        bad = ~(np.abs(got.double().cpu().numpy() - want) <= tol)
        assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got.double().cpu().numpy() - want).max())
    # in place, what lies between the rows untouched
    buf = store.clone()
    B.szo_token_logprobs_bwd(buf[:, :V], *args, scale=0.7, out=buf[:, :V])
    assert torch.equal(buf[:, :V], got) and (buf[:, V:] == 7).all()
    # into rows of another stride
    buf = torch.full((rows, V + 5), 9.0, dtype=DT[dt], device="cuda")
    B.szo_token_logprobs_bwd(store[:, :V], *args, scale=0.7, out=buf[:, :V])
    assert torch.equal(buf[:, :V], got) and (buf[:, V:] == 9).all()
    assert B.device_status() == 0


def test_gradient_against_differences(B):
    """Central differences of the GPU's own results (fp32): step 1/64, so that a difference of the sums carries 64 times
    their error (2^-20 each for these 40 logits) and the third derivative's h^2/6."""
    g = np.random.default_rng(8)
    V, h = 40, 1.0 / 64
    x = torch.from_numpy(g.normal(0, 1, (1, V))).float()
    t = torch.tensor([[3, 9]], dtype=torch.int32).cuda()
    dl, de = torch.tensor([[1.0, -0.5]]).cuda(), torch.tensor([0.7]).cuda()

    def f(z):
        r = B.szo_token_logprobs(z.cuda(), t.expand(z.shape[0], 2).contiguous(), scale=0.9)
        return ((r.logp * dl).sum(1) + r.entropy * de).double().cpu()
    eye = torch.eye(V) * h
    diff = (f(x + eye) - f(x - eye)) / (2 * h)
    r = B.szo_token_logprobs(x.cuda(), t, scale=0.9)
    got = B.szo_token_logprobs_bwd(x.cuda(), t, r.lse, r.entropy, dl, de, scale=0.9).double().cpu()[0]
    assert (got - diff).abs().max() <= 64 * 8 * 2.0 ** -20 + h * h


def test_rows_with_nothing_left_or_nan(B):
    x = torch.randn(4, 500)
    x[1] = float("-inf")
    x[2, 7] = float("nan")
    t = torch.full((4, 1), 3, dtype=torch.int32).cuda()
    r = B.szo_token_logprobs(x.cuda(), t)
    one = torch.ones(4, 1, device="cuda")
    got = B.szo_token_logprobs_bwd(x.cuda(), t, r.lse, r.entropy, one, one[:, 0].contiguous()).cpu()
    assert (got[1] == 0).all() and got[2].isnan().all() and got[0].isfinite().all() and got[3].isfinite().all()


def test_no_rows(B):
    r = B.szo_token_logprobs(torch.empty(0, 10, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"), n_top=3)
    assert r.logp.shape == (0, 2) and r.top_ids.shape == (0, 3)
    z = torch.empty(0, device="cuda")
    assert B.szo_token_logprobs_bwd(torch.empty(0, 10, device="cuda"), None, z, z, None).shape == (0, 10)


def test_captured_and_replayed(B):
    x = torch.randn(6, 32000, device="cuda").bfloat16()
    t = torch.randint(0, 32000, (6, 2), dtype=torch.int32, device="cuda")
    B.szo_token_logprobs(x, t, n_top=5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = B.szo_token_logprobs(x, t, n_top=5)
        d = B.szo_token_logprobs_bwd(x, t, r.lse, r.entropy, torch.ones_like(r.logp))
    for i in range(3):
        x.copy_(torch.randn(6, 32000, device="cuda") * (i + 1))
        graph.replay()
        want = B.szo_token_logprobs(x, t, n_top=5)
        for a, b in zip(r, want):
            assert torch.equal(a, b)
        assert torch.equal(d, B.szo_token_logprobs_bwd(x, t, want.lse, want.entropy, torch.ones_like(want.logp)))


def test_binding_refusals(B):
    x = torch.randn(4, 50, device="cuda")
    t = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    for bad in (lambda: B.szo_token_logprobs(x.t(), None), lambda: B.szo_token_logprobs(x, t.long()), lambda: B.szo_token_logprobs(x, t[:3]),
                lambda: B.szo_token_logprobs(x.double()), lambda: B.szo_token_logprobs(x, t.cpu()),
                lambda: B.szo_token_logprobs_bwd(x, t, torch.zeros(3, device="cuda"), None, torch.zeros(4, device="cuda")),
                lambda: B.szo_token_logprobs_bwd(x, t, x[:, 0].contiguous(), None, x[:, 0].contiguous(), out=x.half())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.szo_token_logprobs(x, t, n_top=33), lambda: B.szo_token_logprobs(x, t, scale=0.0),
                lambda: B.szo_token_logprobs_bwd(x, t, x[:, 0].contiguous(), None, x[:, 0].contiguous(), x[:, 0].contiguous())):
        with pytest.raises(B.SzoError):
            bad()


def masked_rows(g, V, dt):
    """Rows as masks make them: half masked, none, everything, all but one, half at the type's lowest value, all but two."""
    x = values(g, 6, V, dt)
    x[0, g.random(V) < 0.5] = float("-inf")
    x[2] = float("-inf")
    x[3] = float("-inf")
    x[3, V // 2] = 0.5
    x[4, g.random(V) < 0.5] = torch.finfo(DT[dt]).min
    x[5, 2:] = float("-inf")
    return x


def f32(v):
    return float(np.float32(v))                          # (the scale that the kernel gets)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 0.02, 0.021, 50.0, 100.0, 1e4, 1e30])
@pytest.mark.parametrize("V,pad", [(1003, 0), (40003, 2)])
def test_masked_rows_at_every_scale(B, dt, scale, V, pad):
    """Odd widths too: the ends of a row that is no whole number of vectors are filled up with -inf."""
    g = np.random.default_rng(V)
    x = masked_rows(g, V, dt)
    store = torch.full((6, V + pad), float("nan"), dtype=DT[dt], device="cuda")
    store[:, :V] = x.cuda()
    t = torch.from_numpy(g.integers(-1, V, (6, 3)).astype(np.int32))
    t[3, 0] = V // 2
    for top in (0, 5):
        check(B, x, t, top, f32(scale), store[:, :V])
    check(B, x.repeat(60, 1), t.repeat(60, 1), 0, f32(scale))          # (a block per row)


GRADIENTS = {"wide": [(1e-30, None), (1e-30, 1.0), (1e-3, None), (0.02, 1.0), (0.021, 1.0), (1.0, 100.0), (1.0, 1e4), (1.0, 1e6),
                      (1.0, 1e36), (1.0, 1e37), (1e-3, 1e37), (50.0, 1.0), (50.0, 100.0), (100.0, 1e6), (1e4, 1.0), (1e30, None)],
             "f16": [(1e-30, None), (1e-3, None), (0.02, 1.0), (0.02, 1e4), (1.0, 100.0), (50.0, 1.0), (50.0, None)]}      # (results within fp16)


@pytest.mark.parametrize("dt,scale,size", [(d, *c) for d in ("f32", "bf16", "f16") for c in GRADIENTS["f16" if d == "f16" else "wide"]])
@pytest.mark.parametrize("V,pad", [(1003, 0), (40003, 2)])
def test_gradient_of_masked_rows_at_every_scale_and_weight(B, dt, scale, size, V, pad):
    """A masked token's gradient is 0 (its target's share apart), whatever the scale and the weight of the entropy.  On top of
    grad_bound: a probability below the fp32 range (2^-126) counts as 0, so its term is off by at most that much (twice: what
    is below it is 2^y, of which p is 2^y times a number next to 1)."""
    g = np.random.default_rng(V + 1)
    scale = f32(scale)
    x = masked_rows(g, V, dt)
    store = torch.full((6, V + pad), 7.0, dtype=DT[dt], device="cuda")
    store[:, :V] = x.cuda()
    t = g.integers(-1, V, (6, 2)).astype(np.int32)
    t[0, 0] = int(np.flatnonzero(np.isneginf(x[0].double().numpy()))[0])             # a masked target
    dl = g.normal(0, 1, (6, 2)).astype(np.float32)
    de = None if size is None else (size * g.uniform(-1, 1, 6)).astype(np.float32)
    d_t = torch.from_numpy(t).cuda()
    r = B.szo_token_logprobs(store[:, :V], d_t, scale=scale)
    got = B.szo_token_logprobs_bwd(store[:, :V], d_t, r.lse, r.entropy, torch.from_numpy(dl).cuda(), None if de is None else torch.from_numpy(de).cuda(),
                                   scale=scale).double().cpu().numpy()
    assert (got[2] == 0).all()                           # nothing left
    use = np.array([0, 1, 3, 4, 5])
    xs, de64 = x.double().numpy()[use], None if de is None else de[use].astype(np.float64)
    want = ref.logprobs_grad(xs, scale, t[use], dl[use].astype(np.float64), de64)
    tol = grad_bound(want, xs, scale, t[use], dl[use].astype(np.float64), de64, dt)
    lp, _, ent = ref.logprobs(xs, scale)
    weight = np.abs(dl[use].astype(np.float64)).sum(1, keepdims=True)
    if de64 is not None:
        weight = weight + np.abs(de64)[:, None] * (np.abs(np.where(np.isneginf(lp), 0, lp)) + np.abs(ent)[:, None])
    tol = tol + scale * 2.0 ** -125 * weight
    bad = ~(np.abs(got[use] - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], got[use][bad][:4], want[bad][:4])
