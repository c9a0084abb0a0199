"""Token generation from the 8-bit cache (szo_model_enable_decode_kv8) and scoring (szo_model_token_logprobs) against the
oracle: its incremental decode with every key and value passed through the cache's number format, in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from paper_2406_02913_b200 import workloads as wl
from tests import kv8_reference as ref
from tests.fixtures import DecoderFixture

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding
    binding.lib()
    return binding


class Stored(list):
    """A layer list of the oracle's cache whose entries go through the 8-bit format as they are appended."""

    def __init__(self, n_layers, which, page, as_stored):
        super().__init__([None] * n_layers)
        self.which, self.page, self.as_stored, self.caches = which, page, as_stored, {}

    def __setitem__(self, l, x):
        nseq, n, hkv, hd = x.shape
        old = 0 if self[l] is None else self[l].shape[1]
        out = torch.empty_like(x)
        for b in range(nseq):
            c = self.caches.setdefault((l, b), ref.Cache(np.zeros((2, 64, hkv, self.page, hd), np.uint8), np.zeros((64, hkv, 2))))
            c.write(range(64), old, self.as_stored(x[b, old:]).numpy(), self.which)
            out[b] = torch.from_numpy(c.values(range(64), n, self.which))
        super().__setitem__(l, out)


def kv8_cache(n_layers, page, as_stored):
    cache = mo.KVCache(n_layers)
    cache.k, cache.v = Stored(n_layers, 0, page, as_stored), Stored(n_layers, 1, page, as_stored)
    return cache


@pytest.mark.parametrize("name,page", [("tiny", 16), ("tiny_gqa", 32), ("tiny_opt", 16), ("tiny_lut", 128)])
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_decode_steps_match_the_oracle_with_the_cache_format(B, name, page, act):
    """Prompts, chunks and single tokens over several pages.  A key or value whose computed value lies within its own error of
    a border between two codes may take the other one: the fp32 path (1e-6) hardly meets one (a step of one element in a
    thousand times as many moves a logit by well below 2e-3 of the largest), the bf16 path (2^-8) in one element of 30, a
    thirtieth of the cache's own rounding noise on top of its 2e-2 without an 8-bit cache."""
    fx = DecoderFixture(name, seed=6, mask="random", B=3, S=64)
    om = fx.oracle_model()
    S_np = om.S + np.float32(1e-3)
    toks = fx.batch(0)[:, :60]
    lin_W = om.lin_W(S_np)
    a, md, tol = (B.SZO_F32, B.MODE_FP32_VALIDATE, 2e-3) if act == "f32" else (B.SZO_BF16, B.MODE_SPARSE_ADD, 4e-2)
    as_stored = (lambda x: x.float().double()) if act == "f32" else (lambda x: x.bfloat16().double())
    S = torch.from_numpy(S_np.copy()).cuda()
    m = B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), S, act_dtype=a, linear_mode=md, max_batch=fx.B, max_seq=fx.S)
    m.enable_decode(kv8_page_tokens=page)
    m.enable_decode(kv8_page_tokens=page)                # (again: nothing happens)
    far = 0.0
    for calls in ((5, 3, 1, 1, 1, 20, 1), (40, 1, 16, 1)):
        cache, plain, at = kv8_cache(om.cfg.n_layers, page, as_stored), mo.KVCache(om.cfg.n_layers), 0
        for T in calls:
            want = mo.decode_step(om.cfg, om.params, lin_W, toks[:, at:at + T], cache).numpy()
            exact = mo.decode_step(om.cfg, om.params, lin_W, toks[:, at:at + T], plain).numpy()
            got = m.decode_step(torch.from_numpy(np.ascontiguousarray(toks[:, at:at + T])).cuda(), at).cpu().numpy()
            at += T
            top = np.max(np.abs(want))
            assert np.max(np.abs(got - want)) <= tol * top, (name, act, at, np.max(np.abs(got - want)) / top)
            far = max(far, np.max(np.abs(want - exact)) / top)
    assert far > 0                                       # (the format does show: the comparison is with it and not without)
    assert B.device_status() == 0
    m.close()


def test_graph_replay_equals_the_launch_by_launch_form(B):
    fx = DecoderFixture("small_gqa", seed=12, mask="random", B=2, S=48)
    toks = torch.from_numpy(fx.batch(0)).cuda()
    out = []
    for graphs in (False, True):
        S = torch.from_numpy(fx.S_init.copy()).cuda()
        m = B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), S, act_dtype=B.SZO_BF16, linear_mode=B.MODE_SPARSE_ADD, max_batch=2, max_seq=48)
        m.enable_decode(kv8_page_tokens=16)
        stream = torch.cuda.Stream() if graphs else torch.cuda.default_stream()
        stream.wait_stream(torch.cuda.default_stream())
        with torch.cuda.stream(stream):
            got, at = [], 0
            for T in (17, 1, 1, 1, 2, 1, 1, 20):
                got.append(m.decode_step(toks[:, at:at + T].contiguous(), at).clone())
                at += T
        torch.cuda.synchronize()
        out.append(got)
        m.close()
    for x, y in zip(*out):
        assert torch.equal(x, y)
    assert B.device_status() == 0


def test_kv8_decode_refusals(B):
    fx = DecoderFixture("tiny", seed=6, mask="random", B=2, S=16, n_layers=1)
    make = lambda: B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), torch.from_numpy(fx.S_init.copy()).cuda(), act_dtype=B.SZO_BF16,
                           linear_mode=B.MODE_SPARSE_ADD, max_batch=fx.B, max_seq=fx.S)
    toks = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    m = make()
    with pytest.raises(B.SzoError):
        m.enable_decode(kv8_page_tokens=20)
    with pytest.raises(B.SzoError):                      # no cache yet
        m.decode_step(toks, 0)
    m.enable_decode(kv8_page_tokens=16)
    for other in (None, 32):
        with pytest.raises(B.SzoError):
            m.enable_decode(kv8_page_tokens=other)
    with pytest.raises(B.SzoError):                      # beyond max_seq
        m.decode_step(toks, 14)
    m.decode_step(toks, 12)
    m.close()
    m = make()
    m.enable_decode()
    with pytest.raises(B.SzoError):
        m.enable_decode(kv8_page_tokens=16)
    m.close()


@pytest.mark.parametrize("name", ["tiny", "tiny_gqa", "tiny_opt"])
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_token_logprobs_of_a_model(B, name, act):
    """Next-token log probabilities against the oracle's logits (as the decode tests: 1e-4 of the largest logit on the fp32
    path, 2e-2 on the bf16 path, twice for a difference of two), their mean against the library's own loss of the same
    logits, and given candidates and alternatives."""
    fx = DecoderFixture(name, seed=6, mask="random", B=3, S=20)
    om = fx.oracle_model()
    toks = fx.batch(0)
    lin_W = om.lin_W(om.S)
    hs = mo.hidden_states(om.cfg, om.params, lin_W, toks)
    logits = (hs @ torch.as_tensor(np.asarray(om.params["lm_head"]), dtype=torch.float64).T).reshape(60, -1)
    want = torch.log_softmax(logits, -1)
    a, md, tol = (B.SZO_F32, B.MODE_FP32_VALIDATE, 1e-4) if act == "f32" else (B.SZO_BF16, B.MODE_PAIRED, 2e-2)
    m = B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), torch.from_numpy(fx.S_init.copy()).cuda(), act_dtype=a, linear_mode=md, max_batch=3,
                max_seq=20)
    d_toks = torch.from_numpy(toks).cuda()
    tol *= 2 * logits.abs().max().item()
    r = m.token_logprobs(d_toks, n_top=4)
    nxt = np.concatenate([toks[:, 1:], np.full((3, 1), -1)], 1).reshape(-1)
    live = nxt >= 0
    got = r.logp.cpu().double()[:, 0]
    assert (got[~live] == 0).all()
    assert (got[live] - want[np.flatnonzero(live), nxt[live]]).abs().max() <= tol
    ent = -(want.exp() * want).sum(1)
    assert (r.entropy.cpu().double() - ent).abs().max() <= 2 * tol * (1 + ent.max())
    loss = m.loss(d_toks).item()
    assert abs(-got[live].mean().item() - loss) <= 1e-5 * abs(loss)
    best = torch.topk(want, 4).values
    assert (r.top_logp.cpu().double() - best).abs().max() <= tol
    assert (want.gather(1, r.top_ids.cpu().long()) - r.top_logp.cpu().double()).abs().max() <= tol
    t = torch.randint(-1, fx.shape["vocab"], (60, 5), dtype=torch.int32)
    r = m.token_logprobs(d_toks, targets=t.cuda())
    for i in range(5):
        use = (t[:, i] >= 0).numpy()
        assert (r.logp.cpu().double()[use, i] - want[np.flatnonzero(use), t[use, i].long()]).abs().max() <= tol
    with pytest.raises(B.SzoError):
        m.token_logprobs(d_toks, n_top=33)
    with pytest.raises(ValueError):
        m.token_logprobs(d_toks, targets=t[:59].cuda())
    with pytest.raises(ValueError):
        m.token_logprobs(d_toks.long(), targets=t.cuda())
    assert B.device_status() == 0
    m.close()


def test_token_logprobs_needs_the_next_token_loss(B):
    fx = DecoderFixture("tiny", seed=6, mask="random", B=2, S=16, n_layers=1)
    m = B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), torch.from_numpy(fx.S_init.copy()).cuda(), act_dtype=B.SZO_BF16,
                linear_mode=B.MODE_SPARSE_ADD, loss_kind=B.LOSS_CLS2, max_batch=2, max_seq=16)
    with pytest.raises(B.SzoError) as ei:
        m.token_logprobs(torch.zeros((2, 8), dtype=torch.int32, device="cuda"))
    assert ei.value.name == "SZO_ERR_UNSUPPORTED"
    m.close()


def test_generate_and_score_together(B):
    """A run as a program makes it: a ragged batch of prompts written and attended, tokens appended one by one, every step's
    logits scored with alternatives, the scores' gradient taken; against the same run in 64 bits."""
    g = np.random.default_rng(40)
    hkv, H, d, page, V = 2, 8, 64, 16, 997
    lens = [37, 5, 64]
    caps = [n + 6 for n in lens]
    counts = [-(-c // page) for c in caps]
    order = g.permutation(sum(counts) + 1)
    table = np.full((3, max(counts)), -1, np.int32)
    pages, at = [], 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        pages.append(order[at:at + c])
        at += c
    cache = B.Kv8Cache.empty(sum(counts) + 1, hkv, page, d)
    mine = ref.Cache(np.zeros((2, sum(counts) + 1, hkv, page, d), np.uint8), np.zeros((sum(counts) + 1, hkv, 2)))
    kv_len = torch.zeros(3, dtype=torch.int32, device="cuda")
    start = torch.zeros(4, dtype=torch.int32, device="cuda")
    d_table = torch.from_numpy(table).cuda()
    W = torch.from_numpy(g.normal(0, 0.3, (H * d, V))).float()
    now = [0, 0, 0]
    for step in range(6):
        news = lens if step == 0 else [1, 1, 1]
        now = [a + n for a, n in zip(now, news)]
        rows = sum(news)
        kv_len.copy_(torch.tensor(now, dtype=torch.int32))
        start.copy_(torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32))
        batch = B.Kv8Batch(d_table, kv_len, rows, start, max(news))
        qkv = torch.from_numpy(g.normal(0, 1, (rows, (H + 2 * hkv) * d))).bfloat16()
        dev = qkv.cuda()
        k, v = dev[:, H * d:(H + hkv) * d], dev[:, (H + hkv) * d:]
        B.szo_kv8_write(cache, batch, k, v)
        o = B.szo_attention_kv8(cache, batch, dev[:, :H * d])
        last = torch.tensor(np.cumsum(news) - 1).cuda()
        logits = o[last].float() @ W.cuda()
        t = torch.from_numpy(g.integers(0, V, (3, 2)).astype(np.int32)).cuda()
        r = B.szo_token_logprobs(logits, t, n_top=3, scale=0.9)
        grad = B.szo_token_logprobs_bwd(logits, t, r.lse, r.entropy, torch.ones_like(r.logp), torch.ones_like(r.entropy), scale=0.9)
        x = qkv.double().numpy()
        o_ref, wide = np.zeros((3, H * d)), np.zeros((3, H * d))
        for b in range(3):
            rr = slice(int(start[b]), int(start[b + 1]))
            for which in (0, 1):
                lo = (H + which * hkv) * d
                mine.write(pages[b], now[b] - news[b], x[rr, lo:lo + hkv * d].reshape(-1, hkv, d), which)
            oo, ww, _, _ = ref.attention(x[rr, :H * d].reshape(-1, H, d)[-1:], mine.values(pages[b], now[b], 0), mine.values(pages[b], now[b], 1), now[b] - 1, d ** -0.5)
            o_ref[b], wide[b] = oo.reshape(-1), ww.reshape(-1)
        # attention: its 11-bit weights (2^-11 and as much again for everything else) and the one rounding of o; then the product
        # with W in fp32 (512 terms)
        want = o_ref @ W.double().numpy()
        err = (wide * 2.0 ** -10 + np.abs(o_ref) * 2.0 ** -8) @ np.abs(W.double().numpy())
        slack = err + 512 * 2.0 ** -24 * (np.abs(o_ref) @ np.abs(W.double().numpy()))
        assert (np.abs(logits.double().cpu().numpy() - want) <= slack).all()
        # the scores are those of the logits at hand
        lg = logits.double().cpu().numpy()
        lp, lse, ent = ref.logprobs(lg, 0.9)
        tt = t.cpu().numpy()
        assert np.abs(np.take_along_axis(lp, tt, 1) - r.logp.double().cpu().numpy()).max() <= 1e-5 * (1 + np.abs(lse).max())
        assert np.array_equal(r.top_ids.cpu().numpy(), np.argsort(-lg, 1, kind="stable")[:, :3])
        gw = ref.logprobs_grad(lg, 0.9, tt, np.ones((3, 2)), np.ones(3))
        assert np.abs(grad.double().cpu().numpy() - gw).max() <= 2e-5
    assert B.device_status() == 0


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("nseq,seq", [(1, 40), (3, 33)])
def test_one_key_value_head_and_an_odd_number_of_pages(B, act, nseq, seq, monkeypatch):
    """Every layer's scales start where szo_kv8_write takes them, whatever pages x heads is (tolerances: above)."""
    monkeypatch.setitem(wl.MODEL_SHAPES, "tiny_one_kv_head", dict(wl.MODEL_SHAPES["tiny"], n_kv_heads=1, n_layers=3))
    fx = DecoderFixture("tiny_one_kv_head", seed=6, mask="random", B=nseq, S=seq)
    om = fx.oracle_model()
    toks = fx.batch(0)
    lin_W = om.lin_W(om.S)
    a, md, tol = (B.SZO_F32, B.MODE_FP32_VALIDATE, 2e-3) if act == "f32" else (B.SZO_BF16, B.MODE_SPARSE_ADD, 4e-2)
    as_stored = (lambda x: x.float().double()) if act == "f32" else (lambda x: x.bfloat16().double())
    m = B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), torch.from_numpy(fx.S_init.copy()).cuda(), act_dtype=a, linear_mode=md, max_batch=nseq,
                max_seq=seq)
    m.enable_decode(kv8_page_tokens=16)
    cache, at = kv8_cache(om.cfg.n_layers, 16, as_stored), 0
    for T in (20, 1, 5, 1, 1, 4):
        want = mo.decode_step(om.cfg, om.params, lin_W, toks[:, at:at + T], cache).numpy()
        got = m.decode_step(torch.from_numpy(np.ascontiguousarray(toks[:, at:at + T])).cuda(), at).cpu().numpy()
        at += T
        assert np.max(np.abs(got - want)) <= tol * np.max(np.abs(want))
    assert B.device_status() == 0
    m.close()
