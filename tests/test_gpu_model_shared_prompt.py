"""A model whose sequences continue one prompt (szo_model_decode_share), and its next-token losses without logits
(szo_model_token_losses), against the same model without either."""
import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from tests.fixtures import DecoderFixture

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding
    binding.lib()
    return binding


def make(B, fx, act="bf16", **kw):
    a, md = (B.SZO_F32, B.MODE_FP32_VALIDATE) if act == "f32" else (B.SZO_BF16, B.MODE_SPARSE_ADD)
    kw.setdefault("max_batch", fx.B)
    kw.setdefault("max_seq", fx.S)
    return B.Model(fx.shape, fx.names, fx.gpu_tensors(torch, None), torch.from_numpy(fx.S_init.copy()).cuda(), act_dtype=a, linear_mode=md, **kw)


# room for 65536 positions makes the attention read shared pages apart; with little room a batch goes to the attention that shares nothing
@pytest.mark.parametrize("name,page,max_seq", [("tiny", 16, 64), ("tiny_gqa", 32, 64), ("tiny_opt", 16, 64), ("tiny", 16, 65536), ("tiny_gqa", 32, 131072)])
@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("graphs", [False, True])
def test_sequences_continue_one_prompt(B, name, page, max_seq, act, graphs):
    """Every sequence gets the logits that it has when the prompt was its own.  Codes of positions that differ by the roundings of another
    batch size may fall on the other side of a border: bounds as in test_decode_steps_match_the_oracle_with_the_cache_format."""
    fx = DecoderFixture(name, seed=6, mask="random", B=4, S=64, **({"n_layers": 1} if max_seq > 64 else {}))
    toks = torch.from_numpy(fx.batch(0)).cuda()
    tol = 2e-3 if act == "f32" else 4e-2
    stream = torch.cuda.Stream() if graphs else torch.cuda.default_stream()
    stream.wait_stream(torch.cuda.default_stream())
    for n in (2 * page + 5, page, page - 3):
        if n > 50:
            continue
        got, want = [], []
        for shared in (True, False):
            m = make(B, fx, act, max_seq=max_seq, max_batch=4) if max_seq == 64 else make(B, fx, act, max_seq=max_seq, max_batch=4, loss_kind=B.LOSS_CLS2)
            m.enable_decode(kv8_page_tokens=page)
            with torch.cuda.stream(stream):
                prompt = toks[:1, :n].contiguous()
                if shared:
                    m.decode_step(prompt, 0)
                    m.decode_share(4, n)
                else:
                    m.decode_step(prompt.expand(4, n).contiguous(), 0)
                at = n
                for T in (1, 1, 3, 1):
                    (got if shared else want).append(m.decode_step(toks[:, at:at + T].contiguous(), at).clone())
                    at += T
                # fewer sequences than share the prompt
                (got if shared else want).append(m.decode_step(toks[:2, at:at + 1].contiguous(), at).clone())
            torch.cuda.synchronize()
            assert B.device_status() == 0
            m.close()
        for x, y in zip(got, want):
            assert (x - y).abs().max() <= tol * y.abs().max()


def test_sharing_ends_and_protects_its_pages(B):
    fx = DecoderFixture("tiny", seed=7, mask="random", B=3, S=64)
    toks = torch.from_numpy(fx.batch(0)).cuda()
    m = make(B, fx)
    with pytest.raises(B.SzoError):                      # no 8-bit cache yet
        m.decode_share(2, 16)
    m.enable_decode(kv8_page_tokens=16)
    for args in ((0, 16), (4, 16), (2, -1), (2, 65)):
        with pytest.raises(B.SzoError):
            m.decode_share(*args)
    m.decode_step(toks[:, :40].contiguous(), 0)          # each its own
    own = m.decode_step(toks[:, 40:41].contiguous(), 40)
    m.decode_share(3, 40)
    with pytest.raises(B.SzoError):                      # would write a shared page
        m.decode_step(toks[:, 31:32].contiguous(), 31)
    other = m.decode_step(toks[:, 40:41].contiguous(), 40)
    assert torch.allclose(other[0], own[0], atol=float(own.abs().max()) * 4e-2) and not torch.allclose(other[1], own[1], atol=1e-3)
    m.decode_share(1, 0)                                 # their own pages again (the third page, which was copied to, written anew)
    again = m.decode_step(toks[:, 32:41].contiguous(), 32)
    assert torch.allclose(again, own, atol=float(own.abs().max()) * 4e-2)
    m.decode_step(toks[:, :5].contiguous(), 0)
    assert B.device_status() == 0
    m.close()


def test_long_chunks_after_sharing(B, monkeypatch):
    """Chunks of so many tokens that sharing gains nothing, at a length whose attention takes the most workspace."""
    from paper_2406_02913_b200 import workloads as wl
    monkeypatch.setitem(wl.MODEL_SHAPES, "tiny_one_kv_head", dict(wl.MODEL_SHAPES["tiny_gqa"], n_kv_heads=1, n_layers=1))
    fx = DecoderFixture("tiny_one_kv_head", seed=8, mask="random", B=2, S=64)
    toks = torch.from_numpy(wl.token_batch(512, 2, 4096, 8, wl.PURPOSE_MASK_BATCH, 0)).cuda()
    got = []
    for shared in (True, False):
        m = make(B, fx, max_batch=2, max_seq=4096, loss_kind=B.LOSS_CLS2)
        m.enable_decode(kv8_page_tokens=32)
        prompt = toks[:1, :32].contiguous()
        if shared:
            m.decode_step(prompt, 0)
            m.decode_share(2, 32)
        else:
            m.decode_step(prompt.expand(2, 32).contiguous(), 0)
        got.append([m.decode_step(toks[:, 32:32 + n].contiguous(), 32).clone() for n in (2362, 300)])
        assert B.device_status() == 0
        m.close()
    for x, y in zip(*got):
        assert (x - y).abs().max() <= 4e-2 * y.abs().max()


@pytest.mark.parametrize("name", ["tiny", "tiny_gqa", "tiny_opt", "tiny_lut", "small_gqa"])
@pytest.mark.parametrize("kind", [0, 1])
def test_token_losses_match_the_oracle_and_the_stored_logits(B, name, kind):
    fx = DecoderFixture(name, seed=9, mask="random", B=3, S=48)
    m = make(B, fx, loss_kind=kind)
    toks_np = fx.batch(0)
    toks = torch.from_numpy(toks_np).cuda()
    r = m.token_losses(toks)
    loss = r.loss.view(3, 48)
    assert (loss[:, -1] == 0).all() and (loss[:, :-1] > 0).all() and r.lse.isfinite().all()
    if kind == 0:
        # the same hidden states through stored fp32 logits: sums of d products (2^-23 each in tensor cores) of logits below 30
        lp = m.token_logprobs(toks)
        err = 2 * (fx.shape["d_model"] / 16 + 30) * 2.0 ** -23 * 30
        assert torch.allclose(loss.reshape(-1), -lp.logp[:, 0], rtol=0, atol=err) and torch.allclose(r.lse, lp.lse, rtol=0, atol=err)
        # and their mean is the model's loss, to the bf16 path's own tolerance against the oracle
        om = fx.oracle_model()
        want = float(mo.loss_fn(om.cfg, om.params, om.lin_W(om.S), toks_np))
        assert abs(float(loss.sum()) / (3 * 47) - want) <= 2e-3 * abs(want)
    # targets of one's own, on another stream and captured
    t = torch.randint(0, fx.shape["vocab"], (3 * 48,), dtype=torch.int32, device="cuda")
    t[::5] = -1
    first = m.token_losses(toks, t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = m.token_losses(toks, t)
    side.synchronize()
    assert torch.equal(first.loss, again.loss) and torch.equal(first.lse, again.lse) and (first.loss[::5] == 0).all()
    # (the target's term is added last, so other targets mean another order of the sum: 600 additions of 2^-24 and a few roundings each)
    assert (first.lse - r.lse).abs().max() <= 2 * (600 * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -21 * 8)
    assert B.device_status() == 0
    m.close()


def test_token_losses_refusals(B):
    fx = DecoderFixture("tiny", seed=9, mask="random", B=2, S=16, n_layers=1)
    m = make(B, fx, "f32")
    toks = torch.zeros((2, 16), dtype=torch.int32, device="cuda")
    with pytest.raises(B.SzoError):
        m.token_losses(toks)
    m.close()
    m = make(B, fx)
    with pytest.raises(B.SzoError):
        m.token_losses(torch.zeros((2, 17), dtype=torch.int32, device="cuda"))
    with pytest.raises(B.SzoError):
        m.token_losses(torch.zeros((3, 16), dtype=torch.int32, device="cuda"))
    for bad in (toks.long(), toks[0]):
        with pytest.raises(ValueError):
            m.token_losses(bad)
    with pytest.raises(ValueError):
        m.token_losses(toks, torch.zeros(31, dtype=torch.int32, device="cuda"))
    m.close()


def test_scores_of_answers_to_one_prompt(B):
    """The three together: candidates continue a shared prompt, their tokens' losses come from the hidden states, and the gradient of
    their sum with respect to those states is that of the formula."""
    fx = DecoderFixture("tiny", seed=10, mask="random", B=4, S=64)
    m = make(B, fx)
    toks = torch.from_numpy(fx.batch(0)).cuda()
    toks[:, :20] = toks[:1, :20]
    t = torch.full_like(toks, -1)
    t[:, 19:-1] = toks[:, 20:]
    whole = m.token_losses(toks, t.view(-1)).loss.view(4, 64)
    m.enable_decode(kv8_page_tokens=16)
    m.decode_step(toks[:1, :20].contiguous(), 0)
    m.decode_share(4, 20)
    # the first answer token's loss from the decode step's logits of position 20 on: the cache's rounding apart the same numbers
    logits = m.decode_step(toks[:, 20:21].contiguous(), 20)
    lp = B.szo_token_logprobs(logits, toks[:, 21:22].contiguous())
    assert torch.allclose(-lp.logp[:, 0], whole[:, 20], rtol=0.1, atol=0.2)
    assert B.device_status() == 0
    m.close()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("page,n", [(16, 40), (16, 5), (32, 40), (16, 32)])
def test_sequences_get_back_what_they_held(B, act, page, n):
    """A part of a page that was taken over for the time of sharing is not lost: afterwards every sequence continues its own positions with
    the logits that it had, to the bit."""
    fx = DecoderFixture("tiny_gqa", seed=11, mask="random", B=4, S=64)
    toks = torch.from_numpy(fx.batch(0)).cuda()
    m = make(B, fx, act)
    m.enable_decode(kv8_page_tokens=page)
    m.decode_step(toks[:, :40].contiguous(), 0)
    step = toks[:, 40:41].contiguous()
    own = m.decode_step(step, 40).clone()
    for sharers in (4, 3):
        m.decode_share(sharers, n)
        if n == 40:
            shared = m.decode_step(step, 40)
            assert not torch.allclose(shared[1], own[1], atol=1e-3) and not torch.allclose(shared[2], own[2], atol=1e-3)
            if sharers == 3:                              # (the fourth has its own again)
                assert (shared[3] - own[3]).abs().max() <= (2e-3 if act == "f32" else 4e-2) * own.abs().max()
    m.decode_share(1, 0)
    assert torch.equal(m.decode_step(step, 40), own)
    assert B.device_status() == 0
    m.close()


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_captured_steps_follow_the_sharing_of_their_replay(B, act):
    """A step captured by its caller while four sequences share a prompt, replayed when two of them do, when none does and when the prompt is
    another one: every time the logits of the same step made then."""
    fx = DecoderFixture("tiny_gqa", seed=12, mask="random", B=4, S=64, n_layers=2)
    toks = torch.from_numpy(fx.batch(0)).cuda()
    m = make(B, fx, act, max_seq=131072, max_batch=4, loss_kind=B.LOSS_CLS2)      # (room: shared pages are read apart)
    m.enable_decode(kv8_page_tokens=16)
    m.decode_step(toks[:, :40].contiguous(), 0)
    step, out = toks[:, 40:41].contiguous(), torch.empty(4, fx.shape["vocab"], device="cuda")
    m.decode_share(4, 32)
    m.decode_step(step, 40)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.decode_step(step, 40, logits=out)
    seen = []
    for sharers, n in ((4, 32), (2, 32), (1, 32), (3, 16), (4, 0), (4, 35)):
        m.decode_share(sharers, n)
        graph.replay()
        torch.cuda.synchronize()
        want = m.decode_step(step, 40)
        assert (out - want).abs().max() <= (2e-3 if act == "f32" else 4e-2) * want.abs().max(), (sharers, n)
        seen.append(want)
    assert (seen[0] - seen[2]).abs().max() > 0.1 * seen[0].abs().max()            # (whose pages are read does matter)
    assert B.device_status() == 0
    m.close()


@pytest.mark.parametrize("dt,count,new", [("bf16", 12, 1), ("f16", 5, 3), ("bf16", 20, 9)])
def test_attention_losses_and_gradient_of_answers_to_one_prompt(B, dt, count, new):
    """The operators as they follow one another: answers attend to a prompt that they share, what comes out are the hidden states whose losses
    are taken, and the gradient of these goes back to them; by themselves, and captured into one graph that then serves other contents."""
    from tests import test_gpu_head_ce as head
    H, hkv, d, page, prefix, vocab = 8, 2, 64, 32, 4000, 1203
    g = torch.Generator("cuda").manual_seed(count)
    lens, whole = [prefix + new + (37 * b) % 150 for b in range(count)], prefix // page
    per = -(-(96 << 20) // (count * page * hkv * d * 2)) + 1      # (room: shared pages are read apart)
    order = torch.randperm(whole + count * 8, device="cuda", generator=g).int()
    table = torch.full((count, max(per, whole + 8)), -7, dtype=torch.int32, device="cuda")
    table[:, :whole] = order[:whole]
    table[:, whole:whole + 8] = order[whole:].view(count, 8)
    codes = torch.randint(0, 256, (2, whole + count * 8, hkv, page, d), dtype=torch.uint8, device="cuda", generator=g)
    codes[(codes & 127) == 127] = 3
    scales = torch.exp2(torch.randint(-9, -6, (whole + count * 8, hkv, 2), device="cuda", generator=g).float())
    cache, rows = B.Kv8Cache(codes, scales), count * new
    batch = B.Kv8Batch(table, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows)
    shared = B.Kv8Prefix(torch.tensor([prefix], dtype=torch.int32, device="cuda"))
    q = torch.randn(rows, H, d, device="cuda", generator=g).to(head.DT[dt])
    W = (torch.randn(vocab, H * d, device="cuda", generator=g) / 8).to(head.DT[dt])
    t = torch.randint(-1, vocab, (rows,), dtype=torch.int32, device="cuda", generator=g)
    a = torch.randn(rows, device="cuda", generator=g)

    def both():
        o = B.szo_attention_kv8_prefix(cache, batch, shared, q)
        r = B.szo_head_ce(o.view(rows, H * d), W, t)
        return (o, r.loss, r.lse) + B.szo_head_ce_bwd(o.view(rows, H * d), W, t, r.lse, a)
    o, loss, lse, dh, dW = first = both()
    # (the bound of test_agrees_with_attention_that_shares_nothing: values up to 3.5, two results of the same kind)
    logit = ((d + 8) * 2.0 ** -23 + 2.0 ** -20) * 6 * 3.5 * d ** 0.5
    each = 3.5 * (2.0 ** -11 + 2 * logit + (max(lens) + 16) * 2.0 ** -23 + torch.finfo(o.dtype).eps / 2)
    assert (B.szo_attention_kv8(cache, batch, q).double() - o.double()).abs().max() <= 2 * each
    h = o.view(rows, H * d)
    head.check_forward(B.HeadCe(loss, lse), h, W, t, 1.0)
    wh, eh, wW, eW = head.backward_bounds(h, W, t, lse, a, None, 1.0, dt)
    head.within(dh, wh, eh)
    head.within(dW, wW, eW)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, captured))
    q.neg_()
    shared.length.fill_(prefix // 2)
    t.copy_(t.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(captured, both()))
    assert B.device_status() == 0
