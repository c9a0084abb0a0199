"""8-bit key/value cache and token log probabilities: what the host refuses, and the reference the GPU tests use."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import kv8_reference as ref


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _cache(B, **kw):
    d = dict(k_codes=16, v_codes=16, scales=16, n_pages=4, page_tokens=16, n_kv_heads=2, head_dim=64)
    d.update(kw)
    return B.Kv8CacheStruct(*(d[n] for n, _ in B.Kv8CacheStruct._fields_))


def _batch(B, **kw):
    d = dict(page_table=16, kv_len=16, start=None, rows=2, batch=2, max_pages=2, max_new=1)
    d.update(kw)
    return B.Kv8BatchStruct(*(d[n] for n, _ in B.Kv8BatchStruct._fields_))


OK, ARG, SHAPE, ALIGN, UNSUP = 0, -1, -2, -3, -4


@pytest.mark.parametrize("cache,batch,code", [
    (dict(k_codes=None), {}, ARG), (dict(scales=None), {}, ARG), ({}, dict(page_table=None), ARG), ({}, dict(kv_len=None), ARG),
    (dict(page_tokens=24), {}, UNSUP), (dict(page_tokens=256), {}, UNSUP), (dict(page_tokens=0), {}, UNSUP), (dict(head_dim=96), {}, UNSUP),
    (dict(n_kv_heads=0), {}, SHAPE), (dict(n_pages=0), {}, SHAPE), (dict(n_pages=1 << 31), {}, SHAPE),
    ({}, dict(batch=-1), SHAPE), ({}, dict(rows=-1), SHAPE), ({}, dict(max_pages=0), SHAPE), ({}, dict(max_new=-1), SHAPE),
    ({}, dict(max_pages=1 << 27), SHAPE), ({}, dict(rows=1), SHAPE), (dict(v_codes=8), {}, ALIGN), ({}, dict(kv_len=20), ALIGN),
    ({}, dict(start=4), ALIGN)])
def test_cache_and_batch_are_checked_before_any_launch(B, cache, batch, code):
    c_, b_ = _cache(B, **cache), _batch(B, **batch)
    c, b = C.addressof(c_), C.addressof(b_)
    L = B.lib()
    assert L.szo_kv8_write(c, b, 16, 16, 1, 128, 128, None) == code
    assert L.szo_kv8_read(c, b, 16, 16, 1, 128, 128, None) == code
    assert L.szo_attention_kv8(c, b, 16, 256, 16, 256, 1, 4, 0.125, None, 0, None) == code
    assert L.szo_last_error()


def test_row_buffers_are_checked(B):
    c_, b_, e_ = _cache(B), _batch(B), _batch(B, batch=0, rows=0)
    c, b, e = C.addressof(c_), C.addressof(b_), C.addressof(e_)
    L = B.lib()
    for f in (L.szo_kv8_write, L.szo_kv8_read):
        assert f(None, b, 16, 16, 1, 128, 128, None) == ARG and f(c, None, 16, 16, 1, 128, 128, None) == ARG
        assert f(c, b, None, 16, 1, 128, 128, None) == ARG
        assert f(c, b, 16, 16, 3, 128, 128, None) == UNSUP
        assert f(c, b, 16, 16, 1, 120, 128, None) == SHAPE
        assert f(c, b, 16, 24, 1, 128, 128, None) == ALIGN and f(c, b, 16, 16, 1, 128, 132, None) == ALIGN
        assert f(c, b, 16, 16, 0, 128, 130, None) == ALIGN
        assert f(c, e, 16, 16, 1, 128, 128, None) == OK                       # nothing to do, nothing launched
    a = L.szo_attention_kv8
    assert a(c, b, None, 256, 16, 256, 1, 4, 0.125, None, 0, None) == ARG
    assert a(c, b, 16, 256, 16, 256, 7, 4, 0.125, None, 0, None) == UNSUP
    assert a(c, b, 16, 256, 16, 256, 1, 3, 0.125, None, 0, None) == SHAPE              # 3 query heads on 2 key/value heads
    assert a(c, b, 16, 248, 16, 256, 1, 4, 0.125, None, 0, None) == SHAPE
    assert a(c, b, 16, 260, 16, 256, 1, 4, 0.125, None, 0, None) == ALIGN
    assert a(c, b, 16, 256, 16, 256, 1, 4, float("nan"), None, 0, None) == ARG and a(c, b, 16, 256, 16, 256, 1, 4, float("inf"), None, 0, None) == ARG
    assert a(c, e, 16, 256, 16, 256, 1, 4, 0.125, None, 0, None) == OK


def test_attention_workspace(B):
    """One sequence with a long page table needs one; whether it does is a matter of shapes alone."""
    L = B.lib()
    c_, b_ = _cache(B, n_pages=10000), _batch(B, max_pages=8192, batch=1, rows=1)
    c, b = C.addressof(c_), C.addressof(b_)
    need = L.szo_attention_kv8_workspace_bytes(c, b, 4)
    assert 0 < need < 20 << 20
    a = L.szo_attention_kv8
    assert a(c, b, 16, 256, 16, 256, 1, 4, 0.125, None, need, None) == -5
    assert a(c, b, 16, 256, 16, 256, 1, 4, 0.125, 16, need - 1, None) == -5
    assert a(c, b, 16, 256, 16, 256, 1, 4, 0.125, 24, need, None) == ALIGN
    s_, e_ = _batch(B), _batch(B, batch=0, rows=0)
    assert L.szo_attention_kv8_workspace_bytes(c, C.addressof(s_), 4) == 0 and L.szo_attention_kv8_workspace_bytes(c, C.addressof(e_), 4) == 0
    assert L.szo_attention_kv8_workspace_bytes(None, b, 4) == 0 and L.szo_attention_kv8_workspace_bytes(c, b, 3) == 0
    big_ = _cache(B, n_pages=1 << 28)
    assert a(C.addressof(big_), C.addressof(s_), 16, 256, 16, 256, 1, 4, 0.125, None, 0, None) == SHAPE      # 2^33 tokens


def test_logprob_arguments_are_checked(B):
    L = B.lib()

    def fwd(logits=16, dt=1, rows=2, vocab=100, ld=100, scale=1.0, targets=16, nt=1, top=0, logp=16, ids=16, tl=16):
        return L.szo_token_logprobs(logits, dt, rows, vocab, ld, scale, targets, nt, top, logp, 16, 16, ids, tl, None)

    def bwd(logits=16, dt=1, rows=2, vocab=100, ld=100, scale=1.0, targets=16, nt=1, lse=16, ent=16, dl=16, de=16, out=32, old=100):
        return L.szo_token_logprobs_bwd(logits, dt, rows, vocab, ld, scale, targets, nt, lse, ent, dl, de, out, old, None)

    for f in (fwd, bwd):
        assert f(dt=5) == UNSUP and f(rows=-1) == SHAPE and f(vocab=0) == SHAPE and f(ld=99) == SHAPE
        assert f(scale=0.0) == ARG and f(scale=-1.0) == ARG and f(scale=float("nan")) == ARG and f(scale=float("inf")) == ARG
        assert f(nt=65) == UNSUP and f(nt=-1) == UNSUP and f(logits=None) == ARG and f(targets=None) == ARG
        assert f(logits=18) == ALIGN and f(targets=20) == ALIGN
        assert f(rows=0) == OK
    assert fwd(top=33) == UNSUP and fwd(top=-1) == UNSUP and fwd(vocab=20, ld=20, top=21) == UNSUP
    assert fwd(logp=None) == ARG and fwd(top=1, ids=None) == ARG and fwd(top=1, tl=None) == ARG and fwd(logp=8) == ALIGN
    assert bwd(lse=None) == ARG and bwd(out=None) == ARG and bwd(dl=None) == ARG and bwd(ent=None) == ARG
    assert bwd(old=90) == SHAPE and bwd(out=16, old=128) == ARG and bwd(out=40) == ALIGN


def test_binding_refuses_cpu_tensors(B):
    with pytest.raises(ValueError):
        B.Kv8Cache(torch.zeros((2, 1, 1, 16, 64), dtype=torch.uint8), torch.zeros((1, 1, 2)))
    with pytest.raises(ValueError):
        B.szo_token_logprobs(torch.zeros(2, 8))


def test_reference_codes_agree_with_the_format():
    every = torch.arange(256, dtype=torch.uint8)
    t = every.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(ref.TABLE, nan=-1), np.nan_to_num(t, nan=-1))
    g = np.random.default_rng(3)
    y = np.concatenate([g.normal(0, 1, 4000) * 2.0 ** g.integers(-12, 8, 4000), ref.TABLE[:127], (ref.TABLE[:126] + ref.TABLE[1:127]) / 2])
    y = np.clip(y, -448, 448)
    got = ref.encode(y)
    assert np.array_equal(got, torch.from_numpy(y).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert [ref.needed_exponent(a) for a in (0.0, 448.0, 448.0001, 1.0, 1.75, 1.76, 3.5)] == [-63, 0, 1, -8, -8, -7, -7]


def test_reference_gradient_against_differences():
    g = np.random.default_rng(5)
    x = g.normal(0, 2, (4, 11))
    x[1, 3] = -np.inf
    x[2, 1:] = -np.inf
    t = np.array([[2, 2, -1], [0, 10, 4], [0, 0, 0], [1, 2, 3]])
    dl, de = g.normal(0, 1, t.shape), g.normal(0, 1, 4)

    def f(z):
        lp, _, ent = ref.logprobs(z, 0.8)
        return sum(dl[r, i] * lp[r, t[r, i]] for r in range(4) for i in range(3) if t[r, i] >= 0) + (de * ent).sum()
    got = ref.logprobs_grad(x, 0.8, t, dl, de)
    for r in range(4):
        for j in range(11):
            if np.isneginf(x[r, j]):
                continue
            a, b = x.copy(), x.copy()
            a[r, j] += 1e-5
            b[r, j] -= 1e-5
            # central difference: error h^2/6 |f'''| (below 1e-9 here) + 1e-16 |f| / h (below 1e-9)
            assert abs((f(a) - f(b)) / 2e-5 - got[r, j]) < 1e-8
