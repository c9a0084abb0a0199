"""Cross entropy from hidden states, and attention over shared prompts: what the host refuses, and the formulas against differences."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from tests import head_ce_reference as ref

OK, ARG, SHAPE, ALIGN, UNSUP, WS = 0, -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _forward(L, **kw):
    a = dict(h=16, hs=64, W=16, ws_=64, dtype=1, rows=4, vocab=100, d=64, scale=1.0, targets=16, loss=16, lse=16, ws=None, n=0)
    a.update(kw)
    return L.szo_head_ce(a["h"], a["hs"], a["W"], a["ws_"], a["dtype"], a["rows"], a["vocab"], a["d"], a["scale"], a["targets"], a["loss"], a["lse"],
                         a["ws"], a["n"], None)


def _backward(L, **kw):
    a = dict(h=16, hs=64, W=16, ws_=64, dtype=1, rows=4, vocab=100, d=64, scale=1.0, targets=16, lse=16, d_loss=16, d_lse=None, dh=16, dhs=64, dW=16,
             dws=64, ws=None, n=0)
    a.update(kw)
    return L.szo_head_ce_bwd(a["h"], a["hs"], a["W"], a["ws_"], a["dtype"], a["rows"], a["vocab"], a["d"], a["scale"], a["targets"], a["lse"],
                             a["d_loss"], a["d_lse"], a["dh"], a["dhs"], a["dW"], a["dws"], a["ws"], a["n"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=0), UNSUP), (dict(dtype=3), UNSUP), (dict(rows=-1), SHAPE), (dict(vocab=0), SHAPE), (dict(d=0), SHAPE), (dict(d=60, hs=64), SHAPE),
    (dict(rows=1 << 31), SHAPE), (dict(vocab=1 << 31), SHAPE), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=math.nan), ARG),
    (dict(scale=1e31), ARG), (dict(h=None), ARG), (dict(W=None), ARG), (dict(targets=None), ARG), (dict(hs=56), SHAPE), (dict(ws_=56), SHAPE),
    (dict(h=24), ALIGN), (dict(W=8), ALIGN), (dict(hs=68), ALIGN), (dict(ws_=68), ALIGN), (dict(targets=20), ALIGN), ({}, WS), (dict(ws=16, n=1), WS)])
def test_arguments_are_checked_before_any_launch(B, kw, code):
    L = B.lib()
    assert _forward(L, **kw) == code and L.szo_last_error()
    assert _backward(L, **kw) == code and L.szo_last_error()


def test_results_are_checked(B):
    L = B.lib()
    assert _forward(L, loss=None) == ARG and _forward(L, loss=20) == ALIGN and _forward(L, lse=20) == ALIGN and _forward(L, ws=8, n=1 << 30) == ALIGN
    assert _backward(L, lse=None) == ARG and _backward(L, d_loss=None) == ARG and _backward(L, d_lse=20) == ALIGN
    assert _backward(L, dhs=56) == SHAPE and _backward(L, dws=56) == SHAPE and _backward(L, dhs=68) == ALIGN and _backward(L, dws=68) == ALIGN
    assert _backward(L, dh=8) == ALIGN and _backward(L, dW=8) == ALIGN
    # what is not wanted is not looked at; nothing to do is no error
    assert _backward(L, dh=None, dhs=0, dW=None, dws=0) == OK
    assert _forward(L, rows=0, h=None, targets=None, loss=None, lse=None) == OK
    assert _backward(L, rows=0, h=None, targets=None, lse=None, d_loss=None, dW=None) == OK


def test_workspaces(B):
    L = B.lib()
    f, b = L.szo_head_ce_workspace_bytes, L.szo_head_ce_bwd_workspace_bytes
    assert f(0, 100, 64) == 0 and f(4, 0, 64) == 0 and f(4, 100, 60) == 0 and b(4, 100, 64, 0, 0) == 0 and b(0, 100, 64, 1, 1) == 0
    assert 0 < b(100, 5000, 64, 1, 0) <= b(100, 5000, 64, 1, 1)
    # far below the logits
    assert f(4096, 50272, 5120) < 4096 * 50272 * 4 / 16
    assert b(4096, 50272, 5120, 1, 1) < 4096 * 50272 * 4 / 2


def _prefix(B, **kw):
    d = dict(len=16, seqs=16, n_groups=1, max_seqs=2)
    d.update(kw)
    return B.Kv8PrefixStruct(*(d[n] for n, _ in B.Kv8PrefixStruct._fields_))


@pytest.mark.parametrize("prefix,code", [
    (dict(n_groups=-1), SHAPE), (dict(max_seqs=-1), SHAPE), (dict(len=None), ARG), (dict(seqs=None, n_groups=2), SHAPE), (dict(len=20), ALIGN),
    (dict(seqs=24), ALIGN)])
def test_groups_are_checked(B, prefix, code):
    c = B.Kv8CacheStruct(16, 16, 16, 4, 16, 2, 64)
    b = B.Kv8BatchStruct(16, 16, None, 2, 2, 2, 1)
    p = _prefix(B, **prefix)
    L = B.lib()
    a = [C.addressof(x) for x in (c, b, p)]
    assert L.szo_attention_kv8_prefix(*a, 16, 256, 16, 256, 1, 4, 0.125, None, 0, None) == code and L.szo_last_error()
    assert L.szo_attention_kv8_prefix_workspace_bytes(*a, 4) == 0


def test_attention_over_shared_prompts_checks_its_rows(B):
    c, b, e, p = B.Kv8CacheStruct(16, 16, 16, 4, 16, 2, 64), B.Kv8BatchStruct(16, 16, None, 2, 2, 2, 1), B.Kv8BatchStruct(16, 16, None, 0, 0, 2, 1), _prefix(B)
    f = B.lib().szo_attention_kv8_prefix
    c_, b_, e_, p_ = (C.addressof(x) for x in (c, b, e, p))
    assert f(None, b_, p_, 16, 256, 16, 256, 1, 4, 0.1, None, 0, None) == ARG and f(c_, b_, None, 16, 256, 16, 256, 1, 4, 0.1, None, 0, None) == ARG
    assert f(c_, b_, p_, None, 256, 16, 256, 1, 4, 0.1, None, 0, None) == ARG and f(c_, b_, p_, 16, 256, 16, 256, 3, 4, 0.1, None, 0, None) == UNSUP
    assert f(c_, b_, p_, 16, 256, 16, 256, 1, 3, 0.1, None, 0, None) == SHAPE and f(c_, b_, p_, 16, 248, 16, 256, 1, 4, 0.1, None, 0, None) == SHAPE
    assert f(c_, b_, p_, 16, 260, 16, 256, 1, 4, 0.1, None, 0, None) == ALIGN and f(c_, b_, p_, 16, 256, 16, 256, 1, 4, math.inf, None, 0, None) == ARG
    assert f(c_, e_, p_, 16, 256, 16, 256, 1, 4, 0.1, None, 0, None) == OK


def test_the_gradient_s_formula_against_differences():
    g = np.random.default_rng(5)
    rows, vocab, d, scale = 5, 11, 6, 1.3
    h, W = torch.from_numpy(g.normal(0, 1, (rows, d))), torch.from_numpy(g.normal(0, 1, (vocab, d)))
    t = torch.tensor([3, -1, 10, 0, 3])
    a, b = torch.from_numpy(g.normal(0, 1, rows)), torch.from_numpy(g.normal(0, 1, rows))

    def total(h_, W_):
        loss, lse = ref.forward(h_, W_, t, scale)
        return float((a * loss).sum() + (b * lse).sum())
    _, lse = ref.forward(h, W, t, scale)
    dh, dW, _ = ref.backward(h, W, t, lse, a, b, scale)
    for x, want in ((h, dh), (W, dW)):
        for i in range(x.shape[0]):
            for j in range(x.shape[1]):
                step = torch.zeros_like(x)
                step[i, j] = 1e-5
                pair = [(x + s * step if x is h else h, x + s * step if x is W else W) for s in (1, -1)]
                diff = (total(*pair[0]) - total(*pair[1])) / 2e-5
                assert abs(diff - float(want[i, j])) < 1e-8 * 50        # third derivatives of order 1 times 1e-10, and 1e-16 / 1e-5


@pytest.mark.parametrize("rows", [129, 4096, 5000, 8192, 8193, 16384, 65536, 300001])
@pytest.mark.parametrize("vocab", [8192, 50272, 200000])
def test_a_gradient_holds_three_pieces_of_g(B, rows, vocab):
    """However many rows: pieces of 64 MB (rounded up to 256 entries), or of 4096 entries where that is more; for dh alone of a large
    vocabulary 8192 rows at a time."""
    d, L = 4096, B.lib()
    others = 16 * rows + 8 * vocab + 4096                          # the rows' weights, counters

    def bound(n):
        # three pieces, and dh in fp32 (in up to 16 shares where there are few tiles)
        return 3 * (max(64 << 20, 2 * 4096 * n) + 2 * 256 * n) + 4 * n * d * (16 if n < 1024 else 1)
    assert L.szo_head_ce_bwd_workspace_bytes(rows, vocab, d, 1, 0) <= bound(rows if vocab == 8192 else min(rows, 8192)) + others
    assert L.szo_head_ce_bwd_workspace_bytes(rows, vocab, d, 1, 1) <= bound(rows) + 2 * rows * d + others
