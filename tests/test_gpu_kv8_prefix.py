"""Attention over shared prompts in the 8-bit paged cache on the GPU, against the definition in 64 bits and against
szo_attention_kv8 on the same cache."""
import math

import numpy as np
import pytest
import torch

from tests import kv8_reference as ref
from tests.test_gpu_kv8 import DT, ERR_ARG, ERR_SHAPE, World, _rows, attention_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding
    binding.lib()
    return binding


class SharedWorld(World):
    """Groups of sequences whose first whole pages are the same: sizes[g] sequences with prefixes[g] shared positions, alone[g] = False;
    every sequence has caps positions of its own cache beyond."""

    def __init__(self, B, sizes, prefixes, caps, hkv, page, d, seed):
        super().__init__(B, caps, hkv, page, d, seed)
        self.sizes, self.prefixes = sizes, prefixes
        at = 0
        for n, p in zip(sizes, prefixes):
            whole = p // page
            for b in range(at + 1, at + n):
                self.pages[b] = np.concatenate([self.pages[at][:whole], self.pages[b][whole:]])
                self.table[b, :len(self.pages[b])] = self.pages[b]
            at += n
        self.d_table.copy_(torch.from_numpy(self.table))
        # the same table with room for so many pages that reading them for every sequence would be a lot: shared pages are then
        # taken apart; with the narrow one a small batch goes to the attention that shares nothing
        self.narrow = self.d_table
        room = -(-(100 << 20) // (len(caps) * page * hkv * d * 2)) + 1
        self.wide = torch.full((len(caps), room), -7, dtype=torch.int32, device="cuda")
        self.wide[:, :self.narrow.shape[1]] = self.narrow
        self.d_table = self.wide

    def fill(self, lens, dt="bf16", loud=1.0, nan=()):
        """Everything that the sequences' first lens positions need; nan: (sequence, position, head, dim, which)."""
        for b, n in enumerate(lens):
            x = [_rows(self.g, n, self.hkv, self.d, dt, loud) for _ in (0, 1)]
            first = sum(self.sizes[:sum(np.cumsum(self.sizes) <= b)])
            whole = self.prefixes[sum(np.cumsum(self.sizes) <= b)] // self.ref.page * self.ref.page if b < sum(self.sizes) and b != first else 0
            whole = min(whole, n)
            for s, p, h, i, which in nan:
                if s == b:
                    x[which][p, h, i] = float("nan")
            batch = self.B.Kv8Batch(self.d_table[b:b + 1].clone(), torch.tensor([n], dtype=torch.int32, device="cuda"), n - whole,
                                    torch.tensor([0, n - whole], dtype=torch.int32, device="cuda"), max(n - whole, 1))
            if n > whole:
                self.B.szo_kv8_write(self.cache, batch, x[0][whole:].cuda(), x[1][whole:].cuda())
                for which in (0, 1):
                    self.ref.write(self.pages[b], whole, x[which][whole:].double().numpy(), which)

    def prefix(self):
        ends = np.concatenate([[0], np.cumsum(self.sizes)]).astype(np.int32)
        return self.B.Kv8Prefix(torch.tensor(self.prefixes, dtype=torch.int32, device="cuda"), torch.from_numpy(ends).cuda(), max(self.sizes))


def check(B, w, lens, news, H, dt, scale=None, spread=1.0, gap=1, prefix=None, q=None, skipped=()):
    w.d_table = w.narrow
    batch, start, rows = w.batch(lens, news, gap)
    if q is None:
        q = torch.from_numpy(w.g.normal(0, spread, (rows, H, w.d))).to(DT[dt])
    got = []
    for table in (w.narrow, w.wide):
        w.d_table = table
        batch, start, rows = w.batch(lens, news, gap)
        out = torch.full_like(q, 3.0).cuda()
        B.szo_attention_kv8_prefix(w.cache, batch, prefix or w.prefix(), q.cuda(), scale=scale, out=out)
        got.append(out.double().cpu().numpy())
    for one in got:
        compare(w, one, q, start, rows, lens, news, H, dt, scale, gap, skipped)


def compare(w, got, q, start, rows, lens, news, H, dt, scale, gap, skipped):
    assert (got[:gap] == 3).all() and (got[rows - gap:] == 3).all()
    sc = scale if scale is not None else 1 / math.sqrt(w.d)
    for b, (n, m) in enumerate(zip(lens, news)):
        if b in skipped:
            assert (got[start[b]:start[b + 1]] == 3).all()
        if m == 0 or b in skipped:
            continue
        k, v = (w.ref.values(w.pages[b], n, which) for which in (0, 1))
        size = 2.0 ** w.ref.e[w.pages[b][np.arange(n) // w.ref.page], :, 1]
        o, wide, big, top = ref.attention(q[start[b]:start[b + 1]].double().numpy(), k, v, n - m, sc, size)
        mine = got[start[b]:start[b + 1]]
        assert np.array_equal(np.isnan(mine), np.isnan(o)), (b, n, m, np.argwhere(np.isnan(mine) != np.isnan(o))[:4])
        bad = np.abs(np.nan_to_num(mine - o)) > np.nan_to_num(attention_bound(o, wide, big, n, w.d, dt, top[..., None]), nan=1.0)
        assert not bad.any(), (b, n, m, np.argwhere(bad)[:4], np.abs(mine - o).max())


SHAPES = [(64, 1, 1, 16), (128, 2, 1, 16), (128, 1, 4, 64), (64, 2, 5, 32), (128, 1, 8, 128), (64, 1, 9, 16), (128, 2, 3, 32)]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,hkv,group,page", SHAPES)
def test_single_tokens(B, dt, d, hkv, group, page):
    """Shared parts of whole pages and of a little more, of less than one page, groups of one and of many."""
    sizes, prefixes = [5, 1, 3, 12], [128 * 3, 128, 131, 7]
    lens = [385, 400, 512, 386, 449, 130, 132, 140, 257] + [8 + 5 * i for i in range(12)]
    w = SharedWorld(B, sizes, prefixes, lens, hkv, page, d, seed=group + page)
    w.fill(lens)
    check(B, w, lens, [1] * len(lens), hkv * group, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,hkv,group,page", SHAPES)
def test_a_few_tokens(B, dt, d, hkv, group, page):
    sizes, prefixes = [4, 2], [256, 128]
    lens = [261, 300, 256 + 3, 290, 200, 131]
    w = SharedWorld(B, sizes, prefixes, lens, hkv, page, d, seed=group * page)
    w.fill(lens)
    check(B, w, lens, [5, 3, 0, 2, 11, 3], hkv * group, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,hkv,group,page", [(128, 1, 4, 64), (64, 2, 1, 16), (128, 1, 3, 32), (64, 1, 8, 128)])
def test_answers_scored_whole(B, dt, d, hkv, group, page):
    sizes, prefixes = [3, 4], [384, 128]
    lens = [384 + 130, 384 + 70, 384 + 1, 128 + 200, 128 + 64, 128 + 33, 128 + 150]
    w = SharedWorld(B, sizes, prefixes, lens, hkv, page, d, seed=3 * group + page)
    w.fill(lens)
    check(B, w, lens, [130, 70, 1, 200, 64, 33, 20], hkv * group, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 60])
def test_rows_inside_the_shared_part(B, dt, new):
    """Sequences that end inside what their group shares, padding rows, sequences of no positions."""
    sizes, prefixes = [6], [192]
    lens = [260, 192, 100, 33, 1, 0]
    w = SharedWorld(B, sizes, prefixes, [260] * 6, 2, 32, 64, seed=21)
    w.fill([260] * 6)
    check(B, w, lens, [new, new, new, min(new, 40), new, new], 4, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 30])
def test_groups_whose_first_sequences_are_short(B, dt, new):
    """Entries of a table that no position of its sequence needs may hold anything: the first sequences end inside the shared part, in one
    group all do."""
    sizes, prefixes = [4, 3], [192, 192]
    lens = [40, 100, 300, 200, 60, 90, 33]
    w = SharedWorld(B, sizes, prefixes, [300] * 7, 2, 32, 64, seed=31)
    w.fill([300] * 7)
    for b, n in enumerate(lens):
        w.wide[b, -(-n // 32):] = 1 << 28
        w.narrow[b, -(-n // 32):] = -5
    check(B, w, lens, [min(new, n) for n in lens], 4, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt,group,count", [("bf16", 4, 300), ("f16", 1, 700), ("f32", 2, 300)])
def test_many_sequences(B, dt, group, count):
    """Groups of more rows than one tile has, and more sequences than a block has threads."""
    sizes, prefixes = [count - 7, 7], [96, 64]
    lens = [97 + (5 * i) % 40 for i in range(count)]
    w = SharedWorld(B, sizes, prefixes, lens, 1, 16, 64, seed=32)
    w.fill(lens)
    check(B, w, lens, [1 + (i % 3 == 0) for i in range(count)], group, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("new,most,hkv", [(1, 4, 4), (2, 4, 4), (2, 8, 4), (4, 2, 4), (1, 3, 1), (6, 3, 2), (18, 2, 4)])
def test_many_prompts_of_few_sequences(B, dt, new, most, hkv):
    """Prompts that fill the SMs by themselves: rows of a group that are cheaper together, and such that are not."""
    sizes = [1 + (most - 1) * (g % 3 != 2) for g in range(40)]
    lens = [49 + new + (7 * i) % 30 for i in range(sum(sizes))]
    w = SharedWorld(B, sizes, [32 + 16 * (g % 2) for g in range(40)], lens, hkv, 16, 64, seed=33)
    w.fill(lens)
    check(B, w, lens, [new - (i % 4 == 3) for i in range(len(lens))], 4 * hkv, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("new,count", [(1, 3), (1, 40), (7, 20), (40, 9)])
def test_sequences_of_no_group_and_batches_without_one(B, dt, new, count):
    lens = [150 + 7 * i for i in range(count)]
    w = SharedWorld(B, [count], [128], lens, 1, 16, 128, seed=22)
    w.fill(lens)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    news = [new] * count
    whole = B.Kv8Prefix(ints(128))                                          # all sequences are one group
    check(B, w, lens, news, 4, dt, prefix=whole)
    some = B.Kv8Prefix(ints(128, 64), ints(1, 2, count - 1 if count > 3 else 2), max_seqs=count)
    check(B, w, lens, news, 4, dt, prefix=some)
    nothing = B.Kv8Prefix(ints(0))
    check(B, w, lens, news, 4, dt, prefix=nothing)
    none = B.Kv8Prefix(ints(), ints(0), max_seqs=0)
    check(B, w, lens, news, 4, dt, prefix=none)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("spread,scale", [(60.0, None), (1.0, 0.0), (1.0, -0.2), (1e4, 1e-5)])
@pytest.mark.parametrize("new", [1, 50])
def test_sharp_flat_and_odd_scales(B, dt, spread, scale, new):
    lens = [300, 280, 310, 257 + new]
    w = SharedWorld(B, [4], [256], lens, 1, 32, 64, seed=23)
    w.fill(lens)
    check(B, w, lens, [new] * 4, 2, dt, scale=scale, spread=spread)


@pytest.mark.parametrize("new", [1, 4, 70])
def test_nan_reaches_only_rows_that_attend_to_it(B, new):
    lens = [200 + new, 230 + new, 100, 260 + new]
    w = SharedWorld(B, [4], [192], [200 + new, 230 + new, 300, 260 + new], 1, 16, 64, seed=24)
    # a value of the shared part (the third sequence ends before it), a key of it, a value of a sequence's own last position
    w.fill([200 + new, 230 + new, 300, 260 + new], nan=[(0, 150, 0, 5, 1), (1, 229 + new, 0, 9, 1)])
    for dt in ("bf16", "f32"):
        check(B, w, lens, [new, new, min(new, 100), new], 2, dt)
    batch, start, rows = w.batch(lens, [new] * 4)
    q = torch.randn(rows, 2, 64, dtype=torch.bfloat16)
    q[1, 0, 3] = float("nan")
    q[start[2], 1, 0] = float("inf")
    o = B.szo_attention_kv8_prefix(w.cache, batch, w.prefix(), q.cuda())
    assert o[1, 0].isnan().all() if start[1] == 1 or new > 1 else True
    bad = torch.zeros(rows, 2, dtype=torch.bool)
    bad[1, 0] = bad[start[2], 1] = True
    live = np.concatenate([np.arange(start[b], start[b + 1]) for b in range(4)])
    dims = [i for i in range(64) if i not in (5, 9)]
    assert torch.equal(o.cpu()[live][:, :, dims].isnan().any(-1), bad[live])


def test_key_nan_of_the_shared_part(B):
    lens = [200, 210, 90]
    w = SharedWorld(B, [3], [128], [200, 210, 140], 1, 16, 64, seed=25)
    w.fill([200, 210, 140], nan=[(0, 100, 0, 5, 0)])
    for new in (1, 60):
        check(B, w, lens, [new] * 3, 2, "bf16")


def test_descriptions_that_do_not_fit_share_nothing(B):
    count = 6
    lens = [150 + 9 * i for i in range(count)]
    w = SharedWorld(B, [count], [128], lens, 1, 16, 64, seed=26)
    w.fill(lens)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cap = w.wide.shape[1] * 16
    for prefix in (B.Kv8Prefix(ints(-1)), B.Kv8Prefix(ints(cap + 1)), B.Kv8Prefix(ints(128), ints(0, count + 1), max_seqs=count + 1),
                   B.Kv8Prefix(ints(128), ints(4, 2), max_seqs=count), B.Kv8Prefix(ints(128), ints(-1, 4), max_seqs=count),
                   B.Kv8Prefix(ints(128), ints(0, count), max_seqs=count - 1)):
        for new in (1, 40):
            check(B, w, lens, [new] * count, 2, "bf16", prefix=prefix)
            assert B.device_status() == ERR_SHAPE
    # a sequence whose own description does not fit is skipped, the others of its group are not
    for new in (1, 40):
        bad = list(lens)
        bad[2] = cap + 1
        check(B, w, bad, [new] * count, 2, "bf16", skipped=(2,))
        assert B.device_status() == ERR_SHAPE
    # page ids of no page, in the shared part and behind it
    for at in (1, 9):
        t = w.d_table.clone()
        t[slice(None) if at == 1 else 3, at] = w.cache.n_pages     # (a shared page stands in every table)
        for new in (1, 40):
            rows = count * new
            batch = B.Kv8Batch(t, ints(*lens), rows)
            o = B.szo_attention_kv8_prefix(w.cache, batch, w.prefix(), torch.randn(rows, 2, 64, dtype=torch.bfloat16, device="cuda"))
            assert B.device_status() == ERR_ARG and o.isfinite().all()


@pytest.mark.parametrize("new,count,prefix", [(1, 64, 2048), (1, 6, 20000), (3, 33, 900), (64, 12, 1500)])
@pytest.mark.parametrize("dt,H,hkv,d,page", [("bf16", 32, 8, 128, 64), ("f16", 10, 2, 64, 16), ("f32", 8, 4, 128, 32)])
def test_agrees_with_attention_that_shares_nothing(B, dt, H, hkv, d, page, new, count, prefix):
    """Larger batches against szo_attention_kv8 on the same cache: both are within their bounds of the truth, so within
    twice the larger of them of each other; the same bits again, on another stream, from a graph."""
    g = torch.Generator("cuda").manual_seed(new + count)
    own = [new + (37 * b) % 150 for b in range(count)]
    lens = [prefix + n for n in own]
    whole = prefix // page
    per = -(-max(lens) // page) + 1
    n_pages = whole + count * (per - whole)
    order = torch.randperm(n_pages, device="cuda", generator=g).int()
    table = torch.cat([order[:whole].expand(count, whole), order[whole:].view(count, per - whole)], 1).contiguous()
    codes = torch.randint(0, 256, (2, n_pages, hkv, page, d), dtype=torch.uint8, device="cuda", generator=g)
    codes[(codes & 127) == 127] = 3
    scales = torch.exp2(torch.randint(-9, -6, (n_pages, hkv, 2), device="cuda", generator=g).float())
    cache = B.Kv8Cache(codes, scales)
    room = -(-(100 << 20) // (count * page * hkv * d * 2)) + 1             # (see SharedWorld)
    if room > per:
        table = torch.cat([table, torch.full((count, room - per), -7, dtype=torch.int32, device="cuda")], 1)
    batch = B.Kv8Batch(table, torch.tensor(lens, dtype=torch.int32, device="cuda"), count * new)
    shared = B.Kv8Prefix(torch.tensor([prefix], dtype=torch.int32, device="cuda"))
    q = torch.randn(count * new, H, d, device="cuda", generator=g).to(DT[dt])
    plain = B.szo_attention_kv8(cache, batch, q)
    o = B.szo_attention_kv8_prefix(cache, batch, shared, q)
    # values are at most 448 * 2^-7 = 3.5; logits' partial sums at most sum |q k| <= 6 * 3.5 * d / sqrt(d)
    logit = ((d + 8) * 2.0 ** -23 + 2.0 ** -20) * 6 * 3.5 * d ** 0.5
    each = 3.5 * ((2.0 ** -20 if dt == "f32" else 2.0 ** -11) + 2 * logit + (max(lens) + 16) * 2.0 ** -23 + torch.finfo(DT[dt]).eps / 2)
    assert (plain.double() - o.double()).abs().max() <= 2 * each
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = B.szo_attention_kv8_prefix(cache, batch, shared, q)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = B.szo_attention_kv8_prefix(cache, batch, shared, q)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, again) and torch.equal(o, replayed)
    # the graph reads lengths and groups when it runs
    batch.kv_len.sub_(torch.arange(count, device="cuda", dtype=torch.int32) % 2 * min(new, 1))
    shared.length.fill_(prefix // 2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(replayed, B.szo_attention_kv8_prefix(cache, batch, shared, q))
    assert B.device_status() == 0


def test_binding_refuses_what_does_not_fit(B):
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for args in [(ints(1).long(),), (ints(1).cpu(),), (ints(1, 2),), (ints(1), ints(0, 1)), (ints(1), ints(0, 1, 2), 2), (ints(1).view(1, 1),)]:
        with pytest.raises(ValueError):
            B.Kv8Prefix(*args)
