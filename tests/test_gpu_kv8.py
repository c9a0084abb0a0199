"""The 8-bit paged key/value cache on the GPU: writing, reading and attention against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}              # half a step, relative
ERR_ARG, ERR_SHAPE = -1, -2


@pytest.fixture(scope="module")
def B():
    from paper_2406_02913_b200 import binding
    binding.lib()
    return binding


class World:
    """A cache with shuffled pages, its reference, and the sequences' page lists."""

    def __init__(self, B, caps, hkv, page, d, seed, extra=2):
        self.g = np.random.default_rng(seed)
        counts = [max(1, -(-c // page)) for c in caps]
        n_pages = sum(counts) + extra
        order = self.g.permutation(n_pages)
        self.pages, at = [], 0
        for c in counts:
            self.pages.append(order[at:at + c])
            at += c
        self.spare = order[at:]
        # memory as an earlier user left it: any codes, NaN among them, and any scales
        codes = self.g.integers(0, 256, (2, n_pages, hkv, page, d), dtype=np.uint8)
        scales = 2.0 ** self.g.integers(-5, 6, (n_pages, hkv, 2)).astype(np.float64)
        self.ref = ref.Cache(codes, scales)
        self.cache = B.Kv8Cache(torch.from_numpy(codes).cuda(), torch.from_numpy(scales.astype(np.float32)).cuda())
        self.table = np.full((len(caps), max(counts) + 1), -7, np.int32)
        for b, p in enumerate(self.pages):
            self.table[b, :len(p)] = p
        self.d_table = torch.from_numpy(self.table).cuda()
        self.hkv, self.d, self.B = hkv, d, B

    def batch(self, lens, news, gap=0):
        start = np.concatenate([[gap], gap + np.cumsum(news)]).astype(np.int32)
        rows = int(start[-1]) + gap
        return self.B.Kv8Batch(self.d_table, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows, torch.from_numpy(start).cuda(),
                               max(max(news), 1)), start, rows

    def check(self):
        got = self.cache.codes.cpu().numpy()
        e = np.log2(self.cache.scales.double().cpu().numpy())
        # codes are numbers: -0 and 0 apart, NaN is 0x7f or 0xff
        assert np.array_equal(e, self.ref.e)
        same = (got == self.ref.codes) | (((got & 127) == 127) & ((self.ref.codes & 127) == 127))
        assert same.all(), np.argwhere(~same)[:5]


def _rows(g, n, heads, d, dt, loud=1.0):
    x = g.normal(0, 1, (n, heads, d)) * np.exp(g.normal(0, 1.2, (n, heads, 1))) * loud
    return torch.from_numpy(x).to(DT[dt])


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,hkv,page", [(64, 1, 16), (64, 3, 128), (128, 2, 16), (128, 5, 32), (128, 1, 64)])
def test_write_and_read_match_the_definition(B, dt, d, hkv, page):
    caps = [1, 17, 70, 200, 33]
    w = World(B, caps, hkv, page, d, seed=d + hkv + page)
    lens = [0] * len(caps)
    # prompts of odd lengths, single tokens, a few at once, none; later ones louder, so that scales have to grow
    for step, news in enumerate([[1, 15, 31, 150, 0], [0, 1, 1, 1, 1], [0, 1, 33, 0, 16], [0, 0, 5, 49, 16]]):
        lens = [a + n for a, n in zip(lens, news)]
        batch, start, rows = w.batch(lens, news, gap=step)
        k, v = _rows(w.g, rows, hkv, d, dt, 3.0 ** step), _rows(w.g, rows, hkv, d, dt, 2.0 ** -step)
        B.szo_kv8_write(w.cache, batch, k.cuda(), v.cuda())
        for b, n in enumerate(news):
            for which, x in enumerate((k, v)):
                w.ref.write(w.pages[b], lens[b] - n, x[start[b]:start[b + 1]].double().numpy(), which)
        w.check()
    batch, start, rows = w.batch(lens, lens)
    for out in ("f32", "bf16", "f16"):
        got = B.szo_kv8_read(w.cache, batch, DT[out])
        for which in (0, 1):
            want = np.concatenate([w.ref.values(w.pages[b], lens[b], which) for b in range(len(caps))])
            assert torch.equal(got[which].cpu(), torch.from_numpy(want).to(DT[out]))
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_special_values(B, dt):
    d, hkv, page = 64, 2, 16
    w = World(B, [40], hkv, page, d, seed=9)
    big = {"f32": 3e38, "bf16": 3e38, "f16": 6e4}[dt]
    tiny = {"f32": 1e-42, "bf16": 1e-39, "f16": 6e-8}[dt]
    x = _rows(w.g, 20, hkv, d, dt)
    x[0] = 0.0                                        # (a page of zeros in head 1 below)
    x[:16, 1] = 0.0
    x[1, 0, 3], x[2, 0, 5], x[3, 0, 7], x[4, 0, 9], x[17, 1, 1], x[18, 0, 2] = float("nan"), float("inf"), -float("inf"), big, big, tiny
    x[5, 0, 0] = -0.0
    batch, _, _ = w.batch([20], [20])
    B.szo_kv8_write(w.cache, batch, x.cuda(), x.cuda())
    for which in (0, 1):
        w.ref.write(w.pages[0], 0, x.double().numpy(), which)
    w.check()
    # the same positions written again, quieter: the first page is fresh again, nothing of it stays
    y = _rows(w.g, 20, hkv, d, dt, 0.01)
    B.szo_kv8_write(w.cache, batch, y.cuda(), x.cuda())
    w.ref.write(w.pages[0], 0, y.double().numpy(), 0)
    w.ref.write(w.pages[0], 0, x.double().numpy(), 1)
    w.check()


def test_padding_rows_slices_and_strangers(B):
    """Rows at negative positions, rows of no sequence, row buffers that are slices of wider ones."""
    d, hkv, page, H = 64, 2, 16, 4
    w = World(B, [20, 20, 20], hkv, page, d, seed=4)
    lens, news = [3, 0, 18], [7, 4, 18]
    batch, start, rows = w.batch(lens, news, gap=2)
    wide = torch.randn(rows, (H + 2 * hkv) * d, dtype=torch.bfloat16)
    dev = wide.cuda()
    k, v = dev[:, H * d:(H + hkv) * d], dev[:, (H + hkv) * d:]
    B.szo_kv8_write(w.cache, batch, k, v)
    for b in (0, 2):
        for which, x in enumerate((k, v)):
            x = x.cpu().double().numpy().reshape(rows, hkv, d)[start[b + 1] - lens[b]:start[b + 1]]
            w.ref.write(w.pages[b], 0, x, which)
    w.check()
    out = torch.full((rows, 2 * hkv * d + 8), 7.0, device="cuda")
    B.szo_kv8_read(w.cache, batch, out=(out[:, :hkv * d], out[:, hkv * d:2 * hkv * d]))
    o = out.cpu().numpy()
    assert (o[:, 2 * hkv * d:] == 7).all() and (o[:2] == 7).all() and (o[-2:] == 7).all()
    for b in range(3):
        pad = news[b] - lens[b]
        assert (o[start[b]:start[b] + pad, :2 * hkv * d] == 0).all()
        for which in (0, 1):
            want = w.ref.values(w.pages[b], lens[b], which).reshape(lens[b], hkv * d)
            assert np.array_equal(o[start[b] + pad:start[b + 1], which * hkv * d:(which + 1) * hkv * d], want)
    # attention: zeros for padding, strangers left alone, q and o slices too
    buf = torch.full((rows, H * d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    B.szo_attention_kv8(w.cache, batch, dev[:, :H * d], out=buf[:, :H * d])
    o = buf.float().cpu().numpy()
    assert (o[:, H * d:] == 7).all() and (o[:2] == 7).all() and (o[-2:] == 7).all()
    for b in range(3):
        assert (o[start[b]:start[b] + news[b] - lens[b], :H * d] == 0).all()
        assert (np.abs(o[start[b] + news[b] - lens[b]:start[b + 1], :H * d]).max(1) > 0).all()
    assert B.device_status() == 0


def attention_bound(o, wide, big, length, d, dt, top=0.0):
    """Allowed error per element.  A logit is off by at most (d + 8) roundings of its largest partial sum (2^-23 each:
    tensor cores truncate) and, relative to its size, by the few roundings of scaling it and of exp2 (2^-21); weights
    are held in 11 bits (fp32 queries: in 21), sums of `length` terms in 24; a weight below the fp16 range is off by at most
    2^-32 of the largest one, times codes of at most 448 (top: the largest weight times its page's scale); then the one
    rounding of the result."""
    logit = ((d + 8) * 2.0 ** -23 + 2.0 ** -20) * big[..., None]
    weight = 2.0 ** -20 if dt == "f32" else 2.0 ** -11
    return (wide * (weight + 2 * logit + (length + 16) * 2.0 ** -23) * 1.01 + length * 2.0 ** -32 * 448 * top + HALF[dt] * np.abs(o)
            + (2.0 ** -25 if dt == "f16" else 1e-30))


def run_attention(B, w, lens, news, H, dt, scale=None, spread=1.0, gap=1):
    batch, start, rows = w.batch(lens, news, gap)
    q = torch.from_numpy(w.g.normal(0, spread, (rows, H, w.d))).to(DT[dt])
    out = torch.full_like(q, 3.0).cuda()
    B.szo_attention_kv8(w.cache, batch, q.cuda(), scale=scale, out=out)
    got = out.double().cpu().numpy()
    assert (got[:gap] == 3).all() and (got[rows - gap:] == 3).all()
    sc = scale if scale is not None else 1 / math.sqrt(w.d)
    for b, (n, m) in enumerate(zip(lens, news)):
        if m == 0:
            continue
        k, v = (w.ref.values(w.pages[b], n, which) for which in (0, 1))
        size = 2.0 ** w.ref.e[w.pages[b][np.arange(n) // w.ref.page], :, 1]             # [n, heads]
        o, wide, big, top = ref.attention(q[start[b]:start[b + 1]].double().numpy(), k, v, n - m, sc, size)
        mine = got[start[b]:start[b + 1]]
        assert np.array_equal(np.isnan(mine), np.isnan(o)), (b, n, m)
        bad = np.abs(np.nan_to_num(mine - o)) > np.nan_to_num(attention_bound(o, wide, big, n, w.d, dt, top[..., None]), nan=1.0)
        assert not bad.any(), (b, n, m, np.argwhere(bad)[:4], np.abs(mine - o).max())
    return batch, q


def fill(B, w, lens, dt="bf16", loud=1.0):
    batch, start, rows = w.batch(lens, lens)
    k, v = _rows(w.g, rows, w.hkv, w.d, dt, loud), _rows(w.g, rows, w.hkv, w.d, dt, loud)
    B.szo_kv8_write(w.cache, batch, k.cuda(), v.cuda())
    for b in range(len(lens)):
        for which, x in enumerate((k, v)):
            w.ref.write(w.pages[b], 0, x[start[b]:start[b + 1]].double().numpy(), which)


SHAPES = [(64, 1, 1, 16), (128, 2, 1, 16), (128, 1, 4, 64), (64, 2, 5, 32), (128, 1, 8, 128), (64, 1, 9, 16), (128, 2, 3, 32)]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,hkv,group,page", SHAPES)
def test_attention_of_single_tokens(B, dt, d, hkv, group, page):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 129, 700]
    w = World(B, lens, hkv, page, d, seed=group + page)
    fill(B, w, lens)
    run_attention(B, w, lens, [1] * len(lens), hkv * group, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,hkv,group,page", SHAPES)
def test_attention_of_a_few_tokens(B, dt, d, hkv, group, page):
    lens = [5, 9, 64, 130, 259, 300]
    w = World(B, lens, hkv, page, d, seed=group * page)
    fill(B, w, lens)
    run_attention(B, w, lens, [5, 3, 0, 2, 11, 1], hkv * group, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,hkv,group,page", [(128, 1, 4, 64), (64, 2, 1, 16), (128, 1, 3, 32), (64, 1, 8, 128)])
def test_attention_of_prompts_and_chunks(B, dt, d, hkv, group, page):
    lens = [200, 333, 1, 257, 520]
    w = World(B, lens, hkv, page, d, seed=3 * group + page)
    fill(B, w, lens)
    run_attention(B, w, lens, [200, 130, 1, 129, 300], hkv * group, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("new", [1, 6, 150])
def test_attention_pages_of_very_different_sizes(B, dt, new):
    """Scales from 2^-40 to 2^40 in one sequence: weights must not be lost because another page's values are large."""
    w = World(B, [400], 1, 16, 64, seed=8)
    batch, _, rows = w.batch([400], [400])
    k = _rows(w.g, rows, 1, 64, "f32", 0.3)
    v = _rows(w.g, rows, 1, 64, "f32") * (2.0 ** torch.from_numpy(np.repeat(w.g.integers(-40, 41, 25), 16)).double())[:, None, None].float()
    B.szo_kv8_write(w.cache, batch, k.cuda(), v.float().cuda())
    w.ref.write(w.pages[0], 0, k.double().numpy(), 0)
    w.ref.write(w.pages[0], 0, v.double().numpy(), 1)
    w.check()
    if dt != "f16":                                     # (fp16 cannot hold the results)
        run_attention(B, w, [400], [new], 2, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("spread,scale", [(60.0, None), (1e-3, None), (1.0, 0.0), (1.0, -0.2), (1e4, 1e-5), (1e-6, 1e4)])
@pytest.mark.parametrize("new", [1, 7, 140])
def test_attention_sharp_flat_and_odd_scales(B, dt, spread, scale, new):
    w = World(B, [300], 1, 32, 64, seed=12)
    fill(B, w, [300])
    run_attention(B, w, [300], [new], 2, dt, scale=scale, spread=spread)


@pytest.mark.parametrize("new", [4, 16, 150])
def test_nan_reaches_only_rows_that_attend_to_it(B, new):
    w = World(B, [170, 170], 1, 16, 64, seed=13)
    lens = [170, 170]
    batch, start, rows = w.batch(lens, lens)
    k, v = _rows(w.g, rows, 1, 64, "bf16"), _rows(w.g, rows, 1, 64, "bf16")
    v[168, 0, 5] = float("nan")                          # value of position 168 of sequence 0
    k[170 + 169, 0, 7] = float("inf")                    # key of the last position of sequence 1
    B.szo_kv8_write(w.cache, batch, k.cuda(), v.cuda())
    for b in (0, 1):
        for which, x in enumerate((k, v)):
            w.ref.write(w.pages[b], 0, x[start[b]:start[b + 1]].double().numpy(), which)
    for dt in ("bf16", "f32"):
        run_attention(B, w, lens, [new, new], 2, dt)
    # a NaN query: its row, no other
    batch, start, rows = w.batch(lens, [new, new])
    q = torch.randn(rows, 2, 64, dtype=torch.bfloat16, device="cuda")
    q[1, 0, 3] = float("nan")
    o = B.szo_attention_kv8(w.cache, batch, q)
    assert o[1, 0].isnan().all() and not o[0].isnan().any() and not o[1, 1].isnan().any()


def test_prefix_pages_shared_by_sequences(B):
    w = World(B, [96, 96], 2, 32, 128, seed=14)
    fill(B, w, [96, 96])
    w.table[1, :2] = w.table[0, :2]
    w.pages[1] = np.concatenate([w.pages[0][:2], w.pages[1][2:]])
    w.d_table.copy_(torch.from_numpy(w.table))
    run_attention(B, w, [96, 96], [1, 1], 8, "bf16")
    run_attention(B, w, [96, 80], [40, 3], 8, "bf16")


def test_descriptions_that_do_not_fit_are_reported_and_skipped(B):
    """Lengths beyond the table, starts out of order, page ids of no page: the status word says so, nothing else moves."""
    w = World(B, [40, 40, 40], 1, 16, 64, seed=15)
    fill(B, w, [40, 40, 40])
    H = 2

    def run(lens, start, rows, max_new, table=None):
        t = w.d_table if table is None else table
        batch = B.Kv8Batch(t, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows, torch.tensor(start, dtype=torch.int32, device="cuda"), max_new)
        x = torch.ones(rows, 1, 64, device="cuda")
        before = w.cache.codes.clone(), w.cache.scales.clone()
        B.szo_kv8_write(w.cache, batch, x, x)
        s0 = B.device_status()
        moved = not torch.equal(before[0], w.cache.codes)
        w.cache.codes.copy_(before[0])
        w.cache.scales.copy_(before[1])
        o = torch.full((rows, H, 64), 3.0, device="cuda")
        B.szo_attention_kv8(w.cache, batch, torch.ones_like(o), out=o)
        s1 = B.device_status()
        r = torch.full((rows, 1, 64), 3.0, device="cuda")
        B.szo_kv8_read(w.cache, batch, out=(r, r.clone()))
        s2 = B.device_status()
        assert s0 == s1 == s2
        return s0, moved, o.cpu(), r.cpu()

    cap = w.table.shape[1] * 16
    for lens, start, rows, max_new in [([cap + 1, 40, 40], [0, 1, 1, 1], 1, 1), ([-3, 40, 40], [0, 1, 1, 1], 1, 1), ([40, 40, 40], [2, 1, 1, 1], 2, 2),
                                       ([40, 40, 40], [-1, 1, 1, 1], 2, 2), ([40, 40, 40], [0, 3, 3, 3], 2, 4), ([40, 40, 40], [0, 3, 3, 3], 4, 2)]:
        st, moved, o, r = run(lens, start, rows, max_new)
        assert st == ERR_SHAPE and not moved and (o == 3).all() and (r == 3).all()
    for bad in (-1, w.cache.n_pages, 1 << 30):
        t = w.d_table.clone()
        t[0, 2] = bad                                    # positions 32 .. 39 of sequence 0
        st, moved, o, r = run([40, 40, 40], [0, 1, 1, 1], 1, 1, t)
        assert st == ERR_ARG and not moved and (r == 0).all() and o.isfinite().all()
        k, v = (w.ref.values(w.pages[0], 32, i) for i in (0, 1))
        want, wide, big, _ = ref.attention(np.ones((1, H, 64)), k, v, 31, 0.125)      # the 32 positions that there are
        assert (np.abs(o.numpy() - want) <= attention_bound(want, wide, big, 32, 64, "f32")).all()


def test_offsets_beyond_32_bits(B):
    """A cache of more than 2^32 codes (keys alone), pages at its far end."""
    n_pages, hkv, page, d = 36000, 8, 128, 128
    assert n_pages * hkv * page * d > 1 << 32
    cache = B.Kv8Cache.empty(n_pages, hkv, page, d)
    g = np.random.default_rng(1)
    small = ref.Cache(np.zeros((2, 4, hkv, page, d), np.uint8), np.zeros((4, hkv, 2)))
    far = [n_pages - 1, 17, n_pages - 3, n_pages - 2]
    table = torch.tensor([far], dtype=torch.int32, device="cuda")
    n = 400
    k, v = _rows(g, n, hkv, d, "bf16"), _rows(g, n, hkv, d, "bf16")
    kv_len = torch.tensor([n], dtype=torch.int32, device="cuda")
    batch = B.Kv8Batch(table, kv_len, n)
    B.szo_kv8_write(cache, batch, k.cuda(), v.cuda())
    for which, x in enumerate((k, v)):
        small.write(range(4), 0, x.double().numpy(), which)
    got = B.szo_kv8_read(cache, batch, torch.float32)
    for which in (0, 1):
        assert np.array_equal(got[which].cpu().double().numpy(), small.values(range(4), n, which))
    for new in (1, 40):
        q = torch.from_numpy(g.normal(0, 1, (new, 2 * hkv, d))).bfloat16()
        o = B.szo_attention_kv8(cache, B.Kv8Batch(table, kv_len, new), q.cuda()).double().cpu().numpy()
        size = 2.0 ** small.e[np.arange(n) // page, :, 1]
        want, wide, big, top = ref.attention(q.double().numpy(), small.values(range(4), n, 0), small.values(range(4), n, 1), n - new, d ** -0.5, size)
        assert not (np.abs(o - want) > attention_bound(want, wide, big, n, d, "bf16", top[..., None])).any()


def test_no_rows_no_sequences(B):
    w = World(B, [16], 1, 16, 64, seed=2)
    empty = B.Kv8Batch(w.d_table[:0], torch.empty(0, dtype=torch.int32, device="cuda"), 0)
    none = B.Kv8Batch(w.d_table, torch.zeros(1, dtype=torch.int32, device="cuda"), 0)
    for b in (empty, none):
        z = torch.empty(0, 1, 64, device="cuda")
        B.szo_kv8_write(w.cache, b, z, z)
        assert B.szo_kv8_read(w.cache, b)[0].shape == (0, 1, 64)
        assert B.szo_attention_kv8(w.cache, b, z).shape == (0, 1, 64)
    w.check()
    assert B.device_status() == 0


def test_captured_and_replayed_with_other_lengths_on_two_streams(B):
    """One captured write + attention serves every later length; two graphs of two batches replay side by side."""
    worlds = [World(B, [80, 50], 2, 16, 64, seed=30 + i) for i in range(2)]
    H, graphs, state = 4, [], []
    for w in worlds:
        fill(B, w, [37, 20])
        lens = torch.tensor([37, 20], dtype=torch.int32, device="cuda")
        batch = B.Kv8Batch(w.d_table, lens, 2)
        k, v, q = (torch.zeros(2, h, 64, dtype=torch.bfloat16, device="cuda") for h in (2, 2, H))
        o = torch.zeros_like(q)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.szo_kv8_write(w.cache, batch, k, v)
            B.szo_attention_kv8(w.cache, batch, q, out=o)
        graphs.append((graph, s))
        state.append((lens, k, v, q, o))
    for step in range(6):
        torch.cuda.synchronize()
        for w, (lens, k, v, q, o) in zip(worlds, state):
            lens += 1
            for t in (k, v, q):
                t.copy_(torch.from_numpy(w.g.normal(0, 1 + step, tuple(t.shape))))
        torch.cuda.synchronize()
        for graph, s in graphs:
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for w, (lens, k, v, q, o) in zip(worlds, state):
            for b in (0, 1):
                n = int(lens[b])
                for which, x in enumerate((k, v)):
                    w.ref.write(w.pages[b], n - 1, x[b:b + 1].double().cpu().numpy(), which)
                size = 2.0 ** w.ref.e[w.pages[b][np.arange(n) // 16], :, 1]
                want, wide, big, top = ref.attention(q[b:b + 1].double().cpu().numpy(), w.ref.values(w.pages[b], n, 0), w.ref.values(w.pages[b], n, 1), n - 1,
                                                     0.125, size)
                assert not (np.abs(o[b:b + 1].double().cpu().numpy() - want) > attention_bound(want, wide, big, n, 64, "bf16", top[..., None])).any()
            w.check()


@pytest.mark.parametrize("d,hkv,group,page", [(128, 2, 4, 16), (64, 1, 7, 128), (64, 8, 1, 32)])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_long_contexts_of_few_sequences(B, dt, d, hkv, group, page):
    """Page tables long enough for the form that joins its blocks' results in a second launch."""
    lens = [13001, 31]
    w = World(B, lens, hkv, page, d, seed=d + group)
    fill(B, w, lens)
    run_attention(B, w, lens, [1, 1], hkv * group, dt)
    run_attention(B, w, [12999, 20], [8 // group, 0], hkv * group, dt)


@pytest.mark.parametrize("d,hkv,group,page", [(128, 1, 4, 32), (64, 2, 3, 64)])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_chunks_of_few_sequences_with_long_contexts(B, dt, d, hkv, group, page):
    """Few blocks of query rows: their positions are cut and joined."""
    lens = [2900, 700]
    w = World(B, lens, hkv, page, d, seed=d + group)
    fill(B, w, lens)
    run_attention(B, w, lens, [130, 60], hkv * group, dt)
    run_attention(B, w, [2100, 30], [97, 100], hkv * group, dt)           # (and padding rows in a cut sequence)
    assert B.device_status() == 0


@pytest.mark.parametrize("d,group", [(128, 4), (64, 5)])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_cut_chunks_with_empty_shares(B, dt, d, group):
    """The table allows many shares, the lengths leave most of them nothing: sequences of a few positions, none at all, padding."""
    lens = [2900, 5, 0, 129, 1]
    w = World(B, lens, 1, 32, d, seed=d + group)
    fill(B, w, lens)
    run_attention(B, w, lens, [61, 70, 66, 64, 1], group, dt)
    run_attention(B, w, [2899, 0, 0, 128, 0], [1, 90, 0, 128, 3], group, dt)
    assert B.device_status() == 0


@pytest.mark.parametrize("new", [8, 9, 16, 17, 33])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
def test_rows_around_the_choice_of_kernel(B, dt, new):
    lens = [40, 300, 64, 129, 511, 17]
    w = World(B, lens, 4, 16, 128, seed=new)
    fill(B, w, lens)
    run_attention(B, w, lens, [min(new, n) for n in lens], 16, dt)
    run_attention(B, w, lens, [new, new - 1, 0, 0, 1, 0], 16, dt)


def test_same_call_same_bits(B):
    w = World(B, [14000, 900], 2, 32, 128, seed=21)
    fill(B, w, [14000, 900])
    for dt, news in (("bf16", [1, 1]), ("f32", [3, 2]), ("f16", [200, 150])):
        batch, _, rows = w.batch([14000, 900], news)
        q = torch.randn(rows, 8, 128, device="cuda").to(DT[dt])
        first = B.szo_attention_kv8(w.cache, batch, q)
        for _ in range(5):
            assert torch.equal(first, B.szo_attention_kv8(w.cache, batch, q))


def test_binding_refusals(B):
    w = World(B, [40], 2, 16, 64, seed=1)
    batch, _, _ = w.batch([40], [2])
    ok = torch.zeros(2, 2, 64, device="cuda")
    with pytest.raises(ValueError):
        B.szo_kv8_write(w.cache, batch, ok, ok.half())
    with pytest.raises(ValueError):
        B.szo_kv8_write(w.cache, batch, ok[:1], ok[:1])
    with pytest.raises(ValueError):
        B.szo_kv8_write(w.cache, batch, ok.transpose(1, 2).contiguous().transpose(1, 2), ok)
    with pytest.raises(ValueError):
        B.szo_kv8_write(w.cache, batch, ok.double(), ok.double())
    with pytest.raises(ValueError):
        B.szo_attention_kv8(w.cache, batch, ok.cpu())
    with pytest.raises(B.SzoError):
        B.szo_attention_kv8(w.cache, batch, torch.zeros(2, 3, 64, device="cuda"))        # 3 heads on 2
    with pytest.raises(B.SzoError):
        B.szo_attention_kv8(w.cache, batch, ok, scale=float("nan"))
    with pytest.raises(ValueError):
        B.Kv8Batch(w.d_table, torch.zeros(2, dtype=torch.int32, device="cuda"), 2)
    with pytest.raises(ValueError):
        B.Kv8Batch(w.d_table.long(), torch.zeros(1, dtype=torch.int32, device="cuda"), 2)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("new", [3, 9, 150])
@pytest.mark.parametrize("cap", [200, 13000])
def test_padding_rows_of_any_content_are_zeros(B, dt, new, cap):
    """Rows at negative positions hold whatever was in memory, NaN and infinities among it: zeros come out, and the other rows are
    those of padding rows of zeros.  With the long page table the positions are cut and joined."""
    caps, lens = [cap, 200, 200], [2, 0, 64]
    w = World(B, caps, 1, 16, 64, seed=new)
    fill(B, w, lens)
    news = [new, new, min(new, 64) + 1]
    batch, start, rows = w.batch(lens, news)
    q = torch.randn(rows, 2, 64, device="cuda").to(DT[dt])
    dirty = q.clone()
    pad = torch.zeros(rows, dtype=torch.bool)
    for b in range(3):
        pad[start[b]:start[b + 1] - min(lens[b], news[b])] = True
    at = torch.nonzero(pad)[:, 0].cuda()
    q[at] = 0
    dirty[at] = float("inf")
    dirty[at[::2], :, ::3] = float("nan")
    dirty[at[1::3], 0] = -float("inf")
    want, got = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
    B.szo_attention_kv8(w.cache, batch, q, out=want)
    B.szo_attention_kv8(w.cache, batch, dirty, out=got)
    assert (want[at] == 0).all() and not want[start[0]:start[3]].isnan().any()
    assert torch.equal(got, want)
    assert B.device_status() == 0


@pytest.mark.parametrize("dt,new", [("bf16", 1), ("f32", 1), ("bf16", 9), ("bf16", 150)])
@pytest.mark.parametrize("cap", [300, 13000])
def test_every_page_id_of_no_page_is_reported(B, dt, new, cap):
    """A needed entry outside [0, n_pages), -2 like any other, is reported by every operator, and its positions are left out."""
    w = World(B, [cap, 200], 1, 16, 64, seed=6)
    fill(B, w, [290, 200])
    out = []
    for bad in (-1, -2, -3, w.cache.n_pages, -2 ** 31, 2 ** 31 - 1):
        t = w.d_table.clone()
        t[0, 2] = bad
        batch = B.Kv8Batch(t, torch.tensor([290, 200], dtype=torch.int32, device="cuda"), 2 * new)
        q = torch.from_numpy(np.random.default_rng(1).normal(0, 1, (2 * new, 2, 64))).to(DT[dt]).cuda()
        assert B.device_status() == 0
        o = B.szo_attention_kv8(w.cache, batch, q)
        assert B.device_status() == ERR_ARG, bad
        B.szo_kv8_read(w.cache, B.Kv8Batch(t, batch.kv_len, 2 * 290))
        assert B.device_status() == ERR_ARG, bad
        out.append(o)
    assert all(torch.equal(o, out[0]) for o in out) and out[0].isfinite().all()
    # entries that no position needs are not read: -2 behind the last page
    t = w.d_table.clone()
    t[0, -(-290 // 16):] = -2
    B.szo_attention_kv8(w.cache, B.Kv8Batch(t[:1], torch.tensor([290], dtype=torch.int32, device="cuda"), new), q[:new])
    assert B.device_status() == 0


def test_same_bits_for_ragged_batches_and_chunks(B):
    """Single tokens of many ragged sequences, chunks with a cut last round: the same bits again, with other calls in between."""
    g = np.random.default_rng(3)
    lens = [int(n) for n in g.integers(300, 2500, 32)]
    w = World(B, lens, 8, 64, 128, seed=23)
    batch, _, rows = w.batch(lens, lens)
    B.szo_kv8_write(w.cache, batch, *torch.randn(2, rows, 8, 128, device="cuda").unbind(0))
    for dt, news in (("bf16", [1] * 32), ("f16", [1] * 32), ("bf16", [200] * 4 + [0] * 28)):
        batch, _, rows = w.batch(lens, news)
        q, other = (torch.randn(rows, 32, 128, device="cuda").to(DT[dt]) for _ in range(2))
        want, got = torch.zeros_like(q), torch.zeros_like(q)
        B.szo_attention_kv8(w.cache, batch, q, out=want)
        for _ in range(10):
            B.szo_attention_kv8(w.cache, batch, other, out=got)
            B.szo_attention_kv8(w.cache, batch, q, out=got)
            assert torch.equal(got, want)
