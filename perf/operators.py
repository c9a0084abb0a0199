"""The operators of token generation from an 8-bit key/value cache and of scoring what was generated.

An operator's pass in its plain form (elementary torch operations in 32 bits) and through the library's
entry points, on the same inputs:

  write     keys and values of new tokens stored in a paged cache of e4m3 codes with one power-of-two scale
            per (page, key/value head)
  read      cached positions read back as ordinary numbers
  attend    attention of each sequence's newest tokens over its cache
  score     log probabilities of given tokens, entropy and the best alternatives of rows of logits
  grad      the gradient of those log probabilities and entropies with respect to the logits

Cache: codes uint8 [2 (keys, values), pages, heads, page_tokens, head_dim], scales fp32 [pages, heads, 2].
A batch: page_table int32 [batch, max_pages]; kv_len int32 [batch], the positions of each sequence that are
cached once its new tokens are; start int32 [batch + 1], the rows of each sequence in the row buffers.  The
n-th last row of a sequence stands at the n-th last of its positions.
"""
import math

import torch

own = False

E_MIN, E_MAX = -63, 63                       # exponents of the cache's scales
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------------------ the cases
def _cache_case(name, op, dtype, batch, length, length_min, new, new_min, heads, kv_heads, head_dim, page):
    c = dict(op=op, dtype=dtype, batch=batch, len=length, len_min=length_min, new=new, new_min=new_min, heads=heads,
             kv_heads=kv_heads, head_dim=head_dim, page=page)
    return dict(c, name=name) if name else c


def _row_case(name, op, dtype, rows, vocab, pad, targets, top, scale):
    c = dict(op=op, dtype=dtype, rows=rows, vocab=vocab, pad=pad, targets=targets, top=top, scale=scale)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a batch of prompts of the grouped-query 7B shape enters the cache
        _cache_case("write_prompts_8x2048", "write", "bf16", 8, 2048, 1601, 2048, 1601, 32, 8, 128, 64),
        # one layer of a token step of the 7B shape without grouped queries, 32 sequences
        _cache_case("write_token_32", "write", "f16", 32, 1100, 300, 1, 1, 32, 32, 128, 16),
        # contexts handed to a part of the program that wants ordinary numbers
        _cache_case("read_contexts_4x8192", "read", "bf16", 4, 8192, 8000, 8192, 8000, 32, 8, 128, 32),
        # a few short odd ones, for checking
        _cache_case("read_short_odd", "read", "f32", 3, 517, 1, 517, 1, 8, 4, 64, 16),
        # several new tokens per sequence (drafts being verified) in the fp32 form, odd group of heads: latency
        _cache_case("attend_drafts_f32", "attend", "f32", 3, 777, 65, 5, 2, 10, 2, 64, 16),
        # a token step of a ragged batch, grouped-query 7B shape
        _cache_case("attend_token_32_ragged", "attend", "bf16", 32, 8192, 513, 1, 1, 32, 8, 128, 64),
        # one sequence with a very long context
        _cache_case("attend_token_1x131071", "attend", "f16", 1, 131071, 131071, 1, 1, 32, 8, 128, 32),
        # the last chunks of two long prompts
        _cache_case("attend_prompt_2x2048_at_8192", "attend", "bf16", 2, 8192, 7700, 2048, 2000, 32, 8, 128, 64),
        # the distribution of a token step's next tokens, with the 20 best
        _row_case("score_step_8x32000", "score", "f32", 8, 32000, 0, 1, 20, 1.25),
        # log likelihood of whole sequences, vocabulary of the 13B shape, two candidates per position
        _row_case("score_prompts_4096x50272", "score", "bf16", 4096, 50272, 0, 2, 0, 1.0),
        # the gradient of a batch's log likelihood
        _row_case("grad_2048x32000", "grad", "bf16", 2048, 32000, 0, 1, 0, 1.0),
        # a few rows of odd width that lie apart
        _row_case("grad_24x50271", "grad", "f32", 24, 50271, 9, 3, 0, 0.7),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    while True:
        op = rng.choice(("write", "read", "attend", "attend", "attend", "score", "grad"))
        dtype = rng.choice(("bf16", "f16", "f32"))
        if op in ("score", "grad"):
            case = _row_case(None, op, dtype, _log_int(rng, 1, 4096), _log_int(rng, 500, 160000), rng.choice((0, 0, 1, 8, 57)),
                             rng.randint(1, 4), rng.choice((0, 1, 5, 20, 32)) if op == "score" else 0,
                             round(rng.uniform(0.5, 1.5), 3))
            if work(case)["bytes"] <= 4.2e8:
                return case
            continue
        kv_heads, group = rng.choice((1, 2, 4, 8, 16, 32)), rng.choice((1, 2, 3, 4, 5, 7, 8))
        length = _log_int(rng, 1, 131072)
        length_min = rng.randint(max(1, length // 16), length)
        new = length
        if op != "read":
            new = min(length_min, rng.choice((1, 1, 1, rng.randint(2, 8), _log_int(rng, 1, 4096), _log_int(rng, 16, 4096))))
        case = _cache_case(None, op, dtype, _log_int(rng, 1, 64), length, length_min, new, rng.randint(1, min(new, length_min)),
                           kv_heads * group, kv_heads, rng.choice((64, 128)), rng.choice((16, 32, 64)))
        cached = case["batch"] * length * kv_heads * case["head_dim"]
        w = work(case)
        if cached > 1.4e8 or w["bytes"] > 3.5e8:
            continue
        if op == "attend" and (case["batch"] * case["heads"] * new * length > 1.0e9 or w["flops"] > 4.8e11):
            continue
        return case


def _spread(top, low, n):
    return [top - (top - low) * b // max(n - 1, 1) for b in range(n)]


def _lens(case):
    """Cached positions and new rows of every sequence."""
    lens = _spread(case["len"], case["len_min"], case["batch"])
    if case["op"] == "read":
        return lens, list(lens)
    return lens, _spread(case["new"], case["new_min"], case["batch"])


def work(case):
    e = SIZES[case["dtype"]]
    if case["op"] in ("score", "grad"):
        n = case["rows"] * case["vocab"]
        small = case["rows"] * (case["targets"] * 8 + 8 + case["top"] * 8)
        if case["op"] == "score":
            return {"bytes": n * e + small, "flops": 6 * n}
        return {"bytes": 2 * n * e + small + case["rows"] * 4, "flops": 6 * n}
    lens, news = _lens(case)
    d, hkv, h, p = case["head_dim"], case["kv_heads"], case["heads"], case["page"]
    pages = lambda a, b: max(0, -(-b // p) - a // p) if b > a else 0  # noqa: E731  pages that hold positions [a, b)
    tables = 4 * case["batch"] * 2
    if case["op"] == "write":
        rows = sum(news)
        touched = sum(pages(a - n, a) for a, n in zip(lens, news))
        return {"bytes": 2 * rows * hkv * d * (e + 1) + touched * (16 * hkv + 4) + tables, "flops": 4 * rows * hkv * d}
    if case["op"] == "read":
        rows = sum(lens)
        return {"bytes": 2 * rows * hkv * d * (e + 1) + sum(pages(0, a) for a in lens) * (8 * hkv + 4) + tables,
                "flops": 2 * rows * hkv * d}
    pairs = sum(n * a - n * (n - 1) // 2 for a, n in zip(lens, news))
    return {"bytes": 2 * sum(news) * h * d * e + 2 * sum(lens) * hkv * d + sum(pages(0, a) for a in lens) * (8 * hkv + 4) + tables,
            "flops": 4 * pairs * h * d}


# ------------------------------------------------------------------------------ the inputs
def _pow2(e):
    """2^e of whole numbers in [-126, 127], exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(amax):
    """The smallest e in [E_MIN, E_MAX] with amax <= 448 * 2^e."""
    m, k = torch.frexp(amax)
    return (k - 9 + (m > 0.875).to(k.dtype)).clamp(E_MIN, E_MAX)


def _codes(x, e):
    """e4m3 codes of x / 2^e (e broadcast to x)."""
    return (x * _pow2(-e)).to(torch.float8_e4m3fn)


def _kv_values(shape, gen):
    """Keys or values as layers make them: heads apart in size, a few loud channels, some loud tokens; shape [..., heads, head_dim]."""
    x = torch.randn(shape, device="cuda", generator=gen)
    head = torch.exp(0.5 * torch.randn(shape[-2], 1, device="cuda", generator=gen))
    loud = 1 + 6 * (torch.rand(shape[-1], device="cuda", generator=gen) < 0.03).float()
    token = torch.exp(0.7 * torch.randn(*shape[:-2], 1, 1, device="cuda", generator=gen).clamp(-2, 2))
    return x.mul_(head).mul_(loud).mul_(token)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    if case["op"] in ("score", "grad"):
        rows, vocab, nt = case["rows"], case["vocab"], case["targets"]
        store = torch.randn(rows, vocab + case["pad"], device="cuda", generator=gen).mul_(2.5).to(dtype)
        logits = store[:, :vocab]
        s = {"case": case, "logits": logits,
             "targets": torch.randint(0, vocab, (rows, nt), device="cuda", generator=gen, dtype=torch.int32)}
        # some positions have no target (padding), some rows a masked vocabulary, as a constrained sampler makes it
        s["targets"][torch.rand(rows, nt, device="cuda", generator=gen) < 0.05] = -1
        masked = torch.rand(rows, 1, device="cuda", generator=gen) < 0.1
        logits.masked_fill_(masked & (torch.rand(rows, vocab, device="cuda", generator=gen) < 0.5), float("-inf"))
        if case["op"] == "grad":
            s["d_logp"] = torch.randn(rows, nt, device="cuda", generator=gen)
            s["d_entropy"] = torch.randn(rows, device="cuda", generator=gen) * 0.1
            s["lse"], s["entropy"] = (t.clone() for t in _statistics(logits, case["scale"])[:2])
        if own:
            from paper_2406_02913_b200 import binding
            s["lib"] = binding
        return s
    lens, news = _lens(case)
    b, p, hkv, d = case["batch"], case["page"], case["kv_heads"], case["head_dim"]
    counts = [-(-n // p) for n in lens]
    n_pages, max_pages = sum(counts) + 3, max(counts) + 1
    order = torch.randperm(n_pages, device="cuda", generator=gen, dtype=torch.int64).to(torch.int32)
    first = torch.tensor([sum(counts[:i]) for i in range(b)], device="cuda")
    have = torch.tensor(counts, device="cuda")
    j = torch.arange(max_pages, device="cuda")
    table = torch.where(j < have[:, None], order[(first[:, None] + j).clamp(max=n_pages - 1)], -1).to(torch.int32)
    codes = torch.empty(2, n_pages, hkv, p, d, dtype=torch.uint8, device="cuda")
    scales = torch.empty(n_pages, hkv, 2, device="cuda")
    for which in (0, 1):
        x = _kv_values((n_pages, p, hkv, d), gen).transpose(1, 2)
        e = _exponent(x.abs().amax((2, 3)))
        codes[which] = _codes(x, e[:, :, None, None]).view(torch.uint8)
        scales[:, :, which] = _pow2(e)
        del x
    s = {"case": case, "codes": codes, "scales": scales, "table": table, "kv_len": torch.tensor(lens, device="cuda", dtype=torch.int32),
         "start": torch.tensor([sum(news[:i]) for i in range(b + 1)], device="cuda", dtype=torch.int32), "rows": sum(news), "max_new": max(news)}
    if case["op"] == "write":
        s["k"] = _kv_values((s["rows"], hkv, d), gen).mul_(1.5).to(dtype)
        s["v"] = _kv_values((s["rows"], hkv, d), gen).mul_(1.5).to(dtype)
    if case["op"] == "attend":
        s["q"] = torch.randn(s["rows"], case["heads"], d, device="cuda", generator=gen).to(dtype)
    if own:
        from paper_2406_02913_b200 import binding
        s["lib"] = binding
        s["cache"] = binding.Kv8Cache(codes, scales)
        s["batch"] = binding.Kv8Batch(table, s["kv_len"], rows=s["rows"], start=s["start"], max_new=s["max_new"])
    return s


# ------------------------------------------------------------------------------ the plain forms
def _rows(s):
    """Sequence, position of every row, and the page and slot it stands in."""
    start, p = s["start"].long(), s["case"]["page"]
    n = start[1:] - start[:-1]
    b = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n, output_size=s["rows"])
    pos = s["kv_len"].long()[b] - start[1:][b] + torch.arange(s["rows"], device="cuda")
    at = pos.clamp(min=0)
    return b, pos, s["table"].long()[b, at // p], at % p


def _plain_write(s):
    c, p = s["case"], s["case"]["page"]
    start, end = s["start"].long(), s["kv_len"].long()
    n = start[1:] - start[:-1]
    pos0 = (end - n).clamp(min=0)
    # every page that takes a new token: [sequence, j] flattened to the ones there are
    j = (pos0 // p)[:, None] + torch.arange((c["new"] + p - 2) // p + 1, device="cuda")
    b, jj = torch.nonzero((j * p < end[:, None]) & (n > 0)[:, None], as_tuple=True)
    j = j[b, jj]
    pages = s["table"].long()[b, j]
    pos = (j * p)[:, None] + torch.arange(p, device="cuda")
    is_new = (pos >= pos0[b][:, None]) & (pos < end[b][:, None])
    is_old = pos < pos0[b][:, None]
    row = (start[1:][b][:, None] - end[b][:, None] + pos).clamp(0, s["rows"] - 1)
    fresh = (j * p >= pos0[b])[:, None]
    for which, x in enumerate((s["k"], s["v"])):
        x = torch.where(is_new[:, :, None, None], x[row].float(), 0.0).transpose(1, 2)      # [pages, heads, slots, head_dim]
        have = s["scales"][pages, :, which].view(torch.int32)
        have = (((have >> 23) & 255) - 127).clamp(E_MIN, E_MAX)
        want = _exponent(x.abs().amax((2, 3)))
        e = torch.where(fresh, want, torch.maximum(have, want))
        old = s["codes"][which, pages]
        again = (old.view(torch.float8_e4m3fn).float() * _pow2((have - e).clamp(min=-126))[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        new = _codes(x, e[:, :, None, None]).view(torch.uint8)
        out = torch.where(is_new[:, None, :, None], new, torch.where((is_old & ~fresh)[:, None, :, None], again, old))
        s["codes"][which, pages] = out
        s["scales"][pages, :, which] = _pow2(e)
    return _cache_values(s)


def _cache_values(s):
    """The cache as values: e4m3 numbers and the scales they are to be multiplied by."""
    c = s["codes"].view(torch.float8_e4m3fn)
    return {"keys": c[0], "values": c[1], "scales": s["scales"]}


def _plain_read(s):
    _, pos, page, slot = _rows(s)
    out = []
    for which in (0, 1):
        x = s["codes"][which].view(torch.float8_e4m3fn)[page, :, slot].float() * s["scales"][page, :, which][:, :, None]
        out.append(torch.where((pos >= 0)[:, None, None], x, 0.0).to(DTYPES[s["case"]["dtype"]]))
    return out


def _plain_attend(s):
    c, d, hkv = s["case"], s["case"]["head_dim"], s["case"]["kv_heads"]
    g, nb, t = c["heads"] // hkv, c["batch"], s["max_new"]
    start, end = s["start"].long(), s["kv_len"].long()
    n = start[1:] - start[:-1]
    i = torch.arange(t, device="cuda")
    q = s["q"][(start[:-1, None] + i).clamp(max=s["rows"] - 1)].float()                  # [batch, t, heads, d]
    q = q.view(nb, t, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(nb, hkv, g * t, d)
    table = s["table"].long().clamp(min=0)
    k, v = ((s["codes"][w][table].view(torch.float8_e4m3fn).float() * s["scales"][table][..., w, None, None])
            .transpose(1, 2).reshape(nb, hkv, -1, d) for w in (0, 1))
    place = torch.arange(k.shape[2], device="cuda")
    v = torch.where((place < end[:, None])[:, None, :, None], v, 0.0)
    seen = (place <= (end - n)[:, None, None] + i[:, None])[:, None, None]                # [batch, 1, 1, t, places]
    x = (q @ k.transpose(2, 3)).view(nb, hkv, g, t, -1) * (1.0 / math.sqrt(d))
    x = torch.where(seen, x, float("-inf"))
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == float("-inf"), 0.0, top))
    total = x.sum(-1, keepdim=True)
    o = (x.view(nb, hkv, g * t, -1) @ v).view(nb, hkv, g, t, d) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(nb, t, c["heads"], d)
    b, _, _, _ = _rows(s)
    return o[b, torch.arange(s["rows"], device="cuda") - start[b]].to(s["q"].dtype)


def _statistics(logits, scale):
    """log sum exp and entropy of scale * logits, and those scaled logits."""
    x = logits.float() * scale
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1)
    entropy = torch.log(total) - torch.where(p > 0, p * (x - top), 0.0).sum(-1) / total
    return top[:, 0] + torch.log(total), entropy, x


def _plain_score(s):
    lse, entropy, x = _statistics(s["logits"], s["case"]["scale"])
    t = s["targets"].long()
    logp = torch.where(t >= 0, x.gather(1, t.clamp(min=0)) - lse[:, None], 0.0)
    out = {"logp": logp, "entropy": entropy, "lse": lse}
    if s["case"]["top"]:
        at = torch.sort(s["logits"], dim=1, descending=True, stable=True).indices[:, : s["case"]["top"]]
        out["top_ids"], out["top_logp"] = at.to(torch.int32), x.gather(1, at) - lse[:, None]
    return out


def _plain_grad(s):
    scale = s["case"]["scale"]
    logp = s["logits"].float() * scale - s["lse"][:, None]
    p = torch.exp(logp)
    t = s["targets"].long()
    g = torch.where(t >= 0, s["d_logp"], 0.0)
    d = -p * g.sum(1, keepdim=True) - s["d_entropy"][:, None] * torch.where(p > 0, p * (logp + s["entropy"][:, None]), 0.0)
    d.scatter_add_(1, t.clamp(min=0), g)
    return (d * scale).to(s["logits"].dtype)


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend, "score": _plain_score, "grad": _plain_grad}[op](state)
    lib, c = state["lib"], state["case"]
    if op == "write":
        lib.szo_kv8_write(state["cache"], state["batch"], state["k"], state["v"])
        return _cache_values(state)
    if op == "read":
        return list(lib.szo_kv8_read(state["cache"], state["batch"], DTYPES[c["dtype"]]))
    if op == "attend":
        return lib.szo_attention_kv8(state["cache"], state["batch"], state["q"])
    if op == "score":
        r = lib.szo_token_logprobs(state["logits"], state["targets"], n_top=c["top"], scale=c["scale"])
        out = {"logp": r.logp, "entropy": r.entropy, "lse": r.lse}
        if c["top"]:
            out["top_ids"], out["top_logp"] = r.top_ids, r.top_logp
        return out
    return lib.szo_token_logprobs_bwd(state["logits"], state["targets"], state["lse"], state["entropy"], state["d_logp"],
                                      state["d_entropy"], scale=c["scale"])


# ------------------------------------------------------------------------------ the definitions in 64 bits
def _e4m3_numbers(codes):
    """The numbers that e4m3 codes stand for, from sign, exponent and fraction."""
    c = codes.to(torch.int32)
    frac, ex = (c & 7).double(), (c >> 3) & 15
    mag = torch.where(ex == 0, frac / 512, (1 + frac / 8) * torch.exp2((ex - 7).double()))
    mag = torch.where((c & 127) == 127, float("nan"), mag)
    return torch.where((c & 128) != 0, -mag, mag)


def _nearest_e4m3(y):
    """The e4m3 number nearest to y (ties to the even fraction); |y| <= 448."""
    ex = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -60))).clamp(min=-6)
    step = torch.exp2(ex - 3)
    return torch.round(y / step) * step


def _exact_write(s):
    p = s["case"]["page"]
    lens, news = _lens(s["case"])
    codes = s["codes"]
    keys, scales = [], s["scales"].double()
    out = [codes[0].view(torch.float8_e4m3fn), codes[1].view(torch.float8_e4m3fn)]
    table, start = s["table"].tolist(), 0
    todo = {}                                            # pages by (new tokens, first slot): alike ones together
    for b, (end, n) in enumerate(zip(lens, news)):
        for j in range((end - n) // p, -(-end // p)):
            lo, hi = max(end - n, j * p), min(end, (j + 1) * p)
            todo.setdefault((lo - j * p, hi - lo), []).append((table[b][j], start + lo - (end - n)))
        start += n
    for (slot, m), group in todo.items():
        page = torch.tensor([g[0] for g in group], device="cuda")
        row = torch.tensor([g[1] for g in group], device="cuda")[:, None] + torch.arange(m, device="cuda")
        for w, x in enumerate((s["k"], s["v"])):
            x = x[row].double().transpose(1, 2)
            amax = x.abs().amax((2, 3))
            e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -200) / 448)) - 1           # one too low, or off by log2's rounding
            for _ in range(2):
                e = torch.where(amax > 448 * torch.exp2(e), e + 1, e)
            e = e.clamp(E_MIN, E_MAX)
            old = torch.round(torch.log2(scales[page, :, w]))
            if slot:
                e = torch.maximum(e, old)
                back = _e4m3_numbers(codes[w, page][:, :, :slot]) * torch.exp2(old - e)[:, :, None, None]
                part = out[w][page]
                part[:, :, :slot] = _nearest_e4m3(back).float().to(torch.float8_e4m3fn)
                out[w][page] = part
            part = out[w].view(torch.uint8)[page]
            part[:, :, slot:slot + m] = _nearest_e4m3(x * torch.exp2(-e)[:, :, None, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
            out[w].view(torch.uint8)[page] = part
            scales[page, :, w] = torch.exp2(e)
    return {"keys": out[0], "values": out[1], "scales": scales}


def _exact_read(s):
    p, outs = s["case"]["page"], []
    for w in (0, 1):
        parts = []
        for b, n in enumerate(_lens(s["case"])[0]):
            pages = s["table"][b, : -(-n // p)].long()
            x = _e4m3_numbers(s["codes"][w][pages]) * s["scales"][pages][:, :, w, None, None].double()
            parts.append(x.transpose(1, 2).reshape(-1, x.shape[1], x.shape[3])[:n])
        outs.append(torch.cat(parts))
    return outs


def _exact_attend(s):
    c, p, d = s["case"], s["case"]["page"], s["case"]["head_dim"]
    g = c["heads"] // c["kv_heads"]
    lens, news = _lens(c)
    out, start = torch.zeros(s["rows"], c["heads"], d, dtype=torch.float64, device="cuda"), 0
    for b, (end, n) in enumerate(zip(lens, news)):
        pages = s["table"][b, : -(-end // p)].long()
        later = torch.arange(end, device="cuda")[None, :] > torch.arange(end - n, end, device="cuda")[:, None]
        for h in range(c["kv_heads"]):
            k, v = (((_e4m3_numbers(s["codes"][w][pages, h]) * s["scales"][pages, h, w].double()[:, None, None]).reshape(-1, d)[:end]) for w in (0, 1))
            for i in range(h * g, (h + 1) * g):
                x = s["q"][start:start + n, i].double() @ k.T / math.sqrt(d)
                x.masked_fill_(later, float("-inf"))
                out[start:start + n, i] = torch.softmax(x, -1) @ v
        start += n
    return out


def _exact_score(s):
    c, outs = s["case"], []
    for part, t in zip(s["logits"].split(256), s["targets"].long().split(256)):
        x = part.double() * c["scale"]
        logp = torch.log_softmax(x, -1)
        p = logp.exp()
        o = {"logp": torch.where(t >= 0, logp.gather(1, t.clamp(min=0)), 0.0), "entropy": -(p * logp.clamp(min=-1e300)).sum(-1),
             "lse": torch.logsumexp(x, -1)}
        if c["top"]:
            at = torch.argsort(part.double(), dim=1, descending=True, stable=True)[:, : c["top"]]
            o["top_ids"], o["top_logp"] = at.to(torch.int32), logp.gather(1, at)
        outs.append(o)
    return {k: torch.cat([o[k] for o in outs]) for k in outs[0]}


def _exact_grad(s):
    """By differentiating the sum of d_logp * logp + d_entropy * entropy."""
    c, outs = s["case"], []
    for lo in range(0, c["rows"], 256):
        part = slice(lo, lo + 256)
        x = s["logits"][part].double().clamp(min=-1e6).requires_grad_(True)
        logp = torch.log_softmax(x * c["scale"], -1)
        t = s["targets"][part].long()
        total = (torch.where(t >= 0, s["d_logp"][part].double(), 0.0) * logp.gather(1, t.clamp(min=0))).sum()
        total = total - (s["d_entropy"][part].double()[:, None] * logp.exp() * logp).sum()
        total.backward()
        outs.append(x.grad)
    return torch.cat(outs)


def exact(case, seed):
    s = prepare(case, seed)
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend, "score": _exact_score, "grad": _exact_grad}[case["op"]](s)
