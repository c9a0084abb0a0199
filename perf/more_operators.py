"""The operators of training and scoring on many answers to one prompt.

An operator's pass in its plain form (elementary torch operations in 32 bits) and through the library's
entry points, on the same inputs:

  ce        next-token cross entropy of hidden states through a vocabulary matrix, without keeping the logits
  grad      its gradient with respect to the hidden states, and to the vocabulary matrix where that is trained
  attend    attention of the newest tokens of sequences that continue shared prompts over the 8-bit paged
            cache, the shared positions taken once for all sequences of a prompt

Cache: codes uint8 [2 (keys, values), pages, heads, page_tokens, head_dim], scales fp32 [pages, heads, 2].
A batch: page_table int32 [batch, max_pages]; kv_len int32 [batch], the positions of each sequence with its
new tokens; start int32 [batch + 1], the rows of each sequence in the row buffers.  Groups: seqs int32 [groups +
1], the sequences of each group; prefix int32 [groups], the positions that they share from position 0 on.
"""
import math

import torch

own = False

E_MIN, E_MAX = -63, 63                       # exponents of the cache's scales
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------------------ the cases
def _head_case(name, op, dtype, rows, vocab, d, scale=1.0, zloss=False, weights=False):
    c = dict(op=op, dtype=dtype, rows=rows, vocab=vocab, d=d, scale=scale, zloss=zloss, weights=weights)
    return dict(c, name=name) if name else c


def _shared_case(name, dtype, groups, seqs, prefix, own_len, own_min, new, new_min, heads, kv_heads, head_dim, page):
    c = dict(op="attend", dtype=dtype, groups=groups, seqs=seqs, prefix=prefix, own=own_len, own_min=own_min, new=new,
             new_min=new_min, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the last positions of a batch of 8 sequences are scored: the 7B vocabulary matrix is read for a few rows
        _head_case("ce_last_8x32000", "ce", "bf16", 8, 32000, 4096),
        # the small decoder's batch of 4 x 64 tokens: latency
        _head_case("ce_small_256x1024", "ce", "f16", 256, 1024, 256, scale=1.25),
        # the loss of a training batch of 16 x 256 tokens, 7B width
        _head_case("ce_batch_4096x32000", "ce", "bf16", 4096, 32000, 4096),
        # a ragged batch, 13B width, a vocabulary of odd size
        _head_case("ce_ragged_1021x50271", "ce", "f16", 1021, 50271, 5120, scale=0.8),
        # a few rows' gradient down to the hidden states, frozen vocabulary matrix
        _head_case("grad_last_16x32000", "grad", "bf16", 16, 32000, 4096),
        # everything odd, matrix trained, for checking
        _head_case("grad_small_odd", "grad", "f16", 77, 1111, 264, scale=1.5, zloss=True, weights=True),
        # a training batch of 16 x 256 tokens with a frozen matrix: the gradient that the layers below take
        _head_case("grad_batch_4096x32000", "grad", "bf16", 4096, 32000, 4096),
        # a batch of 4 x 512 tokens, 13B width, both gradients, with a term on lse
        _head_case("grad_both_2048x50272", "grad", "bf16", 2048, 50272, 5120, zloss=True, weights=True),
        # a token step of 64 samples of one prompt, grouped-query 7B shape
        _shared_case("attend_token_64_of_8192", "bf16", 1, 64, 8192, 512, 1, 1, 1, 32, 8, 128, 64),
        # a token step of 8 answers to a very long prompt
        _shared_case("attend_token_8_of_65536", "f16", 1, 8, 65536, 200, 30, 1, 1, 32, 8, 128, 32),
        # drafts of a few tokens, fp32, two short prompts, odd group of heads: latency
        _shared_case("attend_drafts_f32", "f32", 2, 3, 400, 70, 9, 5, 2, 10, 2, 64, 16),
        # candidate answers to two prompts, scored whole
        _shared_case("attend_answers_2x16_of_4096", "bf16", 2, 16, 4096, 128, 64, 128, 64, 32, 8, 128, 64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    while True:
        op = rng.choice(("ce", "grad", "attend", "attend"))
        if op != "attend":
            case = _head_case(None, op, rng.choice(("bf16", "f16")), _log_int(rng, 1, 8192), _log_int(rng, 500, 160000),
                              8 * _log_int(rng, 8, 1024), round(rng.uniform(0.5, 1.5), 3), op == "grad" and rng.random() < 0.5,
                              op == "grad" and rng.random() < 0.5)
            if case["rows"] * case["vocab"] <= 2.2e8 and work(case)["flops"] <= 3.1e12 and case["vocab"] * case["d"] <= 5e8:
                return case
            continue
        kv_heads, group = rng.choice((1, 2, 4, 8, 16, 32)), rng.choice((1, 2, 3, 4, 5, 7, 8))
        new = rng.choice((1, 1, 1, rng.randint(2, 8), _log_int(rng, 1, 512)))
        own_len = new + rng.choice((0, _log_int(rng, 1, 2048)))
        case = _shared_case(None, rng.choice(("bf16", "f16", "f32")), rng.choice((1, 1, 1, 2, 3, 5)), _log_int(rng, 1, 128),
                            _log_int(rng, 16, 65536), own_len, rng.randint(new, own_len), new, rng.randint(1, new), kv_heads * group, kv_heads,
                            rng.choice((64, 128)), rng.choice((16, 32, 64)))
        prefixes, groups, _, news = _shape(case)
        scores = sum(n * p for n, p in zip([sum(news[a:b]) for a, b in groups], prefixes)) * case["heads"]
        if scores > 6e8 or len(news) * own_len * kv_heads * case["head_dim"] > 1.4e8 or sum(prefixes) * kv_heads * case["head_dim"] > 1.4e8:
            continue
        if case["dtype"] == "f32" and work(case)["flops"] > 4e10:
            continue
        return case


def _spread(top, low, n):
    return [top - (top - low) * b // max(n - 1, 1) for b in range(n)]


def _shape(case):
    """Shared positions and (first, last + 1) sequence of every group; own positions and new rows of every sequence."""
    sizes = _spread(case["seqs"], max(1, case["seqs"] * 2 // 3), case["groups"])
    prefixes = _spread(case["prefix"], max(1, case["prefix"] * 3 // 4), case["groups"])
    ends = [sum(sizes[:g + 1]) for g in range(len(sizes))]
    owns, news = _spread(case["own"], case["own_min"], ends[-1]), _spread(case["new"], case["new_min"], ends[-1])
    return prefixes, [(e - n, e) for e, n in zip(ends, sizes)], [max(a, n) for a, n in zip(owns, news)], news


def work(case):
    e = SIZES[case["dtype"]]
    if case["op"] != "attend":
        m, v, d = case["rows"], case["vocab"], case["d"]
        if case["op"] == "ce":
            return {"bytes": (m + v) * d * e + m * 12, "flops": 2 * m * v * d}
        outs = m * d + (v * d if case["weights"] else 0)
        return {"bytes": ((m + v) * d + outs) * e + m * (16 if case["zloss"] else 12), "flops": (6 if case["weights"] else 4) * m * v * d}
    prefixes, groups, owns, news = _shape(case)
    d, hkv, h, p = case["head_dim"], case["kv_heads"], case["heads"], case["page"]
    cached = sum(prefixes) + sum(owns)
    pairs = sum(n * (prefixes[g] + a) - n * (n - 1) // 2 for g, (lo, hi) in enumerate(groups) for a, n in zip(owns[lo:hi], news[lo:hi]))
    return {"bytes": 2 * sum(news) * h * d * e + 2 * cached * hkv * d + (cached // p) * (8 * hkv + 4) + 8 * len(owns), "flops": 4 * pairs * h * d}


# ------------------------------------------------------------------------------ the inputs
def _pow2(e):
    """2^e of whole numbers in [-126, 127], exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(amax):
    """The smallest e in [E_MIN, E_MAX] with amax <= 448 * 2^e."""
    m, k = torch.frexp(amax)
    return (k - 9 + (m > 0.875).to(k.dtype)).clamp(E_MIN, E_MAX)


def _kv_values(shape, gen):
    """Keys or values as layers make them: heads apart in size, a few loud channels, some loud tokens; shape [..., heads, head_dim]."""
    x = torch.randn(shape, device="cuda", generator=gen)
    head = torch.exp(0.5 * torch.randn(shape[-2], 1, device="cuda", generator=gen))
    loud = 1 + 6 * (torch.rand(shape[-1], device="cuda", generator=gen) < 0.03).float()
    token = torch.exp(0.7 * torch.randn(*shape[:-2], 1, 1, device="cuda", generator=gen).clamp(-2, 2))
    return x.mul_(head).mul_(loud).mul_(token)


def _prepare_head(case, gen):
    m, v, d, dtype = case["rows"], case["vocab"], case["d"], DTYPES[case["dtype"]]
    W = torch.randn(v, d, device="cuda", generator=gen).mul_(2.5 / math.sqrt(d)).to(dtype)
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen, dtype=torch.int32)
    # hidden states that know something of their target, from nothing to nearly everything
    known = torch.rand(m, 1, device="cuda", generator=gen) * 2.2
    h = torch.randn(m, d, device="cuda", generator=gen).add_(known * W[targets.long()].float()).to(dtype)
    # the prompt's positions have no target, nor have those behind the last token
    targets[torch.rand(m, device="cuda", generator=gen) < 0.15] = -1
    s = {"case": case, "h": h, "W": W, "targets": targets}
    if case["op"] == "grad":
        # the mean over the positions with a target, some sequences weighted; 16-bit floats take the usual loss scale
        weight = torch.where(torch.rand(m, device="cuda", generator=gen) < 0.2, 0.5, 1.0)
        scale = 4096.0 if case["dtype"] == "f16" else 1.0
        s["d_loss"] = weight * (scale / max(m, 1))
        s["lse"], _ = _statistics(s)
        if case["zloss"]:
            s["d_lse"] = s["lse"] * (2e-3 * scale / max(m, 1))
    return s


def _prepare_shared(case, gen):
    prefixes, groups, owns, news = _shape(case)
    b, p, hkv, d = len(owns), case["page"], case["kv_heads"], case["head_dim"]
    common = [n // p for n in prefixes]                                     # whole pages are shared, what is left of a prefix is each one's own
    lens = [prefixes[g] + owns[i] for g, (lo, hi) in enumerate(groups) for i in range(lo, hi)]
    of = [g for g, (lo, hi) in enumerate(groups) for _ in range(lo, hi)]
    counts = [-(-n // p) for n in lens]
    n_pages, max_pages = sum(common) + sum(c - common[g] for c, g in zip(counts, of)) + 3, max(counts) + 1
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(gen.initial_seed())).tolist()
    rows, at = [], sum(common)
    for i, g in enumerate(of):
        first = sum(common[:g])
        mine = counts[i] - common[g]
        rows.append(order[first:first + common[g]] + order[at:at + mine] + [-1] * (max_pages - counts[i]))
        at += mine
    codes = torch.empty(2, n_pages, hkv, p, d, dtype=torch.uint8, device="cuda")
    scales = torch.empty(n_pages, hkv, 2, device="cuda")
    for which in (0, 1):
        x = _kv_values((n_pages, p, hkv, d), gen).transpose(1, 2)
        e = _exponent(x.abs().amax((2, 3)))
        codes[which] = (x * _pow2(-e)[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scales[:, :, which] = _pow2(e)
        del x
    ints = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    return {"case": case, "codes": codes, "scales": scales, "table": ints(rows), "kv_len": ints(lens),
            "start": ints([sum(news[:i]) for i in range(b + 1)]), "rows": sum(news), "max_new": max(news),
            "prefix": ints(prefixes), "seqs": ints([0] + [hi for _, hi in groups]), "max_seqs": max(hi - lo for lo, hi in groups),
            "q": torch.randn(sum(news), case["heads"], d, device="cuda", generator=gen).to(DTYPES[case["dtype"]])}


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(int(seed))
    s = (_prepare_shared if case["op"] == "attend" else _prepare_head)(case, gen)
    if own:
        from paper_2406_02913_b200 import binding
        s["lib"] = binding
        if case["op"] == "attend":
            s["cache"] = binding.Kv8Cache(s["codes"], s["scales"])
            s["batch"] = binding.Kv8Batch(s["table"], s["kv_len"], rows=s["rows"], start=s["start"], max_new=s["max_new"])
            s["shared"] = binding.Kv8Prefix(s["prefix"], seqs=s["seqs"], max_seqs=s["max_seqs"])
    return s


# ------------------------------------------------------------------------------ the plain forms
def _statistics(s):
    """log sum exp of every row's scaled logits, and those logits."""
    x = (s["h"].float() @ s["W"].float().T) * s["case"]["scale"]
    top = x.amax(-1, keepdim=True)
    return top[:, 0] + torch.log(torch.exp(x - top).sum(-1)), x


def _plain_ce(s):
    lse, x = _statistics(s)
    t = s["targets"].long()
    return {"loss": torch.where(t >= 0, lse - x.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0), "lse": lse}


def _plain_grad(s):
    _, x = _statistics(s)
    t = s["targets"].long()
    a = torch.where(t >= 0, s["d_loss"], 0.0)
    g = torch.exp(x - s["lse"][:, None]) * (a + s["d_lse"] if "d_lse" in s else a)[:, None]
    g.scatter_add_(1, t.clamp(min=0)[:, None], -a[:, None])
    g *= s["case"]["scale"]
    out = {"dh": (g @ s["W"].float()).to(s["h"].dtype)}
    if s["case"]["weights"]:
        out["dW"] = (g.T @ s["h"].float()).to(s["h"].dtype)
    return out


def _cached(s, pages):
    """Keys and values of pages [..., n] as fp32 [..., heads, n * page_tokens, head_dim]."""
    outs = []
    for w in (0, 1):
        x = s["codes"][w][pages].view(torch.float8_e4m3fn).float() * s["scales"][pages][..., w, None, None]
        outs.append(x.transpose(-4, -3).flatten(-3, -2))
    return outs


def _plain_attend(s):
    c, d, hkv, p, t = s["case"], s["case"]["head_dim"], s["case"]["kv_heads"], s["case"]["page"], s["max_new"]
    r = c["heads"] // hkv
    prefixes, groups, _, _ = _shape(c)
    start, end = s["start"].long(), s["kv_len"].long()
    n = start[1:] - start[:-1]
    i = torch.arange(t, device="cuda")
    out = torch.empty_like(s["q"])
    for (lo, hi), prefix in zip(groups, prefixes):
        nb, pre = hi - lo, prefix // p
        at = start[lo:hi, None] + i                                                      # rows of each sequence
        there = i < n[lo:hi, None]
        q = s["q"][at.clamp(max=s["rows"] - 1)].float().view(nb, t, hkv, r, d).permute(2, 0, 3, 1, 4).reshape(hkv, nb, r * t, d)
        k0, v0 = _cached(s, s["table"][lo, :pre].long())                                 # [hkv, shared, d]
        last = -(-(prefix + c["own"]) // p)
        k1, v1 = (x.transpose(0, 1) for x in _cached(s, s["table"][lo:hi, pre:last].long().clamp(min=0)))      # [hkv, nb, own, d]
        place = pre * p + torch.arange(k1.shape[2], device="cuda")
        seen = place <= (end - n)[lo:hi, None, None] + i[:, None]                        # [nb, t, own]
        x0 = (q.reshape(hkv, -1, d) @ k0.transpose(1, 2)).view(hkv, nb, r, t, -1) * (1.0 / math.sqrt(d))
        x1 = (q @ k1.transpose(2, 3)).view(hkv, nb, r, t, -1) * (1.0 / math.sqrt(d))
        x1 = torch.where(seen[None, :, None], x1, float("-inf"))
        top = x1.amax(-1, keepdim=True)
        if pre:
            top = torch.maximum(top, x0.amax(-1, keepdim=True))
        x0, x1 = torch.exp(x0 - top), torch.exp(x1 - top)
        total = x0.sum(-1, keepdim=True) + x1.sum(-1, keepdim=True)
        o = (x0.view(hkv, -1, pre * p) @ v0).view(hkv, nb, r, t, d) + (x1.view(hkv, nb, r * t, -1) @ v1).view(hkv, nb, r, t, d)
        o = (o / total).permute(1, 3, 0, 2, 4).reshape(nb, t, c["heads"], d)
        out[at[there]] = o[there].to(out.dtype)
    return out


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"ce": _plain_ce, "grad": _plain_grad, "attend": _plain_attend}[op](state)
    lib, c = state["lib"], state["case"]
    if op == "ce":
        r = lib.szo_head_ce(state["h"], state["W"], state["targets"], scale=c["scale"])
        return {"loss": r.loss, "lse": r.lse}
    if op == "grad":
        dh, dW = lib.szo_head_ce_bwd(state["h"], state["W"], state["targets"], state["lse"], state["d_loss"], state.get("d_lse"),
                                     scale=c["scale"], need_dW=c["weights"])
        return {"dh": dh, "dW": dW} if c["weights"] else {"dh": dh}
    return lib.szo_attention_kv8_prefix(state["cache"], state["batch"], state["shared"], state["q"])


# ------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_ce(s):
    loss, lse, W = [], [], s["W"].double()
    for h, t in zip(s["h"].split(512), s["targets"].long().split(512)):
        logp = torch.log_softmax(h.double() @ W.T * s["case"]["scale"], -1)
        loss.append(torch.where(t >= 0, -logp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0))
        lse.append(h.double() @ W[0] * s["case"]["scale"] - logp[:, 0])
    return {"loss": torch.cat(loss), "lse": torch.cat(lse)}


def _exact_grad(s):
    """The gradient of sum d_loss loss + d_lse lse, lse being what it is given as in the formula of p."""
    c, W = s["case"], s["W"].double()
    dh, dW = [], torch.zeros(W.shape if c["weights"] else (0,), dtype=torch.float64, device="cuda")
    for lo in range(0, c["rows"], 512):
        part = slice(lo, lo + 512)
        h, t, d_loss = s["h"][part].double(), s["targets"][part].long(), s["d_loss"][part].double()
        hit = torch.nn.functional.one_hot(t.clamp(min=0), W.shape[0]).mul_((t >= 0)[:, None])
        p = torch.exp(h @ W.T * c["scale"] - s["lse"][part].double()[:, None])
        g = (p - hit) * torch.where(t >= 0, d_loss, 0.0)[:, None]
        if c["zloss"]:
            g += p * s["d_lse"][part].double()[:, None]
        g *= c["scale"]
        dh.append(g @ W)
        if c["weights"]:
            dW += g.T @ h
    return {"dh": torch.cat(dh), "dW": dW} if c["weights"] else {"dh": torch.cat(dh)}


def _e4m3_numbers(codes):
    """The numbers that e4m3 codes stand for, from sign, exponent and fraction."""
    c = codes.to(torch.int32)
    frac, ex = (c & 7).double(), (c >> 3) & 15
    mag = torch.where(ex == 0, frac / 512, (1 + frac / 8) * torch.exp2((ex - 7).double()))
    mag = torch.where((c & 127) == 127, float("nan"), mag)
    return torch.where((c & 128) != 0, -mag, mag)


def _exact_attend(s):
    c, d = s["case"], s["case"]["head_dim"]
    g = c["heads"] // c["kv_heads"]
    prefixes, groups, owns, news = _shape(c)
    lens = [prefixes[k] + owns[i] for k, (lo, hi) in enumerate(groups) for i in range(lo, hi)]
    if len(lens) * c["kv_heads"] * max(lens) > 6e7:
        return None
    out, start = torch.zeros(s["rows"], c["heads"], d, dtype=torch.float64, device="cuda"), 0
    for b, (end, n) in enumerate(zip(lens, news)):
        pages = s["table"][b, : -(-end // c["page"])].long()
        later = torch.arange(end, device="cuda")[None, :] > torch.arange(end - n, end, device="cuda")[:, None]
        k, v = ((_e4m3_numbers(s["codes"][w][pages]) * s["scales"][pages, :, w].double()[:, :, None, None]).transpose(0, 1).flatten(1, 2)[:, :end]
                for w in (0, 1))
        for h in range(c["kv_heads"]):
            x = s["q"][start:start + n, h * g:(h + 1) * g].double().transpose(0, 1) @ k[h].T / math.sqrt(d)
            out[start:start + n, h * g:(h + 1) * g] = (torch.softmax(x.masked_fill_(later, float("-inf")), -1) @ v[h]).transpose(0, 1)
        start += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"ce": _exact_ce, "grad": _exact_grad, "attend": _exact_attend}[case["op"]](s)
