"""The operators around a KV cache held in 8 bits, as cases that can be timed: rows of K and V written to it and read back, ragged
attention over it, and the log probabilities of the tokens that a rollout from it emitted.

The cache: pages of 64 tokens, e4m3 codes, and for K and V a scale 2^e per page and KV head, so that a value is code * 2^e.  e is the
least one in -15 .. 7 with which every row written fits (448 * 2^e); a page that had rows before the write keeps its scale if that is
larger, and has its rows rounded again if it is smaller.

`own` False computes the operators in elementary torch operations in 32 bits; True calls the framework."""
import math
import random
from statistics import NormalDist

import torch

own = False

DEVICE = "cuda:0"
PAGE = 64
E_MIN, E_MAX = -15, 7
HEADS = {  # query heads, KV heads, head size
    "tiny": (4, 4, 64), "mini_bf16": (6, 2, 128), "s1p5b": (12, 2, 128), "s7b": (28, 4, 128), "mqa": (8, 1, 64), "mha": (8, 8, 128)}
MAX_CONTEXT = 32768


def _swap(name, heads, batch, rows, context, ragged=False):
    return dict(name=name, path="cache", heads=heads, batch=batch, rows=rows, context=context, ragged=ragged)


def _attend(name, heads, batch, rows, context, ragged=False, spread=0.0):
    return dict(name=name, path="attention", heads=heads, batch=batch, rows=rows, context=context, ragged=ragged, spread=spread)


def _score(name, batch, k, vocab, dtype, top, temperature=1.0, ragged=False, masked=0.0):
    return dict(name=name, path="logprobs", batch=batch, k=k, vocab=vocab, dtype=dtype, top=top, temperature=temperature, ragged=ragged, masked=masked)


def listed():
    return [
        # one row for each of 64 sequences, as plain decoding appends it: pages are partly filled, some scales grow
        _swap("cache_s7b_b64_n1", "s7b", 64, 1, 4096),
        # the rows of a verify step, ragged
        _swap("cache_s7b_b128_n1to17", "s7b", 128, 17, 2000, ragged=True),
        # prompts imported whole, or sequences swapped back in
        _swap("cache_s7b_b16_n4001", "s7b", 16, 4001, 37, ragged=True),
        # a handful of short sequences with small heads: a test or a first integration; latency
        _attend("attention_tiny_b4_q5_c128", "tiny", 4, 5, 128),
        # the one long rollout that a batch waits for
        _attend("attention_s1p5b_b1_q1_c30000", "s1p5b", 1, 1, 30000),
        # plain decoding of a mid-sized batch
        _attend("attention_s7b_b64_q1_c4096", "s7b", 64, 1, 4096),
        # a uniform verify batch
        _attend("attention_s7b_b32_q9_c8192", "s7b", 32, 9, 8192),
        # the long-tail verify batch: contexts and draft lengths differ by sequence
        _attend("attention_s7b_longtail_b128_q1to17", "s7b", 128, 17, 4096, ragged=True, spread=1.0),
        # a piece of a prompt behind what is cached of it already
        _attend("attention_s1p5b_b4_q509_c1000", "s1p5b", 4, 509, 1000, ragged=True, spread=0.7),
        # one token each of a few short sequences over a small vocabulary; latency
        _score("logprobs_b4_v4096", 4, 0, 4096, "f32", 5),
        # one verified block, logits of a program with its own model in bf16
        _score("logprobs_b1_k8_v151936_bf16", 1, 8, 151936, "bf16", 20, temperature=0.7),
        # all rows of the long-tail verify batch; part of the vocabulary masked
        _score("logprobs_b128_k0to16_v152064", 128, 16, 152064, "f32", 20, temperature=0.8, ragged=True, masked=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    path = rng.choice(["cache", "cache", "attention", "attention", "attention", "attention", "logprobs", "logprobs", "logprobs"])
    if path == "logprobs":
        vocab, k = _log_int(rng, 1000, 152064), rng.choice([0, 0, 4, 8, rng.randint(1, 16)])
        c = _score("", _log_int(rng, 1, min(512, max(1, 1100 * 152064 // vocab // (k + 1)))), k, vocab, rng.choice(["f32", "bf16"]), rng.randint(0, 20),
                   temperature=round(rng.uniform(0.5, 1.3), 2), ragged=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.1, 0.6]))
    elif path == "cache":
        rows = _log_int(rng, 1, 6000)
        heads = rng.choice(list(HEADS))
        most = (1 << 24) // ((rows + 32) * HEADS[heads][1] * HEADS[heads][2])
        c = _swap("", heads, _log_int(rng, 1, max(1, min(256, most))), rows, _log_int(rng, 1, 8000), ragged=rng.random() < 0.5)
    else:
        heads = rng.choice(list(HEADS) + ["s1p5b", "s7b"])
        rows = rng.choice([1, 1, rng.randint(2, 17), rng.randint(2, 17), _log_int(rng, 18, 700)])
        spread = rng.choice([0.0, 0.0, 0.3, 1.0])
        batch = _log_int(rng, 1, 256 if rows < 18 else 6)
        most = (400000 if rows < 18 else 10000) / batch / math.exp(spread ** 2 / 2) * 4 / max(4, HEADS[heads][1])
        c = _attend("", heads, batch, rows, _log_int(rng, 1, min(MAX_CONTEXT // (4 if spread else 1), max(2, int(most)))), ragged=rng.random() < 0.5, spread=spread)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ sizes
def _spread_out(n, median, sigma, hi):
    """n lengths of a lognormal law (its quantiles, in an order of their own), all `median` at sigma 0."""
    nd = NormalDist(math.log(max(median, 1)), sigma) if sigma > 0 else None
    v = [min(hi, int(math.exp(nd.inv_cdf((i + 0.5) / n)))) if nd else median for i in range(n)]
    random.Random(n * 7919 + median).shuffle(v)
    return v


def _counts(n, most, ragged):
    """Rows of n sequences: `most`, or 1 .. most spread evenly, in an order of their own."""
    v = [1 + (most - 1) * i // max(1, n - 1) if ragged and n > 1 else most for i in range(n)]
    random.Random(n * 104729 + most).shuffle(v)
    return v


def _lengths(case):
    """(rows, committed tokens) of every sequence."""
    rows = _counts(case["batch"], case["rows"], case["ragged"])
    if case["path"] == "cache":
        r = random.Random(case["context"] * 31 + case["batch"])
        return rows, [r.randint(0, 2 * case["context"]) for _ in rows]     # anywhere in a page
    return rows, _spread_out(case["batch"], case["context"], case["spread"], MAX_CONTEXT)


def work(case):
    if case["path"] == "logprobs":
        rows = sum(_counts(case["batch"], case["k"] + 1, case["ragged"]))
        return {"bytes": rows * (case["vocab"] * (4 if case["dtype"] == "f32" else 2) + 12 + 8 * case["top"]), "flops": 4.0 * rows * case["vocab"]}
    Hq, Hkv, D = HEADS[case["heads"]]
    rows, ctx = _lengths(case)
    if case["path"] == "cache":
        back = sum(n + c % PAGE for n, c in zip(rows, ctx))
        blocks = sum((n + c % PAGE + PAGE - 1) // PAGE for n, c in zip(rows, ctx)) * Hkv
        return {"bytes": (sum(rows) + back) * Hkv * D * 2 * 3 + blocks * 16, "flops": 2.0 * (sum(rows) + back) * Hkv * D * 2}
    cached = sum(n + c for n, c in zip(rows, ctx))
    seen = sum(n * c + n * (n + 1) // 2 for n, c in zip(rows, ctx))
    return {"bytes": cached * Hkv * D * 2 + (cached // PAGE + len(rows)) * (Hkv * 8 + 4) + 2 * sum(rows) * Hq * D * 2, "flops": 4.0 * seen * Hq * D}


# ------------------------------------------------------------------------------------------------ inputs
def _normal(shape, g, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEVICE).normal_(0.0, std, generator=g)


def _kv_rows(n, Hkv, D, g):
    """K with a few channels that are much larger than the others, as rotary decoders have them, and V."""
    k, v = _normal((n, Hkv, D), g), _normal((n, Hkv, D), g, 0.7)
    k[:, :, 5] *= 6.0
    k[:, :, D // 2 + 3] *= 9.0
    return k, v


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _plain_cache(n_pages, Hkv, D):
    return {x: {"codes": torch.zeros(n_pages, Hkv, PAGE, D, dtype=torch.uint8, device=DEVICE),
                "e": torch.full((n_pages, Hkv), E_MIN, dtype=torch.int32, device=DEVICE)} for x in "kv"}


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    if case["path"] == "logprobs":
        k, V, n = case["k"], case["vocab"], case["batch"]
        counts = _counts(n, k + 1, case["ragged"])
        logits = _normal((sum(counts), V), g, 2.5, torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        if case["masked"]:                       # tokens that a grammar or a filter rules out
            logits[:, torch.rand(V, generator=g, device=DEVICE) < case["masked"]] = -math.inf
        s = dict(path="logprobs", logits=logits, draft_len=_ints([c - 1 for c in counts]), n_tokens=_ints(counts), k=k, top=case["top"], temperature=case["temperature"],
                 tokens=torch.randint(0, V, (n, k + 1), generator=g, device=DEVICE).to(torch.int32))
        if own:
            from paper_2605_08862_amd.runtime import LogprobScorer
            s["scorer"] = LogprobScorer(n, k, V, case["top"])
        return s
    Hq, Hkv, D = HEADS[case["heads"]]
    rows, ctx = _lengths(case)
    n = len(rows)
    slots = torch.randperm(n, generator=g, device=DEVICE).to(torch.int32)
    order = slots.tolist()
    total = [0] * n
    for b in range(n):
        total[order[b]] = rows[b] + ctx[b]
    if own:
        from paper_2605_08862_amd.runtime import KvqCache
        cache = KvqCache(1, Hq, Hkv, D, n, max(total), q_max=max(rows), device=DEVICE, page_perm_seed=seed, slot_tokens=total)
    else:
        pages = [(t + PAGE - 1) // PAGE for t in total]
        ids = torch.randperm(sum(pages), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        table, at = torch.full((n, max(pages)), -1, dtype=torch.int32), 0
        for b, p in enumerate(pages):
            table[b, :p], at = ids[at:at + p], at + p
        cache = dict(_plain_cache(sum(pages), Hkv, D), table=table.to(DEVICE))
    s = dict(path=case["path"], cache=cache, slots=slots, ctx=_ints(ctx), rows=_ints(rows), most=max(rows), dims=(Hq, Hkv, D))
    # what is in the cache before the pass: the committed tokens, or, for attention, those and the rows' own
    held = ctx if case["path"] == "cache" else [r + c for r, c in zip(rows, ctx)]
    zeros = _ints([0] * n)
    if sum(held):
        k, v = _kv_rows(sum(held), Hkv, D, g)
        if own:
            cache.write(0, slots, zeros, _ints(held), max(held), k, v)
        else:
            _plain_write(cache, slots, zeros, _ints(held), k, v)
    if case["path"] == "attention":
        s["q"] = _normal((sum(rows), Hq, D), g, 0.6)
    else:
        s["k"], s["v"] = _kv_rows(sum(rows), Hkv, D, g)
        s["k"] *= 1.5                            # some pages need a larger scale than before
        back = [r + c % PAGE for r, c in zip(rows, ctx)]
        s |= dict(from_=_ints([c - c % PAGE for c in ctx]), back=_ints(back), most_back=max(back), n_back=sum(back))
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _places(cache, slots, pos0, n_rows, n):
    """(page, token in the page) of n packed rows."""
    ends = torch.cumsum(n_rows, 0)
    r = torch.arange(n, device=DEVICE)
    b = torch.searchsorted(ends, r, right=True)
    pos = pos0[b] + r - (ends - n_rows)[b]
    return cache["table"][slots[b], pos // PAGE].long(), pos % PAGE


def _exponent(a):
    """Least e in E_MIN .. E_MAX with a <= 448 * 2^e."""
    m, x = torch.frexp(a)                        # a = m * 2^x, m in [0.5, 1);  448 = 0.875 * 2^9
    return torch.where(a > 0, x - 9 + (m > 0.875), E_MIN).clamp(E_MIN, E_MAX).to(torch.int32)


def _codes(x):
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_write(cache, slots, pos0, n_rows, k_rows, v_rows):
    page, tok = _places(cache, slots, pos0, n_rows, k_rows.shape[0])
    first = cache["table"][slots, pos0 // PAGE].long()
    partial = pos0 % PAGE != 0                   # the first page had rows before
    older = torch.zeros(cache["k"]["e"].shape[0], dtype=torch.bool, device=DEVICE).scatter_(0, first, partial)
    for x, rows in (("k", k_rows), ("v", v_rows)):
        c, rows = cache[x], rows.float()
        need = _exponent(torch.zeros(c["e"].shape, device=DEVICE).index_reduce_(0, page, rows.abs().amax(-1), "amax"))
        e = c["e"].clone()
        e[page] = torch.where(older[:, None], torch.maximum(c["e"], need), need)[page]
        held = c["codes"][first]
        again = _codes(torch.ldexp(held.view(torch.float8_e4m3fn).float(), (c["e"] - e)[first][:, :, None, None]))
        c["codes"][first] = torch.where(partial[:, None, None, None], again, held)
        c["codes"][page, :, tok] = _codes(torch.ldexp(rows, -e[page][:, :, None]))
        c["e"] = e


def _plain_read(cache, slots, pos0, n_rows, n):
    page, tok = _places(cache, slots, pos0, n_rows, n)
    return [torch.ldexp(cache[x]["codes"][page, :, tok].view(torch.float8_e4m3fn).float(), cache[x]["e"][page][:, :, None]).to(torch.bfloat16) for x in "kv"]


def _plain_attention(s):
    Hq, Hkv, D = s["dims"]
    G, n, most, cache = Hq // Hkv, s["rows"].shape[0], s["most"], s["cache"]
    pages = cache["table"][s["slots"]].clamp(min=0).long()
    T = pages.shape[1] * PAGE

    def dense(x):                                # [n * Hkv, T, D]
        c = torch.ldexp(cache[x]["codes"][pages].view(torch.float8_e4m3fn).float(), cache[x]["e"][pages][..., None, None])
        return c.permute(0, 2, 1, 3, 4).reshape(n * Hkv, T, D)

    start = torch.cumsum(s["rows"], 0) - s["rows"]
    i = torch.arange(most, device=DEVICE)
    at = (start[:, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().view(n, most, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(n * Hkv, most * G, D)
    p = torch.bmm(q, dense("k").transpose(1, 2).contiguous()).view(n, Hkv, most, G, T)
    hidden = torch.arange(T, device=DEVICE) > (s["ctx"][:, None] + i)[..., None]
    p.mul_(1.0 / math.sqrt(D)).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    p.div_(p.sum(-1, keepdim=True))
    o = torch.bmm(p.view(n * Hkv, most * G, T), dense("v")).view(n, Hkv, most, G, D).permute(0, 2, 1, 3, 4).reshape(n, most, Hq, D)
    r = torch.arange(s["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(torch.cumsum(s["rows"], 0), r, right=True)
    return o[b, r - start[b]].to(torch.bfloat16)


def _plain_logprobs(s):
    z, V, top = s["logits"], s["logits"].shape[1], s["top"]
    n, most = s["tokens"].shape
    start = torch.cumsum(s["draft_len"] + 1, 0) - s["draft_len"] - 1
    i = torch.arange(most, device=DEVICE)
    live = i < s["n_tokens"][:, None]
    row = torch.where(live, start[:, None] + i, 0)
    m = z.amax(-1, keepdim=True)
    y = (z.float() - m.float()) / s["temperature"]
    e = y.exp()
    total = e.sum(-1)
    lse = total.log()
    entropy = lse - (e * torch.where(e > 0, y, 0.0)).sum(-1) / total
    out = {"logprob": torch.where(live, y[row, s["tokens"].long()] - lse[row], 0.0), "entropy": torch.where(live, entropy[row], 0.0)}
    if top:
        bits = z.float().view(torch.int32)
        key = (torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() << 32) + (V - 1 - torch.arange(V, device=DEVICE))   # larger: a larger logit, then a lower index
        best = V - 1 - (torch.topk(key, top, dim=-1).values & 0xffffffff)
        out["top_logprobs"] = torch.where(live[..., None], (torch.gather(y, 1, best) - lse[:, None])[row], 0.0)
        out["top_tokens"] = torch.where(live[..., None], best[row], -1).to(torch.int32)
    return out


def run(state):
    s = state
    if s["path"] == "logprobs":
        if not own:
            return _plain_logprobs(s)
        return s["scorer"](s["logits"], s["tokens"], s["n_tokens"], s["draft_len"], temperature=s["temperature"])
    if s["path"] == "attention":
        if not own:
            return _plain_attention(s)
        return s["cache"].attention(0, s["q"], s["slots"], s["ctx"], s["rows"], s["most"])
    if not own:
        _plain_write(s["cache"], s["slots"], s["ctx"], s["rows"], s["k"], s["v"])
        return _plain_read(s["cache"], s["slots"], s["from_"], s["back"], s["n_back"])
    s["cache"].write(0, s["slots"], s["ctx"], s["rows"], s["most"], s["k"], s["v"])
    return s["cache"].read(0, s["slots"], s["from_"], s["back"], s["most_back"], s["n_back"])


# ------------------------------------------------------------------------------------------------ 64 bits
def _round_e4m3(x):
    """Nearest of the values that e4m3 has (ties to even), in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _scale_for(a):
    e = torch.ceil(torch.log2((a / 448.0).clamp(min=2.0 ** -40)))
    return torch.exp2(e.clamp(E_MIN, E_MAX))


def _blocks(x):
    """[n, H, D] rows of one sequence from its first token on -> values held, page by page of 64."""
    n, H, D = x.shape
    full = torch.cat([x.double(), torch.zeros(-n % PAGE, H, D, dtype=torch.float64, device=x.device)]).view(-1, PAGE, H, D)
    scale = _scale_for(full.abs().amax((1, 3), keepdim=True))
    return (_round_e4m3(full / scale) * scale).view(-1, H, D)[:n], scale


def exact(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    if case["path"] == "logprobs":
        k, V, n = case["k"], case["vocab"], case["batch"]
        counts = _counts(n, k + 1, case["ragged"])
        z = _normal((sum(counts), V), g, 2.5, torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        if case["masked"]:
            z[:, torch.rand(V, generator=g, device=DEVICE) < case["masked"]] = -math.inf
        tokens = torch.randint(0, V, (n, k + 1), generator=g, device=DEVICE)
        out = {"logprob": torch.zeros(n, k + 1, dtype=torch.float64, device=DEVICE), "entropy": torch.zeros(n, k + 1, dtype=torch.float64, device=DEVICE)}
        if case["top"]:
            out["top_logprobs"] = torch.zeros(n, k + 1, case["top"], dtype=torch.float64, device=DEVICE)
        at = 0
        for b, c in enumerate(counts):
            lp = torch.log_softmax(z[at:at + c].double() / case["temperature"], -1)
            at += c
            out["logprob"][b, :c] = lp.gather(1, tokens[b, :c, None])[:, 0]
            out["entropy"][b, :c] = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(-1)
            if case["top"]:
                out["top_logprobs"][b, :c] = lp.topk(case["top"], -1).values
        return out
    Hq, Hkv, D = HEADS[case["heads"]]
    rows, ctx = _lengths(case)
    torch.randperm(len(rows), generator=g, device=DEVICE)
    held = ctx if case["path"] == "cache" else [r + c for r, c in zip(rows, ctx)]
    k, v = _kv_rows(sum(held), Hkv, D, g) if sum(held) else (None, None)
    at = new = 0
    if case["path"] == "attention":
        q, out = _normal((sum(rows), Hq, D), g, 0.6), []
        for r, h in zip(rows, held):
            kd, vd = (_blocks(x[at:at + h])[0].permute(1, 0, 2) for x in (k, v))
            qd = q[new:new + r].double().view(r, Hkv, Hq // Hkv, D).permute(1, 0, 2, 3).reshape(Hkv, -1, D)
            z = (torch.bmm(qd, kd.transpose(1, 2).contiguous()) / math.sqrt(D)).view(Hkv, r, -1, h)
            z.masked_fill_((torch.arange(h, device=DEVICE) > torch.arange(h - r, h, device=DEVICE)[:, None])[None, :, None], -math.inf)
            o = torch.bmm(torch.softmax(z, -1).view(Hkv, -1, h), vd.contiguous())
            out.append(o.view(Hkv, r, Hq // Hkv, D).permute(1, 0, 2, 3).reshape(r, Hq, D))
            at, new = at + h, new + r
        return torch.cat(out)
    kn, vn = _kv_rows(sum(rows), Hkv, D, g)
    kn *= 1.5
    got = [[], []]
    for r, h in zip(rows, held):
        for x, xn, o in ((k, kn, got[0]), (v, vn, got[1])):
            t = h % PAGE                         # rows that the first page had
            fresh = torch.cat([torch.zeros(t, Hkv, D, dtype=torch.float64, device=DEVICE), xn[new:new + r].double()])
            if t:
                was, scale = _blocks(x[at + h - t:at + h])
                first = torch.maximum(scale[0], _scale_for(fresh[:PAGE].abs().amax((0, 2), keepdim=True)))
                part = torch.cat([was, fresh[t:PAGE]])
                o.append(_round_e4m3(part / first) * first)
                fresh = fresh[PAGE:]
            if fresh.shape[0]:
                o.append(_blocks(fresh)[0])
        at, new = at + h, new + r
    return [torch.cat(o) for o in got]
