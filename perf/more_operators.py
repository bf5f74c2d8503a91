"""Operators to measure: a paged cache of keys and values and the attention that reads it.

Each case names its operator in "op":

  append  queries and keys rotated; keys and values written into the pages of a cache of 16 or 8 bits, with the
          mean key of every page that the call fills
  attend  attention over a sequence's own pages and over a prefix that the whole batch shares
  sparse  blocks chosen for every token by the mean keys of the pages, and attention over the chosen ones

A batch holds the tokens of its sequences one after the other (`start`, or one token each); `length` counts a
sequence's keys in its own pages (`table`), the call's tokens the last of them.  Pages are
[page][kv head][token][dimension].  8-bit pages are E4M3 codes with a power of two for every token and head,
kept as its exponent + 127.

With `own` false run() computes the plain form in elementary torch operations; with `own` true it calls the library.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
MOST_F16 = 61440.0  # the largest E4M3 value times a power of two that fp16 holds
THETA = 5e5
MAX_SEQ = 1 << 16


# ---------------------------------------------------------------- cases
# heads, kv_heads, head_dim: the 8B shape has 32, 8, 128, the 1B shape 32, 8, 64, the tiny one 4, 4, 64.
# seqs: sequences; new: (least, most) tokens of one in the call; keys: (least, most) keys of one before it;
# prefix: keys that all share; page: tokens of a page; cache: f16, bf16 (the tokens' type) or e4m3.
def _case(name, op, heads, kv_heads, head_dim, dtype, cache, page, seqs, new, keys, **more):
    return dict(name=name, op=op, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, cache=cache,
                page=page, seqs=seqs, new_lo=new[0], new_hi=new[1], keys_lo=keys[0], keys_hi=keys[1], **more)


def listed():
    return [
        # a decode step of nine rows behind a prefix: one layer's keys and values
        _case("append_decode_step", "append", 32, 8, 128, "f16", "f16", 64, 9, (1, 1), (24, 64), prefix=512, means=False),
        # a default batch of 16,384 tokens in rows of a filter's lengths, into 8-bit pages
        _case("append_rows_8b", "append", 32, 8, 128, "f16", "e4m3", 64, 272, (8, 112), (0, 0), prefix=512, means=False),
        # one long prompt of the 1B shape, whose pages get their means
        _case("append_prompt_1b", "append", 32, 8, 64, "bf16", "bf16", 64, 1, (8448, 8448), (0, 0), prefix=0, means=True),
        # one row's decode step: 512 + 60 keys in pages of its own
        _case("attend_one_token", "attend", 32, 8, 128, "f16", "f16", 64, 1, (1, 1), (572, 572), prefix=0),
        # a decode step of 256 rows behind a long shared prefix (instruction and many examples)
        _case("attend_decode_shared", "attend", 32, 8, 128, "f16", "f16", 64, 256, (1, 1), (8, 112), prefix=8192),
        # a decode step of 32 long contexts of different lengths, 8-bit pages
        _case("attend_decode_8bit", "attend", 32, 8, 128, "f16", "e4m3", 64, 32, (1, 1), (1000, 32000), prefix=0),
        # the tiny model's rows, a few tokens each, small pages
        _case("attend_rows_tiny", "attend", 4, 4, 64, "bf16", "bf16", 16, 64, (16, 48), (0, 0), prefix=96),
        # a default batch of rows behind the filter's prefix, 8B
        _case("attend_rows_8b", "attend", 32, 8, 128, "f16", "f16", 64, 272, (8, 112), (0, 0), prefix=512),
        # one prompt over a whole subset of a table, 8B
        _case("attend_prompt_8b", "attend", 32, 8, 128, "bf16", "bf16", 64, 1, (8448, 8448), (0, 0), prefix=0),
        # a decode step of a few long contexts, an eighth of the 1B shape's keys
        _case("sparse_few_1b", "sparse", 32, 8, 64, "bf16", "bf16", 64, 4, (1, 1), (4000, 8448), blocks=16),
        # a decode step of 32 contexts of up to 32,000 tokens
        _case("sparse_decode_8b", "sparse", 32, 8, 128, "f16", "f16", 64, 32, (1, 1), (16000, 32000), blocks=16),
        # the last 2,000 tokens of such a context
        _case("sparse_prompt_8b", "sparse", 32, 8, 128, "f16", "f16", 64, 1, (2000, 2000), (30000, 30000), blocks=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "sparse"))
    kv_heads = rng.choice((1, 2, 4, 8))
    head_dim, dtype = rng.choice((64, 128)), rng.choice(("f16", "bf16"))
    lay = (kv_heads * rng.choice((1, 2, 3, 4, 7, 8)), kv_heads, head_dim, dtype, rng.choice((dtype, dtype, "e4m3")),
           rng.choice((16, 32, 64, 128)))
    if op == "append":
        seqs = _log_int(rng, 1, 256)
        most = _log_int(rng, 1, 16384 // seqs)
        before = rng.choice((0, _log_int(rng, 1, 2000)))
        return _case("", op, *lay, seqs, (rng.randint(1, most), most), (0, before),
                     prefix=rng.choice((0, _log_int(rng, 1, 8192))), means=rng.random() < 0.5)
    if op == "attend" and rng.random() < 0.5:  # a decode step
        seqs = _log_int(rng, 1, 256)
        most = _log_int(rng, 1, min(32000, 262144 // seqs))
        return _case("", op, *lay, seqs, (1, rng.choice((1, 1, 1, 4))), (rng.randint(0, most), most),
                     prefix=rng.choice((0, _log_int(rng, 16, 8192))))
    if op == "attend":
        seqs = _log_int(rng, 1, 256)
        # the products of all its tokens are no more than the long prompt's
        most = _log_int(rng, 2, min(16384 // seqs, int(6000 * math.sqrt(32 / (max(lay[0], 32) * seqs)))))
        return _case("", op, *lay, seqs, (rng.randint(1, most), most), (0, rng.choice((0, _log_int(rng, 1, 400)))),
                     prefix=rng.choice((0, _log_int(rng, 16, 800))))
    seqs = _log_int(rng, 1, 32)
    most = _log_int(rng, 200, 32000)
    new = rng.choice((1, 1, _log_int(rng, 2, max(2, min(1000 // seqs, 30000000 // (seqs * most))))))
    return _case("", op, *lay, seqs, (1, new), (rng.randint(100, most), most), blocks=rng.choice((4, 8, 16, 32)))


def _spread(n, lo, hi, turn=0.0):
    """n whole numbers over [lo, hi] in a mixed order, the last of them hi."""
    return [lo + int(((i + 1) * 0.6180339887 + turn) % 1 * (hi - lo + 1)) for i in range(n - 1)] + [hi]


def _batch(case):
    """Tokens of each sequence in the call, and its keys with them."""
    new = _spread(case["seqs"], case["new_lo"], case["new_hi"])
    return new, [b + n for b, n in zip(_spread(case["seqs"], case["keys_lo"], case["keys_hi"], 0.37), new)]


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _pages(case, n, g):
    """Pages of keys and values: [n][kv heads][page][head_dim], and the exponents of 8-bit ones."""
    shape = (n, case["kv_heads"], case["page"], case["head_dim"])
    k, v = (torch.empty(shape, dtype=E4M3 if case["cache"] == "e4m3" else DTYPES[case["dtype"]], device="cuda")
            for _ in range(2))
    means = torch.empty(n, case["kv_heads"], case["head_dim"], dtype=DTYPES[case["dtype"]], device="cuda")
    for at in range(0, n, 4096):
        m = min(4096, n - at)
        # a page's keys have something in common, one unit of it beside one of their own
        topic = _randn(g, m, case["kv_heads"], 1, case["head_dim"])
        key = topic + _randn(g, m, *shape[1:])
        value = _randn(g, m, *shape[1:])
        if case["cache"] == "e4m3":
            key, value = (key * 64).clamp(-E4M3_MAX, E4M3_MAX), (value * 96).clamp(-E4M3_MAX, E4M3_MAX)
        k[at:at + m], v[at:at + m] = key.to(k.dtype), value.to(v.dtype)
        means[at:at + m] = topic.squeeze(2).to(means.dtype)
    s = dict(k=k, v=v, means=means)
    if case["cache"] == "e4m3":
        s["k_exp"] = torch.full(shape[:3], 121, dtype=torch.uint8, device="cuda")  # 2^-6
        s["v_exp"] = torch.randint(119, 122, shape[:3], generator=g, device="cuda", dtype=torch.uint8)
    return s


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    nq, nkv, hd, page, dt = case["heads"], case["kv_heads"], case["head_dim"], case["page"], DTYPES[case["dtype"]]
    new, length = _batch(case)
    prefix = case.get("prefix", 0)
    tokens = sum(new)
    s["new"], s["len"], s["tokens"] = new, length, tokens
    used = [-(-n // page) for n in length]
    shared = -(-prefix // page)
    pool = sum(used) + shared + 3
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    s["prefix_pages"] = order[:shared].contiguous()
    # a table has room for a page more than the longest sequence; what is not used names no page
    table = torch.full((case["seqs"], max(used) + 1), -1, dtype=torch.int32)
    at = shared
    host = order.cpu()
    for i, u in enumerate(used):
        table[i, :u] = host[at:at + u]
        at += u
    s["table"] = table.cuda()
    s["length"] = torch.tensor(length, dtype=torch.int32, device="cuda")
    s["start"] = None
    if max(new) > 1:
        s["start"] = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    if case["op"] == "append":
        # what a fused q|k|v projection leaves: one tensor, the three parts side by side
        s["qkv"] = (_randn(g, tokens, (nq + 2 * nkv) * hd) * 2).to(dt)
        shape = (pool, nkv, page, hd)
        if case["cache"] == "e4m3":
            s["k"], s["v"] = (torch.zeros(shape, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
            s["k_exp"], s["v_exp"] = (torch.full(shape[:3], 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        else:
            s["k"], s["v"] = (torch.zeros(shape, dtype=dt, device="cuda") for _ in range(2))
        # keys of before the call: whatever a page's earlier tokens left
        if any(b > n for b, n in zip(length, new)):
            s.update({n: t for n, t in _pages(case, pool, g).items() if n != "means"})
        s["means"] = torch.zeros(pool, nkv, hd, dtype=dt, device="cuda") if case["means"] else None
    else:
        s.update(_pages(case, pool, g))
        q = _randn(g, tokens, nkv, nq // nkv, hd)
        if case["op"] == "sparse":
            # tokens look for something that a few pages have, neighbours for the same
            q = q + 0.5 * _randn(g, -(-tokens // 16), nkv, 1, hd).repeat_interleave(16, 0)[:tokens]
        s["q"] = (q * 1.5).view(tokens, nq * hd).to(dt)
    if own:
        from types import SimpleNamespace

        from paper_2606_31808_amd import lmop as L
        shape = SimpleNamespace(n_layers=0, d_model=64, n_heads=nq, n_kv_heads=nkv, head_dim=hd, d_ff=64, vocab=2,
                                group_size=32, rms_eps=1e-5, rope_theta=THETA)
        s["ctx"] = L.Context(shape, device=torch.cuda.current_device(),
                             stream=torch.cuda.current_stream().cuda_stream, max_seq=MAX_SEQ)
        s["cache_own"] = L.PagedCache(s["k"], s["v"], s.get("k_exp"), s.get("v_exp"), s["means"])
    elif case["op"] == "append":
        angle = torch.arange(MAX_SEQ, device="cuda", dtype=torch.float64)[:, None] * _frequencies(hd)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def _frequencies(hd):
    return THETA ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)


# ---------------------------------------------------------------- one pass
def run(s):
    return {"append": _run_append, "attend": _run_attend, "sparse": _run_sparse}[s["op"]](s)


def _run_append(s):
    nq, nkv, hd = s["heads"], s["kv_heads"], s["head_dim"]
    q, k, v = s["qkv"].split((nq * hd, nkv * hd, nkv * hd), 1)
    kept = [s[n] for n in ("k", "v", "k_exp", "v_exp", "means") if s.get(n) is not None]
    if own:
        out = s["ctx"].cache_append(s["cache_own"], k, v, q=q, table=s["table"], length=s["length"], start=s["start"],
                                    first=s["prefix"])
        return out, *kept
    page, dt = s["page"], s["qkv"].dtype
    seq, index = _places(s)
    half = hd // 2
    cos, sin = (s[c][s["prefix"] + index].unsqueeze(1) for c in ("cos", "sin"))

    def turned(x):
        x = x.float().view(x.shape[0], -1, hd)
        x1, x2 = x[..., :half], x[..., half:]
        return torch.cat((x1 * cos - x2 * sin, x1 * sin + x2 * cos), -1)

    page_of, in_page = s["table"][seq, index // page].long(), index % page
    for store, y in (("k", turned(k)), ("v", v.float().view(-1, nkv, hd))):
        if s["cache"] == "e4m3":
            code, exponent = _codes(y, dt)
            s[store][page_of, :, in_page] = code
            s[store + "_exp"][page_of, :, in_page] = exponent
        else:
            s[store][page_of, :, in_page] = y.to(dt)
    if s["means"] is not None:
        full = page_of[in_page == page - 1]
        x = _values(s, "k", full)
        s["means"][full] = (x.double().sum(2) / page).to(dt)
    return turned(q).view(-1, nq * hd).to(dt), *kept


def _codes(y, dt):
    """E4M3 codes and exponents (+ 127) of heads y in 32 bits: the least power of two that fits the largest."""
    if dt == torch.float16:
        y = y.clamp(-MOST_F16, MOST_F16)
    top, e = torch.frexp(y.abs().amax(-1))
    e = torch.where(top > E4M3_MAX / 512, e - 8, e - 9).clamp(min=-126)
    return (y * torch.ldexp(torch.ones_like(top), -e).unsqueeze(-1)).to(E4M3), (e + 127).to(torch.uint8)


def _values(s, store, pages):
    """The pages' values [pages][kv heads][page][head_dim] in 32 bits."""
    x = s[store].view(torch.uint8)[pages].view(E4M3).float() if s["cache"] == "e4m3" else s[store][pages].float()
    if s["cache"] == "e4m3":
        x = x * torch.ldexp(torch.ones((), device="cuda"), s[store + "_exp"][pages].int() - 127).unsqueeze(-1)
    return x


def _places(s):
    """For every token its sequence and its index among that one's keys."""
    new = torch.tensor(s["new"], device="cuda")
    seq = torch.repeat_interleave(torch.arange(s["seqs"], device="cuda"), new, output_size=s["tokens"])
    first = new.cumsum(0) - new
    return seq, (s["length"] - new - first)[seq] + torch.arange(s["tokens"], device="cuda")


def _by_head(s, store, pages, n):
    """The first n keys or values of these pages: [kv heads][n][head_dim]."""
    x = _values(s, store, pages)
    return x.transpose(0, 1).reshape(s["kv_heads"], -1, s["head_dim"])[:, :n]


def _run_attend(s):
    if own:
        return s["ctx"].attend(s["cache_own"], s["q"], table=s["table"], length=s["length"], start=s["start"],
                               max_tokens=max(s["new"]), max_length=max(s["len"]), prefix=s["prefix_pages"],
                               prefix_length=s["prefix"])
    nkv, hd, page, shared = s["kv_heads"], s["head_dim"], s["page"], s["prefix"]
    group = s["heads"] // nkv
    q = s["q"].float().view(-1, nkv, group, hd).permute(1, 0, 2, 3) * hd ** -0.5
    pk, pv = (_by_head(s, c, s["prefix_pages"].long(), shared) for c in "kv")
    out = torch.empty_like(q)
    at = 0
    for i, (n, m) in enumerate(zip(s["new"], s["len"])):
        pages = s["table"][i, :-(-m // page)].long()
        k, v = torch.cat((pk, _by_head(s, "k", pages, m)), 1), torch.cat((pv, _by_head(s, "v", pages, m)), 1)
        # token j of n sees the prefix and its sequence's keys up to its own
        hidden = (torch.arange(shared + m, device="cuda") > shared + m - n + torch.arange(n, device="cuda")[:, None])
        step = nkv if n < 256 else 1  # heads at a time
        for h in range(0, nkv, step):
            z = torch.bmm(q[h:h + step, at:at + n].reshape(step, n * group, hd), k[h:h + step].transpose(1, 2))
            if n > 1:
                z.masked_fill_(hidden.repeat_interleave(group, 0), -math.inf)
            p = (z - z.amax(-1, keepdim=True)).exp_()
            o = torch.bmm(p, v[h:h + step].contiguous()) / p.sum(-1, keepdim=True)
            out[h:h + step, at:at + n] = o.view(step, n, group, hd)
        at += n
    return out.permute(1, 0, 2, 3).reshape(s["q"].shape).to(s["q"].dtype)


def _run_sparse(s):
    if own:
        blocks = s["ctx"].select_blocks(s["cache_own"], s["q"], s["blocks"], table=s["table"], length=s["length"],
                                        start=s["start"], max_length=max(s["len"]))
        return blocks, s["ctx"].attend(s["cache_own"], s["q"], table=s["table"], length=s["length"], start=s["start"],
                                       max_tokens=max(s["new"]), max_length=max(s["len"]), blocks=blocks)
    nkv, hd, page, want = s["kv_heads"], s["head_dim"], s["page"], s["blocks"]
    group = s["heads"] // nkv
    seq, index = _places(s)
    q = s["q"].view(-1, nkv, group, hd)
    mean = s["means"][s["table"].clamp(min=0).long()].permute(0, 2, 3, 1)  # [seqs][kv heads][head_dim][blocks]
    n_blocks = mean.shape[3]
    mine = index // page
    chosen, out = [], []
    least = min(want, n_blocks)
    for i in range(s["seqs"]):
        here = slice(sum(s["new"][:i]), sum(s["new"][:i + 1]))
        # borders between chosen blocks and others are narrow: 64 bits
        score = torch.matmul(q[here].double().sum(2).unsqueeze(2).transpose(0, 1).reshape(nkv, -1, hd),
                             mean[i].double().contiguous()).transpose(0, 1)
        b = torch.arange(n_blocks, device="cuda")
        last = mine[here, None, None]
        score = torch.where(b > last, -math.inf, torch.where(b == last, math.inf, score))
        ids = score.sort(dim=-1, descending=True, stable=True)[1][..., :least]
        ids = torch.where(ids <= last, ids, n_blocks).sort(-1)[0]
        ids = torch.nn.functional.pad(ids, (0, want - least), value=n_blocks)
        chosen.append(torch.where(ids < n_blocks, ids, -1).to(torch.int32))
    chosen = torch.cat(chosen)
    head = torch.arange(nkv, device="cuda")[None, :, None]
    in_page = torch.arange(page, device="cuda")
    step = max(1, (1 << 28) // (nkv * want * page * hd))  # tokens at a time
    for at in range(0, s["tokens"], step):
        t = slice(at, min(s["tokens"], at + step))
        ids = chosen[t].long()
        pages = s["table"][seq[t, None, None], ids.clamp(min=0)].long().clamp(min=0)
        k, v = (_some(s, c, pages, head) for c in "kv")  # [tokens][kv heads][keys][head_dim]
        seen = (ids[..., None] >= 0) & (ids[..., None] * page + in_page <= index[t, None, None, None])
        z = torch.matmul(q[t].float() * hd ** -0.5, k.transpose(2, 3))
        z = torch.where(seen.view(z.shape[0], nkv, 1, -1), z, -math.inf)
        p = (z - z.amax(-1, keepdim=True)).exp_()
        out.append(torch.matmul(p, v) / p.sum(-1, keepdim=True))
    return chosen, torch.cat(out).view(s["q"].shape).to(s["q"].dtype)


def _some(s, store, pages, head):
    """The values of one head of each page: [tokens][kv heads][blocks * page][head_dim]."""
    if s["cache"] == "e4m3":
        x = s[store].view(torch.uint8)[pages, head].view(E4M3).float()
        x = x * torch.ldexp(torch.ones((), device="cuda"), s[store + "_exp"][pages, head].int() - 127).unsqueeze(-1)
    else:
        x = s[store][pages, head].float()
    return x.view(*pages.shape[:2], -1, s["head_dim"])


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    nq, nkv, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    new, length = _batch(case)
    tokens, prefix = sum(new), case.get("prefix", 0)
    one = nkv * (hd * 2 if case["cache"] != "e4m3" else hd + 1)  # a token's keys, or its values
    if case["op"] == "append":
        means = 2 * nkv * hd * sum(m // page - (m - n) // page for n, m in zip(new, length)) if case["means"] else 0
        return {"bytes": tokens * (4 * nq * hd + 4 * nkv * hd + 2 * one + 4 * hd) + means,
                "flops": tokens * (3.0 * (nq + nkv) * hd + (3.0 * 2 * nkv * hd if case["cache"] == "e4m3" else 0))}
    ends = 4 * tokens * nq * hd  # queries and outputs
    if case["op"] == "attend":
        seen = sum(n * prefix + n * m - n * (n - 1) // 2 for n, m in zip(new, length))
        return {"bytes": ends + 2 * one * (prefix + sum(length)), "flops": 4.0 * nq * hd * seen}
    want = case["blocks"]
    seen = read = scored = 0
    for n, m in zip(new, length):
        counts = [min(want - 1, i // page) * page + i % page + 1 for i in range(m - n, m)]
        seen += sum(counts)
        read += min(m, sum(counts))
        scored += sum(i // page for i in range(m - n, m))
    return {"bytes": ends + 2 * one * read + 2 * nkv * hd * sum(m // page for m in length) + 4 * tokens * nkv * want,
            "flops": 4.0 * nq * hd * seen + 2.0 * nkv * hd * scored}


# ---------------------------------------------------------------- the definition in 64 bits
def _e4m3(y):
    """The E4M3 value nearest to y (float64), ties to the even one: 3 fraction bits, least exponent -6."""
    e = torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4
    step = torch.pow(2.0, e.double())
    return (torch.round(y / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sparse": _exact_sparse}[case["op"]](s)


def _whole(s, store):
    """The store in 64 bits."""
    x = s[store].double()
    if s["cache"] == "e4m3":
        x = x * torch.pow(2.0, s[store + "_exp"].double() - 127).unsqueeze(-1)
    return x


def _exact_append(s):
    nq, nkv, hd, page = s["heads"], s["kv_heads"], s["head_dim"], s["page"]
    x = s["qkv"].double().view(-1, nq + 2 * nkv, hd)
    where = [(i, m - n + j) for i, (n, m) in enumerate(zip(s["new"], s["len"])) for j in range(n)]
    seq, index = torch.tensor(where, device="cuda").unbind(1)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       (s["prefix"] + index).double()[:, None, None] * _frequencies(hd))
    z = torch.complex(x[:, :nq + nkv, :hd // 2].contiguous(), x[:, :nq + nkv, hd // 2:].contiguous()) * turn
    turned = torch.cat((z.real, z.imag), -1)
    at = s["table"].long()[seq, torch.div(index, page, rounding_mode="floor")]
    slot = index.remainder(page)
    # the means are those of the keys as they are kept
    out, kept = {}, {}
    for store, y in (("k", turned[:, nq:]), ("v", x[:, nq + nkv:])):
        kept[store] = _whole(s, store)
        if s["cache"] == "e4m3":
            if s["dtype"] == "f16":
                y = y.clamp(-MOST_F16, MOST_F16)
            e = torch.ceil(torch.log2(y.abs().amax(-1) / E4M3_MAX)).clamp(min=-126)
            code = _e4m3(y / torch.pow(2.0, e).unsqueeze(-1))
            out[store], out[store + "_exp"] = s[store].double(), s[store + "_exp"].clone()
            out[store][at, :, slot], out[store + "_exp"][at, :, slot] = code, (e + 127).to(torch.uint8)
            kept[store][at, :, slot] = code * torch.pow(2.0, e).unsqueeze(-1)
        else:
            kept[store][at, :, slot] = y
            out[store] = kept[store]
    kept_out = [out[n] for n in ("k", "v", "k_exp", "v_exp") if n in out]
    if s["means"] is not None:
        mean = s["means"].double()
        full = at[slot == page - 1]
        mean[full] = kept["k"][full].mean(2)
        kept_out.append(mean if s["cache"] != "e4m3" else None)  # a code on the other side of a tie moves it
    return turned[:, :nq].reshape(len(where), -1), *kept_out


def _exact_attend(s):
    nq, nkv, hd, page, shared = s["heads"], s["kv_heads"], s["head_dim"], s["page"], s["prefix"]
    new, length = s["new"], s["len"]
    if nq * hd * sum(n * (shared + m) for n, m in zip(new, length)) > 2e12:
        return None
    q = s["q"].double().view(-1, nq, hd)
    out = torch.zeros_like(q)
    for i, (n, m) in enumerate(zip(new, length)):
        ids = torch.cat((s["prefix_pages"], s["table"][i])).long().clamp(min=0)
        # the place of every key: the prefix's pages, then the sequence's own
        spot = torch.cat((torch.arange(shared), len(s["prefix_pages"]) * page + torch.arange(m))).cuda()
        first = sum(new[:i])
        ends = shared + m - n + 1 + torch.arange(n, device="cuda")
        k, v = (_dequantised(s, c, ids[spot // page], spot % page) for c in "kv")
        for h in range(nq):
            z = torch.mm(q[first:first + n, h], k[:, h * nkv // nq].t().contiguous()) / math.sqrt(hd)
            z = z.masked_fill(torch.arange(shared + m, device="cuda") >= ends[:, None], -math.inf)
            out[first:first + n, h] = torch.mm(torch.softmax(z, -1), v[:, h * nkv // nq].contiguous())
    return out.view(-1, nq * hd)


def _dequantised(s, store, page, slot):
    """Keys or values at these places, in 64 bits: [places][kv heads][head_dim]."""
    if s["cache"] != "e4m3":
        return s[store][page, :, slot].double()
    return (s[store].view(torch.uint8)[page, :, slot].view(E4M3).double()
            * torch.pow(2.0, s[store + "_exp"][page, :, slot].double() - 127).unsqueeze(-1))


def _exact_sparse(s):
    nq, nkv, hd, page, want = s["heads"], s["kv_heads"], s["head_dim"], s["page"], s["blocks"]
    q = s["q"].double().view(-1, nkv, nq // nkv, hd)
    chosen = torch.full((s["tokens"], nkv, want), -1, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    t = 0
    for i, (n, m) in enumerate(zip(s["new"], s["len"])):
        ids = s["table"][i].long().clamp(min=0)
        spot = torch.arange(m, device="cuda")
        k, v = (_dequantised(s, c, ids[spot // page], spot % page) for c in "kv")
        mean = s["means"][ids].double()
        for h in range(nkv):
            score = torch.mm(q[t:t + n, h].sum(1), mean[:, h].t().contiguous())
            mine = (m - n + torch.arange(n, device="cuda")) // page
            block = torch.arange(len(ids), device="cuda")
            score.masked_fill_(block >= mine[:, None], -math.inf)
            # the best of the earlier blocks, of equals the first, and the token's own
            order = torch.argsort(-score, dim=-1, stable=True)
            place = torch.empty_like(order).scatter_(1, order, block.expand_as(order).contiguous())
            taken = (place < want - 1) & (block < mine[:, None]) | (block == mine[:, None])
            rank = taken.cumsum(1) - 1
            row, col = taken.nonzero().unbind(1)
            chosen[t + row, h, rank[row, col]] = col.to(torch.int32)
            at = max(1, (1 << 27) // (m * (nq // nkv)))  # tokens at a time
            for a in range(0, n, at):
                e = min(n, a + at)
                seen = taken[a:e].repeat_interleave(page, 1)[:, :m] & (
                    torch.arange(m, device="cuda") <= (m - n + torch.arange(a, e, device="cuda"))[:, None])
                z = torch.mm(q[t + a:t + e, h].reshape(-1, hd), k[:, h].t().contiguous()) / math.sqrt(hd)
                z = z.masked_fill(~seen.repeat_interleave(nq // nkv, 0), -math.inf)
                out[t + a:t + e, h] = torch.mm(torch.softmax(z, -1), v[:, h].contiguous()).view(e - a, -1, hd)
        t += n
    return chosen, out.view(-1, nq * hd)
