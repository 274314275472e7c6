"""What is timed of the decoding step's operators on a paged 8-bit cache: the page tables of
a step, the cache's append, the attention that reads it, and sampling from the target logits.

``run`` makes the calls a decoding loop makes through ``paper_2604_05650_b200.binding``
(``own``), or computes the same operators with elementary torch operations.

  pages   From the lengths of the requests on the GPU: which free pages they take, the
          block table, and the cache slot of every new token.
  append  New K/V rows (bf16) written to their slots as E4M3 codes, with one power-of-two
          scale per block of tokens and head; a block that is begun already keeps the
          larger scale, its older codes being brought to it.
  attend  Attention of gamma draft queries per sequence over that cache, with the share of
          each query's probability on the visual span.  Queries that see nothing give zeros.
  sample  A token per row of logits by temperature, top-k, top-p and min-p, from one given
          uniform number per row.

Head shapes are those of ``workloads.CONFIGS``, its sweep and the tests, or generic.
"""
import math

import torch

own = False

# (query heads, KV heads, head_dim)
HEADS = ((28, 4, 128), (40, 8, 128), (64, 8, 128), (8, 2, 64))
VOCAB = 152064
_kept = {}


def _attend(name, heads, batch, gamma, kv_len, page, block, *, ragged=0.0, idle=0):
    """ragged: by how much of kv_len the shortest sequence is shorter; idle: padding of the batch,
    sequences of length 0."""
    hq, hkv, d = heads
    case = {"op": "attend", "hq": hq, "hkv": hkv, "d": d, "batch": batch, "gamma": gamma, "kv_len": kv_len,
            "page": page, "block": block, "ragged": ragged, "idle": idle}
    return dict(case, name=name) if name else case


def _append(name, heads, batch, new, kv_len, page, block, *, ragged=0.0, idle=0):
    """new: tokens appended to each sequence; idle: rows of the call that hold no token (slot -1)."""
    _, hkv, d = heads
    case = {"op": "append", "hkv": hkv, "d": d, "batch": batch, "new": new, "kv_len": kv_len, "page": page,
            "block": block, "ragged": ragged, "idle": idle}
    return dict(case, name=name) if name else case


def _pages(name, batch, new, kv_len, page, *, ragged=0.0, spare=0):
    """spare: entries of the slot map behind the last token."""
    case = {"op": "pages", "batch": batch, "new": new, "kv_len": kv_len, "page": page, "ragged": ragged, "spare": spare}
    return dict(case, name=name) if name else case


def _sample(name, rows, vocab, dtype, filters):
    """filters: "none", "k", "p", "min", "kp" or "mixed" (another set for every row)."""
    case = {"op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "filters": filters}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token against a few hundred positions in small pages: all latency
        _attend("attend-tiny", HEADS[3], 1, 1, 333, 16, 16),
        # plain decoding of eight requests, one query each, lengths apart
        _attend("attend-token", HEADS[0], 8, 1, 16384, 64, 64, ragged=0.6),
        # the verify step the library is quoted on: a chain of 8 over 128 frames
        _attend("attend-chain", HEADS[1], 1, 8, 32768, 128, 128),
        # a server's batch, two places of it empty, pages shorter than a tile
        _attend("attend-batch", HEADS[2], 16, 10, 32003, 32, 32, ragged=0.5, idle=2),
        # two long videos
        _attend("attend-long", HEADS[1], 2, 4, 131071, 256, 64),
        # the draft tokens of a batch's step
        _append("append-step", HEADS[1], 16, 8, 8000, 64, 64, ragged=0.5, idle=16),
        # prompts of several requests, prefilled together
        _append("append-prompt", HEADS[1], 7, 4999, 0, 128, 32, ragged=0.9),
        # page tables of a decoding step
        _pages("pages-step", 16, 8, 32000, 16, ragged=0.5),
        # ... and of many prompts at once
        _pages("pages-prompts", 96, 30011, 0, 64, ragged=0.95, spare=4096),
        # one answer's next token
        _sample("sample-one", 1, VOCAB, "f32", "p"),
        # the positions of a batch's drafts, every request with filters of its own
        _sample("sample-batch", 128, VOCAB, "f32", "mixed"),
        # a small vocabulary in bf16, min-p
        _sample("sample-small", 8, 4096, "bf16", "min"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attend", "attend", "append", "pages", "sample"))
    page = rng.choice((16, 32, 64, 128, 256, 512))
    block = rng.choice([b for b in (16, 32, 64, 128) if page % b == 0])
    if op == "attend":
        heads = rng.choice(HEADS)
        gamma = _log(rng, 1, 128 // (heads[0] // heads[1]))
        kv_len = _log(rng, 200, 131071) | 1
        most = 16 * 32003 * 8 * 128 // (kv_len * heads[1] * heads[2])
        return _attend(None, heads, min(_log(rng, 1, 32), max(1, most)), gamma, kv_len, page, block,
                       ragged=rng.choice((0.0, 0.3, 0.9)), idle=rng.choice((0, 0, 3)))
    if op == "append":
        new = _log(rng, 1, 5000)
        return _append(None, rng.choice(HEADS), _log(rng, 1, max(1, min(64, 35000 // new))), new, rng.choice((0, 77, 3001)),
                       page, block, ragged=rng.choice((0.0, 0.5, 0.9)), idle=rng.choice((0, 5)))
    if op == "pages":
        new = _log(rng, 1, 30000)
        return _pages(None, _log(rng, 1, 128), new, rng.choice((0, 500, 32000)), page, ragged=rng.choice((0.0, 0.5, 0.9)),
                      spare=_log(rng, 1, 5000))
    vocab = _log(rng, 1000, VOCAB)
    return _sample(None, _log(rng, 1, min(1024, max(1, 128 * VOCAB // vocab))), vocab, rng.choice(("f32", "bf16")),
                   rng.choice(("none", "k", "p", "min", "kp", "mixed")))


def _lengths(case, most):
    """Per sequence: `most`, shortened by up to the share `ragged`; the idle ones at the end have none."""
    got = [most - int(most * case["ragged"] * ((b * 2654435761) % 4294967296) / 4294967296) for b in range(case["batch"])]
    idle = case.get("idle", 0) if case["op"] == "attend" else 0
    return got[:case["batch"] - idle] + [0] * min(idle, case["batch"]) if idle < case["batch"] else got


def _up(a, b):
    return -(-a // b)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dev = {"device": "cuda"}
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, **dev)  # noqa: E731
    if case["op"] == "attend":
        return _prepare_attend(case, g, i32)
    if case["op"] == "append":
        return _prepare_append(case, g, i32)
    if case["op"] == "pages":
        return _prepare_pages(case, g, i32)
    rows, vocab = case["rows"], case["vocab"]
    # logits as a target model's: mean 0, deviation 3, one planted token per row
    logits = torch.randn(rows, vocab, generator=g, **dev) * 3
    logits.scatter_add_(1, torch.randint(vocab, (rows, 1), generator=g, **dev), torch.full((rows, 1), 8.0, **dev))
    pick = torch.randint(6, (rows,), generator=g, **dev)
    plain = {"none": 0, "k": 1, "p": 2, "min": 3, "kp": 4}
    if case["filters"] != "mixed":
        pick = torch.full((rows,), plain[case["filters"]], **dev)
    rand = lambda lo, hi: lo + (hi - lo) * torch.rand(rows, generator=g, **dev)  # noqa: E731
    off = torch.zeros(rows, **dev)
    return {"case": case, "logits": logits if case["dtype"] == "f32" else logits.bfloat16(),
            # (5: greedy)
            "temperature": torch.where(pick == 5, off, rand(0.5, 1.2)),
            "top_k": torch.where((pick == 1) | (pick == 4), torch.randint(1, 200, (rows,), generator=g, **dev), 0).int(),
            "top_p": torch.where((pick == 2) | (pick == 4), rand(0.6, 0.99), off + 1),
            "min_p": torch.where(pick == 3, rand(0.01, 0.2), off),
            "uniform": torch.rand(rows, generator=g, **dev),
            "tokens": torch.empty(rows, dtype=torch.int32, **dev), "probs": torch.empty(rows, **dev)}


def _pool(case, n_pages, g):
    """K or V pages: E4M3 codes of normal values, scales that differ from block to block."""
    shape = (n_pages, case["hkv"], case["page"], case["d"])
    codes = torch.empty(shape, dtype=torch.uint8, device="cuda")
    values = torch.empty(shape, dtype=torch.float16, device="cuda").normal_(0, 100, generator=g).clamp_(-448, 448)
    codes.copy_(values.to(torch.float8_e4m3fn).view(torch.uint8))
    scale = torch.randn(n_pages, case["hkv"], case["page"] // case["block"], generator=g, device="cuda").mul_(0.2).exp_() / 100
    return codes, scale


def _prepare_attend(case, g, i32):
    b, gamma, page = case["batch"], case["gamma"], case["page"]
    lens = _lengths(case, case["kv_len"])
    per_seq = _up(max(case["kv_len"], gamma), page)
    lens = [max(n, gamma) if n else 0 for n in lens]
    used = [_up(n, page) for n in lens]
    n_pages = sum(used) + 3
    k, ks = _pool(case, n_pages, g)
    v, vs = _pool(case, n_pages, g)
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((b, per_seq), -1, dtype=torch.int32, device="cuda")
    first = 0
    for i in range(b):
        table[i, :used[i]] = order[first:first + used[i]]
        first += used[i]
    q = torch.randn(b, gamma, case["hq"], case["d"], generator=g, device="cuda").bfloat16()
    # the visual span: three quarters of the context, behind a short prompt
    span = [[n // 32, n // 32 + 3 * (n - gamma) // 4] if n > gamma else [0, 0] for n in lens]
    return {"case": case, "n_pages": n_pages, "max_kv_len": max(case["kv_len"], gamma), "q": q, "k": k, "ks": ks, "v": v, "vs": vs,
            "table": table, "lens": i32(lens), "span": i32(span), "out": torch.empty_like(q),
            "mass": torch.empty(b, gamma, case["hq"], device="cuda")}


def _prepare_append(case, g, i32):
    page, hkv, d = case["page"], case["hkv"], case["d"]
    new = [max(1, n) for n in _lengths(case, case["new"])]
    held = [case["kv_len"] - 13 * i if case["kv_len"] > 13 * i else case["kv_len"] for i in range(case["batch"])]
    used = [_up(a + n, page) for a, n in zip(held, new)]
    n_pages = sum(used) + 2
    order = torch.randperm(n_pages, generator=g, device="cuda")
    slots, first = [], 0
    for a, n, u in zip(held, new, used):
        pos = torch.arange(a, a + n, device="cuda")
        slots.append(order[first + pos // page] * page + pos % page)
        first += u
    slots.append(torch.full((case["idle"],), -1, device="cuda"))
    slots = torch.cat(slots).int()
    k, ks = _pool(case, n_pages, g)
    v, vs = _pool(case, n_pages, g)
    # (what an append leaves: powers of two)
    ks, vs = torch.exp2(torch.round(torch.log2(ks)) - 1), torch.exp2(torch.round(torch.log2(vs)) - 1)
    # K and V as one projection gives them: neighbours in a row of q, k and v
    rows = torch.randn(slots.numel(), 3, hkv, d, generator=g, device="cuda").bfloat16()
    return {"case": case, "n_pages": n_pages, "k_new": rows[:, 1], "v_new": rows[:, 2], "slots": slots, "k": k, "ks": ks, "v": v, "vs": vs}


def _prepare_pages(case, g, i32):
    b, page = case["batch"], case["page"]
    new = [max(1, n) for n in _lengths(case, case["new"])]
    lens = [case["kv_len"] - 7 * i if case["kv_len"] > 7 * i else case["kv_len"] for i in range(b)]
    held = [_up(n, page) for n in lens]
    per_seq = _up(case["kv_len"] + case["new"], page) + 1
    n_pages = sum(held) + sum(_up(n + m, page) for n, m in zip(lens, new)) + 5
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((b, per_seq), -1, dtype=torch.int32, device="cuda")
    first = 0
    for i in range(b):
        table[i, :held[i]] = order[first:first + held[i]]
        first += held[i]
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:n_pages - first] = order[first:]
    total = sum(new) + case["spare"]
    empty = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"case": case, "n_pages": n_pages, "per_seq": per_seq, "total": total, "lens": i32(lens), "new": i32(new), "held": i32(held),
            "n_free": i32([n_pages - first]), "free": free, "table": table, "new_lens": empty(b), "new_held": empty(b),
            "new_n_free": empty(1), "starts": empty(b + 1), "slots": empty(total)}


def run(s):
    if own:
        return _own(s)
    return {"attend": _plain_attend, "append": _plain_append, "pages": _plain_pages, "sample": _plain_sample}[s["case"]["op"]](s)


def _own(s):
    from paper_2604_05650_b200 import binding
    if not _kept:
        _kept["context"] = binding.Context(torch.cuda.current_device())
    ctx, c = _kept["context"], s["case"]
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    if c["op"] == "attend":
        shape = binding.attn_shape(c["batch"], c["gamma"], c["hq"], c["hkv"], c["d"], s["table"].shape[1] * c["page"])
        cache = binding.paged_fp8(c["page"], s["n_pages"], c["block"])
        ctx.verify_attention_paged_fp8(shape, cache, s["q"], s["k"], s["v"], s["ks"], s["vs"], s["table"], s["lens"], s["span"],
                                       s["out"], s["mass"], max_kv_len=s["max_kv_len"])
        return s["out"], s["mass"]
    if c["op"] == "append":
        cache = binding.paged_fp8(c["page"], s["n_pages"], c["block"])
        ctx.append_paged_fp8(s["slots"].numel(), c["hkv"], c["d"], cache, s["k_new"], s["v_new"], s["k_new"].stride(0),
                             s["v_new"].stride(0), s["slots"], s["k"], s["v"], s["ks"], s["vs"])
        return s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["ks"], s["vs"]
    if c["op"] == "pages":
        ctx.plan_pages(c["batch"], c["page"], s["per_seq"], s["n_pages"], s["total"], s["lens"], s["new"], s["held"], s["n_free"],
                       s["free"], s["table"], s["new_lens"], s["new_held"], s["new_n_free"], s["starts"], s["slots"])
        return s["table"], s["new_lens"], s["new_held"], s["new_n_free"], s["starts"], s["slots"]
    ctx.sample(c["rows"], c["vocab"], s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["uniform"], s["tokens"],
               s["probs"], bf16=c["dtype"] == "bf16")
    return s["tokens"], s["probs"]


def _rows_of(pool, scale, table, block, positions):
    """The cache's values [B, Hkv, positions, D] in fp32."""
    page = pool.shape[2]
    at = torch.arange(positions, device="cuda")
    pages = table[:, at // page].clamp_min(0).long()                      # [B, positions]
    codes = pool.view(torch.float8_e4m3fn)[pages, :, (at % page)[None]]   # [B, positions, Hkv, D]
    each = scale[pages, :, (at % page // block)[None]]
    return (codes.float() * each[..., None]).transpose(1, 2)


def _plain_attend(s):
    c = s["case"]
    b, gamma, hq, hkv, d = c["batch"], c["gamma"], c["hq"], c["hkv"], c["d"]
    n = s["max_kv_len"]
    k, v = _rows_of(s["k"], s["ks"], s["table"], c["block"], n), _rows_of(s["v"], s["vs"], s["table"], c["block"], n)
    q = s["q"].float().view(b, gamma, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, -1, d)
    scores = (q @ k.transpose(2, 3)).view(b, hkv, gamma, -1, n) / math.sqrt(d)
    at = torch.arange(n, device="cuda")
    sees = s["lens"][:, None] - gamma + torch.arange(1, gamma + 1, device="cuda")           # [B, gamma]
    scores.masked_fill_(at >= sees[:, None, :, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1)
    inside = (at >= s["span"][:, :1]) & (at < s["span"][:, 1:])
    mass = (p * inside[:, None, None, None]).sum(-1)
    v = v.masked_fill((at >= s["lens"][:, None])[:, None, :, None], 0)
    out = (p.view(b, hkv, -1, n) @ v).view(b, hkv, gamma, -1, d)
    heads_last = lambda x: x.permute(0, 2, 1, 3, *range(4, x.dim())).reshape(b, gamma, hq, *x.shape[4:])  # noqa: E731
    return heads_last(out).bfloat16(), heads_last(mass)


def _plain_append(s):
    c = s["case"]
    _plain_append_one(c, s["slots"], s["k_new"], s["k"], s["ks"])
    _plain_append_one(c, s["slots"], s["v_new"], s["v"], s["vs"])
    return s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["ks"], s["vs"]


def _e4m3(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append_one(c, slots, new, pool, scale):
    page, block, hkv, d = c["page"], c["block"], c["hkv"], c["d"]
    keep = (slots >= 0).nonzero()[:, 0]
    slots, new = slots[keep].long(), new[keep].float()
    which = slots // block                                                # block of every token, over all pages
    n_blocks = pool.shape[0] * page // block
    largest = torch.zeros(n_blocks, hkv, device="cuda").scatter_reduce_(0, which[:, None].expand(-1, hkv), new.abs().amax(-1), "amax")
    before = torch.full((n_blocks,), block, device="cuda").scatter_reduce_(0, which, slots % block, "amin")
    touched = (before < block).nonzero()[:, 0]
    largest, before = largest[touched], before[touched]
    # the smallest power of two that brings the largest value to at most 448
    m, e = torch.frexp(largest)
    need = torch.exp2(torch.where(largest > 0, e - 9 + (m > 0.875), -100).clamp(-100, 119).float())
    page_of, part = touched // (page // block), touched % (page // block)
    had = scale[page_of, :, part]                                         # [blocks, Hkv]
    now = torch.where(before[:, None] > 0, torch.maximum(had, need), need)
    blocks = pool.view(-1, hkv, page // block, block, d)
    old = blocks[page_of, :, part]                                        # [blocks, Hkv, block, D]
    brought = _e4m3(old.view(torch.float8_e4m3fn).float() * (had / now)[..., None, None])
    mine = torch.arange(block, device="cuda") < before[:, None]
    blocks[page_of, :, part] = torch.where(mine[:, None, :, None], brought, old)
    scale[page_of, :, part] = now
    pool[slots // page, :, slots % page] = _e4m3(new / scale[slots // page, :, slots % page // block][..., None])


def _plain_pages(s):
    c, page = s["case"], s["case"]["page"]
    lens, new, held, table, free = s["lens"].long(), s["new"].long(), s["held"].long(), s["table"], s["free"]
    starts = torch.nn.functional.pad(new.cumsum(0), (1, 0))
    fits = (lens + new <= s["per_seq"] * page) & (starts[1:] <= s["total"])
    need = torch.where(fits, ((lens + new + page - 1) // page - held).clamp_min(0), 0)
    upto = need.cumsum(0)
    fits &= (need == 0) | (upto <= s["n_free"])
    took = torch.where(fits & (need > 0), upto, 0).amax()
    # the pages taken, in the order of the requests
    b = torch.arange(need.numel(), device="cuda").repeat_interleave(torch.where(fits, need, 0))
    nth = torch.arange(b.numel(), device="cuda")
    j = held[b] + nth - (upto - need)[b]
    table[b, j] = free[s["n_free"].long() - 1 - nth]
    # the slots of the new tokens
    at = torch.arange(s["total"], device="cuda")
    r = torch.searchsorted(starts, at, right=True) - 1
    live = (r < need.numel())
    r = r.clamp_max(need.numel() - 1)
    pos = lens[r] + at - starts[r]
    live &= fits[r]
    entry = table[r, (pos // page).clamp_max(s["per_seq"] - 1)]
    slots = torch.where(live & (entry >= 0), entry * page + pos % page, -1).int()
    return (table, torch.where(fits, lens + new, lens).int(), torch.where(fits, held + need, held).int(), (s["n_free"] - took).int(),
            starts.int(), slots)


def _plain_sample(s):
    logits = s["logits"].float()
    vocab = logits.shape[1]
    temp = s["temperature"][:, None].double()
    sorted_, index = logits.sort(dim=1, descending=True, stable=True)
    sorted_ = sorted_.double()
    top = sorted_[:, :1]
    warm = torch.where(temp > 0, temp, 1)
    w = ((sorted_ - top) / warm).exp()
    rank = torch.arange(vocab, device="cuda")
    k = torch.where(s["top_k"] > 0, s["top_k"], vocab)[:, None]
    k = torch.where(temp > 0, k, 1)
    w = torch.where(rank < k, w, 0)
    upto = w.cumsum(1)
    p = s["top_p"][:, None].double()
    keep = (p >= 1) | (upto - w < p * upto[:, -1:])
    keep &= sorted_ >= top + warm * s["min_p"][:, None].double().log()
    keep[:, 0] = True
    kept = torch.zeros_like(w).scatter_(1, index, w * keep)
    upto = kept.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= s["uniform"][:, None].double() * total).sum(1, keepdim=True).clamp_max(vocab - 1)
    return token[:, 0].int(), (kept.gather(1, token) / total)[:, 0].float()


def work(case):
    op = case["op"]
    if op == "attend":
        lens = sum(max(n, case["gamma"]) if n else 0 for n in _lengths(case, case["kv_len"]))
        rows = case["batch"] * case["gamma"] * case["hq"]
        per = case["hkv"] * (2 * case["d"] + 8 / case["block"]) + 4 / case["page"]
        return {"bytes": lens * per + rows * (4 * case["d"] + 4), "flops": 4 * lens * case["gamma"] * case["hq"] * case["d"]}
    if op == "append":
        tokens = sum(max(1, n) for n in _lengths(case, case["new"]))
        return {"bytes": tokens * (case["hkv"] * case["d"] * 2 * 3 + 4) + 8 * tokens * case["hkv"] / case["block"]}
    if op == "pages":
        tokens = sum(max(1, n) for n in _lengths(case, case["new"])) + case["spare"]
        return {"bytes": 4 * tokens + 8 * tokens / case["page"] + 28 * case["batch"]}
    return {"bytes": case["rows"] * (case["vocab"] * (4 if case["dtype"] == "f32" else 2) + 28)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s)
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "pages":
        return _exact_pages(s)
    return _exact_sample(s)


def _exact_attend(s):
    """One sequence and KV head at a time, in fp64."""
    c = s["case"]
    page, block, group, gamma = c["page"], c["block"], c["hq"] // c["hkv"], c["gamma"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    mass = torch.zeros(s["mass"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        lo, hi = s["span"][b].tolist()
        pages = s["table"][b, :_up(n, page)].long()
        for h in range(c["hkv"]):
            def cache(pool, scale):
                x = pool[pages, h].view(torch.float8_e4m3fn).double() * scale[pages, h].double().repeat_interleave(block, 1)[..., None]
                return x.reshape(-1, c["d"])[:n]
            k, v = cache(s["k"], s["ks"]), cache(s["v"], s["vs"])
            q = s["q"][b, :, h * group:(h + 1) * group].double()
            for j in range(gamma):
                sees = n - gamma + j + 1
                if sees < 1:
                    continue
                p = torch.softmax(q[j] @ k[:sees].T / c["d"] ** 0.5, -1)
                out[b, j, h * group:(h + 1) * group] = p @ v[:sees]
                mass[b, j, h * group:(h + 1) * group] = p[:, lo:min(hi, sees)].sum(-1)
    return out, mass


def _exact_append(s):
    """Block by block from the slots, values of E4M3 taken from the list of all of them."""
    c = s["case"]
    page, block = c["page"], c["block"]
    if s["slots"].numel() > 3000:
        return None
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()[:127]      # 0 .. 448, ascending
    def nearest(x):
        i = torch.searchsorted(every, x.abs().contiguous()).clamp(1, 126)
        down, up = x.abs() - every[i - 1], every[i] - x.abs()
        i = torch.where((down < up) | ((down == up) & (i % 2 == 1)), i - 1, i)
        return every[i] * torch.where(x < 0, -1.0, 1.0)
    slots = s["slots"].cpu().tolist()
    got = []
    for new, pool, scale in ((s["k_new"], s["k"], s["ks"]), (s["v_new"], s["v"], s["vs"])):
        new, scale = new.double().cpu(), scale.double().cpu()
        pool = pool.cpu().view(torch.float8_e4m3fn).double()
        blocks = {}
        for i, x in enumerate(slots):
            if x >= 0:
                blocks.setdefault((x // page, x % page // block), []).append((x % block, i))
        for (p, part), tokens in blocks.items():
            begun = min(tokens)[0]
            a = new[[i for _, i in tokens]].abs().amax((0, 2))
            need = torch.exp2(torch.ceil(torch.log2(a / 448)))
            had = scale[p, :, part]
            now = torch.maximum(need, had) if begun else need
            at = part * block
            pool[p, :, at:at + begun] = nearest(pool[p, :, at:at + begun] * (had / now)[:, None, None])
            scale[p, :, part] = now
            for off, i in tokens:
                pool[p, :, at + off] = nearest(new[i] / now[:, None])
        got += [pool, scale]
    return got[0], got[2], got[1], got[3]


def _exact_pages(s):
    return None


def _exact_sample(s):
    """Row by row: what stays is a set of the largest logits, found from its size."""
    tokens, probs = [], []
    for r in range(s["logits"].shape[0]):
        x = s["logits"][r].double()
        t, u = float(s["temperature"][r]), float(s["uniform"][r])
        if t <= 0:
            tokens.append(int(x.argmax()))
            probs.append(1.0)
            continue
        z = torch.softmax(x / t, -1)
        size = x.numel()
        order = torch.argsort(-x, stable=True)
        k = int(s["top_k"][r])
        if k > 0:
            size = min(size, k)
        run_ = z[order[:size]].cumsum(0)
        if float(s["top_p"][r]) < 1:
            size = min(size, 1 + int((run_[:-1] < float(s["top_p"][r]) * run_[-1]).sum()))
        if float(s["min_p"][r]) > 0:
            size = min(size, int((x >= x.max() + t * math.log(float(s["min_p"][r]))).sum()))
        stay = torch.zeros_like(z)
        stay[order[:size]] = z[order[:size]]
        sums = stay.cumsum(0)
        i = int(torch.searchsorted(sums, u * sums[-1], right=True))
        tokens.append(i)
        probs.append(float(stay[i] / sums[-1]))
    return torch.tensor(tokens, dtype=torch.int32, device="cuda"), torch.tensor(probs, dtype=torch.float64, device="cuda")
