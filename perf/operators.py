"""The paged cache held in 8 bits, as a serving program uses it: block tables and slots from request lengths, the
quantising append, and single-token attention (entmax and softmax) over the 8-bit pages.

Kinds of a pass:
  map       new tokens per sequence -> pages from the free list, block table, slot / sequence / position of every token
  append    new K and V rows -> 8-bit codes in their pages, one power-of-two scale per page and KV head, page statistics
  entmax    one query token per sequence over every page ("full"), a page list per query head ("heads") or a page list
            shared by the query heads of a KV head ("group"): alpha-entmax with its exact threshold
  softmax   the same with softmax and its log-sum-exp, over every page or a page list per query head

`own`: False computes the passes with elementary torch operations, True through the framework's entry points."""
import math

import torch

own = False

D = 128
MAX_CODE = 448.0                       # largest finite value of the 8-bit format (OCP E4M3)
LOW, HIGH = -100, 119                  # exponents a scale may have


def _case(name, kind, **kw):
    c = dict(kind=kind, **kw)
    return dict(c, name=name) if name else c


def _attention(name, kind, over, batch, heads, tokens, page=16, dtype="bf16", alpha=1.5, flat=1.0, budget=0.02, stagger=0):
    """heads: (query heads, KV heads).  stagger: sequence b is b * stagger tokens shorter than the longest, down to an
    empty one.  flat: factor on the score scale.  budget: share of the longest sequence's pages in a list."""
    return _case(name, kind, over=over, batch=batch, q_heads=heads[0], kv_heads=heads[1], tokens=tokens, page=page,
                 dtype=dtype, alpha=alpha, flat=flat, budget=budget, stagger=stagger)


def _append(name, batch, kv_heads, total, page=16, dtype="bf16", held=1000, stats=True):
    """total: new tokens of all sequences together, dealt unevenly.  held: tokens of the longest sequence before."""
    return _case(name, "append", batch=batch, kv_heads=kv_heads, total=total, page=page, dtype=dtype, held=held, stats=stats)


def _map(name, batch, total, page=16, held=4096, short=False):
    """short: the free list does not hold pages for everybody."""
    return _case(name, "map", batch=batch, total=total, page=page, held=held, short=short)


def listed():
    return [
        # a decode step of a serving batch: one token for each of 64 sequences, one in sixteen of which begins a page
        _map("map-64x1", 64, 64),
        # prompts of a large batch mapped at once, with the free list running out on the way
        _map("map-256-prompts-128k", 256, 131072, page=32, held=0, short=True),
        # the decode step's append, statistics brought up to date: latency
        _append("append-64x1", 64, 8, 64),
        # a few prompts, 32K tokens together, statistics with them: bandwidth
        _append("append-prompts-32k", 6, 8, 32768, held=0),
        # chunks of prompts that go on in partly filled pages, float32 rows, an odd page size, no statistics
        _append("append-chunks-5k-f32-p12", 5, 2, 5003, page=12, dtype="f32", held=777, stats=False),
        # the smallest attention: one short sequence, no grouped heads, float32 queries, an odd page size, a small alpha
        _attention("entmax-1x777-f32-p12", "entmax", "full", 1, (8, 8), 777, page=12, dtype="f32", alpha=1.25),
        # the headline workload of the framework on an 8-bit cache: 2 % of a million tokens, a list per query head
        _attention("entmax-heads-1x1m", "entmax", "heads", 1, (32, 8), 1048576),
        # a batch of short chats with lists shared per KV head, sparsemax; every length different
        _attention("entmax-group-64x8k", "entmax", "group", 64, (32, 8), 8192, alpha=2.0, budget=0.0625, stagger=37),
        # every page of four long sequences
        _attention("entmax-full-4x128k", "entmax", "full", 4, (32, 8), 131072, stagger=9001),
        # softmax over everything: eight heads to a KV head, uneven lengths, pages of 32; the largest call
        _attention("softmax-full-8x128k-p32", "softmax", "full", 8, (64, 8), 131072, page=32, stagger=5003),
        # an ordinary batch, multi-query
        _attention("softmax-full-16x2k", "softmax", "full", 16, (8, 1), 2049, stagger=131),
        # softmax over a selection
        _attention("softmax-heads-4x128k", "softmax", "heads", 4, (32, 8), 131072, budget=0.04, stagger=9001),
    ]


def _near(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm, odd ones among them."""
    return max(1, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(("map", "append", "append", "entmax", "entmax", "entmax", "softmax", "softmax"))
    page = rng.choice((4, 8, 12, 16, 16, 16, 32, 32, 48, 64))
    if kind == "map":
        batch = _near(rng, 1, 1024)
        return _map(None, batch, _near(rng, max(1, batch // 2), 131072), page, rng.choice((0, 100, 4096)), rng.random() < 0.3)
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "append":
        total = _near(rng, 1, 16384 if dtype == "f32" else 32768)
        return _append(None, _near(rng, 1, min(128, 2 * total)), rng.choice((1, 2, 4, 8)), total, page, dtype,
                       rng.choice((0, 100, 1000, 4000)), rng.random() < 0.6)
    heads = rng.choice(((8, 8), (16, 8), (32, 8), (32, 8), (64, 8), (8, 1), (4, 4), (3, 3), (10, 5)))
    over = rng.choice(("full", "heads", "group") if kind == "entmax" else ("full", "heads"))
    tokens = _near(rng, 1, 1 << 20)
    most = 7000000 if over == "full" else 4000000              # tokens times KV heads in the cache of a draw
    while tokens * heads[1] > most:
        tokens = tokens // 2 + 1
    batch = _near(rng, 1, max(1.0, min(64, most / (tokens * heads[1]))))
    stagger = 0 if batch == 1 or rng.random() < 0.3 else rng.randint(1, max(1, 3 * tokens // (2 * batch)))
    return _attention(None, kind, over, batch, heads, tokens, page, dtype, rng.choice((1.25, 1.5, 1.5, 2.0, 1.7)),
                      rng.choice((1.0, 1.0, 0.25)), rng.choice((0.01, 0.02, 0.0625, 0.25)), stagger)


# ---- sizes --------------------------------------------------------------------------------------------------------
def _shares(c):
    """New tokens per sequence: uneven, some without any where there are more sequences than tokens."""
    b, left = c["batch"], c["total"]
    if c["total"] <= b:
        return [1 if i < c["total"] else 0 for i in range(b)]
    w = [1.0 + (i * 7 % 5) / 2.0 for i in range(b)]
    n = [max(1, int((left - b) * x / sum(w))) for x in w]
    n[-1] += left - sum(n)
    return n


def _held(c):
    return [max(0, c["held"] - 61 * i % (c["held"] + 1)) if c["held"] else 0 for i in range(c["batch"])]


def _lens(c):
    return [max(0, c["tokens"] - b * c["stagger"]) for b in range(c["batch"])]


def _row_pages(c):
    """Length of a block table's row."""
    if c["kind"] in ("map", "append"):
        return max(-(-(h + n) // c["page"]) for h, n in zip(_held(c), _shares(c))) + 1
    return -(-c["tokens"] // c["page"])


def _list_pages(c):
    return max(1, math.ceil(c["budget"] * _row_pages(c)))


def work(case):
    c = case
    if c["kind"] == "map":
        pages = sum(-(-(h + n) // c["page"]) - -(-h // c["page"]) for h, n in zip(_held(c), _shares(c)))
        return {"bytes": 20 * c["batch"] + 16 * c["total"] + 8 * pages, "flops": 0}
    esz = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "append":
        fresh, partly, touched = c["total"], 0, 0
        for h, n in zip(_held(c), _shares(c)):
            if n:
                touched += -(-(h + n) // c["page"]) - h // c["page"]
                partly += h % c["page"]
        hk = c["kv_heads"]
        # new rows and their codes; the old keys of partly filled pages where statistics are wanted; scales
        return {"bytes": 2 * fresh * hk * D * (esz + 1) + 16 * fresh + touched * hk * (8 + (4 * D * esz if c["stats"] else 0))
                + (partly * hk * D if c["stats"] else 0), "flops": 0}
    hq, hk, p = c["q_heads"], c["kv_heads"], c["page"]
    if c["over"] == "full":
        rows = sum(_lens(c)) * hk
        scored = sum(_lens(c)) * hq
    else:
        lists = hk if c["over"] == "group" else hq
        rows = sum(min(_list_pages(c) * p, n) for n in _lens(c)) * lists
        scored = rows * (hq // hk if c["over"] == "group" else 1)
    io = c["batch"] * hq * D * (esz + 4)
    values = rows * D if c["kind"] == "softmax" else min(rows, 32 * c["batch"] * hq) * D    # entmax reads its support's rows
    return {"bytes": rows * D + rows // p * 8 + values + io, "flops": 2 * scored * D * (2 if c["kind"] == "softmax" else 1)}


# ---- inputs -------------------------------------------------------------------------------------------------------
def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _scale_for(amax):
    """The least power of two s with amax <= 448 s, kept in its range; amax finite, 0 for nothing."""
    m, e = torch.frexp(amax)                                       # amax = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875).to(e.dtype), torch.full_like(e, LOW)).clamp(LOW, HIGH)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes(x, s):
    """Codes of x / s: to nearest, ties to even; what is no finite number becomes the format's NaN."""
    c = (x / s).clamp(-MAX_CODE, MAX_CODE).to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(x.isfinite(), c, torch.full_like(c, 0x7F))


def _values(codes, s):
    return codes.view(torch.float8_e4m3fn).float() * s


def _quantised(x):
    """[pages, heads, P, D] -> codes and scales [pages, heads]."""
    s = _scale_for(x.abs().amax((-1, -2)))
    return _codes(x, s[..., None, None]), s


def _pools(c, n_phys, g, key_rows=None):
    """K and V pools of n_phys pages: ordinary keys with a few channels far from zero, as models have them.
    key_rows: (page, head, token, row [., D]) of keys that the queries look for."""
    hk, p = c["kv_heads"], c["page"]
    offs = torch.zeros(D, device="cuda")
    offs[torch.randperm(D, generator=g, device="cuda")[:4]] = 5.0
    pool = {}
    for name in ("k", "v"):
        code = torch.empty(n_phys, hk, p, D, dtype=torch.uint8, device="cuda")
        scale = torch.empty(n_phys, hk, device="cuda")
        step = max(1, (1 << 27) // (hk * p * D))
        for lo in range(0, n_phys, step):
            x = torch.randn(min(step, n_phys - lo), hk, p, D, generator=g, device="cuda")
            if name == "k":
                x += offs
                if key_rows is not None:
                    page, head, tok, row = key_rows
                    here = (page >= lo) & (page < lo + x.shape[0])
                    x[page[here] - lo, head[here], tok[here]] = row[here] + offs
            code[lo:lo + x.shape[0]], scale[lo:lo + x.shape[0]] = _quantised(x)
        pool[name + "_pool"], pool[name + "_scale"] = code, scale
    return pool


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    b_, p, m = c["batch"], c["page"], _row_pages(c)
    if c["kind"] in ("map", "append"):
        held, new = _held(c), _shares(c)
        have = [-(-n // p) for n in held]
        need = sum(-(-(h + n) // p) for h, n in zip(held, new)) - sum(have)
        n_phys = sum(have) + need + 5
        ids = torch.randperm(n_phys, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros(b_, m, dtype=torch.int32, device="cuda")
        mapped = torch.arange(m, device="cuda")[None, :] < _ints(have)[:, None]
        table[mapped] = ids[:sum(have)]
        n_free = (need * 3) // 4 if c.get("short") else need + 5
        s = dict(case=c, seq_lens=_ints(held), n_new=_ints(new), block_table=table, free_pages=ids[sum(have):].contiguous(),
                 n_free=_ints([n_free]), pages=need, total=c["total"])
        if c["kind"] == "append":
            dt, hk = _type(c), c["kv_heads"]
            s.update(_pools(c, n_phys, g))
            # the step's tokens as mapped: slots, sequences and positions of the packed rows
            seq = torch.repeat_interleave(torch.arange(b_, device="cuda"), _ints(new).long())
            first = (torch.cumsum(_ints(new), 0) - _ints(new)).long()
            pos = _ints(held).long()[seq] + torch.arange(c["total"], device="cuda") - first[seq]
            fresh = torch.arange(m, device="cuda")[None, :] < _ints([-(-(h + n) // p) for h, n in zip(held, new)])[:, None]
            table[fresh & ~mapped] = ids[sum(have):sum(have) + need]
            s["slots"] = table[seq, pos // p].long() * p + pos % p
            s["seq"], s["pos"] = seq.to(torch.int32), pos.to(torch.int32)
            s["runs"] = sum(-(-(h + n) // p) - h // p for h, n in zip(held, new) if n)
            # K and V are parts of one projection's rows; now and then a token is larger than what its page has seen
            rows = torch.randn(c["total"], 3, hk, D, generator=g, device="cuda")
            rows *= torch.where(torch.rand(c["total"], 1, 1, 1, generator=g, device="cuda") < 0.1, 4.0, 1.0)
            rows = rows.to(dt)
            s["k_new"], s["v_new"] = rows[:, 1], rows[:, 2]
            if c["stats"]:
                s["box"] = torch.zeros(b_, hk, m, 2, D, dtype=dt, device="cuda")
                s["gauss"] = torch.zeros_like(s["box"])
        if own:
            s.update(_held_by_a_program(s))
        return s
    hq, hk, lens = c["q_heads"], c["kv_heads"], _lens(c)
    q = torch.randn(b_, hq, D, generator=g, device="cuda").to(_type(c))
    n_phys = b_ * m
    table = torch.randperm(n_phys, generator=g, device="cuda").view(b_, m).to(torch.int32)
    # keys near the query's direction: 32 a head, the same number for every head of a group
    n_pl = 32
    at = (torch.rand(b_, hq, n_pl, generator=g, device="cuda") * _ints(lens)[:, None, None]).long()
    at = torch.minimum(at, _ints(lens)[:, None, None] - 1).clamp(min=0)
    qf = q.float()
    row = 3.0 * qf / qf.norm(dim=-1, keepdim=True)
    row = row[:, :, None] + 0.3 * torch.randn(b_, hq, n_pl, D, generator=g, device="cuda")
    page = torch.gather(table.long()[:, None].expand(b_, hq, m), 2, at // p)
    head = (torch.arange(hq, device="cuda") // (hq // hk))[None, :, None].expand_as(at)
    # of two queries that look for one place the first has it
    order = ((page * hk + head) * p + at % p).flatten()
    first = torch.full((n_phys * hk * p,), order.numel(), device="cuda").scatter_reduce(0, order, torch.arange(order.numel(), device="cuda"), "amin")
    mine = first[order] == torch.arange(order.numel(), device="cuda")
    pool = _pools(c, n_phys, g, (page.flatten()[mine], head.flatten()[mine], (at % p).flatten()[mine], row.flatten(0, 2)[mine]))
    s = dict(case=c, q=q, block_table=table, seq_lens=_ints(lens), scale=c["flat"] / math.sqrt(D), **pool)
    if c["over"] != "full":
        # lists as a selection leaves them: the pages of the planted keys first of all, then others, ascending
        lists, k = (hk if c["over"] == "group" else hq), _list_pages(c)
        score = torch.rand(b_, lists, m, generator=g, device="cuda")
        into = (at // p).view(b_, lists, -1)
        score.scatter_reduce_(2, into, 2.0 + torch.rand(into.shape, generator=g, device="cuda"), "amax")
        pages = _ints([-(-n // p) for n in lens])[:, None, None]
        score = torch.where(torch.arange(m, device="cuda") < pages, score, torch.full_like(score, -1.0))
        idx = score.topk(k, dim=-1).indices
        count = torch.minimum(pages, torch.full_like(pages, k))
        idx = torch.where(torch.arange(k, device="cuda") < count, idx, torch.full_like(idx, m)).sort(-1).values.clamp(max=m - 1)
        s["page_idx"], s["n_sel"] = idx.to(torch.int32), count[..., 0].expand(b_, lists).to(torch.int32).contiguous()
    if own:
        s.update(_held_by_a_program(s))
    return s


def _held_by_a_program(s):
    """Configuration, views, workspace and output buffers, which a program makes once and keeps."""
    from paper_2605_21649_amd import binding as ekv
    c = s["case"]
    f32, i32 = dict(device="cuda", dtype=torch.float32), dict(device="cuda", dtype=torch.int32)
    b_, m, hk = c["batch"], s["block_table"].shape[1], c.get("kv_heads", 1)
    hq = c.get("q_heads", hk)
    cap = s["page_idx"].shape[2] if "page_idx" in s else m
    h = {"ekv": ekv, "cfg": ekv.make_config(b_, hq, hk, D, c["page"], c.get("dtype", "bf16"), c.get("alpha", 1.5),
                                            s.get("scale", 1.0), m, cap)}
    if c["kind"] == "map":
        t = s["total"]
        h.update(slots=torch.empty(t, device="cuda", dtype=torch.int64), seq=torch.empty(t, **i32), pos=torch.empty(t, **i32),
                 start=torch.empty(b_ + 1, **i32), n_mapped=torch.empty(b_, **i32), new_lens=torch.empty(b_, **i32),
                 n_left=torch.empty(1, **i32))
        h["tokens"] = ekv.token_map(h["slots"], h["seq"], h["pos"], h["start"], h["n_mapped"])
        return h
    h["cache"] = ekv.cache8_view(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["block_table"], s["seq_lens"])
    if c["kind"] == "append":
        h["tokens"] = ekv.token_map(s["slots"], s["seq"], s["pos"])
        h["stats"] = ekv.stats_view(s["box"], s["gauss"]) if c["stats"] else None
        return h
    h.update(out=torch.empty(b_, hq, D, **f32), tau=torch.empty(b_, hq, **f32), supp=torch.empty(b_, hq, **i32))
    op = {("entmax", True): ekv.EKV_OP_DECODE_FULL, ("entmax", False): ekv.EKV_OP_DECODE_SPARSE,
          ("softmax", True): ekv.EKV_OP_DECODE8_FULL_SOFTMAX, ("softmax", False): ekv.EKV_OP_DECODE8_SPARSE_SOFTMAX}
    n = ekv.ekv_workspace_bytes(h["cfg"], op[c["kind"], c["over"] == "full"])
    h["ws"] = torch.empty(max(256, n), device="cuda", dtype=torch.uint8)
    return h


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(s):
    """The number of support tokens, which the last bit of one score moves by one, is not among the outputs of an entmax
    pass; its threshold and output show what it stands for.  Codes are returned as values of their 8-bit type, with the
    scales beside them."""
    return _own(s) if own else PLAIN[s["case"]["kind"]](s)


def _state_of(s):
    r = {k: s[k].view(torch.float8_e4m3fn) for k in ("k_pool", "v_pool")}
    r.update({k: s[k] for k in ("k_scale", "v_scale", "box", "gauss") if k in s})
    return r


def _own(s):
    c, ekv = s["case"], s["ekv"]
    if c["kind"] == "map":
        ekv.ekv_map_tokens(s["cfg"], s["seq_lens"], s["n_new"], s["block_table"], s["free_pages"], s["n_free"], s["tokens"],
                           s["new_lens"], s["n_left"])
        return {k: s[k] for k in ("block_table", "slots", "seq", "pos", "start", "n_mapped", "new_lens", "n_left")}
    if c["kind"] == "append":
        ekv.ekv_cache8_append(s["cfg"], s["cache"], s["stats"], s["tokens"], s["k_new"], s["v_new"])
        return _state_of(s)
    if c["kind"] == "softmax":
        if c["over"] == "full":
            ekv.ekv_decode8_full_softmax(s["cfg"], s["q"], s["cache"], s["out"], s["tau"], s["ws"])
        else:
            ekv.ekv_decode8_sparse_softmax(s["cfg"], s["q"], s["cache"], s["page_idx"], s["n_sel"], s["out"], s["tau"], s["ws"])
        return {"out": s["out"], "lse": s["tau"]}
    if c["over"] == "full":
        ekv.ekv_decode8_full(s["cfg"], s["q"], s["cache"], s["out"], s["tau"], s["supp"], s["ws"])
    else:
        call = ekv.ekv_decode8_sparse_group if c["over"] == "group" else ekv.ekv_decode8_sparse
        call(s["cfg"], s["q"], s["cache"], s["page_idx"], s["n_sel"], s["out"], s["tau"], s["supp"], s["ws"])
    return {"out": s["out"], "tau": s["tau"]}


def _plain_map(s):
    c, t = s["case"], s["total"]
    p, m, b_ = c["page"], s["block_table"].shape[1], c["batch"]
    n, new, free = s["seq_lens"].long(), s["n_new"].long().clamp(min=0), s["n_free"].long()
    ends = torch.cumsum(new, 0)
    start = torch.cat((torch.zeros_like(ends[:1]), ends))
    have = (n + p - 1) // p
    fits = (new > 0) & (n + new <= m * p) & (ends <= t)
    need = torch.where(fits, (n + new + p - 1) // p - have, 0)
    taken = torch.cumsum(need, 0)
    fits &= (need == 0) | (taken <= free)
    mapped = torch.where(fits, new, 0)
    i = torch.arange(t, device=n.device)
    b = torch.searchsorted(ends, i, right=True).clamp(max=b_ - 1)
    live = (i < ends[-1]) & fits[b]
    pos = torch.where(live, n[b] + i - start[b], 0)
    page = pos // p
    fresh = live & (page >= have[b])
    at = free - 1 - (taken[b] - need[b] + page - have[b])
    phys = torch.where(fresh, s["free_pages"].long()[at.clamp(0, s["free_pages"].numel() - 1)], s["block_table"].long()[b, page])
    table = torch.cat((s["block_table"].flatten(), torch.zeros_like(s["seq_lens"][:1])))     # one place for what is not written
    table[torch.where(fresh, b * m + page, b_ * m)] = phys.to(torch.int32)
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return {"block_table": table[:-1].view(b_, m), "slots": torch.where(live, phys * p + pos % p, -1), "seq": i32(torch.where(live, b, -1)),
            "pos": i32(torch.where(live, pos, -1)), "start": i32(start), "n_mapped": i32(mapped), "new_lens": i32(n + mapped),
            "n_left": i32(free - torch.where(fits, need, 0).sum())}


def _plain_append(s):
    c, r_ = s["case"], s["runs"]
    p, slots = c["page"], s["slots"]
    t = torch.arange(slots.numel(), device=slots.device)
    page, off = slots // p, slots % p
    begins = (off == 0) | (t == 0) | (slots != torch.cat((slots[:1], slots[:-1])) + 1)
    run_of = torch.cumsum(begins, 0) - 1
    to = torch.where(begins, run_of, r_)                            # one place for what begins nothing
    of_run = lambda v: torch.zeros(r_ + 1, dtype=torch.int64, device=v.device).scatter(0, to, v)[:-1]  # noqa: E731
    phys, kept, seq, lpage = of_run(page), of_run(off), of_run(s["seq"].long()), of_run(s["pos"].long() // p)
    count = kept + torch.zeros(r_, dtype=torch.int64, device=page.device).scatter_add(0, run_of, torch.ones_like(t))
    tok = torch.arange(p, device=page.device)
    old, valid = (tok < kept[:, None])[:, None, :, None], (tok < count[:, None])[:, None, :, None]
    for name in ("k", "v"):
        new, pool, scale = s[name + "_new"].float(), s[name + "_pool"], s[name + "_scale"]
        was, s_was = pool[phys], scale[phys]
        x = torch.where(old, _values(was, s_was[..., None, None]), 0.0)
        top = torch.zeros(r_, new.shape[1], device=new.device).scatter_reduce(
            0, run_of[:, None].expand(-1, new.shape[1]), torch.where(new.isfinite(), new.abs(), 0.0).amax(-1), "amax")
        s_now = _scale_for(top)
        s_now = torch.where(kept[:, None] > 0, torch.maximum(s_now, s_was), s_now)
        x[run_of, :, off] = new
        code = torch.where(valid, _codes(x, s_now[..., None, None]), was)
        pool[phys], scale[phys] = code, s_now
        if name == "k" and c["stats"]:
            x = _values(code, s_now[..., None, None])
            n = count[:, None, None].float()
            lo, hi = torch.where(valid, x, math.inf).amin(2), torch.where(valid, x, -math.inf).amax(2)
            mean = torch.where(valid, x, 0.0).sum(2) / n
            var = torch.where(valid, (x - mean[:, :, None]).square(), 0.0).sum(2) / n
            dt = s["box"].dtype
            s["box"][seq, :, lpage] = torch.stack((lo, hi), 2).to(dt)
            s["gauss"][seq, :, lpage] = torch.stack((mean, var), 2).to(dt)
    return _state_of(s)


def _candidates(s):
    """Keys and values [B, lists, n, D] that the pass looks at, and which of them count."""
    c = s["case"]
    p, hk, table, n = c["page"], c["kv_heads"], s["block_table"].long(), s["seq_lens"].long()
    if "page_idx" in s:
        idx = s["page_idx"].long()
        lists = idx.shape[1]
        head = (torch.arange(lists, device=idx.device) // (lists // hk))[None, :, None]
        phys = torch.gather(table[:, None].expand(-1, lists, -1), 2, idx)
        taken = torch.arange(idx.shape[2], device=idx.device) < s["n_sel"][..., None]
    else:
        head, phys = torch.arange(hk, device=table.device)[None, :, None], table[:, None]
        idx = torch.arange(table.shape[1], device=table.device)[None, None]
        taken = torch.ones_like(idx, dtype=torch.bool)
    tok = idx[..., None] * p + torch.arange(p, device=idx.device)
    counts = (taken[..., None] & (tok < n[:, None, None, None])).flatten(2)
    side = lambda x: _values(s[x + "_pool"][phys, head], s[x + "_scale"][phys, head][..., None, None]).flatten(2, 3)  # noqa: E731
    return side, counts


def _plain_scores(s, side, counts):
    c = s["case"]
    k = side("k")
    q = s["q"].float().view(c["batch"], k.shape[1], -1, D)
    return torch.where(counts[:, :, None], s["scale"] * (q @ k.transpose(-1, -2)), -math.inf)


def _plain_entmax(s):
    c = s["case"]
    a = c["alpha"] - 1.0
    beta = 1.0 / a
    side, counts = _candidates(s)
    z = _plain_scores(s, side, counts) * a
    top = z.amax(-1, keepdim=True)
    empty = top == -math.inf
    u = torch.where(empty, -math.inf, z - torch.where(empty, 0.0, top))
    t = torch.full_like(top, -1.0)
    for _ in range(24):                  # Newton's steps on the norm of (u - t)_+ from the left, where they stay
        x = (u - t).clamp(min=0.0)
        f = x.pow(beta).sum(-1, keepdim=True)
        slope = x.pow(beta - 1.0).mul_(x > 0).sum(-1, keepdim=True)
        r = f.pow(a)
        t = torch.where(empty, t, t + (r - 1.0).clamp(min=0.0) * f / (r * slope))
    w = (u - t).clamp(min=0.0).pow(beta)
    out = (w @ side("v")).reshape(c["batch"], c["q_heads"], D)
    return {"out": out, "tau": torch.where(empty, math.inf, t + top).reshape(c["batch"], c["q_heads"])}


def _plain_softmax(s):
    c = s["case"]
    side, counts = _candidates(s)
    z = _plain_scores(s, side, counts)
    top = z.amax(-1, keepdim=True)
    empty = top == -math.inf
    e = torch.where(empty, 0.0, torch.exp(z - torch.where(empty, 0.0, top)))
    total = e.sum(-1, keepdim=True)
    out = (e @ side("v")) / torch.where(empty, 1.0, total)
    return {"out": out.reshape(c["batch"], c["q_heads"], D), "lse": (top + torch.log(total)).reshape(c["batch"], c["q_heads"])}


PLAIN = {"map": _plain_map, "append": _plain_append, "entmax": _plain_entmax, "softmax": _plain_softmax}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _table64():
    """Values of the 256 codes: sign, 4 bits of exponent with bias 7, 3 of mantissa."""
    v = []
    for code in range(128):
        e, m = code >> 3, code & 7
        v.append(math.nan if code == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return torch.tensor(v + [-x for x in v], dtype=torch.float64, device="cuda")


def _two_to(e):
    """2^e for whole e, by its bits: a power function may be off in its last place."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round64(x):
    """x to the nearest value of the 8-bit format, ties to an even last place, not beyond +-448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -60)))
    e = torch.where(_two_to(e) > x.abs(), e - 1, e).clamp(min=-6)
    step = _two_to(e - 3)
    return (torch.round(x / step) * step).clamp(-MAX_CODE, MAX_CODE)


def exact(case, seed):
    if case["kind"] == "map":
        return None                                     # whole numbers alone
    s = prepare(case, seed)
    return _exact_append(s) if case["kind"] == "append" else _exact_attention(s)


def _exact_append(s):
    c, value = s["case"], _table64()
    p, total = c["page"], s["total"]
    slots, seq, pos = s["slots"].tolist(), s["seq"].tolist(), s["pos"].tolist()
    groups = []                                         # (page, first kept, rows lo..hi, sequence, logical page)
    for i in range(total):
        if i and slots[i] == slots[i - 1] + 1 and slots[i] % p:
            groups[-1][3] = i + 1
        else:
            groups.append([slots[i] // p, slots[i] % p, i, i + 1, seq[i], pos[i] // p])
    if len(groups) > 20000:
        return None
    r = {}
    stored = {}
    # a touched page at a time in whole-number arithmetic would take long: pages of one shape (kept, count) go together
    shapes = {}
    for gr in groups:
        shapes.setdefault((gr[1], gr[3] - gr[2]), []).append(gr)
    for name in ("k", "v"):
        code, scale, new = s[name + "_pool"], s[name + "_scale"].double(), s[name + "_new"].double()
        pool = value[code.int()]                        # codes as values, without the scales
        for (kept, count), grs in shapes.items():
            page = torch.tensor([gr[0] for gr in grs], device="cuda")
            lo = torch.tensor([gr[2] for gr in grs], device="cuda")
            x = new[lo[:, None] + torch.arange(count, device="cuda")].transpose(1, 2)      # [., heads, count, D]
            top = x.abs().amax((2, 3))
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -300) / MAX_CODE))
            e = torch.where(MAX_CODE * _two_to(e - 1) >= top, e - 1, torch.where(MAX_CODE * _two_to(e) < top, e + 1, e))
            sc = _two_to(e.clamp(LOW, HIGH))
            if kept:
                sc = torch.maximum(sc, scale[page])
                pool[page, :, :kept] = _round64(pool[page, :, :kept] * (scale[page] / sc)[..., None, None])
            pool[page, :, kept:kept + count] = _round64(x / sc[..., None, None])
            scale[page] = sc
            if name == "k" and c["stats"]:
                y = pool[page, :, :kept + count] * sc[..., None, None]
                mean = y.mean(2)
                stored[kept, count] = (torch.stack((y.amin(2), y.amax(2)), 2), torch.stack((mean, (y - mean[:, :, None]).square().mean(2)), 2))
        r[name + "_pool"], r[name + "_scale"] = pool, scale
    if c["stats"]:
        r["box"], r["gauss"] = s["box"].double(), s["gauss"].double()
        for key, grs in shapes.items():
            b, lp = (torch.tensor([gr[j] for gr in grs], device="cuda") for j in (4, 5))
            r["box"][b, :, lp], r["gauss"][b, :, lp] = stored[key]
    return r


def _exact_attention(s):
    c, value = s["case"], _table64()
    p, hq, hk = c["page"], c["q_heads"], c["kv_heads"]
    grp = hq // hk
    a = c["alpha"] - 1.0
    lens = s["seq_lens"].tolist()
    out = torch.zeros(c["batch"], hq, D, dtype=torch.float64, device="cuda")
    top = torch.full((c["batch"], hq), math.inf if c["kind"] == "entmax" else -math.inf, dtype=torch.float64, device="cuda")
    lists = s["page_idx"].shape[1] if "page_idx" in s else hk
    for b, n in enumerate(lens):
        for i in range(lists if n else 0):
            h, mine = i // (lists // hk), slice(i * (hq // lists), (i + 1) * (hq // lists))
            pages = torch.arange(-(-n // p), device="cuda") if "page_idx" not in s else s["page_idx"][b, i, :int(s["n_sel"][b, i])].long()
            tok = (pages[:, None] * p + torch.arange(p, device="cuda")).flatten()
            rows = s["block_table"][b].long()[pages]
            k, v = ((value[s[x + "_pool"][rows, h].int()] * s[x + "_scale"][rows, h].double()[:, None, None]).flatten(0, 1)[tok < n] for x in ("k", "v"))
            if not k.shape[0]:
                continue
            z = s["scale"] * (s["q"][b, mine].double() @ k.T)
            if c["kind"] == "softmax":
                out[b, mine], top[b, mine] = torch.softmax(z, -1) @ v, torch.logsumexp(z, -1)
                continue
            z = a * z
            hi = z.amax(-1, keepdim=True)
            lo = hi - 1.0
            near = (z > lo).any(0)                      # nothing below the largest score less one has any weight
            z, v = z[:, near], v[near]
            for _ in range(60):
                mid = 0.5 * (lo + hi)
                over = (z - mid).clamp(min=0.0).pow(1.0 / a).sum(-1, keepdim=True) >= 1.0
                lo, hi = torch.where(over, mid, lo), torch.where(over, hi, mid)
            w = (z - lo).clamp(min=0.0).pow(1.0 / a)
            out[b, mine], top[b, mine] = w @ v, lo[:, 0]
    return {"out": out, "tau" if c["kind"] == "entmax" else "lse": top}
