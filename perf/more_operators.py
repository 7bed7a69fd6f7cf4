"""A step of drafted tokens over the paged cache, as a serving program takes it: queries and keys of the drafted rows
normalised and rotated, attention of every sequence's tree of drafted tokens over its cache (16, 32 or 8 bits an element),
and the rows that were accepted appended to the cache.

Kinds of a pass:
  rotate    rows of a fused projection -> queries and keys, each head divided by its root mean square, weighted, and
            rotated by the angles of its row's position
  append    new K and V rows, taken in the order of a row index -> the pages that their slots name, page statistics
  tree      the drafted rows of every sequence attend to the cache ("full": every page, "heads": a page list per query
            head, "group": a list per KV head) and to the drafted rows that their masks name; form "entmax" or "softmax"

`own`: False computes the passes with elementary torch operations, True through the framework's entry points."""
import math

import torch

own = False

D = 128
MAX_CODE = 448.0                       # largest finite value of the 8-bit format (OCP E4M3)
LOW, HIGH = -100, 119                  # exponents a scale may have
EPS = 1e-6


def _case(name, kind, **kw):
    c = dict(kind=kind, **kw)
    return dict(c, name=name) if name else c


def _rotate(name, tokens, heads, dtype="bf16", turned=128, pairs=False, far=4096):
    """turned: channels of a head that are rotated.  pairs: neighbours are rotated, not halves.  far: largest position."""
    return _case(name, "rotate", tokens=tokens, q_heads=heads[0], kv_heads=heads[1], dtype=dtype, turned=turned, pairs=pairs,
                 far=far)


def _append(name, batch, kv_heads, total, page=16, dtype="bf16", held=1000, stats=True, picked=0):
    """total: new tokens of all sequences together, dealt unevenly.  held: tokens of the longest sequence before.
    picked: rows to pick the new tokens from by an index, in ascending stretches (0: the rows themselves)."""
    return _case(name, "append", batch=batch, kv_heads=kv_heads, total=total, page=page, dtype=dtype, held=held, stats=stats,
                 picked=picked)


def _tree(name, form, over, batch, heads, tokens, drafted, page=16, dtype="bf16", cache="same", alpha=1.5, budget=0.02,
          stagger=0, chain=False):
    """heads: (query heads, KV heads).  tokens: of the longest sequence, sequence b is b * stagger shorter, down to an empty
    one.  drafted: rows of the largest tree; the others have fewer, some none.  dtype: of queries and drafted rows, cache:
    "same" or "e4m3".  budget: share of the longest sequence's pages in a list.  chain: every row follows the one before."""
    return _case(name, "tree", form=form, over=over, batch=batch, q_heads=heads[0], kv_heads=heads[1], tokens=tokens,
                 drafted=drafted, page=page, dtype=dtype, cache=cache, alpha=alpha, budget=budget, stagger=stagger, chain=chain)


def listed():
    return [
        # a chain of a few drafted tokens of one sequence, float32, neighbours rotated in half of the channels: latency
        _rotate("rotate-5-f32", 5, (8, 8), dtype="f32", turned=64, pairs=True),
        # the drafted rows of a serving batch, sixteen sequences with trees of sixteen, far into a long context
        _rotate("rotate-256", 256, (32, 8), far=1048576),
        # prompts, 32K tokens together: bandwidth
        _rotate("rotate-prompts-32k", 32768, (32, 8), far=32768),
        # the accepted paths of 64 sequences, two or three rows each of trees of sixteen: latency
        _append("append-paths-64", 64, 8, 157, picked=1024),
        # chunks of prompts that go on in partly filled pages, float32 rows, an odd page size: bandwidth
        _append("append-chunks-16k-f32-p12", 7, 8, 16411, page=12, dtype="f32", held=777),
        # the smallest attention: a chain of five, one short sequence, no grouped heads, float32, a small alpha
        _tree("entmax-1x777-f32-p12", "entmax", "full", 1, (8, 8), 777, 5, page=12, dtype="f32", alpha=1.25, chain=True),
        # the framework's headline workload with a tree of sixteen: 2 % of a million tokens, a list per query head
        _tree("entmax-heads-1x1m", "entmax", "heads", 1, (32, 8), 1048576, 16),
        # a batch of chats on an 8-bit cache, lists shared per KV head, sparsemax; every length different
        _tree("entmax-group-64x8k-e4m3", "entmax", "group", 64, (32, 8), 8192, 8, cache="e4m3", alpha=2.0, budget=0.0625, stagger=37),
        # every page of four long sequences
        _tree("entmax-full-4x128k", "entmax", "full", 4, (32, 8), 131072, 16, stagger=9001),
        # softmax over everything with the largest trees: the most arithmetic
        _tree("softmax-full-8x32k-64", "softmax", "full", 8, (32, 8), 32768, 64, page=32, stagger=1009),
        # an ordinary batch, multi-query, on an 8-bit cache
        _tree("softmax-full-16x2k-e4m3", "softmax", "full", 16, (8, 1), 2049, 24, cache="e4m3", stagger=131),
        # softmax over a selection per query head
        _tree("softmax-heads-4x128k", "softmax", "heads", 4, (32, 8), 131072, 32, budget=0.04, stagger=9001),
    ]


def _near(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm, odd ones among them."""
    return max(1, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


HEADS = ((8, 8), (16, 8), (32, 8), (32, 8), (64, 8), (8, 1), (4, 4), (3, 3), (10, 5))


def draw(rng):
    kind = rng.choice(("rotate", "append", "tree", "tree", "tree", "tree"))
    page = rng.choice((4, 8, 12, 16, 16, 16, 32, 32, 48, 64))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "rotate":
        return _rotate(None, _near(rng, 1, 12288 if dtype == "f32" else 32768), rng.choice(HEADS), dtype,
                       rng.choice((128, 128, 64, 32, 96)), rng.random() < 0.4, _near(rng, 64, 1 << 20))
    if kind == "append":
        total = _near(rng, 1, 12288 if dtype == "f32" else 24576)
        batch = _near(rng, 1, min(128, 2 * total))
        return _append(None, batch, rng.choice((1, 2, 4, 8)), total, page, dtype, rng.choice((0, 100, 1000, 4000)),
                       rng.random() < 0.7, rng.choice((0, total + 3, 5 * total)))
    form = rng.choice(("entmax", "softmax"))
    heads, over = rng.choice(HEADS), rng.choice(("full", "heads", "group") if form == "entmax" else ("full", "heads"))
    cache = rng.choice(("same", "same", "e4m3"))
    drafted, tokens, budget = _near(rng, 1, 64), _near(rng, 1, 1 << 20), rng.choice((0.01, 0.02, 0.0625, 0.25))
    share = 1.0 if over == "full" else budget
    # keys of all caches together and scores of all rows together stay below the largest listed cases'
    keys = (3 << 20) // ((2 if dtype == "f32" and cache == "same" else 1) * (2 if form == "softmax" else 1))
    lists = heads[0] if over == "heads" else heads[1]
    cost = lambda b: max(b * tokens * max(heads[1], share * lists) / keys, b * tokens * share * heads[0] * drafted / 2.2e8)  # noqa: E731
    while cost(1) > 1:
        tokens, drafted = tokens // 2 + 1, max(1, drafted * 3 // 4)
    batch = _near(rng, 1, max(1.0, min(64, 1 / cost(1))))
    stagger = 0 if batch == 1 or rng.random() < 0.3 else rng.randint(1, max(1, 3 * tokens // (2 * batch)))
    return _tree(None, form, over, batch, heads, tokens, drafted, page, dtype, cache, rng.choice((1.25, 1.5, 1.5, 2.0, 1.7)),
                 budget, stagger, rng.random() < 0.3)


# ---- sizes --------------------------------------------------------------------------------------------------------
def _shares(c):
    """New tokens per sequence: uneven, some without any where there are more sequences than tokens."""
    b, left = c["batch"], c["total"]
    if left <= b:
        return [1 if i < left else 0 for i in range(b)]
    w = [1.0 + (i * 7 % 5) / 2.0 for i in range(b)]
    n = [max(1, int((left - b) * x / sum(w))) for x in w]
    n[-1] += left - sum(n)
    return n


def _held(c):
    return [max(0, c["held"] - 61 * i % (c["held"] + 1)) if c["held"] else 0 for i in range(c["batch"])]


def _lens(c):
    return [max(0, c["tokens"] - b * c["stagger"]) for b in range(c["batch"])]


def _trees(c):
    """Drafted rows per sequence: the first has the most, every seventh is idle."""
    return [0 if b % 7 == 5 else max(1, c["drafted"] - 3 * b % c["drafted"]) for b in range(c["batch"])]


def _row_pages(c):
    if c["kind"] == "append":
        return max(-(-(h + n) // c["page"]) for h, n in zip(_held(c), _shares(c))) + 1
    return -(-c["tokens"] // c["page"])


def _list_pages(c):
    return max(1, math.ceil(c["budget"] * _row_pages(c)))


def work(case):
    c = case
    esz = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rotate":
        heads = c["tokens"] * (c["q_heads"] + c["kv_heads"])
        return {"bytes": 2 * heads * D * esz + 4 * c["tokens"], "flops": 8 * heads * D}
    if c["kind"] == "append":
        touched = partly = 0
        for h, n in zip(_held(c), _shares(c)):
            if n:
                touched += -(-(h + n) // c["page"]) - h // c["page"]
                partly += h % c["page"]
        row = c["kv_heads"] * D * esz
        return {"bytes": 4 * c["total"] * row + (16 + (4 if c["picked"] else 0)) * c["total"]
                + ((4 * touched + partly) * row if c["stats"] else 0), "flops": 6 * c["total"] * c["kv_heads"] * D if c["stats"] else 0}
    hq, hk, lens, rows = c["q_heads"], c["kv_heads"], _lens(c), _trees(c)
    lists = hq if c["over"] == "heads" else hk
    most = max(lens) if c["over"] == "full" else _list_pages(c) * c["page"]
    keys = sum(min(most, n) for n, t in zip(lens, rows) if t) * lists
    scored = sum((min(most, n) + t) * t for n, t in zip(lens, rows)) * hq
    drafted = sum(rows)
    values = keys if c["form"] == "softmax" else min(keys, 32 * drafted * hq)       # entmax reads its support's rows
    esz_cache = 1 if c["cache"] == "e4m3" else esz
    io = drafted * (hq * D * (esz + 4) + 2 * hk * D * esz + 8)
    return {"bytes": (keys + values) * D * esz_cache + io, "flops": 2 * scored * D * (2 if c["form"] == "softmax" else 1)}


# ---- inputs -------------------------------------------------------------------------------------------------------
def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _scale_for(amax):
    """The least power of two s with amax <= 448 s, kept in its range; amax finite, 0 for nothing."""
    m, e = torch.frexp(amax)                                       # amax = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875).to(e.dtype), torch.full_like(e, LOW)).clamp(LOW, HIGH)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _values(codes, s):
    return codes.view(torch.float8_e4m3fn).float() * s


def _pools(c, n_phys, g, planted=None):
    """K and V pools: ordinary keys with a few channels far from zero, as models have them.  planted: (page, head, token,
    row [., D]) of keys that the queries look for."""
    hk, p, codes = c["kv_heads"], c["page"], c.get("cache") == "e4m3"
    offs = torch.zeros(D, device="cuda")
    offs[torch.randperm(D, generator=g, device="cuda")[:4]] = 5.0
    got = {"offs": offs}
    for name in ("k", "v"):
        pool = torch.empty(n_phys, hk, p, D, dtype=torch.uint8 if codes else _type(c), device="cuda")
        scale = torch.empty(n_phys, hk, device="cuda")
        step = max(1, (1 << 27) // (hk * p * D))
        for lo in range(0, n_phys, step):
            x = torch.randn(min(step, n_phys - lo), hk, p, D, generator=g, device="cuda")
            if name == "k":
                x += offs
                if planted is not None:
                    page, head, tok, row = planted
                    here = (page >= lo) & (page < lo + x.shape[0])
                    x[page[here] - lo, head[here], tok[here]] = row[here] + offs
            if codes:
                s = _scale_for(x.abs().amax((-1, -2)))
                scale[lo:lo + x.shape[0]] = s
                pool[lo:lo + x.shape[0]] = (x / s[..., None, None]).clamp(-MAX_CODE, MAX_CODE).to(torch.float8_e4m3fn).view(torch.uint8)
            else:
                pool[lo:lo + x.shape[0]] = x.to(pool.dtype)
        got[name + "_pool"] = pool
        if codes:
            got[name + "_scale"] = scale
    return got


def prepare(case, seed):
    s = {"rotate": _prepare_rotate, "append": _prepare_append, "tree": _prepare_tree}[case["kind"]](case, _generator(seed))
    if own:
        s.update(_held_by_a_program(s))
    return s


def _prepare_rotate(c, g):
    n, hq, hk, dt = c["tokens"], c["q_heads"], c["kv_heads"], _type(c)
    # queries and keys are parts of one projection's rows, with values behind them
    rows = torch.randn(n, hq + 2 * hk, D, generator=g, device="cuda")
    rows *= torch.exp(torch.randn(n, hq + 2 * hk, 1, generator=g, device="cuda"))
    rows = rows.to(dt)
    weight = lambda: (1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dt)  # noqa: E731
    freq = 10000.0 ** (-torch.arange(c["turned"] // 2, device="cuda", dtype=torch.float64) * 2.0 / c["turned"])
    return dict(case=c, x_q=rows[:, :hq], x_k=rows[:, hq:hq + hk], w_q=weight(), w_k=weight(), freq=freq.float(),
                pos=torch.randint(0, c["far"], (n,), generator=g, device="cuda", dtype=torch.int32))


def _prepare_append(c, g):
    b_, p, m, held, new = c["batch"], c["page"], _row_pages(c), _held(c), _shares(c)
    have, need = [-(-n // p) for n in held], [-(-(h + n) // p) for h, n in zip(held, new)]
    n_phys = sum(need) + 5
    table = torch.zeros(b_, m, dtype=torch.int32, device="cuda")
    at = torch.arange(m, device="cuda")[None, :] < _ints(need)[:, None]
    table[at] = torch.randperm(n_phys, generator=g, device="cuda").to(torch.int32)[:sum(need)]
    # the step's tokens as mapped: slots, sequences and positions
    seq = torch.repeat_interleave(torch.arange(b_, device="cuda"), _ints(new).long())
    first = (torch.cumsum(_ints(new), 0) - _ints(new)).long()
    pos = _ints(held).long()[seq] + torch.arange(c["total"], device="cuda") - first[seq]
    s = dict(case=c, slots=table[seq, pos // p].long() * p + pos % p, seq=seq.to(torch.int32), pos=pos.to(torch.int32),
             runs=sum(-(-(h + n) // p) - h // p for h, n in zip(held, new) if n), block_table=table)
    s.update(_pools(c, n_phys, g))
    n_rows = c["picked"] or c["total"]
    rows = torch.randn(n_rows, 3, c["kv_heads"], D, generator=g, device="cuda").to(_type(c))
    s["k_new"], s["v_new"] = rows[:, 1], rows[:, 2]                 # parts of one projection's rows
    if c["picked"]:
        s["rows"] = torch.randperm(n_rows, generator=g, device="cuda")[:c["total"]].sort().values.to(torch.int32)
    if c["stats"]:
        s["box"] = torch.zeros(b_, c["kv_heads"], m, 2, D, dtype=_type(c), device="cuda")
        s["gauss"] = torch.zeros_like(s["box"])
    return s


def _masks(c, trees, g):
    """Which drafted rows each row sees: itself and the rows it follows, as bits; a row follows the one before or, in a
    tree, one of the rows before."""
    n, pick, seen = sum(trees), torch.rand(sum(trees), generator=g, device="cuda").tolist(), []
    for t in trees:
        at = len(seen)
        for i in range(t):
            parent = i - 1 if c["chain"] or i == 0 else int(pick[at + i] * i)
            seen.append((1 << i) | (seen[at + parent] if i else 0))
    signed = [v - (1 << 64) if v >> 63 else v for v in seen]
    return torch.tensor(signed, dtype=torch.int64, device="cuda").view(n)


def _prepare_tree(c, g):
    b_, p, m, hq, hk, lens, trees = c["batch"], c["page"], _row_pages(c), c["q_heads"], c["kv_heads"], _lens(c), _trees(c)
    n, grp = sum(trees), hq // hk
    q = torch.randn(n, hq, D, generator=g, device="cuda").to(_type(c))
    seq = torch.repeat_interleave(torch.arange(b_, device="cuda"), _ints(trees).long())
    table = torch.randperm(b_ * m, generator=g, device="cuda").view(b_, m).to(torch.int32)
    # keys near the query's direction, a few for every row and head
    n_pl, long = 8, _ints(lens).long()[seq][:, None, None]
    at = torch.minimum((torch.rand(n, hq, n_pl, generator=g, device="cuda") * long).long(), long - 1).clamp(min=0)
    qf = q.float()
    near = 3.0 * qf / qf.norm(dim=-1, keepdim=True)
    row = near[:, :, None] + 0.3 * torch.randn(n, hq, n_pl, D, generator=g, device="cuda")
    page = table.long()[seq[:, None, None], at // p]
    head = (torch.arange(hq, device="cuda") // grp)[None, :, None].expand_as(at)
    # of two queries that look for one place the first has it
    place = ((page * hk + head) * p + at % p).flatten()
    order = torch.arange(place.numel(), device="cuda")
    first = torch.full((b_ * m * hk * p,), place.numel(), device="cuda").scatter_reduce(0, place, order, "amin")
    mine = first[place] == order
    s = dict(case=c, q=q, block_table=table, seq_lens=_ints(lens), scale=1.0 / math.sqrt(D), seq=seq, visible=_masks(c, trees, g),
             start=_ints([sum(trees[:b]) for b in range(b_ + 1)]), rows=n, most=max(trees + [1]))
    s.update(_pools(c, b_ * m, g, (page.flatten()[mine], head.flatten()[mine], (at % p).flatten()[mine], row.flatten(0, 2)[mine])))
    # drafted keys, now and then one near its own query; parts of one projection's rows
    rows = torch.randn(n, 3, hk, D, generator=g, device="cuda")
    rows[:, 1] = torch.where(torch.rand(n, 1, 1, generator=g, device="cuda") < 0.25, near[:, ::grp], rows[:, 1]) + s.pop("offs")
    rows = rows.to(_type(c))
    s["k_new"], s["v_new"] = rows[:, 1], rows[:, 2]
    if c["over"] != "full":
        # lists as a selection leaves them: the pages of the planted keys first of all, then others, ascending
        lists, k = (hk if c["over"] == "group" else hq), _list_pages(c)
        score = torch.rand(b_, lists, m, generator=g, device="cuda")
        into = (torch.arange(lists, device="cuda")[None, :, None] * m + (at // p).view(n, lists, -1) + seq[:, None, None] * lists * m).flatten()
        score.view(-1).scatter_reduce_(0, into, 2.0 + torch.rand(into.shape, generator=g, device="cuda"), "amax")
        pages = _ints([-(-x // p) for x in lens])[:, None, None]
        score = torch.where(torch.arange(m, device="cuda") < pages, score, torch.full_like(score, -1.0))
        idx = score.topk(k, dim=-1).indices
        count = torch.minimum(pages, torch.full_like(pages, k))
        idx = torch.where(torch.arange(k, device="cuda") < count, idx, torch.full_like(idx, m)).sort(-1).values.clamp(max=m - 1)
        s["page_idx"], s["n_sel"] = idx.to(torch.int32), count[..., 0].expand(b_, lists).to(torch.int32).contiguous()
    return s


def _held_by_a_program(s):
    """Configuration, views, workspace and output buffers, which a program makes once and keeps."""
    from paper_2605_21649_amd import binding as ekv
    c = s["case"]
    f32 = dict(device="cuda", dtype=torch.float32)
    m = s["block_table"].shape[1] if "block_table" in s else 1
    cap = s["page_idx"].shape[2] if "page_idx" in s else m
    h = {"ekv": ekv, "cfg": ekv.make_config(c.get("batch", 1), c.get("q_heads", c["kv_heads"]), c["kv_heads"], D, c.get("page", 16), c["dtype"],
                                            c.get("alpha", 1.5), s.get("scale", 1.0), m, cap)}
    if c["kind"] == "rotate":
        h.update(q_out=torch.empty(c["tokens"], c["q_heads"], D, device="cuda", dtype=_type(c)),
                 k_out=torch.empty(c["tokens"], c["kv_heads"], D, device="cuda", dtype=_type(c)))
        return h
    if c["kind"] == "append":
        h["cache"] = ekv.cache_view(s["k_pool"], s["v_pool"], s["block_table"], torch.zeros_like(s["block_table"][:, 0]).contiguous())
        h["tokens"] = ekv.token_map(s["slots"], s["seq"], s["pos"])
        h["stats"] = ekv.stats_view(s["box"], s["gauss"]) if c["stats"] else None
        return h
    n, hq, codes = s["rows"], c["q_heads"], c["cache"] == "e4m3"
    if codes:
        h["cache"] = ekv.cache8_view(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["block_table"], s["seq_lens"])
    else:
        h["cache"] = ekv.cache_view(s["k_pool"], s["v_pool"], s["block_table"], s["seq_lens"])
    h["tree"] = ekv.tree_view(s["start"], s["visible"], s["k_new"], s["v_new"], s["most"])
    h.update(out=torch.empty(n, hq, D, **f32), norm=torch.empty(n, hq, **f32), supp=torch.empty(n, hq, device="cuda", dtype=torch.int32))
    op = {("entmax", True): ekv.EKV_OP_TREE_FULL, ("entmax", False): ekv.EKV_OP_TREE_SPARSE,
          ("softmax", True): ekv.EKV_OP_TREE_FULL_SOFTMAX, ("softmax", False): ekv.EKV_OP_TREE_SPARSE_SOFTMAX}
    size = ekv.ekv_tree_workspace_bytes(h["cfg"], op[c["form"], c["over"] == "full"], n, s["most"])
    h["ws"] = torch.empty(max(256, size), device="cuda", dtype=torch.uint8)
    name = "ekv_tree8_" if codes else "ekv_tree_"
    name += {"full": "full", "heads": "sparse", "group": "sparse_group"}[c["over"]] + ("_softmax" if c["form"] == "softmax" else "")
    h["call"] = getattr(ekv, name)
    return h


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(s):
    """The number of support tokens, which the last bit of one score moves by one, is not among the outputs of an entmax
    pass; its threshold and output show what it stands for."""
    return _own(s) if own else PLAIN[s["case"]["kind"]](s)


def _own(s):
    c, ekv = s["case"], s["ekv"]
    if c["kind"] == "rotate":
        ekv.ekv_norm_rotate(s["cfg"], s["x_q"], s["x_k"], s["w_q"], s["w_k"], EPS, s["freq"], s["pos"], s["q_out"], s["k_out"], pairs=c["pairs"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "append":
        ekv.ekv_cache_append(s["cfg"], s["cache"], s["stats"], s["tokens"], s["k_new"], s["v_new"], rows=s.get("rows"))
        return {k: s[k] for k in ("k_pool", "v_pool", "box", "gauss") if k in s}
    lists = () if c["over"] == "full" else (s["page_idx"], s["n_sel"])
    if c["form"] == "softmax":
        s["call"](s["cfg"], s["q"], s["cache"], s["tree"], *lists, s["out"], s["norm"], s["ws"])
        return {"out": s["out"], "lse": s["norm"]}
    s["call"](s["cfg"], s["q"], s["cache"], s["tree"], *lists, s["out"], s["norm"], s["supp"], s["ws"])
    return {"out": s["out"], "tau": s["norm"]}


def _plain_rotate(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * s["freq"].double()
    cos, sin, r = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None], c["turned"]
    turned = lambda x: _turn(x, cos, sin, r, c["pairs"])  # noqa: E731
    head = lambda x, w: (x.float() / torch.sqrt(x.float().square().mean(-1, keepdim=True) + EPS)) * w.float()  # noqa: E731
    return {"q": turned(head(s["x_q"], s["w_q"])).to(_type(c)), "k": turned(head(s["x_k"], s["w_k"])).to(_type(c))}


def _turn(x, cos, sin, r, pairs):
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if pairs else (x[..., :r // 2], x[..., r // 2:r])
    u, v = a * cos - b * sin, b * cos + a * sin
    t = torch.stack((u, v), -1).flatten(-2) if pairs else torch.cat((u, v), -1)
    return torch.cat((t, x[..., r:]), -1)


def _plain_append(s):
    c, slots, p = s["case"], s["slots"], s["case"]["page"]
    k, v = (s[x + "_new"][s["rows"].long()] if "rows" in s else s[x + "_new"] for x in ("k", "v"))
    page, off = slots // p, slots % p
    s["k_pool"][page, :, off] = k
    s["v_pool"][page, :, off] = v
    if c["stats"]:
        # the last row that a page gets says how many tokens it has: one place for the others
        t = torch.arange(slots.numel(), device=slots.device)
        goes_on = torch.cat((slots[1:], slots[-1:])) == slots + 1
        ends = ~goes_on | (off == p - 1) | (t == slots.numel() - 1)
        run = torch.cumsum(ends, 0) - ends.long()
        to = torch.where(ends, run, s["runs"])
        of_run = lambda x: torch.zeros(s["runs"] + 1, dtype=torch.int64, device=x.device).scatter(0, to, x)[:-1]  # noqa: E731
        phys, count, seq, lpage = of_run(page), of_run(off) + 1, of_run(s["seq"].long()), of_run(s["pos"].long() // p)
        x = s["k_pool"][phys].float()
        valid = (torch.arange(p, device=x.device) < count[:, None])[:, None, :, None]
        n = count[:, None, None].float()
        mean = torch.where(valid, x, 0.0).sum(2) / n
        var = torch.where(valid, (x - mean[:, :, None]).square(), 0.0).sum(2) / n
        lo, hi = torch.where(valid, x, math.inf).amin(2), torch.where(valid, x, -math.inf).amax(2)
        s["box"][seq, :, lpage] = torch.stack((lo, hi), 2).to(s["box"].dtype)
        s["gauss"][seq, :, lpage] = torch.stack((mean, var), 2).to(s["box"].dtype)
    return {k: s[k] for k in ("k_pool", "v_pool", "box", "gauss") if k in s}


def _plain_tree(s):
    """Scores [B, lists, rows of a tree times heads of a list, keys], the sequences' rows padded to the largest tree."""
    c = s["case"]
    p, hq, hk, b_, t = c["page"], c["q_heads"], c["kv_heads"], c["batch"], s["most"]
    table, n, start = s["block_table"].long(), s["seq_lens"].long(), s["start"].long()
    dev = table.device
    lists = hq if c["over"] == "heads" else hk
    idx = s["page_idx"].long() if "page_idx" in s else torch.arange(table.shape[1], device=dev)[None, None]
    kv = (torch.arange(lists, device=dev) // (lists // hk))[None, :, None]
    phys = torch.gather(table[:, None].expand(-1, lists, -1), 2, idx) if "page_idx" in s else table[:, None]
    counts = (idx[..., None] * p + torch.arange(p, device=dev)) < n[:, None, None, None]
    if "n_sel" in s:
        counts &= (torch.arange(idx.shape[2], device=dev) < s["n_sel"][..., None])[..., None]
    row = torch.arange(t, device=dev)
    live = row < (start[1:] - start[:-1])[:, None]                              # [B, t]
    at = torch.where(live, start[:-1, None] + row, 0)
    seen = ((s["visible"][at][..., None] >> row) & 1).bool() & live[:, :, None] & live[:, None]      # [B, t, t]

    def side(x):
        pool = s[x + "_pool"][phys, kv]
        pool = _values(pool, s[x + "_scale"][phys, kv][..., None, None]) if c["cache"] == "e4m3" else pool.float()
        new = torch.where(live[..., None, None], s[x + "_new"][at].float(), 0.0)[:, :, kv[0, :, 0]].transpose(1, 2)
        return torch.cat((pool.flatten(2, 3).expand(b_, -1, -1, -1), new), 2)

    q = s["q"][at].float().view(b_, t, lists, -1, D).transpose(1, 2).reshape(b_, lists, -1, D)
    may = torch.cat((counts.flatten(2)[:, :, None].expand(b_, lists, t, -1), seen[:, None].expand(-1, lists, -1, -1)), 3)
    may = may.repeat_interleave(hq // lists, 2)
    z = torch.where(may, s["scale"] * (q @ side("k").transpose(-1, -2)), -math.inf)
    del may
    top, w, norm = _weights_entmax(z, c["alpha"]) if c["form"] == "entmax" else _weights_softmax(z)
    rows = lambda x: x.reshape(b_, lists, t, hq // lists, -1).transpose(1, 2).reshape(b_, t, hq, -1)[live]  # noqa: E731
    return {"out": rows(w @ side("v")), ("tau" if c["form"] == "entmax" else "lse"): rows(norm)[..., 0]}


def _weights_entmax(z, alpha):
    a = alpha - 1.0
    beta = 1.0 / a
    z *= a
    top = z.amax(-1, keepdim=True)
    empty = top == -math.inf
    u = torch.where(empty, -math.inf, z - torch.where(empty, 0.0, top))
    t = torch.full_like(top, -1.0)
    for _ in range(24):                  # Newton's steps on the norm of (u - t)_+ from the left, where they stay
        x = (u - t).clamp(min=0.0)
        slope = x.pow(beta - 1.0).mul_(x > 0).sum(-1, keepdim=True)
        f = x.pow_(beta).sum(-1, keepdim=True)
        r = f.pow(a)
        t = torch.where(empty, t, t + (r - 1.0).clamp(min=0.0) * f / (r * slope))
    return top, (u - t).clamp_(min=0.0).pow_(beta), torch.where(empty, math.inf, t + top)


def _weights_softmax(z):
    top = z.amax(-1, keepdim=True)
    empty = top == -math.inf
    e = torch.where(empty, 0.0, torch.exp(z - torch.where(empty, 0.0, top)))
    total = e.sum(-1, keepdim=True)
    return top, e / torch.where(empty, 1.0, total), top + torch.log(total)


PLAIN = {"rotate": _plain_rotate, "append": _plain_append, "tree": _plain_tree}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "tree": _exact_tree}[case["kind"]](s)


def _exact_rotate(s):
    c, got = s["case"], {}
    turns = s["pos"].double()[:, None] * s["freq"].double()
    unit = torch.polar(torch.ones_like(turns), turns)[:, None]
    for name in ("q", "k"):
        x = s["x_" + name].double()
        y = x * torch.rsqrt(x.square().sum(-1, keepdim=True) / D + EPS) * s["w_" + name].double()
        r = c["turned"]
        if c["pairs"]:
            y[..., :r] = torch.view_as_real(torch.view_as_complex(y[..., :r].reshape(*y.shape[:2], r // 2, 2).contiguous()) * unit).flatten(-2)
        else:
            z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * unit
            y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
        got[name] = y
    return got


def _exact_append(s):
    c = s["case"]
    hk, p = c["kv_heads"], c["page"]
    got = {}
    for name in ("k", "v"):
        flat = s[name + "_pool"].double().transpose(1, 2).reshape(-1, hk, D)      # a row for every slot
        new = s[name + "_new"].double()
        flat[s["slots"]] = new.index_select(0, s["rows"].long()) if "rows" in s else new
        got[name + "_pool"] = flat.view(-1, p, hk, D).transpose(1, 2)
    if c["stats"]:
        got["box"], got["gauss"] = s["box"].double(), s["gauss"].double()
        lens = [h + n for h, n in zip(_held(c), _shares(c))]
        for b, (h, n) in enumerate(zip(_held(c), _shares(c))):
            if not n:
                continue
            # whole pages together, the last one by itself
            first, whole = h // p, lens[b] // p
            rows = got["k_pool"][s["block_table"][b].long()]                      # [m, heads, P, D]
            for lo, hi, cnt in ((first, whole, p), (whole, whole + 1, lens[b] % p)):
                if lo < hi and cnt:
                    x = rows[lo:hi, :, :cnt]
                    mean = x.mean(2)
                    got["box"][b, :, lo:hi] = torch.stack((x.amin(2), x.amax(2)), 2).transpose(0, 1)
                    got["gauss"][b, :, lo:hi] = torch.stack((mean, (x - mean[:, :, None]).square().mean(2)), 2).transpose(0, 1)
    return got


def _table64():
    """Values of the 256 codes: sign, 4 bits of exponent with bias 7, 3 of mantissa."""
    v = []
    for code in range(128):
        e, m = code >> 3, code & 7
        v.append(math.nan if code == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return torch.tensor(v + [-x for x in v], dtype=torch.float64, device="cuda")


def _exact_tree(s):
    c, value = s["case"], _table64()
    p, hq, hk, a = c["page"], c["q_heads"], c["kv_heads"], c["alpha"] - 1.0
    lens, start = s["seq_lens"].tolist(), s["start"].tolist()
    out = torch.zeros(s["rows"], hq, D, dtype=torch.float64, device="cuda")
    norm = torch.full((s["rows"], hq), math.inf if c["form"] == "entmax" else -math.inf, dtype=torch.float64, device="cuda")
    lists = hq if c["over"] == "heads" else hk
    for b, n in enumerate(lens):
        r0, r1 = start[b], start[b + 1]
        t = r1 - r0
        bit = torch.arange(t, device="cuda")
        seen = ((s["visible"][r0:r1, None] >> bit) & 1).bool()
        for i in range(lists if t else 0):
            h, mine = i // (lists // hk), slice(i * (hq // lists), (i + 1) * (hq // lists))
            pages = torch.arange(-(-n // p), device="cuda") if "page_idx" not in s else s["page_idx"][b, i, :int(s["n_sel"][b, i])].long()
            tok = (pages[:, None] * p + torch.arange(p, device="cuda")).flatten()
            rows = s["block_table"][b].long()[pages]
            sides = []
            for x in ("k", "v"):
                kept = s[x + "_pool"][rows, h]
                kept = value[kept.int()] * s[x + "_scale"][rows, h].double()[:, None, None] if c["cache"] == "e4m3" else kept.double()
                sides.append(torch.cat((kept.flatten(0, 1)[tok < n], s[x + "_new"][r0:r1, h].double())))
            k, v = sides
            z = s["scale"] * (s["q"][r0:r1, mine].double() @ k.T)                 # [t, heads, keys]
            z[..., k.shape[0] - t:].masked_fill_(~seen[:, None], -math.inf)
            if c["form"] == "softmax":
                out[r0:r1, mine], norm[r0:r1, mine] = torch.softmax(z, -1) @ v, torch.logsumexp(z, -1)
                continue
            z = a * z
            hi = z.amax(-1, keepdim=True)
            lo = hi - 1.0
            near = (z > lo).flatten(0, 1).any(0)        # nothing below the largest score less one has any weight
            z, v = z[..., near], v[near]
            for _ in range(60):
                mid = 0.5 * (lo + hi)
                over = (z - mid).clamp(min=0.0).pow(1.0 / a).sum(-1, keepdim=True) >= 1.0
                lo, hi = torch.where(over, mid, lo), torch.where(over, hi, mid)
            out[r0:r1, mine], norm[r0:r1, mine] = (z - lo).clamp(min=0.0).pow(1.0 / a) @ v, lo[..., 0]
    return {"out": out, "tau" if c["form"] == "entmax" else "lse": norm}
