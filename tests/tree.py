"""Drafted rows over a paged cache: inputs on the host, the definition in 64 bits with limits of the kernels' rounding, and the call."""
import math

import torch

from paper_2605_21649_amd import binding as ekv

D = 128
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def quantised(x):
    """Codes and power-of-two scales of pages [n, heads, P, D]."""
    top = x.abs().amax((-1, -2)).clamp(min=1e-20)
    s = 2.0 ** torch.ceil(torch.log2(top / 448))
    return (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8), s.float()


class Tree:
    """lens: tokens of the cached sequences, trees: drafted rows.  over: "full", "heads" or "group"; chosen: share of the pages in a list."""

    def __init__(self, lens, trees, heads=(4, 2), page=16, dtype="bf16", cache="same", alpha=1.5, over="full", chosen=0.4, seed=0,
                 scale=1 / math.sqrt(D), extra_rows=0, max_tree=None, pool_heads=None, extra_pages=0, masks="tree"):
        g = self.g = torch.Generator().manual_seed(seed)
        self.lens, self.trees, self.page, self.dt, self.dtype = lens, trees, page, TYPE[dtype], dtype
        self.hq, self.hk, self.cache, self.alpha, self.over, self.scale = *heads, cache, alpha, over, scale
        self.b, self.grp, self.n = len(lens), heads[0] // heads[1], sum(trees) + extra_rows
        self.pool_heads = pool_heads or self.hk
        need = [-(-x // page) for x in lens]
        self.m = max(need + [1]) + extra_pages
        self.n_phys = sum(need) + 2
        ids = torch.randperm(self.n_phys, generator=g)
        self.table = torch.full((self.b, self.m), -5, dtype=torch.int32)
        at = 0
        for i, x in enumerate(need):
            self.table[i, :x] = ids[at:at + x].int()
            at += x
        shape = (self.n_phys, self.pool_heads, page, D)
        k, v = torch.randn(*shape, generator=g), torch.randn(*shape, generator=g)
        k[..., :4] += 3.0
        rows = torch.randn(self.n, 3, self.hk, D, generator=g)
        rows[:, 1, :, :4] += 3.0
        self.q = (1.5 * torch.randn(self.n, self.hq, D, generator=g)).to(self.dt)
        if self.n:                                            # some drafted keys near a query
            rows[::3, 1] += self.q[::3, ::self.grp].float() / 4
        rows = rows.to(self.dt)
        self.k_new, self.v_new = rows[:, 1], rows[:, 2]
        self.start = torch.tensor([sum(trees[:i]) for i in range(self.b + 1)], dtype=torch.int32)
        self.max_tree = max_tree or max(trees + [1])
        self.visible = torch.zeros(self.n, dtype=torch.int64)
        for i, t in enumerate(trees):
            seen = []
            for r in range(t):
                if masks == "any":                            # none among them
                    bits = int(torch.randint(0, 1 << 62, (), generator=g)) & int(torch.randint(0, 1 << 62, (), generator=g)) if r % 3 else 0
                    bits |= -1 << 64 if r % 5 == 4 else 0     # bits beyond the tree's rows too
                    seen.append(bits & ((1 << 64) - 1))
                else:
                    parent = r - 1 if masks == "chain" else int(torch.randint(0, max(r, 1), (), generator=g))
                    seen.append((1 << r) | (seen[parent] if r else 0))
                x = seen[r]
                self.visible[int(self.start[i]) + r] = x - (1 << 64) if x >> 63 else x
        if cache == "e4m3":
            (self.k, self.ks), (self.v, self.vs) = quantised(k), quantised(v)
            self.values = [c.view(torch.float8_e4m3fn).double() * s.double()[..., None, None] for c, s in ((self.k, self.ks), (self.v, self.vs))]
        else:
            self.k, self.v = k.to(self.dt), v.to(self.dt)
            self.values = [self.k.double(), self.v.double()]
        self.lists = {"full": self.hk, "heads": self.hq, "group": self.hk}[over]
        self.cap, self.page_idx, self.n_sel = self.m, None, None
        if over != "full":
            self.cap = min(self.m, max(1, math.ceil(chosen * self.m)) + 1)
            self.page_idx = torch.full((self.b, self.lists, self.cap), 1 << 30, dtype=torch.int32)
            self.n_sel = torch.zeros(self.b, self.lists, dtype=torch.int32)
            for i in range(self.b):
                for h in range(self.lists):
                    n = min(need[i], max(0, self.cap - h % 2))
                    self.page_idx[i, h, :n] = torch.randperm(need[i], generator=g)[:n].sort().values.int() if need[i] else 0
                    self.n_sel[i, h] = n

    def keys_of(self, b, h):
        """(keys, values) of the cache that list h of sequence b holds, in 64 bits."""
        n, p = self.lens[b], self.page
        pages = range(-(-n // p)) if self.over == "full" else self.page_idx[b, h, :int(self.n_sel[b, h])].tolist()
        hkv = h // (self.lists // self.hk)
        k, v = [], []
        for lp in pages:
            ph, cnt = int(self.table[b, lp]), min(p, n - lp * p)
            k.append(self.values[0][ph, hkv, :cnt])
            v.append(self.values[1][ph, hkv, :cnt])
        none = torch.zeros(0, D, dtype=torch.float64)
        return torch.cat(k + [none]), torch.cat(v + [none])

    def device(self, form):
        put = lambda t: t.cuda() if t is not None else None  # noqa: E731
        d = {x: put(getattr(self, x)) for x in ("k", "v", "ks", "vs", "table", "start", "visible", "q", "page_idx", "n_sel") if hasattr(self, x)}
        d["lens"] = torch.tensor(self.lens, dtype=torch.int32).cuda()
        rows = torch.zeros(self.n, 3, self.hk, D, dtype=self.dt)             # parts of a fused projection
        rows[:, 1], rows[:, 2] = self.k_new, self.v_new
        d["rows"] = rows.cuda()
        self.cfg = ekv.make_config(self.b, self.hq, self.hk, D, self.page, self.dtype, self.alpha, self.scale, self.m, self.cap, self.pool_heads)
        if self.cache == "e4m3":
            d["cache"] = ekv.cache8_view(d["k"], d["v"], d["ks"], d["vs"], d["table"], d["lens"])
        else:
            d["cache"] = ekv.cache_view(d["k"], d["v"], d["table"], d["lens"])
        d["tree"] = ekv.tree_view(d["start"], d["visible"], d["rows"][:, 1], d["rows"][:, 2], self.max_tree)
        op = {("entmax", True): ekv.EKV_OP_TREE_FULL, ("entmax", False): ekv.EKV_OP_TREE_SPARSE, ("softmax", True): ekv.EKV_OP_TREE_FULL_SOFTMAX,
              ("softmax", False): ekv.EKV_OP_TREE_SPARSE_SOFTMAX}[form, self.over == "full"]
        size = ekv.ekv_tree_workspace_bytes(self.cfg, op, self.n, self.max_tree)
        d["ws"] = torch.full((size,), 255, dtype=torch.uint8, device="cuda")     # NaN to whoever reads what was not written
        d["out"] = torch.full((self.n, self.hq, D), 77.0, device="cuda")
        d["norm"] = torch.full((self.n, self.hq), 77.0, device="cuda")
        d["supp"] = torch.full((self.n, self.hq), 77, dtype=torch.int32, device="cuda")
        return d

    def name(self, form):
        return ("ekv_tree8_" if self.cache == "e4m3" else "ekv_tree_") + {"full": "full", "heads": "sparse", "group": "sparse_group"}[self.over] + \
            ("_softmax" if form == "softmax" else "")

    def call(self, d, form, stream=None):
        lists = () if self.over == "full" else (d["page_idx"], d["n_sel"])
        outs = (d["out"], d["norm"]) + ((d["supp"],) if form == "entmax" else ())
        getattr(ekv, self.name(form))(self.cfg, d["q"], d["cache"], d["tree"], *lists, *outs, d["ws"], stream=stream)

    def run(self, form):
        d = self.device(form)
        self.call(d, form)
        torch.cuda.synchronize()
        return d["out"].cpu(), d["norm"].cpu(), d["supp"].cpu()

    def check(self, form, got, rows_of=None):
        out, norm, supp = got
        a = self.alpha - 1.0
        beta = 1.0 / a
        u = 2.0 ** -24
        taken = torch.zeros(self.n, dtype=torch.bool)
        for b in range(self.b):
            t = min(self.trees[b], self.max_tree)
            r0 = int(self.start[b])
            taken[r0:r0 + t] = True
            for h in range(self.lists if t else 0):
                kc, vc = self.keys_of(b, h)
                n = kc.shape[0]
                hkv = h // (self.lists // self.hk)
                k, v = (torch.cat((x, new[r0:r0 + t, hkv].double())) for x, new in ((kc, self.k_new), (vc, self.v_new)))
                for hq in range(h * self.hq // self.lists, (h + 1) * self.hq // self.lists):
                    for r in range(t):
                        at = (r0 + r, hq)
                        bits = int(self.visible[r0 + r])
                        seen = torch.tensor([True] * n + [bool(bits >> i & 1) for i in range(t)])
                        K, V = k[seen], v[seen]
                        q = self.q[at].double()
                        if not len(K):
                            assert (out[at] == 0).all() and norm[at] == (math.inf if form == "entmax" else -math.inf), at
                            if form == "entmax":
                                assert supp[at] == 0
                            continue
                        s = self.scale * (K @ q)
                        # products' sums: 4 instructions of at most 32 roundings (bf16), 128 roundings in turn (float32); the scale one
                        off = (132 if self.dtype == "f32" else 37) * u * self.scale * (K.abs() @ q.abs())
                        if form == "softmax":
                            p = torch.softmax(s, 0)
                            # a weight is off by its score, the largest score of its row, 2 for the conversion to powers of two and 2 for the
                            # power itself (exponents up to 64 where weights count: 64 u), the rest by the sums: 32 keys an instruction,
                            # partial results of 4 wavefronts and some workgroups
                            rel = off + off.max() + 80 * u + (len(K) / 32 + 100) * u
                            limit = (p * rel) @ V.abs() + (p @ rel) * (p @ V).abs() + 1e-30
                            err = (out[at].double() - p @ V).abs()
                            assert (err <= limit).all(), (at, (err / limit).max().item())
                            ref = torch.logsumexp(s, 0)
                            assert abs(norm[at].double() - ref) <= off.max() + (80 + len(K) / 32) * u + 4 * u * abs(ref), (at, norm[at], ref)
                            continue
                        z = a * s
                        lo, hi = z.max() - 1.0, z.max()
                        for _ in range(60):
                            mid = 0.5 * (lo + hi)
                            lo, hi = (mid, hi) if (z - mid).clamp(min=0).pow(beta).sum() >= 1 else (lo, mid)
                        # the root moves by no more than the scores do; the solve stops at a mass within 4e-7 of 1 or at its last place
                        dz = a * off.max() + 2 * u * z.abs().max()
                        d_tau = dz + 4e-6 * max(1.0, abs(float(lo)))
                        assert abs(norm[at].double() - lo) <= d_tau, (at, norm[at], lo)
                        x = (z - lo + dz + d_tau).clamp(min=0)
                        p = (z - lo).clamp(min=0).pow(beta)
                        moved = beta * x.pow(beta - 1.0) * (x > 0) * (dz + d_tau) if beta >= 1 else x.pow(beta) - p + p * 1e-6 + (x > 0) * (dz + d_tau) ** beta
                        limit = (moved + 40 * u * p * (1 + beta)) @ V.abs() + 1e-30
                        err = (out[at].double() - p @ V).abs()
                        assert (err <= limit).all(), (at, (err / limit).max().item())
                        assert int((z > lo + dz + d_tau).sum()) <= int(supp[at]) <= int((z > lo - dz - d_tau).sum()), at
        # rows of no sequence are left as they were
        assert (out[~taken] == 77).all() and (norm[~taken] == 77).all() and (supp[~taken] == 77).all()


def check(form, got=None, **kw):
    t = Tree(**kw)
    t.check(form, t.run(form))
