"""Device buffers of one workload: everything the entry points read and write, plus the ekv_config.

Plumbing for the tests and the benchmark (torch allocates, the library computes); no part of the method."""
import torch

from paper_2605_21649_amd import binding as ekv
from paper_2605_21649_amd import synth


class DeviceState:
    """All device buffers of one workload plus its ekv_config."""

    def __init__(self, w, inp, cap=None, device="cuda"):
        self.w = w
        dev = torch.device(device)
        self.inp = {k: v.to(dev) for k, v in inp.items()}
        B, Hq, Hkv, d, P = w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, w.page_size
        self.Mmax = w.pages_per_seq
        self.cap = cap if cap is not None else self.Mmax
        self.cfg = ekv.make_config(B, Hq, Hkv, d, P, w.kv_dtype, w.alpha, w.score_scale, self.Mmax, self.cap)
        dt = synth.torch_dtype(w.kv_dtype)
        self.box_stats = torch.zeros(B, Hkv, self.Mmax, 2, d, device=dev, dtype=dt)
        self.gauss_stats = torch.zeros(B, Hkv, self.Mmax, 2, d, device=dev, dtype=dt)
        f32 = dict(device=dev, dtype=torch.float32)
        i32 = dict(device=dev, dtype=torch.int32)
        self.box = torch.zeros(B, Hq, self.Mmax, **f32)
        self.mu = torch.zeros(B, Hq, self.Mmax, **f32)
        self.sigma = torch.zeros(B, Hq, self.Mmax, **f32)
        self.page_idx = torch.zeros(B, Hq, self.cap, **i32)
        self.n_sel = torch.zeros(B, Hq, **i32)
        self.overflow = torch.zeros(B, Hq, **i32)
        self.tau_hat = torch.zeros(B, Hq, **f32)
        self.out = torch.zeros(B, Hq, d, **f32)
        self.tau = torch.zeros(B, Hq, **f32)
        self.supp = torch.zeros(B, Hq, **i32)
        self.ws = {}

    def cache(self):
        i = self.inp
        return ekv.cache_view(i["k_pool"], i["v_pool"], i["block_table"], i["seq_lens"])

    def stats(self):
        return ekv.stats_view(self.box_stats, self.gauss_stats, getattr(self, "box8_stats", None))

    def enable_box8(self):
        """Allocate the optional 8-bit bounds; from then on build/append keep them up to date."""
        w = self.w
        self.box8_stats = torch.zeros(w.batch, w.n_kv_heads, self.Mmax, 16, 2, 8, device=self.box.device,
                                      dtype=torch.uint8)
        return self.box8_stats

    def enable_cache8(self, chunk=65536):
        """The workload's sequences on an 8-bit cache of their own, as a server fills one: pages are mapped from lengths and the
        tokens appended in chunks, with the page statistics of the stored keys.
        The last token of each sequence stays for the step (map_and_append8)."""
        w, dev, i = self.w, self.box.device, self.inp
        B, Hkv, d, P, M = w.batch, w.n_kv_heads, w.head_dim, w.page_size, self.Mmax
        n_phys = B * M
        i32 = dict(device=dev, dtype=torch.int32)
        self.pools8 = [torch.zeros(n_phys, Hkv, P, d, device=dev, dtype=torch.uint8) for _ in range(2)]
        self.scales8 = [torch.ones(n_phys, Hkv, device=dev) for _ in range(2)]
        self.table8, self.free8 = torch.zeros(B, M, **i32), torch.randperm(n_phys, device=dev).to(torch.int32)
        self.box_stats8, self.gauss_stats8 = torch.zeros_like(self.box_stats), torch.zeros_like(self.gauss_stats)
        lens, n_free = torch.zeros(B, **i32), torch.full((1,), n_phys, **i32)
        total = i["seq_lens"].tolist()
        for at in range(0, max(total), chunk):
            counts = [max(0, min(at + chunk, n - 1) - at) for n in total]
            if not sum(counts):
                break
            t = self._tokens8(sum(counts))
            new_lens, left = torch.zeros(B, **i32), torch.zeros(1, **i32)
            ekv.ekv_map_tokens(self.cfg, lens, torch.tensor(counts, **i32), self.table8, self.free8, n_free, t["map"], new_lens, left)
            rows = []
            for name in ("k_pool", "v_pool"):
                part = []
                for b, c in enumerate(counts):
                    pos = torch.arange(at, at + c, device=dev)
                    part.append(i[name][i["block_table"][b].long()[pos // P], :, pos % P])
                rows.append(torch.cat(part))
            lens, n_free = new_lens, left
            ekv.ekv_cache8_append(self.cfg, self.cache8(lens), self.stats8(), t["map"], *rows)
            del rows
        last = i["seq_lens"].long() - 1
        at = (torch.arange(B, device=dev), last // P)
        self.new8 = [i[name][i["block_table"].long()[at], :, last % P].contiguous() for name in ("k_pool", "v_pool")]
        self.lens8, self.free_count8, self.ones8 = lens, n_free, torch.ones(B, **i32)
        self.lens8_now, self.left8 = torch.zeros(B, **i32), torch.zeros(1, **i32)
        self.tokens8 = self._tokens8(B)

    def _tokens8(self, n):
        i32 = dict(device=self.box.device, dtype=torch.int32)
        t = {"slots": torch.zeros(n, device=self.box.device, dtype=torch.int64), "seq": torch.zeros(n, **i32), "pos": torch.zeros(n, **i32),
             "start": torch.zeros(self.w.batch + 1, **i32), "n_mapped": torch.zeros(self.w.batch, **i32)}
        t["map"] = ekv.token_map(t["slots"], t["seq"], t["pos"], t["start"], t["n_mapped"])
        return t

    def cache8(self, lens=None):
        return ekv.cache8_view(*self.pools8, *self.scales8, self.table8, self.lens8_now if lens is None else lens)

    def stats8(self):
        return ekv.stats_view(self.box_stats8, self.gauss_stats8)

    def map_and_append8(self):
        """One token per sequence: its page and slot, its codes, its page's statistics.  The free list and the lengths before it
        stay, so that the step can be repeated."""
        ekv.ekv_map_tokens(self.cfg, self.lens8, self.ones8, self.table8, self.free8, self.free_count8, self.tokens8["map"],
                           self.lens8_now, self.left8)
        ekv.ekv_cache8_append(self.cfg, self.cache8(), self.stats8(), self.tokens8["map"], *self.new8)

    def workspace(self, op):
        if op not in self.ws:
            n = ekv.ekv_workspace_bytes(self.cfg, op)
            self.ws[op] = torch.empty(max(n, 256), device=self.box.device, dtype=torch.uint8)
        return self.ws[op]


class HeadSlice:
    """The KV heads [h0, h1) of a batch-1 DeviceState (and their query heads) as a problem of its own: a config
    with the pools' head stride, pool pointers advanced to h0, and contiguous slices of every per-head array.
    Independent slices can run on separate streams."""

    def __init__(self, st, h0, h1):
        w = st.w
        assert w.batch == 1, "per-head arrays of a head range are contiguous only for batch 1"
        G = w.group
        self.st, self.h0, self.h1 = st, h0, h1
        q0, q1 = h0 * G, h1 * G
        self.cfg = ekv.make_config(1, q1 - q0, h1 - h0, w.head_dim, w.page_size, w.kv_dtype, w.alpha, w.score_scale,
                                   st.Mmax, st.cap, pool_kv_heads=w.n_kv_heads)
        i = st.inp
        self.q = i["q"][:, q0:q1]
        self.seq_lens = i["seq_lens"]
        self.box_stats, self.gauss_stats = st.box_stats[:, h0:h1], st.gauss_stats[:, h0:h1]
        self.box8_stats = st.box8_stats[:, h0:h1] if hasattr(st, "box8_stats") else None
        for name in ("box", "mu", "sigma", "page_idx", "n_sel", "overflow", "tau_hat", "out", "tau", "supp"):
            setattr(self, name, getattr(st, name)[:, q0:q1])
        self.ws = {}

    def cache(self, seq_lens=None):
        i = self.st.inp
        return ekv.cache_view_heads(i["k_pool"], i["v_pool"], i["block_table"],
                                    self.seq_lens if seq_lens is None else seq_lens, self.h0)

    def stats(self):
        return ekv.stats_view(self.box_stats, self.gauss_stats, self.box8_stats)

    def new_token(self, k_new, v_new):
        """[1][Hkv][d] tokens of all heads -> this slice's."""
        return k_new[:, self.h0:self.h1], v_new[:, self.h0:self.h1]

    def workspace(self, op):
        if op not in self.ws:
            n = ekv.ekv_workspace_bytes(self.cfg, op)
            self.ws[op] = torch.empty(max(n, 256), device=self.box.device, dtype=torch.uint8)
        return self.ws[op]
