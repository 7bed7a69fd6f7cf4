"""Plain numpy forms of the 8-bit cache in 64 bits, and the inputs its tests share."""
import numpy as np
import torch

from paper_2605_21649_amd import binding as ekv

D = 128
LOW, HIGH = -100, 119                     # exponents of scales


def code_values():
    v = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = np.nan if code & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[code] = -x if code & 128 else x
    return v


VALUES = code_values()


def round_codes(x):
    """The nearest value of the format, ties to an even last place, at most +-448; NaN for what is no finite number."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    y = np.where(fine, x, 0.0)
    _, e = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    y = np.clip(np.rint(y / step) * step, -448.0, 448.0)
    return np.where(fine, y, np.nan)


def scale_for(x):
    """The least power of two in range with max |x| <= 448 s over the finite elements."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    top = x[np.isfinite(x)].max(initial=0.0)
    for e in range(LOW, HIGH + 1):
        if top <= 448.0 * 2.0 ** e:
            return 2.0 ** e
    return 2.0 ** HIGH


class Cache8:
    """Device buffers of an 8-bit cache; everything that no token has been written to holds NaN codes, and pages that no
    sequence has, NaN scales."""

    def __init__(self, batch, q_heads, kv_heads, page, lens, row_pages=None, dtype="bf16", alpha=1.5, scale=None, cap=None, seed=0,
                 device="cuda", pool_heads=0, spread=True):
        rng = np.random.default_rng(seed)
        self.B, self.Hq, self.Hkv, self.P, self.G, self.dtype = batch, q_heads, kv_heads, page, q_heads // kv_heads, dtype
        self.lens = list(lens)
        self.M = row_pages or max(1, max(-(-n // page) for n in self.lens))
        self.cap = cap or self.M
        self.alpha, self.scale = alpha, scale or 1.0 / np.sqrt(D)
        used = sum(-(-n // page) for n in self.lens)
        self.n_phys = used + 3
        ids = rng.permutation(self.n_phys)[:used]
        table = rng.integers(-5, 5 * self.n_phys, (batch, self.M))            # entries past a sequence may hold anything
        at = 0
        for b, n in enumerate(self.lens):
            m = -(-n // page)
            table[b, :m] = ids[at:at + m]
            at += m
        codes, scales = [], []
        for side in range(2):
            x = rng.standard_normal((self.n_phys, kv_heads, page, D))
            if side == 0:
                x[..., rng.permutation(D)[:4]] += 4.0
            if spread:                                                        # pages of quite different magnitude
                x *= 2.0 ** rng.integers(-3, 3, (self.n_phys, kv_heads, 1, 1))
            s = 2.0 ** np.ceil(np.log2(np.abs(x).max((2, 3)) / 448.0))
            code = torch.from_numpy((x / s[..., None, None]).astype(np.float32)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            codes.append(code.numpy().copy())
            scales.append(s)
        valid = np.zeros((self.n_phys, page), dtype=bool)
        for b, n in enumerate(self.lens):
            for p in range(-(-n // page)):
                valid[table[b, p], :min(page, n - p * page)] = True
        for side in range(2):
            codes[side][~np.broadcast_to(valid[:, None, :], codes[side].shape[:3])] = 0x7F if side else 0xFF
            scales[side][~valid.any(1)] = np.nan
        self.table, self.codes, self.scales, self.valid = table, codes, scales, valid
        q = rng.standard_normal((batch, q_heads, D))
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        dev = torch.device(device)
        self.q = torch.from_numpy(q.astype(np.float32)).to(dt).to(dev)
        self.k_pool, self.v_pool = (torch.from_numpy(x).to(dev) for x in codes)
        self.k_scale, self.v_scale = (torch.from_numpy(x.astype(np.float32)).to(dev) for x in scales)
        self.block_table = torch.from_numpy(table.astype(np.int32)).to(dev)
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32, device=dev)
        self.cfg = ekv.make_config(batch, q_heads, kv_heads, D, page, dtype, alpha, self.scale, self.M, self.cap, pool_heads)
        f32, i32 = dict(device=dev, dtype=torch.float32), dict(device=dev, dtype=torch.int32)
        self.out = torch.full((batch, q_heads, D), float("nan"), **f32)
        self.tau = torch.full((batch, q_heads), float("nan"), **f32)
        self.supp = torch.full((batch, q_heads), -1, **i32)

    def view(self):
        return ekv.cache8_view(self.k_pool, self.v_pool, self.k_scale, self.v_scale, self.block_table, self.seq_lens)

    def workspace(self, op, cfg=None):
        return torch.empty(max(256, ekv.ekv_workspace_bytes(cfg or self.cfg, op)), dtype=torch.uint8, device=self.q.device)

    def keys_values(self, b, h):
        """float64 K, V of a sequence's KV head in logical order."""
        n, P = self.lens[b], self.P
        rows = self.table[b, :-(-n // P)]
        return tuple((VALUES[self.codes[i][rows, h]] * self.scales[i][rows, h][:, None, None]).reshape(-1, D)[:n] for i in range(2))

    def query(self, b, h):
        return self.q[b, h].float().cpu().numpy().astype(np.float64)

    def tokens(self, b, pages):
        t = (np.asarray(pages, dtype=np.int64)[:, None] * self.P + np.arange(self.P)).reshape(-1)
        return t[t < self.lens[b]]


def score_error(q, K, scale):
    """A bound of a score's error: products are exact, 128 of them are added in float32 (half a step, 2^-24, of the
    magnitudes' sum an addition, three times as many for a query of three terms), and two multiplications follow."""
    if not len(K):
        return 0.0
    return float((3 * 128 + 2) * 2.0 ** -24 * scale * (np.abs(K) @ np.abs(q)).max())


class Large:
    """An 8-bit cache of sequences too long to make on the host, for comparisons of samples: signed values of ordinary size, pages of
    different magnitude, NaN codes behind every last token and NaN scales where no token is."""

    def __init__(self, q_heads, kv_heads, page, lens, cap=None, dtype="bf16", seed=0, row_pages=None, flat=1.0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.B, self.Hq, self.Hkv, self.P, self.G = len(lens), q_heads, kv_heads, page, q_heads // kv_heads
        self.lens, self.alpha, self.scale = list(lens), 1.5, flat / np.sqrt(D)
        self.M = row_pages or -(-max(lens) // page)
        self.cap = cap or self.M
        n_phys = self.B * self.M
        self.table = torch.randperm(n_phys, generator=g, device=device).view(self.B, self.M).to(torch.int32)
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32, device=device)
        self.pools, self.scales = [], []
        behind = torch.arange(self.M * page, device=device).view(1, self.M, page) >= self.seq_lens[:, None, None]
        for side in range(2):
            code = torch.empty(n_phys, kv_heads, page, D, dtype=torch.uint8, device=device)
            step = max(1, (1 << 26) // (kv_heads * page * D))
            for lo in range(0, n_phys, step):
                x = torch.randn(min(step, n_phys - lo), kv_heads, page, D, generator=g, device=device)
                code[lo:lo + x.shape[0]] = (x * 100.0).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            scale = 2.0 ** torch.randint(-8, -5, (n_phys, kv_heads), generator=g, device=device).float()      # sizes of 0.4 to 1.6
            for b in range(self.B):
                rows = self.table[b].long()
                code[rows] = torch.where(behind[b][:, None, :, None], 0x7F if side else 0xFF, code[rows])
                scale[rows[behind[b].all(1)]] = float("nan")
            self.pools.append(code)
            self.scales.append(scale)
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.q = torch.randn(self.B, q_heads, D, generator=g, device=device).to(dt)
        self.cfg = ekv.make_config(self.B, q_heads, kv_heads, D, page, dtype, self.alpha, self.scale, self.M, self.cap)
        self.out = torch.full((self.B, q_heads, D), float("nan"), device=device)
        self.tau = torch.full((self.B, q_heads), float("nan"), device=device)
        self.supp = torch.full((self.B, q_heads), -1, dtype=torch.int32, device=device)

    view = lambda self: ekv.cache8_view(*self.pools, *self.scales, self.table, self.seq_lens)  # noqa: E731
    workspace = Cache8.workspace
    query = Cache8.query
    tokens = Cache8.tokens

    def keys_values(self, b, h):
        n, P = self.lens[b], self.P
        rows = self.table[b, :-(-n // P)].long()
        return tuple((VALUES[self.pools[i][rows, h].cpu().numpy()] * self.scales[i][rows, h].cpu().numpy().astype(np.float64)[:, None, None])
                     .reshape(-1, D)[:n] for i in range(2))


def entmax_limits(ref, q, K, V, alpha, scale):
    """How far a threshold, and each channel of the output, may be from the oracle's `ref` (over K and V): tau moves by the scores'
    error times alpha - 1 and the solve stops within 4e-6 max(1, |tau|); weights p = x^beta move with x by twice that, and
    float32 sums of the support follow."""
    a = alpha - 1.0
    e = a * score_error(q, K, scale) + 4e-6 * max(1.0, abs(ref["tau"]))
    x = a * ref["s"] - ref["tau"]
    dp = np.maximum(x + 2 * e, 0.0) ** (1.0 / a) - np.maximum(x - 2 * e, 0.0) ** (1.0 / a)
    return e, dp @ np.abs(V) + (len(ref["support"]) + 8) * 2.0 ** -24 * (ref["p"] @ np.abs(V))


def softmax_limits(ref, q, K, V, scale):
    """The same for a log-sum-exp and its output: weights move by the factor exp(2 e), and float32 sums follow."""
    e = score_error(q, K, scale) + 8 * 2.0 ** -24 * max(1.0, 2.0 * np.abs(ref["s"]).max())
    return (e + 8 * 2.0 ** -24 * max(1.0, abs(ref["lse"])) + len(K) * 2.0 ** -24,
            (np.expm1(2 * e) + (len(K) + 64) * 2.0 ** -24) * (ref["p"] @ np.abs(V)))
