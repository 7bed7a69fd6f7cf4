"""Norm and rotation of queries and keys against the formula in 64 bits."""
import math

import pytest
import torch

from paper_2605_21649_amd import binding as ekv

pytestmark = pytest.mark.gpu
D = 128
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def formula(x, w, eps, freq, pos, pairs):
    """In 64 bits: the result, and the size |a| + |b| of the two products that each channel is the sum of."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * w.double()
    size = y.abs()
    n = 0 if freq is None else freq.numel()
    if n:
        angle = pos.double()[:, None, None] * freq.double()
        cos, sin = torch.cos(angle), torch.sin(angle)
        i, j = (torch.arange(0, 2 * n, 2), torch.arange(1, 2 * n, 2)) if pairs else (torch.arange(n), torch.arange(n, 2 * n))
        a, b = y[..., i].clone(), y[..., j].clone()
        y[..., i], y[..., j] = a * cos - b * sin, b * cos + a * sin
        size[..., i] = size[..., j] = a.abs() + b.abs()
    return y, size


def run(case, seed=0):
    n, hq, hk, dtype, turned, pairs, far, norm = case
    g = torch.Generator().manual_seed(seed)
    dt = TYPE[dtype]
    rows = (torch.randn(n, hq + 2 * hk, D, generator=g) * torch.exp(2 * torch.randn(n, hq + 2 * hk, 1, generator=g))).to(dt)
    x = {"q": rows[:, :hq], "k": rows[:, hq:hq + hk]}
    w = {s: (1 + 0.3 * torch.randn(D, generator=g)).to(dt) if norm else None for s in "qk"}
    freq = (10000.0 ** (-torch.arange(turned // 2, dtype=torch.float64) * 2 / turned)).float() if turned else None
    pos = torch.randint(0, far, (n,), generator=g, dtype=torch.int32)
    pos[::5] = -1
    pos[0] = far - 1
    dev = rows.cuda()
    out = {"q": torch.full((n, hq, D), 7.0, dtype=dt, device="cuda"), "k": torch.full((n, hk, D), 7.0, dtype=dt, device="cuda")}
    put = lambda t: None if t is None else t.cuda()  # noqa: E731
    cfg = ekv.make_config(1, hq, hk, D, 16, dtype, 1.5, 1.0, 1, 1)
    ekv.ekv_norm_rotate(cfg, dev[:, :hq], dev[:, hq:hq + hk], put(w["q"]), put(w["k"]), 1e-6, put(freq), pos.cuda(), out["q"], out["k"],
                        pairs=pairs)
    torch.cuda.synchronize()
    for s in "qk":
        got = out[s].cpu()
        assert (got[pos < 0] == 7.0).all()                              # passed over
        ref, size = formula(x[s], w[s], 1e-6, freq, pos, pairs)
        here = pos >= 0
        # float32: the mean's sum (12 roundings, halved by the root), root, quotient, two products: 10; turns rounded to 24 bits are pi /
        # 2^25 of angle (1.6 u), sine and cosine within two units in the last place (4 u), two products and a sum (3): 20 u, u = 2^-24
        limit = 20 * 2.0 ** -24 * size + (2.0 ** -8 * ref.abs() if dtype == "bf16" else 0)
        off = (got.double() - ref).abs()
        assert (off <= limit)[here].all(), (s, ((off - limit)[here]).max().item())


@pytest.mark.parametrize("case", [
    (1, 1, 1, "f32", 128, False, 1, True), (1, 8, 8, "bf16", 128, False, 2, True), (5, 8, 8, "f32", 64, True, 4096, True),
    (7, 3, 3, "bf16", 32, False, 1 << 20, True), (13, 10, 5, "f32", 96, False, 1 << 20, True), (9, 32, 8, "bf16", 16, True, 1 << 20, True),
    (257, 64, 8, "bf16", 128, True, 1 << 30, True), (300, 32, 8, "f32", 128, False, 1 << 30, True),
    (511, 8, 1, "bf16", 96, True, 100000, False), (1023, 32, 8, "bf16", 128, False, 1 << 20, True), (6, 4, 4, "f32", 0, False, 9, True),
    (410, 32, 8, "f32", 48, True, 1 << 20, False), (2049, 8, 1, "bf16", 64, False, 5000, True),
], ids=lambda c: "-".join(map(str, c)))
def test_against_the_formula(case):
    run(case)


def test_without_norm_and_rotation_rows_are_copied():
    x = torch.randn(3, 6, D).cuda()
    q, k = torch.zeros(3, 4, D, device="cuda"), torch.zeros(3, 2, D, device="cuda")
    cfg = ekv.make_config(1, 4, 2, D, 16, "f32", 1.5, 1.0, 1, 1)
    ekv.ekv_norm_rotate(cfg, x[:, :4], x[:, 4:], None, None, 0.0, None, None, q, k)
    assert torch.equal(q, x[:, :4]) and torch.equal(k, x[:, 4:])


def test_one_side_with_a_norm_and_rows_that_are_zero_infinite_or_no_number():
    x = torch.randn(4, 3, D)
    x[0] = 0.0
    x[1, 0, 5], x[2, 1, 7] = math.inf, math.nan
    w, q, k = torch.ones(D).cuda(), torch.empty(4, 2, D, device="cuda"), torch.empty(4, 1, D, device="cuda")
    cfg = ekv.make_config(1, 2, 1, D, 16, "f32", 1.5, 1.0, 1, 1)
    ekv.ekv_norm_rotate(cfg, x.cuda()[:, :2], x.cuda()[:, 2:], w, None, 1e-6, None, None, q, k)
    assert (q[0] == 0).all() and torch.equal(k.cpu(), x[:, 2:])
    # an infinity makes its head's root infinite: nothing is left of the others, and of itself no number; other heads do not see it
    assert (q[1, 0, torch.arange(D) != 5] == 0).all() and q[1, 0, 5].isnan() and q[2, 1].isnan().all()
    assert q[1, 1].isfinite().all() and q[2, 0].isfinite().all() and q[3].isfinite().all()


def test_the_same_in_a_graph_and_on_another_stream():
    n, hq, hk = 33, 32, 8
    x, pos = torch.randn(n, 48, D, device="cuda").bfloat16(), torch.randint(0, 9999, (n,), device="cuda", dtype=torch.int32)
    w, freq = torch.rand(D, device="cuda").bfloat16(), torch.rand(64, device="cuda")
    cfg = ekv.make_config(1, hq, hk, D, 16, "bf16", 1.5, 1.0, 1, 1)
    call = lambda q, k: ekv.ekv_norm_rotate(cfg, x[:, :32], x[:, 32:40], w, w, 1e-5, freq, pos, q, k)  # noqa: E731
    q, k = torch.empty(n, hq, D, device="cuda").bfloat16(), torch.empty(n, hk, D, device="cuda").bfloat16()
    call(q, k)
    q2, k2 = torch.zeros_like(q), torch.zeros_like(k)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call(q2, k2)
    s.synchronize()
    assert torch.equal(q, q2) and torch.equal(k, k2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(q2, k2)
    for shift in (3, 0):
        pos += shift
        call(q, k)
        q2.zero_(), k2.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, q2) and torch.equal(k, k2)
