"""A step of drafted tokens as a program takes it: rows of a projection are normalised and rotated, the drafted rows attend to the cache and
to their tree, the accepted path is appended; against the single-token calls, which see the same tokens one after the other."""
import pytest
import torch

from paper_2605_21649_amd import binding as ekv

pytestmark = pytest.mark.gpu
D, P, HQ, HK = 128, 16, 8, 2


@pytest.mark.parametrize("eight", [False, True])
def test_accepted_paths_leave_the_cache_that_single_tokens_make(eight):
    g = torch.Generator().manual_seed(3)
    lens, b, m = [37, 160, 0], 3, 16
    n_phys = b * m
    dt = torch.bfloat16
    table = torch.randperm(n_phys, generator=g).view(b, m).int().cuda()
    held = torch.tensor(lens, dtype=torch.int32).cuda()
    cfg = ekv.make_config(b, HQ, HK, D, P, "bf16", 1.5, D ** -0.5, m, m)
    i32 = dict(dtype=torch.int32, device="cuda")

    def cache():
        if eight:
            pools = [torch.zeros(n_phys, HK, P, D, dtype=torch.uint8, device="cuda") for _ in "kv"]
            scales = [torch.ones(n_phys, HK, device="cuda") for _ in "kv"]
            return pools + scales
        return [torch.zeros(n_phys, HK, P, D, dtype=dt, device="cuda") for _ in "kv"]

    def view(c, lengths):
        return ekv.cache8_view(*c, table, lengths) if eight else ekv.cache_view(*c, table, lengths)

    def stats():
        return [torch.zeros(b, HK, m, 2, D, dtype=dt, device="cuda") for _ in range(2)]

    def append(c, s, slots, seq, pos, k, v, rows=None):
        tok = ekv.token_map(slots, seq, pos)
        if eight:
            if rows is not None:
                k, v = k[rows.long()], v[rows.long()]
            ekv.ekv_cache8_append(cfg, view(c, held), ekv.stats_view(*s), tok, k, v)
        else:
            ekv.ekv_cache_append(cfg, view(c, held), ekv.stats_view(*s), tok, k, v, rows=rows)

    def slots_of(seq, pos):
        seq, pos = torch.tensor(seq).cuda(), torch.tensor(pos).cuda()
        return table[seq, pos // P].long() * P + pos % P, seq.int(), pos.int()

    # prompts, normalised and rotated as later tokens are
    w = (1 + 0.1 * torch.randn(2, D, generator=g)).to(dt).cuda()
    freq = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()

    def turned(rows, pos):
        n = rows.shape[0]
        q, k = torch.empty(n, HQ, D, dtype=dt, device="cuda"), torch.empty(n, HK, D, dtype=dt, device="cuda")
        ekv.ekv_norm_rotate(cfg, rows[:, :HQ], rows[:, HQ:HQ + HK], w[0], w[1], 1e-6, freq, pos, q, k)
        return q, k, rows[:, HQ + HK:]

    project = lambda n: torch.randn(n, HQ + 2 * HK, D, generator=g).to(dt).cuda()  # noqa: E731
    seq, pos = [s for s, n in enumerate(lens) for _ in range(n)], [i for n in lens for i in range(n)]
    prompt = slots_of(seq, pos)
    _, k0, v0 = turned(project(len(seq)), prompt[2])
    one, two, s_one, s_two = cache(), cache(), stats(), stats()
    for c, s in ((one, s_one), (two, s_two)):
        append(c, s, *prompt, k0, v0)
    # a tree for every sequence: row i follows parent[i]; the accepted path is 0 -> 2 -> 3 -> 5
    parent = [-1, 0, 0, 2, 1, 3]
    t = len(parent)
    seen, depth = [], []
    for i, p in enumerate(parent):
        seen.append((1 << i) | (seen[p] if p >= 0 else 0))
        depth.append(depth[p] + 1 if p >= 0 else 0)
    path = [0, 2, 3, 5]
    rows = project(b * t)
    where = torch.tensor([n + d for n in lens for d in depth], **i32)
    q, k, v = turned(rows, where)
    start = torch.arange(0, b * t + 1, t, **i32)
    tree = ekv.tree_view(start, torch.tensor(seen * b).cuda(), k, v, t)
    out, tau, supp = torch.empty(b * t, HQ, D, device="cuda"), torch.empty(b * t, HQ, device="cuda"), torch.empty(b * t, HQ, **i32)
    ws = torch.empty(ekv.ekv_tree_workspace_bytes(cfg, ekv.EKV_OP_TREE_FULL, b * t, t), dtype=torch.uint8, device="cuda")
    (ekv.ekv_tree8_full if eight else ekv.ekv_tree_full)(cfg, q, view(one, held), tree, out, tau, supp, ws)
    # the path at once
    rows_of = torch.tensor([s * t + r for s in range(b) for r in path], **i32)
    append(one, s_one, *slots_of([s for s in range(b) for _ in path], [n + i for n in lens for i in range(len(path))]), k, v, rows_of)
    # and token by token, each attending over what was appended before it and itself
    n_now = held.clone()
    o, x, c = torch.empty(b, HQ, D, device="cuda"), torch.empty(b, HQ, device="cuda"), torch.empty(b, HQ, **i32)
    wd = torch.empty(ekv.ekv_workspace_bytes(cfg, ekv.EKV_OP_DECODE_FULL), dtype=torch.uint8, device="cuda")
    for i, r in enumerate(path):
        mine = torch.arange(b, device="cuda") * t + r
        append(two, s_two, *slots_of(list(range(b)), [n + i for n in lens]), k[mine].contiguous(), v[mine].contiguous())
        n_now += 1
        if not eight:                                   # the 8-bit cache holds a token rounded, the tree has it as it is
            ekv.ekv_decode_full(cfg, q[mine].contiguous(), view(two, n_now), o, x, c, wd)
            torch.cuda.synchronize()
            # two kernels' float32 roundings of the same row, scores up to 30: thresholds within 1e-5, outputs 1e-4 of values of size 1
            assert torch.allclose(tau[mine], x, rtol=1e-5, atol=1e-5) and torch.allclose(out[mine], o, rtol=1e-4, atol=1e-4)
    torch.cuda.synchronize()
    for got, want in zip(one + s_one, two + s_two):
        if not eight:
            assert torch.equal(got, want)
    if eight:                                           # codes of a run at once and token by token may differ where a scale grew in between
        a, e = (c[0].view(torch.float8_e4m3fn).float() * c[2][..., None, None] for c in (one, two))
        assert ((a - e).abs() <= 2 * 2.0 ** -4 * torch.maximum(a.abs(), e.abs()) + 2.0 ** -9 * torch.maximum(one[2], two[2])[..., None, None]).all()
