"""A step of drafted tokens over the 8-bit cache, from the projection to the cache: attention against the definition in 64 bits over the stored
values and the drafted rows as they are, statistics against ekv_stats_build of a cache that holds the stored values."""
import pytest
import torch

from paper_2605_21649_amd import binding as ekv
from tests.tree import D, Tree

pytestmark = pytest.mark.gpu
P, HQ, HK = 16, 8, 2
PARENT = [-1, 0, 0, 2, 1, 3]
PATH = [0, 2, 3, 5]


def append(cfg, t, pools, scales, box, gauss, seq, pos, k, v):
    seq, pos = torch.tensor(seq).cuda(), torch.tensor(pos).cuda()
    slots = t.table.cuda()[seq, pos // P].long() * P + pos % P
    tokens = ekv.token_map(slots, seq.int(), pos.int())
    ekv.ekv_cache8_append(cfg, ekv.cache8_view(*pools, *scales), ekv.stats_view(box, gauss), tokens, k, v)
    return tokens, slots


def stored(pool, scale):
    return pool.view(torch.float8_e4m3fn).double() * scale.double()[..., None, None]


@pytest.mark.parametrize("at_once", [True, False])
@pytest.mark.parametrize("lens", [[37, 160, 0], [15, 16, 17], [1, 250, 64]])
def test_attention_and_statistics_of_a_step(lens, at_once):
    g = torch.Generator().manual_seed(sum(lens))
    b, n_tree = len(lens), len(PARENT)
    t = Tree(lens, [n_tree] * b, heads=(HQ, HK), page=P, cache="e4m3", extra_pages=1, seed=5)     # its tables and masks; contents below
    t.m = m = max(lens) // P + 2
    t.n_phys = b * m
    t.table = torch.randperm(b * m, generator=g).view(b, m).int()
    cfg = t.cfg = ekv.make_config(b, HQ, HK, D, P, "bf16", 1.5, t.scale, m, m)
    t.cap = m
    dt = torch.bfloat16
    pools = [torch.zeros(b * m, HK, P, D, dtype=torch.uint8, device="cuda") for _ in "kv"]
    scales = [torch.ones(b * m, HK, device="cuda") for _ in "kv"]
    box, gauss = (torch.zeros(b, HK, m, 2, D, dtype=dt, device="cuda") for _ in range(2))
    w = (1 + 0.1 * torch.randn(2, D, generator=g)).to(dt).cuda()
    freq = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()

    def turned(pos):
        rows = torch.randn(len(pos), HQ + 2 * HK, D, generator=g).to(dt).cuda()
        q, k = torch.empty(len(pos), HQ, D, dtype=dt, device="cuda"), torch.empty(len(pos), HK, D, dtype=dt, device="cuda")
        ekv.ekv_norm_rotate(cfg, rows[:, :HQ], rows[:, HQ:HQ + HK], w[0], w[1], 1e-6, freq, torch.tensor(pos, dtype=torch.int32).cuda(), q, k)
        return q, k, rows[:, HQ + HK:]

    seq, pos = [s for s, n in enumerate(lens) for _ in range(n)], [i for n in lens for i in range(n)]
    _, k0, v0 = turned(pos)
    held = [append(cfg, t, pools, scales, box, gauss, seq, pos, k0, v0)]
    depth, seen = [], []
    for i, p in enumerate(PARENT):
        depth.append(depth[p] + 1 if p >= 0 else 0)
        seen.append((1 << i) | (seen[p] if p >= 0 else 0))
    q, k, v = turned([n + x for n in lens for x in depth])
    torch.cuda.synchronize()
    # the tree's rows over what the cache holds now
    t.values = [stored(pool, scale).cpu() for pool, scale in zip(pools, scales)]
    t.q, t.k_new, t.v_new, t.visible = q.cpu(), k.cpu(), v.cpu(), torch.tensor(seen * b)
    t.k, t.v, t.ks, t.vs = *(x.cpu() for x in pools), *(x.cpu() for x in scales)
    for form in ("entmax", "softmax"):
        t.check(form, t.run(form))
    # the accepted path, at once or token by token
    if at_once:
        rows = torch.tensor([s * n_tree + r for s in range(b) for r in PATH]).cuda()
        held.append(append(cfg, t, pools, scales, box, gauss, [s for s in range(b) for _ in PATH], [n + i for n in lens for i in range(len(PATH))],
                           k[rows], v[rows].contiguous()))
    else:
        for i, r in enumerate(PATH):
            rows = torch.arange(b).cuda() * n_tree + r
            held.append(append(cfg, t, pools, scales, box, gauss, list(range(b)), [n + i for n in lens], k[rows], v[rows].contiguous()))
    torch.cuda.synchronize()
    now = [n + len(PATH) for n in lens]
    plain = stored(pools[0], scales[0]).to(dt)               # exact: a code has four bits
    want = [torch.zeros_like(box), torch.zeros_like(gauss)]
    ekv.ekv_stats_build(cfg, ekv.cache_view(plain, plain, t.table.cuda(), torch.tensor(now, dtype=torch.int32).cuda()), ekv.stats_view(*want))
    torch.cuda.synchronize()
    for s, n in enumerate(now):
        pages = -(-n // P)
        assert torch.equal(box[s, :, :pages], want[0][s, :, :pages]) and torch.equal(gauss[s, :, :pages], want[1][s, :, :pages]), s
    # what was drafted and accepted is in the cache within half a step of its scale
    for side, new in enumerate((k, v)):
        values, scale = stored(pools[side], scales[side]), scales[side].double()
        for s, n in enumerate(lens):
            for i, r in enumerate(PATH):
                page, tok = int(t.table[s, (n + i) // P]), (n + i) % P
                got, x = values[page, :, tok], new[s * n_tree + r].double()
                # half a step of a code is 2^-4 of the value, or 2^-10 of the scale below its normal numbers; a page whose scale grew rounds
                # a row again each time, by a step that is its last one's at most: once for each row behind it
                times = 1 if at_once else len(PATH) - i
                limit = times * torch.maximum(2.0 ** -4 * torch.maximum(x.abs(), got.abs()), 2.0 ** -10 * scale[page][:, None])
                assert ((got - x).abs() <= limit).all(), (side, s, i)
