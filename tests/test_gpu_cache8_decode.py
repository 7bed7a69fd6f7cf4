"""Attention over the 8-bit cache against the oracle on the values that the codes stand for.

Tolerances.  Codes times scales are exact on both sides, so that what differs is float32 arithmetic: e bounds a score's error
(cache8.score_error).  Entmax: tau moves by at most the scores' largest error times alpha - 1 (the mass falls in tau as it rises in
the scores), and the solve stops within 4e-6 max(1, |tau|), the bound of every decode of this library; a weight
p = x^beta moves by beta x^(beta-1) times that.  Softmax: weights move by the factor exp(2 e) and by exp's and the sums'
float32 steps; the log-sum-exp by e and a few of its own steps."""
import numpy as np
import pytest
import torch

from oracle import entmaxkv_oracle as orc
from paper_2605_21649_amd import binding as ekv
from tests.cache8 import Cache8, D, VALUES, score_error

pytestmark = pytest.mark.gpu

HEADS = [(2, 2), (4, 2), (8, 2), (16, 2)]


def check_entmax(c, b, h, tok, out, tau, supp):
    K, V = c.keys_values(b, h // c.G)
    q = c.query(b, h)
    if len(tok) == 0:
        assert np.all(out == 0.0) and tau == np.inf and supp == 0
        return
    ref = orc.entmax_attention(q, K, V, c.alpha, c.scale, tok)
    a = c.alpha - 1.0
    beta = 1.0 / a
    e = a * score_error(q, K[tok], c.scale) + 4e-6 * max(1.0, abs(ref["tau"]))
    assert abs(tau - ref["tau"]) <= e, (tau, ref["tau"], e)
    z = a * ref["s"]
    assert abs(int(supp) - len(ref["support"])) <= int((np.abs(z - ref["tau"]) <= 2 * e).sum())
    # a weight's change over [x - 2e, x + 2e], and sums of up to n terms in float32
    x = np.maximum(z - ref["tau"], 0.0)
    dp = np.maximum(x + 2 * e, 0.0) ** beta - np.maximum(x - 2 * e, 0.0) ** beta
    dp[z - ref["tau"] < -2 * e] = 0.0
    size = ref["p"] @ np.abs(V[tok])
    limit = dp @ np.abs(V[tok]) + (len(ref["support"]) + 8) * 2.0 ** -24 * size
    assert np.all(np.abs(out - ref["o"]) <= limit), (np.abs(out - ref["o"]) / limit).max()


def check_softmax(c, b, h, tok, out, lse):
    K, V = c.keys_values(b, h // c.G)
    q = c.query(b, h)
    if len(tok) == 0:
        assert np.all(out == 0.0) and lse == -np.inf
        return
    ref = orc.softmax_attention(q, K, V, c.scale, tok)
    top = np.abs(ref["s"]).max()
    e = score_error(q, K[tok], c.scale) + 8 * 2.0 ** -24 * max(1.0, 2.0 * top)
    assert abs(lse - ref["lse"]) <= e + 8 * 2.0 ** -24 * max(1.0, abs(ref["lse"])) + len(tok) * 2.0 ** -24
    limit = (np.expm1(2 * e) + (len(tok) + 64) * 2.0 ** -24) * (ref["p"] @ np.abs(V[tok]))
    assert np.all(np.abs(out - ref["o"]) <= limit), (np.abs(out - ref["o"]) / limit).max()


def check_all(c, kind, lists=None):
    out, tau, supp = c.out.cpu().numpy().astype(np.float64), c.tau.cpu().numpy(), c.supp.cpu().numpy()
    for b in range(c.B):
        for h in range(c.Hq):
            tok = np.arange(c.lens[b]) if lists is None else np.concatenate([c.tokens(b, [p]) for p in lists[b][h]] or [np.arange(0)])
            if kind == "entmax":
                check_entmax(c, b, h, tok, out[b, h], tau[b, h], supp[b, h])
            else:
                check_softmax(c, b, h, tok, out[b, h], tau[b, h])


def run_full(c, kind):
    if kind == "entmax":
        ekv.ekv_decode8_full(c.cfg, c.q, c.view(), c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_FULL))
    else:
        ekv.ekv_decode8_full_softmax(c.cfg, c.q, c.view(), c.out, c.tau, c.workspace(ekv.EKV_OP_DECODE8_FULL_SOFTMAX))
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["entmax", "softmax"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [4, 12, 16, 28, 32, 48, 60, 64])
def test_every_page_of_ragged_sequences(page, heads, dtype, kind):
    # empty, one token, a page less one, a page, a page and one, an odd length, several steps
    c = Cache8(7, *heads, page, [0, 1, page - 1, page, page + 1, 131, 777], dtype=dtype, seed=page + heads[0])
    run_full(c, kind)
    check_all(c, kind)


@pytest.mark.parametrize("kind", ["entmax", "softmax"])
@pytest.mark.parametrize("alpha,flat", [(1.25, 1.0), (1.5, 0.05), (1.7, 1.0), (2.0, 1.0), (3.0, 0.3), (1.02, 1.0)])
def test_alphas_and_flat_attention(alpha, flat, kind):
    c = Cache8(2, 4, 1, 16, [3001, 40], alpha=alpha, scale=flat / np.sqrt(D), seed=5)
    run_full(c, kind)
    check_all(c, kind)


@pytest.mark.parametrize("kind", ["entmax", "softmax"])
@pytest.mark.parametrize("heads", [(1, 1), (8, 1), (4, 4)])
def test_long_sequences_beside_short_ones(heads, kind):
    # steps of one sequence over many workgroups, workgroups with many sequences, a block table much longer than the sequences
    c = Cache8(9, *heads, 16, [20011, 0, 3, 0, 0, 260, 4096, 17, 0], row_pages=3000, seed=7, dtype="bf16" if heads[0] > 1 else "f32")
    run_full(c, kind)
    check_all(c, kind)


def page_lists(c, rng, n_lists, most):
    """Ascending lists, empty ones and a full one among them; in the first a page is named twice."""
    lists = []
    for b in range(c.B):
        m = -(-c.lens[b] // c.P)
        row = []
        for i in range(n_lists):
            k = min(m, int(rng.integers(0, most + 1)))
            row.append(sorted(rng.permutation(m)[:k].tolist()))
        lists.append(row)
    return lists


def as_tensors(c, lists, cap, rng):
    n_lists = len(lists[0])
    idx = rng.integers(-3, c.M + 3, (c.B, n_lists, cap))          # what stands behind a list's end may be anything
    n = np.zeros((c.B, n_lists), dtype=np.int32)
    for b in range(c.B):
        for i, pages in enumerate(lists[b]):
            idx[b, i, :len(pages)] = pages
            n[b, i] = len(pages)
    return torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(n).cuda()


@pytest.mark.parametrize("call", ["sparse", "group", "softmax"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [4, 12, 16, 32, 44, 64])
def test_page_lists(page, heads, dtype, call):
    rng = np.random.default_rng(page)
    c = Cache8(5, *heads, page, [0, 1, 5 * page - 2, 9 * page, 700], dtype=dtype, seed=page, cap=9)
    lists = page_lists(c, rng, c.Hkv if call == "group" else c.Hq, 9)
    lists[3][0] = [2, 2, 5]                                        # the same page twice counts twice
    idx, n = as_tensors(c, lists, 9, rng)
    if call == "softmax":
        ekv.ekv_decode8_sparse_softmax(c.cfg, c.q, c.view(), idx, n, c.out, c.tau, c.workspace(ekv.EKV_OP_DECODE8_SPARSE_SOFTMAX))
    else:
        fn = ekv.ekv_decode8_sparse_group if call == "group" else ekv.ekv_decode8_sparse
        fn(c.cfg, c.q, c.view(), idx, n, c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_SPARSE))
    torch.cuda.synchronize()
    per_head = [[row[h // c.G] for h in range(c.Hq)] for row in lists] if call == "group" else lists
    check_all(c, "softmax" if call == "softmax" else "entmax", per_head)


@pytest.mark.parametrize("call", ["sparse", "full", "group"])
@pytest.mark.parametrize("page", [16, 12])
def test_entmax_equals_the_decode_of_a_bf16_cache_with_these_values(page, call):
    """Codes times scales are bf16 numbers: the same calls on a cache that holds them differ by the order of float32 sums."""
    c = Cache8(3, 8, 2, page, [1500, 77, 900], seed=11, cap=20)
    pools = [torch.from_numpy(np.nan_to_num(VALUES[c.codes[i]] * c.scales[i][..., None, None])).to(torch.bfloat16).cuda() for i in range(2)]
    cache = ekv.cache_view(pools[0], pools[1], c.block_table, c.seq_lens)
    rng = np.random.default_rng(3)
    idx, n = as_tensors(c, page_lists(c, rng, c.Hkv if call == "group" else c.Hq, 20), 20, rng)
    toks = [torch.full((3, 8, 64), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    got = []
    for i, (name, view) in enumerate((("ekv_decode_", cache), ("ekv_decode8_", c.view()))):
        ex = ekv.decode_extras(support_tokens=toks[i])
        c.out.fill_(float("nan"))
        if call == "full":
            getattr(ekv, name + "full")(c.cfg, c.q, view, c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_FULL), extras=ex)
        else:
            getattr(ekv, name + ("sparse_group" if call == "group" else "sparse"))(
                c.cfg, c.q, view, idx, n, c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_SPARSE), extras=ex)
        torch.cuda.synchronize()
        got.append((c.out.clone(), c.tau.clone(), c.supp.clone()))
    e = max(score_error(c.query(b, h), c.keys_values(b, h // c.G)[0], c.scale) for b in range(3) for h in range(8))
    fine = torch.isfinite(got[0][1])
    assert torch.equal(fine, torch.isfinite(got[1][1]))
    assert float((got[0][1] - got[1][1])[fine].abs().max()) <= 2 * (0.5 * e + 8e-6)
    assert float((got[0][0] - got[1][0]).norm() / got[0][0].norm()) <= 2e-5
    assert float((got[0][2] - got[1][2]).abs().max()) <= 1


def test_side_outputs():
    c = Cache8(2, 8, 2, 16, [2000, 300], seed=21, cap=125)
    ws = c.workspace(ekv.EKV_OP_DECODE_FULL)
    lse, toks = torch.zeros(2, 8, device="cuda"), torch.full((2, 8, 512), -1, dtype=torch.int32, device="cuda")
    evals, mass, kept = torch.zeros(2, 8, dtype=torch.int32, device="cuda"), torch.zeros(2, 8, device="cuda"), torch.zeros(2, 8, dtype=torch.int32, device="cuda")
    run_full(c, "entmax")
    ref_tau = c.tau.clone()
    ex = ekv.decode_extras(support_tokens=toks, tau_ref=ref_tau, kept_mass_ref=mass, kept_supp_ref=kept, lse=lse, tau_seed=ref_tau,
                           solve_evals=evals)
    ekv.ekv_decode8_full(c.cfg, c.q, c.view(), c.out, c.tau, c.supp, ws, extras=ex)
    torch.cuda.synchronize()
    check_all(c, "entmax")
    assert torch.equal(kept, c.supp) and float((mass - 1).abs().max()) < 1e-5 and int(evals.min()) >= 1
    for b in range(2):
        for h in range(8):
            K, V = c.keys_values(b, h // 4)
            s = orc.softmax_attention(c.query(b, h), K, V, c.scale)
            assert abs(float(lse[b, h]) - s["lse"]) <= score_error(c.query(b, h), K, c.scale) + 1e-5 * max(1.0, abs(s["lse"]))
            z = 0.5 * s["s"]
            t = toks[b, h, :int(c.supp[b, h])].cpu().numpy()
            assert np.all(np.diff(t) > 0) and np.all(z[t] > float(c.tau[b, h]) - 1e-5)


def test_a_range_of_heads_of_a_larger_cache():
    c = Cache8(1, 8, 4, 16, [500], seed=31)
    run_full(c, "entmax")
    whole = c.out.clone(), c.tau.clone()
    for kind in ("entmax", "softmax"):
        run_full(c, kind)
        all_out, all_tau = c.out.clone(), c.tau.clone()
        h0, h1, G = 1, 3, 2
        cfg = ekv.make_config(1, (h1 - h0) * G, h1 - h0, D, 16, "bf16", c.alpha, c.scale, c.M, c.cap, pool_kv_heads=4)
        v = c.view()
        part = ekv.ekv_cache8_view(v.k_pool + h0 * 16 * D, v.v_pool + h0 * 16 * D, v.k_scale + 4 * h0, v.v_scale + 4 * h0, v.block_table,
                                   v.seq_lens, v.n_phys_pages)
        out, tau, supp = torch.zeros(1, 4, D, device="cuda"), torch.zeros(1, 4, device="cuda"), torch.zeros(1, 4, dtype=torch.int32, device="cuda")
        q = c.q[:, h0 * G:h1 * G]
        if kind == "entmax":
            ekv.ekv_decode8_full(cfg, q, part, out, tau, supp, c.workspace(ekv.EKV_OP_DECODE_FULL, cfg))
            assert torch.equal(out, all_out[:, 2:6]) and torch.equal(tau, all_tau[:, 2:6])
        else:                                    # another number of workgroups: other partial sums
            ekv.ekv_decode8_full_softmax(cfg, q, part, out, tau, c.workspace(ekv.EKV_OP_DECODE8_FULL_SOFTMAX, cfg))
            assert float((out - all_out[:, 2:6]).abs().max()) < 1e-5 and float((tau - all_tau[:, 2:6]).abs().max()) < 1e-5
    assert torch.isfinite(whole[0]).all()


@pytest.mark.parametrize("kind", ["entmax", "softmax"])
def test_many_units(kind):
    """More units than a workgroup keeps prefix sums of: 1100 sequences of 8 KV heads."""
    lens = [(7 * b) % 40 for b in range(1100)]
    c = Cache8(1100, 8, 8, 8, lens, seed=41)
    run_full(c, kind)
    rng = np.random.default_rng(1)
    out, tau, supp = c.out.cpu().numpy().astype(np.float64), c.tau.cpu().numpy(), c.supp.cpu().numpy()
    for b in rng.permutation(1100)[:40].tolist() + [0, 1099]:
        h = int(rng.integers(0, 8))
        if kind == "entmax":
            check_entmax(c, b, h, np.arange(lens[b]), out[b, h], tau[b, h], supp[b, h])
        else:
            check_softmax(c, b, h, np.arange(lens[b]), out[b, h], tau[b, h])


def test_large_and_extreme_scores():
    """Scores of hundreds, where a maximum kept from before is far off, and values near the ends of the scales' range."""
    c = Cache8(1, 4, 1, 16, [600], seed=51, scale=4.0, spread=False)
    run_full(c, "softmax")
    check_all(c, "softmax")
    run_full(c, "entmax")
    check_all(c, "entmax")
    for e in (-100, 119):
        c = Cache8(1, 2, 1, 16, [100], seed=52, spread=False)
        c.scales[1][:] = 2.0 ** e
        c.codes[1][:] = (c.codes[1] & 0x80) | 0x38          # +-1
        c.v_pool.copy_(torch.from_numpy(c.codes[1]).cuda())
        c.v_scale.fill_(2.0 ** e)
        for kind in ("softmax", "entmax"):
            run_full(c, kind)
            check_all(c, kind)


def test_a_key_that_is_no_number():
    c = Cache8(1, 2, 1, 16, [100], seed=53)
    c.k_pool[c.table[0, 2], 0, 5, 3] = 0x7F
    run_full(c, "softmax")
    assert torch.isnan(c.out).all() and torch.isnan(c.tau).all()


def test_same_inputs_same_bits():
    c = Cache8(4, 16, 2, 16, [5000, 200, 3, 9000], seed=61)
    for kind in ("entmax", "softmax"):
        seen = []
        for _ in range(3):
            run_full(c, kind)
            seen.append((c.out.clone(), c.tau.clone()))
        assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for s in seen[1:] for a, b in zip(seen[0], s))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(8, 8), (16, 8), (32, 8), (64, 8)])
@pytest.mark.parametrize("page", [8, 16, 32, 64])
def test_large_calls_are_those_of_their_sequences_alone(page, heads, dtype):
    """A batch whose K (over 64 MiB) takes the score pass that holds its stores back, with a sequence that begins and ends anywhere
    in a wavefront's range, an empty one and single tokens, against the sequences one by one: the same sums, to the last bit."""
    lens = [40011, 1, 0, 33, 25000 + page, 3 * page - 1, 8192]
    B, Hq, Hkv = len(lens), *heads
    M = -(-max(lens) // page)
    g = torch.Generator(device="cuda").manual_seed(page)
    n_phys = B * M
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.randn(B, Hq, D, generator=g, device="cuda").to(dt)
    kp, vp = (torch.randint(0, 127, (n_phys, Hkv, page, D), generator=g, device="cuda", dtype=torch.uint8) % 0x60 | (
        torch.randint(0, 2, (n_phys, Hkv, page, D), generator=g, device="cuda", dtype=torch.uint8) << 7) for _ in range(2))
    ks, vs = (2.0 ** torch.randint(-6, -2, (n_phys, Hkv), generator=g, device="cuda").float() for _ in range(2))
    table = torch.randperm(n_phys, generator=g, device="cuda").view(B, M).to(torch.int32)
    assert B * Hkv * M * page * D >= 64 << 20

    def run(rows, m):
        cfg = ekv.make_config(len(rows), Hq, Hkv, D, page, dtype, 1.5, 0.02, m, m)
        out, tau, supp = torch.zeros(len(rows), Hq, D, device="cuda"), torch.zeros(len(rows), Hq, device="cuda"), torch.zeros(len(rows), Hq, dtype=torch.int32, device="cuda")
        ws = torch.empty(ekv.ekv_workspace_bytes(cfg, ekv.EKV_OP_DECODE_FULL), dtype=torch.uint8, device="cuda")
        t, n = table[rows][:, :m].contiguous(), torch.tensor([lens[b] for b in rows], dtype=torch.int32, device="cuda")
        ekv.ekv_decode8_full(cfg, q[rows].contiguous(), ekv.cache8_view(kp, vp, ks, vs, t, n), out, tau, supp, ws)
        torch.cuda.synchronize()
        return out, tau, supp

    whole = run(list(range(B)), M)
    for b in range(B):
        m = max(1, min(M, -(-lens[b] // page)))
        if Hkv * m * page * D >= 64 << 20:
            m = M
        one = run([b], m)
        for x, y in zip(whole[1:], one[1:]):
            assert torch.equal(x[b:b + 1].view(torch.int32), y.view(torch.int32)), b
        assert torch.allclose(whole[0][b], one[0][0], rtol=0, atol=2e-6 * float(one[0].abs().max()) + 1e-12)


@pytest.mark.parametrize("kind", ["full", "sparse", "softmax", "sparse_softmax"])
@pytest.mark.parametrize("page", [4, 12, 20, 44, 16])
def test_wavefronts_with_many_items_are_those_with_one(page, kind):
    """A batch so large that a wavefront has several groups or steps, whose last tokens and page slots fall on any lane, against
    its sequences one by one.  The scores are the same to the last bit, but the kernel that solves a row goes by the number of rows, and
    with it where the solve starts: either threshold is within 4e-6 max(1, |tau|) of the exact one, and so is every weight's base;
    softmax has another order of its partial sums."""
    B, Hq, Hkv, n_max = 48, 8, 8, 200 * page
    g = torch.Generator(device="cuda").manual_seed(page)
    M = 200
    lens = [n_max - (b * 53) % n_max for b in range(B)]
    kp, vp = (torch.randint(0, 0x60, (B * M, Hkv, page, D), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    ks, vs = (2.0 ** torch.randint(-6, -3, (B * M, Hkv), generator=g, device="cuda").float() for _ in range(2))
    table = torch.randperm(B * M, generator=g, device="cuda").view(B, M).to(torch.int32)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    t = torch.arange(M * page, device="cuda").view(1, M, page) >= n[:, None, None]           # slots behind the last token: no numbers
    kp[table.long()] = torch.where(t[:, :, None, :, None], torch.full_like(kp[:1, :1, :1, :1], 0x7F)[:, None], kp[table.long()])
    vp[table.long()] = torch.where(t[:, :, None, :, None], torch.full_like(vp[:1, :1, :1, :1], 0x7F)[:, None], vp[table.long()])
    q = torch.randn(B, Hq, D, generator=g, device="cuda").to(torch.bfloat16)
    cap = 150
    idx = torch.stack([torch.randperm(M, generator=g, device="cuda")[:cap].sort().values for _ in range(B * Hq)]).view(B, Hq, cap).to(torch.int32)
    n_sel = torch.randint(0, cap + 1, (B, Hq), generator=g, device="cuda", dtype=torch.int32)

    def run(rows):
        cfg = ekv.make_config(len(rows), Hq, Hkv, D, page, "bf16", 1.5, 0.02, M, cap)
        out, tau, supp = torch.zeros(len(rows), Hq, D, device="cuda"), torch.zeros(len(rows), Hq, device="cuda"), torch.zeros(len(rows), Hq, dtype=torch.int32, device="cuda")
        op = {"full": ekv.EKV_OP_DECODE_FULL, "sparse": ekv.EKV_OP_DECODE_SPARSE, "softmax": ekv.EKV_OP_DECODE8_FULL_SOFTMAX,
              "sparse_softmax": ekv.EKV_OP_DECODE8_SPARSE_SOFTMAX}[kind]
        ws = torch.empty(max(256, ekv.ekv_workspace_bytes(cfg, op)), dtype=torch.uint8, device="cuda")
        qr, tr, nr = q[rows].contiguous(), table[rows].contiguous(), n[rows].contiguous()
        view = ekv.cache8_view(kp, vp, ks, vs, tr, nr)
        lists = (idx[rows].contiguous(), n_sel[rows].contiguous()) if "sparse" in kind else ()
        if "softmax" in kind:
            getattr(ekv, "ekv_decode8_" + ("sparse_softmax" if lists else "full_softmax"))(cfg, qr, view, *lists, out, tau, ws)
        else:
            getattr(ekv, "ekv_decode8_" + kind)(cfg, qr, view, *lists, out, tau, supp, ws)
        torch.cuda.synchronize()
        return out, tau, supp

    whole = run(list(range(B)))
    assert torch.isfinite(whole[0]).all()
    for b in range(B):
        one = run([b])
        assert torch.allclose(whole[1][b], one[1][0], rtol=8e-6, atol=8e-6), b
        # weights are (z - tau)^2 <= 1: moved by 2 * 8e-6 at most for each of n tokens, and n float32 additions
        limit = 2.4e-5 * lens[b] * 448.0 * 2.0 ** -3 if "softmax" not in kind else 1e-5 * float(one[0].abs().max())
        assert float((whole[0][b] - one[0][0]).abs().max()) <= limit, b


@pytest.mark.parametrize("page", [4, 12, 16, 60])
def test_steps_of_one_workgroup(page):
    """Sequences of every length around the ends of steps, octets and pages, each by the wavefronts of few workgroups."""
    lens = [32 * k + d for k in (1, 5, 8, 9, 24) for d in (-1, 0, 1, 2, 7, 9)]
    c = Cache8(len(lens), 2, 1, page, lens, seed=page)
    run_full(c, "softmax")
    check_all(c, "softmax")


@pytest.mark.parametrize("page", [12, 16])
@pytest.mark.parametrize("rows", [600, 40000])
def test_a_batch_of_empty_sequences(rows, page):
    """Nothing to look at anywhere, in short and in long capacities, with lists and without."""
    c = Cache8(3, 8, 2, page, [0, 0, 0], row_pages=rows, seed=1, cap=min(rows, 500))
    idx, n = torch.zeros(3, 8, c.cap, dtype=torch.int32, device="cuda"), torch.full((3, 8), c.cap, dtype=torch.int32, device="cuda")
    n[1] = 0

    def empty(first):
        torch.cuda.synchronize()
        ok = not c.out.any() and bool((c.tau == first).all())
        c.out.fill_(float("nan"))
        c.tau.fill_(float("nan"))
        return ok

    for kind, first in (("entmax", np.inf), ("softmax", -np.inf)):
        run_full(c, kind)
        assert empty(first)
    ekv.ekv_decode8_sparse(c.cfg, c.q, c.view(), idx, n, c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_SPARSE))
    assert empty(np.inf) and not c.supp.any()
    ekv.ekv_decode8_sparse_group(c.cfg, c.q, c.view(), idx[:, :2].contiguous(), n[:, :2].contiguous(), c.out, c.tau, c.supp,
                                 c.workspace(ekv.EKV_OP_DECODE_SPARSE))
    assert empty(np.inf)
    ekv.ekv_decode8_sparse_softmax(c.cfg, c.q, c.view(), idx, n, c.out, c.tau, c.workspace(ekv.EKV_OP_DECODE8_SPARSE_SOFTMAX))
    assert empty(-np.inf)


@pytest.mark.parametrize("call", ["sparse", "group", "softmax"])
@pytest.mark.parametrize("page", [12, 16, 64])
def test_long_lists_of_grouped_heads(page, call):
    """Lists longer than one workgroup decodes, of heads that share most of their pages, split over the GPU."""
    rng = np.random.default_rng(page)
    cap = 5000 // page
    c = Cache8(2, 8, 2, page, [9000, 4100], seed=page, cap=cap)
    lists = []
    for b in range(2):
        m = -(-c.lens[b] // page)
        shared = [rng.permutation(m) for _ in range(2)]
        lists.append([sorted(shared[i // (1 if call == "group" else 4)][:min(m, cap) - 3 * (i % 4)].tolist()) for i in range(2 if call == "group" else 8)])
    idx, n = as_tensors(c, lists, cap, rng)
    if call == "softmax":
        ekv.ekv_decode8_sparse_softmax(c.cfg, c.q, c.view(), idx, n, c.out, c.tau, c.workspace(ekv.EKV_OP_DECODE8_SPARSE_SOFTMAX))
    else:
        fn = ekv.ekv_decode8_sparse_group if call == "group" else ekv.ekv_decode8_sparse
        fn(c.cfg, c.q, c.view(), idx, n, c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_SPARSE))
    torch.cuda.synchronize()
    check_all(c, "softmax" if call == "softmax" else "entmax", [[row[h // 4] for h in range(8)] for row in lists] if call == "group" else lists)


def test_many_partial_results_of_many_heads():
    """More workgroups to a KV head than the join takes at once, of more query heads than compute units; an uneven batch."""
    c = Cache8(6, 64, 8, 16, [3000, 2990, 2500, 3000, 100, 2000], seed=71)
    run_full(c, "softmax")
    out, tau = c.out.cpu().numpy().astype(np.float64), c.tau.cpu().numpy()
    rng = np.random.default_rng(0)
    for b in range(6):
        for h in rng.permutation(64)[:10].tolist() + [0, 63]:
            check_softmax(c, b, h, np.arange(c.lens[b]), out[b, h], tau[b, h])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [4, 12, 20, 36, 48, 60, 16])
def test_the_longest_rows_of_one_workgroup(page, dtype):
    """Lists and sequences about as long as one workgroup takes from scores to output, and one page beyond, whose wavefronts have
    several groups each; few rows and many, a full list, an empty one and some of every length between."""
    rng = np.random.default_rng(page)
    for B, tokens in ((2, 2048), (8, 4096), (2, 2048 + page), (8, 4096 + page)):
        cap = tokens // page
        c = Cache8(B, 16, 2, page, [2 * tokens - 301 * b for b in range(B)], seed=page, cap=cap, dtype=dtype)
        lists = []
        for b in range(B):
            m = -(-c.lens[b] // page)
            keep = [min(m, cap) if h == 0 else 0 if h == 1 else int(rng.integers(1, min(m, cap))) for h in range(16)]
            lists.append([sorted(rng.permutation(m)[:k].tolist()) for k in keep])
        idx, n = as_tensors(c, lists, cap, rng)
        ekv.ekv_decode8_sparse(c.cfg, c.q, c.view(), idx, n, c.out, c.tau, c.supp, c.workspace(ekv.EKV_OP_DECODE_SPARSE))
        torch.cuda.synchronize()
        check_all(c, "entmax", lists)
    for n in (1024 // page * page, 1024 // page * page - page // 2, 1024 // page * page + 1):
        c = Cache8(3, 16, 2, page, [n, n - 600, 1], seed=n, dtype=dtype)
        run_full(c, "entmax")
        check_all(c, "entmax")
