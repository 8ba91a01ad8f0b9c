"""The operators of include/kv.h on the GPU against the float64 oracle (oracle/kv_ref.py): sizes, layouts, strides, positions,
pages and masks where they can go wrong.  Bounds are derived in kv_util.py and beside the checks."""
import numpy as np
import pytest
import torch

from oracle import kv_ref as orc
from tests import kv_util as ku
from tests.kv_util import NAN, f64

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _A():
    import paper_2605_10905_amd as A

    return A


# ---- rope_qkv ----------------------------------------------------------------------------------

ROPE = [
    # B, N, Hq, Hkv, d, norm, rot, interleaved, positions given, elements between the rows
    (1, 1, 1, 1, 64, True, 64, False, False, 0), (1, 1, 1, 1, 128, False, 0, False, False, 0),
    (2, 5, 3, 1, 128, True, 128, False, True, 8), (2, 37, 6, 2, 64, True, 32, True, True, 0), (1, 33, 32, 8, 128, True, 64, True, False, 24),
    (3, 17, 7, 7, 64, False, 48, False, True, 0), (1, 130, 5, 5, 128, True, 16, False, False, 0), (2, 9, 16, 4, 128, False, 96, True, True, 8),
    (1, 300, 2, 1, 64, True, 16, True, False, 0), (4, 3, 12, 12, 128, True, 112, False, True, 0), (1, 7, 9, 3, 64, True, 0, False, True, 16),
    # rows of a wave's step from one token, from two, from many; steps that end behind the last row
    (5, 1000, 1, 1, 128, True, 128, False, True, 0), (1, 3001, 5, 1, 64, True, 64, False, False, 0), (2, 1500, 6, 1, 128, True, 64, True, True, 8), (3, 700, 12, 2, 64, False, 64, False, True, 0),
]


def _rope_inputs(case, seed):
    B, N, Hq, Hkv, d, norm, rot, inter, given, gap = case
    gen = ku.generator(seed)
    T, width = B * N, (Hq + 2 * Hkv) * d
    npos = max(400, N)
    pos = torch.randint(0, npos, (T,), generator=gen, device="cuda", dtype=torch.int32) if given else None
    at = pos.cpu().tolist() if given else list(range(N)) * B
    tab = ku.table(npos, rot) if rot else None
    qkv = ku.rows(gen, T, width, width + gap, 1.5)
    w = ku.weights(gen, d, norm)
    return gen, T, width, npos, pos, at, tab, qkv, w


def _tokens(x):
    """[B, H, N, d] as [B N, H, d]."""
    return f64(x).transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])


def _host_table(tab):
    return None if tab is None else tab.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("case", ROPE, ids=str)
def test_rope_qkv(case):
    A = _A()
    B, N, Hq, Hkv, d, norm, rot, inter, given, gap = case
    gen, T, width, npos, pos, at, tab, qkv, w = _rope_inputs(case, 11 + sum(case))
    outs = [ku.guarded((B, h, N, d), torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    A.rope_qkv(qkv, width + gap, *w, EPS, tab, npos, rot, inter, pos, *(o for o, _ in outs), B, Hq, Hkv, N, d)
    torch.cuda.synchronize()
    x = f64(qkv).reshape(T, -1, d)
    want = orc.rope_qkv(x, Hq, Hkv, *map(ku.arr, w), EPS, _host_table(tab), at, rot, inter)
    plain = orc.rope_qkv(x, Hq, Hkv, *map(ku.arr, w), EPS, None, at, 0, inter)  # (before the rotation: the size of a row)
    for name, (o, intact), ref, y in zip("qkv", outs, want, plain):
        assert intact(), name
        got = _tokens(o)
        assert np.isfinite(got).all()
        if name == "v":
            assert np.array_equal(got, ref)
        else:
            assert (np.abs(got - ref) <= ku.forward_bound(ref, ku.row_size(y))).all(), name


@pytest.mark.parametrize("case", ROPE, ids=str)
def test_rope_qkv_bwd(case):
    A = _A()
    B, N, Hq, Hkv, d, norm, rot, inter, given, gap = case
    gen, T, width, npos, pos, at, tab, qkv, w = _rope_inputs(case, 12 + sum(case))
    grads = [torch.randn((B, h, N, d), generator=gen, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)]
    dld = width + 16
    dqkv, intact = ku.guarded((T, dld), torch.bfloat16, 5.0)
    dw = [ku.guarded((d,), torch.float32) if norm else (None, lambda: True) for _ in range(2)]
    ws, ws_intact = ku.guarded((A.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4,), torch.float32) if norm else (None, lambda: True)
    args = (*w, EPS, tab, npos, rot, inter, pos)

    def run(out, dws):
        A.rope_qkv_bwd(*grads, qkv if norm else None, width + gap, *args, out, dld, *dws, ws, B, Hq, Hkv, N, d)
        torch.cuda.synchronize()

    run(dqkv[:, :width], [x for x, _ in dw])
    assert intact() and ws_intact() and all(f() for _, f in dw)
    assert bool((dqkv[:, width:] == 5).all())  # what lies between the rows
    x = f64(qkv).reshape(T, -1, d)
    g = [_tokens(t) for t in grads]
    want, *want_w = orc.rope_qkv_bwd(*g, x, Hq, Hkv, *map(ku.arr, w), EPS, _host_table(tab), at, rot, inter)
    got = f64(dqkv[:, :width]).reshape(T, -1, d)
    assert np.array_equal(got[:, Hq + Hkv:], g[2])
    for lo, hi, dz, wt in ((0, Hq, g[0], w[0]), (Hq, Hq + Hkv, g[1], w[1])):
        # at most 48 roundings to 32 bits (2^-24 each) of a row's largest terms: r |g| w and r |xhat| mean(g w xhat), |g| <= 2 max |dz|
        size = 2 * ku.row_size(dz)
        if wt is not None:
            n = orc.rms(x[:, lo:hi], EPS)
            hat = ku.row_size(x[:, lo:hi]) / n
            size = size * np.abs(ku.arr(wt)).max() / n * (1 + hat * hat)
        ref = want[:, lo:hi]
        assert (np.abs(got[:, lo:hi] - ref) <= 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + 2.0 ** -18 * size + 1e-38).all()
        if wt is not None:
            # each term 48 roundings, and it goes through at most 208 additions of sums no larger than that of all magnitudes
            total = (2 * np.abs(dz).max(-1, keepdims=True) * np.ones(d) * np.abs(x[:, lo:hi]) / n).sum((0, 1))
            k = 0 if lo == 0 else 1
            assert (np.abs(f64(dw[k][0]) - want_w[k]) <= 2.0 ** -16 * total).all()
    again, dws = torch.full_like(dqkv, 5.0), [torch.full_like(t, 1e30) if t is not None else None for t, _ in dw]
    if ws is not None:
        ws.fill_(1e30)  # what the workspace held before is not read
    run(again[:, :width], dws)
    assert torch.equal(again.view(torch.int16), dqkv.view(torch.int16)) and all(t is None or torch.equal(t, u) for t, (u, _) in zip(dws, dw))


def test_rope_gradient_against_differences():
    """The directional derivative of the forward oracle (64 bits) along random directions, inputs as they are stored."""
    A = _A()
    B, N, Hq, Hkv, d, rot = 2, 11, 6, 2, 64, 64
    gen = ku.generator(5)
    T, width, npos = B * N, (Hq + 2 * Hkv) * d, 50
    qkv, w, tab = ku.rows(gen, T, width, width), ku.weights(gen, d, True), ku.table(npos, rot)
    pos = torch.randint(0, npos, (T,), generator=gen, device="cuda", dtype=torch.int32)
    grads = [torch.randn((B, h, N, d), generator=gen, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)]
    dqkv, dw = torch.empty_like(qkv), [torch.empty(d, device="cuda") for _ in range(2)]
    ws = torch.empty(A.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4, device="cuda")
    A.rope_qkv_bwd(*grads, qkv, width, *w, EPS, tab, npos, rot, False, pos, dqkv, width, *dw, ws, B, Hq, Hkv, N, d)
    torch.cuda.synchronize()
    g, x, ww, at = [_tokens(t) for t in grads], f64(qkv).reshape(T, -1, d), [f64(t) for t in w], pos.cpu().tolist()
    loss = lambda x, wq, wk: sum((a * b).sum() for a, b in zip(g, orc.rope_qkv(x, Hq, Hkv, wq, wk, EPS, _host_table(tab), at, rot, False)))
    rng, h = np.random.default_rng(6), 1e-4
    dx = f64(dqkv).reshape(T, -1, d)
    for _ in range(4):
        u = rng.standard_normal(x.shape)
        diff = (loss(x + h * u, *ww) - loss(x - h * u, *ww)) / (2 * h)
        assert abs(diff - (dx * u).sum()) <= 2.0 ** -8 * np.abs(dx * u).sum() + 1e-6 * np.abs(diff)  # (each element half a bf16 step off)
        u = rng.standard_normal(d)
        for i in range(2):
            up, down = [list(ww) for _ in range(2)]
            up[i], down[i] = ww[i] + h * u, ww[i] - h * u
            diff = (loss(x, *up) - loss(x, *down)) / (2 * h)
            assert abs(diff - f64(dw[i]) @ u) <= 1e-5 * np.abs(f64(dw[i]) * u).sum() + 1e-6 * np.abs(diff)


def test_positions_outside_the_table_are_nan_and_nothing_else():
    A = _A()
    B, N, Hq, Hkv, d, npos = 2, 6, 4, 2, 128, 20
    gen = ku.generator(7)
    width = (Hq + 2 * Hkv) * d
    qkv, w, tab = ku.rows(gen, B * N, width, width), ku.weights(gen, d, True), ku.table(npos, d)
    pos = torch.arange(B * N, dtype=torch.int32, device="cuda")
    outs = [torch.empty((B, h, N, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    run = lambda: A.rope_qkv(qkv, width, *w, EPS, tab, npos, d, False, pos, *outs, B, Hq, Hkv, N, d)
    run()
    want = [o.clone() for o in outs]
    bad = {1: -1, 5: npos, 7: 2 ** 31 - 1, 10: -2 ** 31}
    for t, v in bad.items():
        pos[t] = v
    run()
    torch.cuda.synchronize()
    for o, ref, rotated in zip(outs, want, (True, True, False)):
        for t in range(B * N):
            row, r = o[t // N, :, t % N], ref[t // N, :, t % N]
            if t in bad and rotated:
                assert bool(row.isnan().all())
            else:
                assert torch.equal(row, r)
    dqkv, dw = torch.empty_like(qkv), [torch.empty(d, device="cuda") for _ in range(2)]
    ws = torch.empty(A.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4, device="cuda")
    A.rope_qkv_bwd(*outs, qkv, width, *w, EPS, tab, npos, d, False, pos, dqkv, width, *dw, ws, B, Hq, Hkv, N, d)
    torch.cuda.synchronize()
    rows = dqkv.view(B * N, -1, d)
    assert bool(rows[list(bad), :Hq + Hkv].isnan().all()) and all(bool(x.isnan().all()) for x in dw)
    good = [t for t in range(B * N) if t not in bad]
    assert bool(rows[good].isfinite().all()) and bool(rows[:, Hq + Hkv:].isfinite().all())


def test_rope_of_more_tokens_than_a_launch_has_waves_for():
    """12 million tokens of three heads: more than 2^31 elements and 2^32 bytes, and more tasks than workgroups start; rows at both ends and between."""
    A = _A()
    N, d, npos = 12_000_000, 64, 90
    gen = ku.generator(9)
    width, w, tab = 3 * d, ku.weights(gen, d, True), ku.table(npos, d)
    qkv = torch.empty((N, width), dtype=torch.bfloat16, device="cuda")
    for i in range(0, N, 1_000_000):
        qkv[i:i + 1_000_000] = torch.randn((min(1_000_000, N - i), width), generator=gen, device="cuda").bfloat16()
    pos = torch.randint(0, npos, (N,), generator=gen, device="cuda", dtype=torch.int32)
    outs = [torch.full((1, 1, N, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    A.rope_qkv(qkv, width, *w, EPS, tab, npos, d, False, pos, *outs, 1, 1, 1, N, d)
    torch.cuda.synchronize()
    assert all(bool(o.isfinite().all()) for o in outs) and torch.equal(outs[2][0, 0], qkv[:, 2 * d:])
    at = torch.cat([torch.arange(50), torch.randint(0, N, (300,), generator=torch.Generator().manual_seed(3)), torch.arange(N - 50, N)]).cuda()
    x, p = f64(qkv[at]).reshape(-1, 3, d), pos[at].cpu().tolist()
    args = (1, 1, *map(ku.arr, w), EPS, _host_table(tab), p, d, False)
    want, plain = orc.rope_qkv(x, *args), orc.rope_qkv(x, *args[:-2], 0, False)
    for o, ref, y in zip(outs[:2], want, plain):
        assert (np.abs(f64(o[0, 0, at])[:, None] - ref) <= ku.forward_bound(ref, ku.row_size(y))).all()
    dqkv, dw = torch.full_like(qkv, NAN), [torch.empty(d, device="cuda") for _ in range(2)]
    ws = torch.empty(A.rope_qkv_bwd_workspace_bytes(1, 1, 1, N, d) // 4, device="cuda")
    A.rope_qkv_bwd(*outs, qkv, width, *w, EPS, tab, npos, d, False, pos, dqkv, width, *dw, ws, 1, 1, 1, N, d)
    torch.cuda.synchronize()
    assert bool(dqkv.isfinite().all()) and torch.equal(dqkv[:, 2 * d:], qkv[:, 2 * d:])
    g = [f64(o[0, 0, at])[:, None] for o in outs]
    ref, _, _ = orc.rope_qkv_bwd(*g, x, *args)
    for h, wt in enumerate(w):  # (the bound of test_rope_qkv_bwd)
        n = orc.rms(x[:, h:h + 1], EPS)
        size = 2 * ku.row_size(g[h]) * np.abs(ku.arr(wt)).max() / n * (1 + (ku.row_size(x[:, h:h + 1]) / n) ** 2)
        got = f64(dqkv[at]).reshape(-1, 3, d)[:, h:h + 1]
        assert (np.abs(got - ref[:, h:h + 1]) <= 2.0 ** -8 * np.abs(ref[:, h:h + 1]) * (1 + 2.0 ** -8) + 2.0 ** -18 * size + 1e-38).all()
    # q's gradient is its output here, and rotations keep lengths: the weight's gradient is w_i times the sum of xhat_i^2 mixed over the pair;
    # summed over all features with those weights, sum_i w_i dw_i = sum of |y|^2 = sum of |z|^2
    for o, wt, got in zip(outs, w, dw):
        total = float(sum(o[0, 0, i:i + 1_000_000].double().square().sum() for i in range(0, N, 1_000_000)))
        assert abs(float((got.double() * wt.double()).sum()) - total) <= 2.0 ** -8 * total  # (z rounded to bf16)


# ---- kv_append ---------------------------------------------------------------------------------

APPEND = [
    # new tokens and keys before of every sequence, Hq, Hkv, d, norm, rot, interleaved, page, fp8
    ([1], [0], 1, 1, 64, True, 64, False, 16, False), ([1, 1, 1], [15, 16, 40], 8, 2, 128, True, 128, False, 16, False),
    ([1, 1, 1], [15, 16, 40], 8, 2, 128, True, 128, False, 16, True), ([33, 1, 20], [0, 31, 5], 6, 3, 64, False, 32, True, 32, True),
    ([70, 130], [3, 0], 32, 8, 128, False, 0, False, 64, False), ([5, 40], [300, 1], 3, 1, 128, True, 96, False, 128, True),
    ([17], [1000], 4, 4, 64, True, 64, True, 256, False), ([9, 2], [0, 2040], 2, 2, 128, True, 128, False, 1024, True),
]


def _append_check(got, ref, y, fp8, descale):
    if not fp8:
        return (np.abs(got - ref) <= ku.forward_bound(ref, ku.row_size(y))).all()
    # codes: half a step, 2^-4 of the value or 2^-10 below 2^-6; the 32-bit value before it as in forward_bound and one quotient more
    lim, err = np.clip(ref / descale, -448, 448), 2.0 ** -18 * ku.row_size(y) / descale
    return (np.abs(got - lim) <= np.maximum(2.0 ** -4 * (np.abs(lim) + err), 2.0 ** -10) + err).all()


@pytest.mark.parametrize("case", APPEND, ids=str)
def test_kv_append(case):
    A = _A()
    new, before, Hq, Hkv, d, norm, rot, inter, page, fp8 = case
    gen = ku.generator(21 + sum(new))
    S, T, width = len(new), sum(new), (Hq + 2 * Hkv) * d
    cache = ku.Cache(gen, [a + b for a, b in zip(new, before)], Hkv, d, page, fp8, fill=False)
    npos = max(a + b for a, b in zip(new, before))
    seq = [s for s, n in enumerate(new) for _ in range(n)]
    pos = [before[s] + i for s, n in enumerate(new) for i in range(n)]
    tab, w, qkv = (ku.table(npos, rot) if rot else None), ku.weights(gen, d, norm), ku.rows(gen, T, width, width + 8, 3.0)
    order = torch.randperm(T, generator=gen, device="cuda").cpu().tolist()  # tokens in no order
    seq, pos = [seq[i] for i in order], [pos[i] for i in order]
    one_each = new == [1] * S
    if one_each:
        seq, pos = list(range(S)), before
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q, intact = ku.guarded((T, Hq, d), torch.bfloat16)
    A.kv_append(qkv, width + 8, *w, EPS, tab, npos, rot, inter, ints(pos), None if one_each else ints(seq), cache.pages, q, cache.k, cache.v, T, S, Hq, Hkv, d,
                cache.width, page, cache.num, A.ATTN_FP8_E4M3 if fp8 else A.ATTN_BF16, *cache.descale)
    torch.cuda.synchronize()
    assert intact()
    x = f64(qkv).reshape(T, -1, d)
    want = orc.rope_qkv(x, Hq, Hkv, *map(ku.arr, w), EPS, _host_table(tab), pos, rot, inter)
    plain = orc.rope_qkv(x, Hq, Hkv, *map(ku.arr, w), EPS, None, pos, 0, inter)
    assert (np.abs(f64(q) - want[0]) <= ku.forward_bound(want[0], ku.row_size(plain[0]))).all()
    pages = cache.pages.cpu().numpy()
    for buf, ref, y, f in ((cache.k, want[1], plain[1], cache.descale[0]), (cache.v, want[2], plain[2], cache.descale[1])):
        held = f64(buf)
        written = np.zeros((cache.num, page), bool)
        for t in range(T):
            at = pages[seq[t], pos[t] // page], pos[t] % page
            written[at] = True
            assert _append_check(held[at[0], :, at[1]], ref[t], y[t], fp8, f), t
        assert np.isnan(held.transpose(0, 2, 1, 3)[~written]).all()  # nothing else is touched


@pytest.mark.parametrize("fp8", [False, True])
def test_kv_append_padding_and_what_does_not_fit(fp8):
    A = _A()
    Hq, Hkv, d, page, npos, S = 4, 2, 64, 16, 60, 3
    gen = ku.generator(31)
    width = (Hq + 2 * Hkv) * d
    cache = ku.Cache(gen, [48, 48, 48], Hkv, d, page, fp8, fill=False)
    cache.pages[1, 1], cache.pages[2, 0] = -1, cache.num  # no page, and one that does not exist
    #        fine     padding  pos>=npos  no such sequence  beyond the table   no page  bad page  fine
    tokens = [(0, 5), (0, -1), (0, npos), (3, 1), (-1, 2), (1, 50), (1, 17), (2, 3), (2, 20), (0, -2 ** 31), (0, 2 ** 31 - 1)]
    kind = ["fine", "skip", "nan", "nan", "nan", "q", "q", "q", "fine", "skip", "nan"]
    T = len(tokens)
    qkv, w, tab = ku.rows(gen, T, width, width), ku.weights(gen, d, True), ku.table(npos, d)
    q = torch.full((T, Hq, d), 3.0, dtype=torch.bfloat16, device="cuda")
    seq, pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*tokens))
    A.kv_append(qkv, width, *w, EPS, tab, npos, d, False, pos, seq, cache.pages, q, cache.k, cache.v, T, S, Hq, Hkv, d, cache.width, page, cache.num,
                A.ATTN_FP8_E4M3 if fp8 else A.ATTN_BF16, *cache.descale)
    torch.cuda.synchronize()
    held, pages = f64(cache.k), cache.pages.cpu().numpy()
    written = ~np.isnan(held).any((1, 3))
    want = np.zeros_like(written)
    for t, (what, (s, p)) in enumerate(zip(kind, tokens)):
        row = q[t].float()
        assert bool({"fine": row.isfinite(), "q": row.isfinite(), "nan": row.isnan(), "skip": row == 3}[what].all()), (t, what)
        if what == "fine":
            want[pages[s, p // page], p % page] = True
    assert np.array_equal(written, want)


def test_kv_append_saturates_and_keeps_nan():
    A = _A()
    d, page = 64, 16
    cache = ku.Cache(ku.generator(41), [1], 1, d, page, True, fill=False)
    row = torch.zeros((1, 3 * d), device="cuda")
    row[0, 2 * d:2 * d + 8] = torch.tensor([1e4, -1e4, float("inf"), -float("inf"), NAN, 448 * 0.021, 2.0 ** -9 * 0.021, 0.0], device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.empty((1, 1, d), dtype=torch.bfloat16, device="cuda")
    A.kv_append(row.bfloat16(), 3 * d, None, None, 0.0, None, 0, 0, False, zero, None, cache.pages, q, cache.k, cache.v, 1, 1, 1, 1, d, cache.width, page,
                cache.num, A.ATTN_FP8_E4M3, 0.013, 0.021)
    torch.cuda.synchronize()
    got = f64(cache.v[cache.pages[0, 0].long(), 0, 0])
    assert got[:4].tolist() == [448, -448, 448, -448] and np.isnan(got[4]) and got[5] == 448 and got[6] == 2.0 ** -9 and not got[7:].any()


# ---- kv_decode ---------------------------------------------------------------------------------


def _decode(q, cache, scale, ws=None, stream=None):
    A = _A()
    B, Hq, d = q.shape
    Hkv = cache.k.shape[1]
    o, o_intact = ku.guarded((B, Hq, d), torch.bfloat16)
    lse, lse_intact = ku.guarded((B, Hq), torch.float32)
    nbytes = A.kv_decode_workspace_bytes(B, Hq, Hkv, d)
    assert nbytes % 4 == 0
    if ws is None:
        ws, ws_intact = ku.guarded((nbytes // 4,), torch.float32)
    else:
        ws_intact = lambda: True
    lens = torch.tensor(cache.lens, dtype=torch.int32, device="cuda")
    A.kv_decode(q, cache.k, cache.v, cache.pages, lens, o, lse, ws, B, Hq, Hkv, d, cache.width, cache.page, cache.num, scale,
                A.ATTN_FP8_E4M3 if cache.fp8 else A.ATTN_BF16, *cache.descale, stream=stream)
    torch.cuda.synchronize()
    assert o_intact() and lse_intact() and ws_intact()
    return o, lse


def _q(gen, B, Hq, d, sigma=1.0):
    return (torch.randn((B, Hq, d), generator=gen, device="cuda") * sigma).bfloat16()


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257, 500, 1023]
DECODE = [(Hq, Hkv, d, page, fp8) for d in (64, 128) for fp8 in (False, True)
          for Hq, Hkv, page in ((1, 1, 16), (8, 1, 16), (6, 2, 32), (16, 1, 64), (5, 5, 128), (40, 2, 256), (17, 1, 1024), (33, 1, 16), (64, 1, 32), (130, 2, 64))]


@pytest.mark.parametrize("Hq,Hkv,d,page,fp8", DECODE)
def test_kv_decode_ragged(Hq, Hkv, d, page, fp8):
    gen = ku.generator(51 + Hq + page)
    cache = ku.Cache(gen, LENS, Hkv, d, page, fp8)
    q = _q(gen, len(LENS), Hq, d)
    o, lse = _decode(q, cache, d ** -0.5)
    ku.decode_check(o, lse, q, cache, d ** -0.5)
    o2, lse2 = _decode(q, cache, d ** -0.5)
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("lens", [[1], [0], [7], [4001], [20000, 3], [0, 0, 5000, 0], [1] * 70, [33] * 300, [5] * 64 + [9000], [0] * 130], ids=lambda x: f"{len(x)}x{max(x)}")
@pytest.mark.parametrize("Hq,Hkv,d,fp8", [(8, 2, 128, False), (4, 4, 64, False), (8, 1, 128, True), (24, 1, 64, True)])
def test_kv_decode_splits(lens, Hq, Hkv, d, fp8):
    """Few long sequences (split over many workgroups), many short ones, both."""
    gen = ku.generator(61 + len(lens))
    cache = ku.Cache(gen, lens, Hkv, d, 16, fp8)
    q = _q(gen, len(lens), Hq, d)
    o, lse = _decode(q, cache, 0.11)
    ku.decode_check(o, lse, q, cache, 0.11)


@pytest.mark.parametrize("lens,Hq,Hkv,d,fp8", [
    ([128] * 32, 16, 8, 128, False),         # as many (sequence, key head) pairs as workgroups: each of them takes one whole
    ([256] * 64, 20, 4, 64, False), ([257] * 32, 8, 8, 128, True), ([100] * 300, 3, 1, 128, False),
    ([70000], 8, 1, 128, False), ([70001], 64, 1, 64, True), ([33000, 33000], 70, 2, 128, False), ([16001, 7, 0, 40000], 33, 1, 128, True),
    ([4000] * 20 + [1] * 9, 32, 1, 64, False), ([999] * 40, 64, 1, 128, True), ([50000, 64], 16, 2, 64, False), ([32768], 4, 1, 128, False),
    ([32 * 1023], 4, 1, 128, False), ([32 * 1025], 4, 1, 128, False), ([32 * 1028, 32 * 4], 5, 1, 128, False),
    # fewer tiles than waves, a number that leaves a workgroup incomplete, as many as workgroups and one more
    ([32 * 1022 - 5], 4, 1, 128, False), ([32 * 901, 40], 6, 1, 128, False), ([32 * 256], 8, 1, 128, False), ([32 * 257], 8, 1, 128, False), ([32 * 100, 32 * 156 - 1, 9], 2, 1, 128, False),
    ([64 * 255, 64], 40, 1, 128, True), ([64 * 130 + 1, 64 * 131], 3, 1, 64, False), ([128 * 300, 0, 128 * 400], 8, 1, 64, True), ([90] * 45, 30, 5, 128, False),
], ids=lambda x: f"{len(x)}x{max(x)}" if isinstance(x, list) else str(x))
def test_kv_decode_pieces_that_share_a_workgroup(lens, Hq, Hkv, d, fp8):
    """Pieces of the work that begin and end with a workgroup's and that do not: sums of four waves, of one, of all."""
    gen = ku.generator(65 + len(lens))
    cache = ku.Cache(gen, lens, Hkv, d, 64, fp8)
    q = _q(gen, len(lens), Hq, d)
    o, lse = _decode(q, cache, d ** -0.5)
    ku.decode_check(o, lse, q, cache, d ** -0.5)
    o2, lse2 = _decode(q, cache, d ** -0.5)
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("fp8", [False, True])
def test_kv_decode_many_short_sequences(fp8):
    gen = ku.generator(63)
    lens = [(37 * i) % 41 for i in range(1500)]
    cache = ku.Cache(gen, lens, 1, 64, 16, fp8)
    q = _q(gen, len(lens), 2, 64)
    o, lse = _decode(q, cache, 0.125)
    ku.decode_check(o, lse, q, cache, 0.125)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 64])
def test_kv_decode_hidden_pages(page, fp8):
    """Entries outside the cache hide their keys; a sequence with none left is empty; lengths beyond the table end with it."""
    gen = ku.generator(71)
    lens = [200, 200, 70, 400, 1, 330]
    cache = ku.Cache(gen, lens, 2, 128, page, fp8)
    cache.pages[0, 0], cache.pages[0, 2] = -1, cache.num
    cache.pages[1, :] = -5  # nothing left
    cache.pages[3, ::2] = 2 ** 31 - 1
    cache.lens = [200, 200, 70, 2 ** 31 - 1, 1, 330]  # the fourth: as long as the table
    if cache.width * page > 400:
        cache.pages[3, 400 // page:] = -1
    cache.lens[4] = -3
    q = _q(gen, len(lens), 8, 128)
    o, lse = _decode(q, cache, 0.09)
    ku.decode_check(o, lse, q, cache, 0.09)
    assert not bool(o[1].any()) and bool(torch.isneginf(lse[1]).all()) and bool(torch.isneginf(lse[4]).all())


@pytest.mark.parametrize("d", [64, 128])
def test_kv_decode_scores_of_every_size(d):
    """One dominant key late or early, equal scores, scores that rise from key to key, very small and very large ones; a feature that
    hides keys with scores of -1e4, of bf16's lowest value, and -inf."""
    gen = ku.generator(81)
    lens = [300] * 8
    cache = ku.Cache(gen, lens, 1, d, 32, False)
    q = _q(gen, 8, 4, d)
    pages = cache.pages.long()

    def keys(b):
        return cache.k[pages[b]].clone()  # [pages, 1, page, d]

    def put(b, k):
        cache.k[pages[b]] = k

    flat = lambda k: k[:, 0].reshape(-1, d)
    for b, change in enumerate(("last", "first", "equal", "rise", "tiny", "hide4", "hidelow", "hideinf")):
        k = keys(b)
        f = k[:, 0].reshape(-1, d).float()
        if change in ("last", "first"):
            f[299 if change == "last" else 0] = 4.0 * q[b, 1].float()
        elif change == "equal":
            f[:] = 0.25
        elif change == "rise":
            f[:, 0] = torch.arange(f.shape[0], device="cuda") * 0.5
            q[b, :, 0] = 8.0
        elif change == "tiny":
            f *= 1e-30
        else:
            q[b, :, 3] = 1.0
            f[:, 3] = 0.0
            f[::3, 3] = {"hide4": -1e4, "hidelow": torch.finfo(torch.bfloat16).min, "hideinf": -float("inf")}[change]
            f[0, 3] = f[::3, 3][1]
        k[:, 0] = f.view(k.shape[0], k.shape[2], d).bfloat16()
        # what lies behind the last key stays poisoned
        k.view(-1, d)[300:] = NAN
        put(b, k)
    o, lse = _decode(q, cache, 0.125)
    got, got_lse = f64(o), lse.cpu().numpy()
    for b in range(8):
        k, v = (x[:, :] for x in cache.visible(b))
        if b >= 6:  # hidden keys weigh nothing: the oracle without them
            seen = np.array([j for j in range(300) if j % 3])
            k, v = k[:, seen], v[:, seen]
        want, want_lse = orc.decode(f64(q[b]), k, v, 0.125)
        # bound as decode_check's, with the largest score magnitude of visible keys
        a = 0.125 * (np.abs(f64(q[b])) @ np.abs(k[0]).T).max()
        rel = 2.0 ** -24 * (2 * (d + 8) * a + 64) + 2.0 ** -20
        p = np.exp(0.125 * f64(q[b]) @ k[0].T - want_lse[:, None])
        bound = (2.0 ** -8 + rel) * (p @ np.abs(v[0])) * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) + 1e-30
        assert (np.abs(got[b] - want) <= bound).all(), b
        assert (np.abs(got_lse[b] - want_lse) <= rel + 2.0 ** -22 * (1 + np.abs(want_lse))).all(), b


def test_kv_decode_not_a_number_stays_in_its_row():
    gen = ku.generator(91)
    cache = ku.Cache(gen, [100, 100, 100, 100], 2, 128, 16, False)
    q = _q(gen, 4, 4, 128)
    clean, clean_lse = _decode(q, cache, 0.1)
    q[1, 2, 5] = NAN                                         # one query row
    cache.k[cache.pages[2, 3].long(), 0, 2, 7] = NAN          # a visible key of head 0
    cache.v[cache.pages[3, 6].long(), 1, 3, 9] = float("inf")  # a visible value (key 99) of head 1
    cache.v[cache.pages[3, 6].long(), 1, 4:] = -float("inf")  # behind the last key
    o, lse = _decode(q, cache, 0.1)
    bad = torch.zeros(o.shape, dtype=torch.bool, device="cuda")
    bad[1, 2], bad[2, :2] = True, True
    assert bool(o[bad].isnan().all())
    assert bool(torch.isposinf(o[3, 2:, 9]).all())
    bad[3, 2:, 9] = True
    assert torch.equal(o[~bad], clean[~bad])
    same = torch.ones(lse.shape, dtype=torch.bool, device="cuda")
    same[1, 2], same[2, :2] = False, False
    assert torch.equal(lse[same], clean_lse[same]) and bool(lse[~same].isnan().all())


def test_kv_decode_in_a_cache_of_more_than_2_to_31_elements():
    """Pages on both sides of 2^31 elements and of 2^32 bytes."""
    A = _A()
    Hkv, d, page = 8, 128, 64
    num = 2 ** 31 // (Hkv * d * page) + 40
    gen = ku.generator(95)
    small = ku.Cache(gen, [700, 90], Hkv, d, page, False)
    big = [torch.empty((num, Hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    where = torch.randperm(small.num, generator=gen, device="cuda")
    where = torch.where(where % 2 == 0, num - 1 - where, num // 2 - 8 + where)  # near the end, and around 2^30 elements
    for dst, src in zip(big, (small.k, small.v)):
        dst[where] = src
    q = _q(gen, 2, 32, d)
    want = _decode(q, small, 0.088)
    ku.decode_check(*want, q, small, 0.088)
    pages = torch.where(small.pages >= 0, where[small.pages.clamp_min(0).long()].int(), -1)
    o, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    ws = torch.empty(A.kv_decode_workspace_bytes(2, 32, Hkv, d) // 4, device="cuda")
    lens = torch.tensor(small.lens, dtype=torch.int32, device="cuda")
    A.kv_decode(q, *big, pages, lens, o, lse, ws, 2, 32, Hkv, d, small.width, page, num, 0.088, A.ATTN_BF16)
    torch.cuda.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    # and new tokens are put there
    width = (32 + 2 * Hkv) * d
    qkv, pos = ku.rows(gen, 2, width, width), lens - 1
    A.kv_append(qkv, width, None, None, 0.0, None, 0, 0, False, pos, None, pages, q, *big, 2, 2, 32, Hkv, d, small.width, page, num, A.ATTN_BF16)
    torch.cuda.synchronize()
    x = qkv.view(2, -1, d)
    for b in range(2):
        at = pages[b, int(pos[b]) // page].long()
        assert torch.equal(big[0][at, :, int(pos[b]) % page], x[b, 32:40]) and torch.equal(big[1][at, :, int(pos[b]) % page], x[b, 40:])


def test_kv_decode_on_two_streams_at_once():
    gen = ku.generator(97)
    caches = [ku.Cache(gen, lens, 2, 128, 16, False) for lens in ([3000, 10], [40, 900, 2000])]
    qs = [_q(gen, len(c.lens), 8, 128) for c in caches]
    want = [_decode(q, c, 0.1) for q, c in zip(qs, caches)]
    A = _A()
    streams = [torch.cuda.Stream() for _ in caches]
    outs = []
    for _ in range(20):
        for s, q, c in zip(streams, qs, caches):
            B = len(c.lens)
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                o, lse = torch.empty_like(q), torch.empty((B, 8), device="cuda")
                ws = torch.empty(A.kv_decode_workspace_bytes(B, 8, 2, 128) // 4, device="cuda")
                lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
                A.kv_decode(q, c.k, c.v, c.pages, lens, o, lse, ws, B, 8, 2, 128, c.width, 16, c.num, 0.1, A.ATTN_BF16)
                outs.append((o, lse))
    torch.cuda.synchronize()
    for i, (o, lse) in enumerate(outs):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


def test_tensors_of_another_device_are_refused():
    """With one GPU: the same call, told that another device is the current one."""
    import importlib

    call, t = importlib.import_module("paper_2605_10905_amd.kv")._call, torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="q is on device 0, the current one is 1"):
        call.kv_decode(1, 0, t, *[4096] * 7, 1, 1, 1, 64, 1, 16, 1, 1.0, 0, 1.0, 1.0)


@pytest.mark.parametrize("d,fp8", [(64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("G", [3, 20, 50, 70])
def test_kv_decode_many_pairs(G, d, fp8):
    """More (sequence, key head) pairs than workgroups share: every number of query blocks, every type."""
    gen = ku.generator(67 + G)
    lens = [(53 * i) % 300 for i in range(150)]
    cache = ku.Cache(gen, lens, 1, d, 32, fp8)
    q = _q(gen, len(lens), G, d)
    o, lse = _decode(q, cache, d ** -0.5)
    ku.decode_check(o, lse, q, cache, d ** -0.5)


def test_two_captured_graphs_share_a_workspace():
    """Calls of other sizes, each in a graph of its own, over one workspace: replayed in turn on one stream, with eager work between."""
    A = _A()
    gen = ku.generator(99)
    caches = [ku.Cache(gen, lens, Hkv, 128, 32, False) for lens, Hkv in (([5000, 30], 2), ([70] * 40, 8), ([1], 1))]
    qs = [_q(gen, len(c.lens), 4 * c.k.shape[1], 128) for c in caches]
    want = [_decode(q, c, 0.09) for q, c in zip(qs, caches)]
    ws = torch.full((max(A.kv_decode_workspace_bytes(len(c.lens), q.shape[1], c.k.shape[1], 128) for q, c in zip(qs, caches)) // 4,), NAN, device="cuda")
    outs, graphs = [(torch.empty_like(o), torch.empty_like(lse)) for o, lse in want], []
    lens = [torch.tensor(c.lens, dtype=torch.int32, device="cuda") for c in caches]

    def call(i, stream=None):
        q, c, (o, lse) = qs[i], caches[i], outs[i]
        A.kv_decode(q, c.k, c.v, c.pages, lens[i], o, lse, ws, len(c.lens), q.shape[1], c.k.shape[1], 128, c.width, 32, c.num, 0.09, A.ATTN_BF16, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(3):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            call(i, torch.cuda.current_stream())
    for i in (0, 1, 0, 2, 1, 1, 0, 2):
        for t in outs[i]:
            t.fill_(7.0)
        graphs[i].replay()
        call((i + 1) % 3)
        torch.cuda.synchronize()
        for k in (i, (i + 1) % 3):
            assert torch.equal(outs[k][0], want[k][0]) and torch.equal(outs[k][1], want[k][1]), (i, k)
        ws.fill_(1e30)


# ---- together ----------------------------------------------------------------------------------


@pytest.mark.parametrize("fp8", [False, True])
def test_a_layer_that_generates(fp8):
    """Projection (gemm_bf16_nt), prompts of odd lengths into the cache, then tokens one by one through a captured step (append and
    decode): the same as causal attention (rope_qkv, attn_fwd) over the whole sequences, and the oracle on what the cache holds."""
    A = _A()
    Hq, Hkv, d, E, page, S, steps = 8, 2, 128, 256, 32, 3, 9
    prompts = [45, 3, 64]
    gen = ku.generator(101)
    width, npos, scale = (Hq + 2 * Hkv) * d, 100, d ** -0.5
    weight = (torch.randn((width, E), generator=gen, device="cuda") * E ** -0.5).bfloat16()
    total = max(prompts) + steps
    x = torch.randn((S, total, E), generator=gen, device="cuda").bfloat16()
    w, tab = ku.weights(gen, d, True), ku.table(npos, d)
    dtype = A.ATTN_FP8_E4M3 if fp8 else A.ATTN_BF16

    qkv = torch.empty((S, total, width), dtype=torch.bfloat16, device="cuda")
    A.gemm_bf16_nt(x, weight, qkv, S * total, width, E)
    q, k, v = (torch.empty((S, h, total, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    A.rope_qkv(qkv, width, *w, EPS, tab, npos, d, False, None, q, k, v, S, Hq, Hkv, total, d)
    o, lse = torch.empty_like(q), torch.empty((S, Hq, total), device="cuda")
    A.attn_fwd(q, k, v, o, lse, S, Hq, Hkv, total, d, True, scale, A.ATTN_BF16)

    cache = ku.Cache(gen, [n + steps for n in prompts], Hkv, d, page, fp8, fill=False)
    seq = torch.tensor([s for s, n in enumerate(prompts) for _ in range(n)], dtype=torch.int32, device="cuda")
    pos = torch.tensor([i for n in prompts for i in range(n)], dtype=torch.int32, device="cuda")
    tail = (cache.width, page, cache.num, dtype, *cache.descale)
    T = len(seq)
    prompt_q = torch.empty((T, Hq, d), dtype=torch.bfloat16, device="cuda")
    rows = torch.cat([qkv[s, :n] for s, n in enumerate(prompts)])
    A.kv_append(rows, width, *w, EPS, tab, npos, d, False, pos, seq, cache.pages, prompt_q, cache.k, cache.v, T, S, Hq, Hkv, d, *tail)
    assert torch.equal(prompt_q, torch.cat([q[s, :, :n].transpose(0, 1) for s, n in enumerate(prompts)]))

    new_x = torch.empty((S, E), dtype=torch.bfloat16, device="cuda")
    new = torch.empty((S, width), dtype=torch.bfloat16, device="cuda")
    at, lens = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2))
    new_q, new_o, new_lse = torch.empty((S, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((S, Hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((S, Hq), device="cuda")
    ws = torch.empty(A.kv_decode_workspace_bytes(S, Hq, Hkv, d) // 4, device="cuda")

    def step():
        A.gemm_bf16_nt(new_x, weight, new, S, width, E)
        A.kv_append(new, width, *w, EPS, tab, npos, d, False, at, None, cache.pages, new_q, cache.k, cache.v, S, S, Hq, Hkv, d, *tail)
        A.kv_decode(new_q, cache.k, cache.v, cache.pages, lens, new_o, new_lse, ws, S, Hq, Hkv, d, cache.width, page, cache.num, scale, dtype, *cache.descale)

    at.fill_(-1)  # (what is run before the capture leaves the cache alone)
    new_x.zero_()
    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(steps):
        now = [n + i for n in prompts]
        new_x.copy_(torch.stack([x[s, p] for s, p in enumerate(now)]))
        at.copy_(torch.tensor(now, dtype=torch.int32))
        lens.copy_(at + 1)
        ws.fill_(NAN)  # eager work between the replays
        new_o.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        cache.lens = [p + 1 for p in now]
        ku.decode_check(new_o, new_lse, new_q, cache, scale, f"step {i}")
        o2, lse2 = _decode(new_q, cache, scale)
        assert torch.equal(o2, new_o) and torch.equal(lse2, new_lse)
        if not fp8:
            # the products of 3 rows and of all of them may sum in another order, so that q, k and v may be one bf16 step (2^-7 of a
            # value) apart: scores by at most twice that of scale |q| |k|; o by that of v, two roundings of P and two of o
            for s, p in enumerate(now):
                kk = k[s, :, :p + 1].float().abs().repeat_interleave(Hq // Hkv, 0)
                score = scale * float((kk @ q[s, :, p, :, None].float().abs()).max())
                assert float((new_lse[s] - lse[s, :, p]).abs().max()) <= 2.0 ** -6 * score + 1e-5
                assert float((new_o[s].float() - o[s, :, p].float()).abs().max()) <= (2.0 ** -5 + 2.0 ** -5 * score) * float(v[s, :, :p + 1].float().abs().max())


def test_a_layer_that_trains():
    """Projection, rope_qkv, attn_fwd, attn_bwd, rope_qkv_bwd: the gradient of the packed rows and of the norm weights against
    differences of the float64 oracles of the whole chain."""
    from oracle import attn_ref

    A = _A()
    B, N, Hq, Hkv, d = 1, 70, 4, 2, 64
    gen = ku.generator(111)
    width, npos, scale = (Hq + 2 * Hkv) * d, 80, d ** -0.5
    qkv, w, tab = ku.rows(gen, B * N, width, width), ku.weights(gen, d, True), ku.table(npos, d)
    q, k, v = (torch.empty((B, h, N, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    A.rope_qkv(qkv, width, *w, EPS, tab, npos, d, False, None, q, k, v, B, Hq, Hkv, N, d)
    o, lse = torch.empty_like(q), torch.empty((B, Hq, N), device="cuda")
    A.attn_fwd(q, k, v, o, lse, B, Hq, Hkv, N, d, True, scale, A.ATTN_BF16)
    do = torch.randn(q.shape, generator=gen, device="cuda").bfloat16()
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    A.attn_bwd(q, k, v, o, do, lse, dq, dk, dv, torch.empty(A.attn_bwd_workspace_bytes(B, Hq, N) // 4, device="cuda"), B, Hq, Hkv, N, d, True, scale, A.ATTN_BF16)
    dqkv, dw = torch.empty_like(qkv), [torch.empty(d, device="cuda") for _ in range(2)]
    A.rope_qkv_bwd(dq, dk, dv, qkv, width, *w, EPS, tab, npos, d, False, None, dqkv, width, *dw,
                   torch.empty(A.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4, device="cuda"), B, Hq, Hkv, N, d)
    torch.cuda.synchronize()
    x, ww, g = f64(qkv).reshape(N, -1, d), [f64(t) for t in w], f64(do)[0]

    def loss(x, wq, wk):
        a = orc.rope_qkv(x, Hq, Hkv, wq, wk, EPS, _host_table(tab), list(range(N)), d, False)
        return float((attn_ref.attn_ref(*(t.transpose(1, 0, 2)[None] for t in a), True, scale)[0][0] * g).sum())

    rng, h = np.random.default_rng(8), 1e-4
    dx = f64(dqkv).reshape(N, -1, d)
    for _ in range(6):
        # roundings of q, k, v, o, P, dS, their gradients and the result to bf16, half a step (2^-8) each and independent: a dozen of them,
        # sqrt(12) * 2^-8 = 1.4e-2 of the 2-norm of dx times the direction's (of unit length per element); six sigma of a sum of signs
        u = rng.standard_normal(x.shape)
        diff = (loss(x + h * u, *ww) - loss(x - h * u, *ww)) / (2 * h)
        assert abs(diff - (dx * u).sum()) <= 6 * 1.4e-2 * np.linalg.norm(dx)
    for i in range(2):
        u = rng.standard_normal(d)
        up, down = list(ww), list(ww)
        up[i], down[i] = ww[i] + h * u, ww[i] - h * u
        diff = (loss(x, *up) - loss(x, *down)) / (2 * h)
        # dweight: a sum over tokens and heads of dq (dk), each about a dozen roundings off, times xhat
        size = np.linalg.norm(f64(dq if i == 0 else dk)) * np.abs(u).max() * 2
        assert abs(diff - f64(dw[i]) @ u) <= 6 * 1.4e-2 * size
