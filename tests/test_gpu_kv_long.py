"""The operators of include/kv.h where a wave takes many steps: rings that are refilled, page entries fetched ahead, rows and positions fetched
ahead, grids that are walked more than once.  References in 64 bits from the definitions, by torch on the GPU (tests/test_gpu_kv.py holds the oracle's
loops to the small cases); bounds as derived in kv_util.py and test_gpu_kv.py."""
import numpy as np
import pytest
import torch

from oracle import kv_ref as orc
from tests import kv_util as ku
from tests.kv_long_cases import APPEND, ROPE
from tests.kv_util import NAN

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _A():
    import paper_2605_10905_amd as A

    return A


def _turned(y, table, pos, rot, inter, sign=1.0):
    if not rot:
        return y
    i, j = (torch.tensor(x, device="cuda") for x in zip(*orc.pairs_of(rot, inter)))
    cs = table.double()[pos.long()][:, None]
    cos, sin, z = cs[..., 0], sign * cs[..., 1], y.clone()
    z[..., i] = y[..., i] * cos - y[..., j] * sin
    z[..., j] = y[..., j] * cos + y[..., i] * sin
    return z


def _size(y):
    return y.abs().amax(-1, keepdim=True)


def _rms(x):
    return (x.square().mean(-1, keepdim=True) + EPS).sqrt()


def _normed(x, w):
    return x if w is None else x / _rms(x) * w.double()


def _forward_check(got, y, table, pos, rot, inter):
    """ku.forward_bound of rows y (before the rotation)."""
    want = _turned(y, table, pos, rot, inter)
    assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -19 * _size(y) + 1e-38).all())


def _inputs(gen, B, N, H, d, norm, rot, given):
    T, npos = B * N, max(N, 500)
    pos = torch.randint(0, npos, (T,), generator=gen, device="cuda", dtype=torch.int32) if given else None
    at = pos if given else torch.arange(N, device="cuda", dtype=torch.int32).repeat(B)
    return T, npos, pos, at, ku.table(npos, rot) if rot else None, ku.weights(gen, d, norm), ku.rows(gen, T, H * d, H * d + 8, 1.5)


@pytest.mark.parametrize("case", ROPE, ids=str)
def test_rope_qkv_of_many_rows(case):
    A = _A()
    B, N, Hq, Hkv, d, norm, rot, inter, given = case
    gen, H = ku.generator(301 + N), Hq + 2 * Hkv
    T, npos, pos, at, tab, w, qkv = _inputs(gen, B, N, H, d, norm, rot, given)
    outs = [ku.guarded((B, h, N, d), torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    A.rope_qkv(qkv, H * d + 8, *w, EPS, tab, npos, rot, inter, pos, *(o for o, _ in outs), B, Hq, Hkv, N, d)
    torch.cuda.synchronize()
    assert all(f() for _, f in outs)
    rows = [o.transpose(1, 2).reshape(T, -1, d) for o, _ in outs]
    x = qkv.reshape(T, H, d)
    assert torch.equal(rows[2], x[:, Hq + Hkv:])
    for got, lo, hi, wt in ((rows[0], 0, Hq, w[0]), (rows[1], Hq, Hq + Hkv, w[1])):
        _forward_check(got, _normed(x[:, lo:hi].double(), wt), tab, at, rot, inter)


@pytest.mark.parametrize("case", ROPE, ids=str)
def test_rope_qkv_bwd_of_many_rows(case):
    A = _A()
    B, N, Hq, Hkv, d, norm, rot, inter, given = case
    gen, H = ku.generator(302 + N), Hq + 2 * Hkv
    T, npos, pos, at, tab, w, qkv = _inputs(gen, B, N, H, d, norm, rot, given)
    grads = [torch.randn((B, h, N, d), generator=gen, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)]
    out, intact = ku.guarded((T, H * d + 16), torch.bfloat16, 5.0)
    dw = [ku.guarded((d,), torch.float32) if norm else (None, lambda: True) for _ in range(2)]
    ws = torch.full((A.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4,), NAN, device="cuda") if norm else None
    A.rope_qkv_bwd(*grads, qkv, H * d + 8, *w, EPS, tab, npos, rot, inter, pos, out[:, :H * d], H * d + 16, *(t for t, _ in dw), ws, B, Hq, Hkv, N, d)
    torch.cuda.synchronize()
    assert intact() and all(f() for _, f in dw) and bool((out[:, H * d:] == 5).all())
    got, x = out[:, :H * d].reshape(T, H, d), qkv.reshape(T, H, d)
    dz = [t.transpose(1, 2).reshape(T, -1, d) for t in grads]
    assert torch.equal(got[:, Hq + Hkv:], dz[2])
    for lo, hi, k in ((0, Hq, 0), (Hq, Hq + Hkv, 1)):
        wt, xx = w[k], x[:, lo:hi].double()
        g = _turned(dz[k].double(), tab, at, rot, inter, -1.0)
        size = 2 * _size(dz[k].double())
        if wt is not None:
            # y_j = x_j w_j / n, n^2 = sum x^2 / d + eps: dx_i = g_i w_i / n - x_i sum_j(g_j w_j x_j) / (d n^3)
            n = _rms(xx)
            # each term 48 roundings and at most 8 + 33 + 24 additions (a lane's rows, a workgroup's lanes, the workgroups)
            off = (dw[k][0].double() - (g * xx / n).sum((0, 1))).abs()
            assert bool((off <= 2.0 ** -16 * (2 * _size(dz[k].double()) * xx.abs() / n).sum((0, 1))).all())
            size = size * wt.double().abs().max() / n * (1 + (_size(xx) / n) ** 2)
            gw = g * wt.double()
            g = gw / n - xx * ((gw * xx).sum(-1, keepdim=True) / (d * n ** 3))
        assert bool(((got[:, lo:hi].double() - g).abs() <= 2.0 ** -8 * g.abs() * (1 + 2.0 ** -8) + 2.0 ** -18 * size + 1e-38).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_kv_append_of_many_tokens(case, fp8):
    A = _A()
    T, Hq, Hkv, d, norm, rot, inter, page = case
    gen, H, S = ku.generator(303 + T), Hq + 2 * Hkv, 5
    # tokens of five sequences in no order; every sixteenth is padding
    per = -(-T // S)
    place = torch.randperm(S * per, generator=gen, device="cuda")[:T]
    seq, pos = (place // per).int(), (place % per).int()
    pad = torch.arange(T, device="cuda") % 16 == 7
    pos[pad] = -1
    width = -(-per // page)
    num = S * width + 2
    pages = torch.randperm(num, generator=gen, device="cuda")[:S * width].int().view(S, width).contiguous()
    shape = (num, Hkv, page, d)
    caches = [torch.full(shape, 0x7F, dtype=torch.uint8, device="cuda") if fp8 else torch.full(shape, NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tab, w, qkv = (ku.table(per, rot) if rot else None), ku.weights(gen, d, norm), ku.rows(gen, T, H * d, H * d + 8, 3.0)
    q, intact = ku.guarded((T, Hq, d), torch.bfloat16, 3.0)
    descale = (0.013, 0.021) if fp8 else (1.0, 1.0)
    A.kv_append(qkv, H * d + 8, *w, EPS, tab, per, rot, inter, pos, seq, pages, q, *caches, T, S, Hq, Hkv, d, width, page, num,
                A.ATTN_FP8_E4M3 if fp8 else A.ATTN_BF16, *descale)
    torch.cuda.synchronize()
    assert intact() and bool((q[pad] == 3).all())
    x, keep = qkv.reshape(T, H, d)[~pad], ~pad
    at = pos[keep]
    y = [_normed(x[:, :Hq].double(), w[0]), _normed(x[:, Hq:Hq + Hkv].double(), w[1]), x[:, Hq + Hkv:].double()]
    _forward_check(q[keep], y[0], tab, at, rot, inter)
    where = pages[seq[keep].long(), at.long() // page].long(), at.long() % page
    written = torch.zeros((num, page), dtype=torch.bool, device="cuda")
    written[where] = True
    assert int(written.sum()) == int(keep.sum())
    for cache, yy, f, turn in ((caches[0], y[1], descale[0], rot), (caches[1], y[2], descale[1], 0)):
        held = (cache.view(torch.float8_e4m3fn) if fp8 else cache).float().transpose(1, 2)  # [page, row, head, feature]
        assert bool(held[~written].isnan().all())
        got = held[where]
        if not fp8:
            _forward_check(got, yy, tab, at, turn, inter)
            continue
        lim, err = (_turned(yy, tab, at, turn, inter) / f).clamp(-448, 448), 2.0 ** -18 * _size(yy) / f
        assert bool(((got.double() - lim).abs() <= (2.0 ** -4 * (lim.abs() + err)).clamp_min(2.0 ** -10) + err).all())


def test_rope_of_more_rows_than_the_largest_grid_takes_at_once():
    """2^20 workgroups of four waves of three steps are 201 million rows of 64 features: behind them waves begin again.  The same bits as calls that
    do not need it, which other tests hold to the definition."""
    A = _A()
    N, d, npos, part = 67_300_000, 64, 90, 1_900_000
    gen = ku.generator(305)
    w, tab = ku.weights(gen, d, True), ku.table(npos, d)
    qkv = torch.empty((N, 3 * d), dtype=torch.bfloat16, device="cuda")
    for i in range(0, N, part):
        qkv[i:i + part] = torch.randn((min(part, N - i), 3 * d), generator=gen, device="cuda", dtype=torch.bfloat16)
    pos = torch.randint(0, npos, (N,), generator=gen, device="cuda", dtype=torch.int32)
    outs = [torch.full((1, 1, N, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    A.rope_qkv(qkv, 3 * d, *w, EPS, tab, npos, d, False, pos, *outs, 1, 1, 1, N, d)
    for i in range(0, N, part):
        n = min(part, N - i)
        want = [torch.empty((1, 1, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        A.rope_qkv(qkv[i:i + n], 3 * d, *w, EPS, tab, npos, d, False, pos[i:i + n], *want, 1, 1, 1, n, d)
        for o, ref in zip(outs, want):
            assert torch.equal(o[0, 0, i:i + n], ref[0, 0]), i


def test_kv_append_of_more_tokens_than_the_largest_grid_takes_at_once():
    """2^20 workgroups of four waves of a token each."""
    A = _A()
    T, d, page, npos = 4_300_000, 64, 1024, 4_300_000
    gen = ku.generator(306)
    W = -(-T // page)
    qkv = torch.randn((T, 3 * d), generator=gen, device="cuda", dtype=torch.bfloat16)
    pos, seq = torch.randperm(T, generator=gen, device="cuda").int(), torch.zeros(T, dtype=torch.int32, device="cuda")
    pages = torch.randperm(W, generator=gen, device="cuda").int().view(1, W)
    tab, w = ku.table(npos, 16), ku.weights(gen, d, True)
    q, (k, v) = torch.full((T, 1, d), NAN, dtype=torch.bfloat16, device="cuda"), (torch.full((W, 1, page, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    A.kv_append(qkv, 3 * d, *w, EPS, tab, npos, 16, False, pos, seq, pages, q, k, v, T, 1, 1, 1, d, W, page, W, A.ATTN_BF16)
    want = [torch.empty((1, 1, T, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    A.rope_qkv(qkv, 3 * d, *w, EPS, tab, npos, 16, False, pos, *want, 1, 1, 1, T, d)
    torch.cuda.synchronize()
    where = pages[0, pos.long() // page].long(), pos.long() % page
    assert torch.equal(q[:, 0], want[0][0, 0]) and torch.equal(k[where[0], 0, where[1]], want[1][0, 0]) and torch.equal(v[where[0], 0, where[1]], want[2][0, 0])


# ---- kv_decode ---------------------------------------------------------------------------------

WORKERS = 1024


def _tile(d, fp8):
    return 8192 // (d * (1 if fp8 else 2))


@pytest.mark.parametrize("B", [9, 40, 150])
@pytest.mark.parametrize("G,Hkv", [(6, 2), (16, 1), (20, 2), (40, 2), (70, 1)])
@pytest.mark.parametrize("d,fp8", [(64, False), (64, True), (128, False), (128, True)])
def test_kv_decode_of_many_tiles(d, fp8, G, Hkv, B):
    """Seven tiles and more for every wave: slots of its ring are refilled two times and more, and sequences change, end inside a tile, have
    no keys and lose pages on refilled slots.  Few pairs of a sequence and a key head (rows joined by whole workgroups), some, and more than
    share workgroups."""
    A = _A()
    tile, units = _tile(d, fp8), Hkv * (2 if G > 64 else 1)
    page = 16 if d == 64 else 64
    gen, rng = ku.generator(311 + G + B), np.random.default_rng(7 + G + B + d)
    mean = 7.6 * WORKERS * tile / (B * units)
    lens = [int(n) for n in rng.uniform(1, 2 * mean, B)]
    for i, n in enumerate((0, 1, tile, tile + 1, tile * 3 - 1)):
        lens[(3 * i + 1) % B] = n
    lens[0] = int(2 * mean)
    tiles = sum(-(-n // tile) for n in lens) * units
    while tiles < 7 * WORKERS:  # (what the short ones took away goes to the last)
        lens[-1] += tile * 64
        tiles += 64 * units
    need = [-(-n // page) for n in lens]
    width, num = max(need), sum(need) + 3
    order = torch.randperm(num, generator=gen, device="cuda").int()
    pages = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    pages[torch.arange(width, device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]] = order[:sum(need)]
    descale = (0.013, 0.021) if fp8 else (1.0, 1.0)
    nan = 0x7F if fp8 else NAN
    caches = []
    for f in descale:
        x = torch.randn((num, Hkv, page, d), generator=gen, device="cuda")
        x = (x / f).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else x.bfloat16()
        x[order[sum(need):].long()] = nan
        for b, n in enumerate(lens):
            if n % page:
                x[pages[b, n // page].long(), :, n % page:] = nan
        caches.append(x)
    hidden = torch.rand((B, width), generator=gen, device="cuda") < 0.03
    hidden[::2] = False
    lost = pages.clone()
    lost[hidden] = torch.where(torch.rand((B, width), generator=gen, device="cuda") < 0.5, -1, num + 5).int()[hidden]
    Hq, scale = Hkv * G, d ** -0.5
    q = torch.randn((B, Hq, d), generator=gen, device="cuda").bfloat16()
    lens_ = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.full((A.kv_decode_workspace_bytes(B, Hq, Hkv, d) // 4,), NAN, device="cuda")

    def run():
        o, intact = ku.guarded((B, Hq, d), torch.bfloat16)
        lse, lse_intact = ku.guarded((B, Hq), torch.float32)
        A.kv_decode(q, *caches, lost, lens_, o, lse, ws, B, Hq, Hkv, d, width, page, num, scale, A.ATTN_FP8_E4M3 if fp8 else A.ATTN_BF16, *descale)
        torch.cuda.synchronize()
        assert intact() and lse_intact()
        return o, lse

    o, lse = run()
    again = run()
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    for b, n in enumerate(lens):
        if n == 0:
            assert not bool(o[b].any()) and bool(torch.isneginf(lse[b]).all())
            continue
        at, seen = pages[b, :need[b]].long(), (~hidden[b, :need[b]]).repeat_interleave(page)[:n]
        k, v = ((c[at].view(torch.float8_e4m3fn) if fp8 else c[at]).double().transpose(0, 1).reshape(Hkv, -1, d)[:, :n] * f for c, f in zip(caches, descale))
        for h in range(Hkv):
            qh, rows = q[b, h * G:(h + 1) * G].double(), slice(h * G, (h + 1) * G)
            kk, vv = k[h][seen], v[h][seen]
            if kk.shape[0] == 0:
                assert not bool(o[b, rows].any()) and bool(torch.isneginf(lse[b, rows]).all())
                continue
            s = scale * (qh @ kk.t().contiguous())
            want_lse = torch.logsumexp(s, -1)
            p = (s - want_lse[:, None]).exp()
            want, pv = p @ vv, p @ vv.abs()
            a = scale * (qh.abs() @ kk.abs().t().contiguous()).amax(-1)
            rel = 2.0 ** -24 * (2 * (d + 8) * a + n / 16 + 32) + 2.0 ** -20
            bound = (2.0 ** -15 + 2.0 ** -18 + rel[:, None]) * pv * (1 + 2.0 ** -7) + 2.0 ** -8 * want.abs() * (1 + 2.0 ** -8) + 1e-38
            off = (o[b, rows].double() - want).abs()
            assert bool((off <= bound).all()), (b, h, n, float((off / bound).max()))
            assert bool(((lse[b, rows].double() - want_lse).abs() <= rel + 2.0 ** -22 * (1 + want_lse.abs())).all()), (b, h, n)
