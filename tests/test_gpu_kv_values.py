"""The operators of include/kv.h on the GPU: what particular values become, and how exact the sums of kv_decode are."""
import numpy as np
import pytest
import torch

from oracle import kv_ref as orc
from tests import kv_util as ku
from tests.kv_util import NAN, f64

pytestmark = pytest.mark.gpu

INF = float("inf")


def _A():
    import paper_2605_10905_amd as A

    return A


# ---- features past `rot` -----------------------------------------------------------------------

UNROTATED = [(d, rot, inter) for d in (64, 128) for rot in (0, 16, d // 2, d - 16) for inter in (False, True)]


def _marked(gen, shape, rot):
    """Rows [.., d] whose features from `rot` on hold infinities, NaN, the largest numbers and both zeros in places of no order: (rows, their
    clean form: zero there)."""
    x = torch.randn(shape, generator=gen, device="cuda").bfloat16()
    values = torch.tensor([INF, -INF, NAN, torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min, -0.0, 0.0, 1.0], device="cuda").bfloat16()
    which = torch.randint(0, len(values), shape, generator=gen, device="cuda")
    put = torch.rand(shape, generator=gen, device="cuda") < 0.2
    put[..., :rot] = False
    clean = torch.where(put, torch.zeros_like(x), x)
    return torch.where(put, values[which], x), clean


def _same(got, want):
    """Bit for bit, one NaN as good as another."""
    nan = got.isnan() & want.isnan()
    return bool((nan | (got.view(torch.int16) == want.view(torch.int16))).all())


@pytest.mark.parametrize("d,rot,inter", UNROTATED)
def test_features_that_are_not_rotated_are_copied(d, rot, inter):
    """Without a norm z = x from feature `rot` on, whatever x is (infinities, NaN, -0), and the rotated features do not see them."""
    A = _A()
    B, N, Hq, Hkv = 2, 21, 5, 1
    gen = ku.generator(201 + rot)
    T, H = B * N, Hq + 2 * Hkv
    tab = ku.table(N, rot) if rot else None
    x, clean = _marked(gen, (T, H, d), rot)
    heads = ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, H))

    def run(x):
        outs = [torch.empty((B, hi - lo, N, d), dtype=torch.bfloat16, device="cuda") for lo, hi in heads]
        A.rope_qkv(x, H * d, None, None, 0.0, tab, N, rot, inter, None, *outs, B, Hq, Hkv, N, d)
        return torch.cat([o.transpose(1, 2).reshape(T, -1, d) for o in outs], 1)

    got, base = run(x.view(T, -1)), run(clean.view(T, -1))
    torch.cuda.synchronize()
    assert _same(got[..., rot:], x[..., rot:])
    assert _same(got[:, :Hq + Hkv, :rot], base[:, :Hq + Hkv, :rot]) and _same(got[:, Hq + Hkv:], x[:, Hq + Hkv:])


@pytest.mark.parametrize("d,rot,inter", UNROTATED)
def test_gradients_of_features_that_are_not_rotated_are_copied(d, rot, inter):
    A = _A()
    B, N, Hq, Hkv = 2, 21, 5, 1
    gen = ku.generator(202 + rot)
    T, H = B * N, Hq + 2 * Hkv
    tab = ku.table(N, rot) if rot else None
    x, clean = _marked(gen, (T, H, d), rot)
    heads = ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, H))

    def run(x):
        grads = [x[:, lo:hi].reshape(B, N, hi - lo, d).transpose(1, 2).contiguous() for lo, hi in heads]
        out = torch.empty((T, H * d), dtype=torch.bfloat16, device="cuda")
        A.rope_qkv_bwd(*grads, None, H * d, None, None, 0.0, tab, N, rot, inter, None, out, H * d, None, None, None, B, Hq, Hkv, N, d)
        return out.view(T, H, d)

    got, base = run(x), run(clean)
    torch.cuda.synchronize()
    assert _same(got[..., rot:], x[..., rot:]) and _same(got[:, :Hq + Hkv, :rot], base[:, :Hq + Hkv, :rot])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,rot,inter", UNROTATED)
def test_features_that_are_not_rotated_enter_the_cache_as_they_are(d, rot, inter, fp8):
    """bf16 as they are; e4m3 saturated at 448 with the value's sign, NaN as NaN."""
    A = _A()
    Hq, Hkv, page = 4, 2, 16
    lens = [20, 1, 33]
    gen = ku.generator(203 + rot)
    T, H = sum(lens), Hq + 2 * Hkv
    tab = ku.table(64, rot) if rot else None
    x, clean = _marked(gen, (T, H, d), rot)
    pos = torch.tensor([i for n in lens for i in range(n)], dtype=torch.int32, device="cuda")
    seq = torch.tensor([s for s, n in enumerate(lens) for _ in range(n)], dtype=torch.int32, device="cuda")
    cache = ku.Cache(gen, lens, Hkv, d, page, fp8, fill=False)
    at = cache.pages[seq.long(), pos.long() // page].long(), pos.long() % page

    def run(x):
        q = torch.empty((T, Hq, d), dtype=torch.bfloat16, device="cuda")
        A.kv_append(x.reshape(T, -1), H * d, None, None, 0.0, tab, 64, rot, inter, pos, seq, cache.pages, q, cache.k, cache.v, T, len(lens), Hq, Hkv, d,
                    cache.width, page, cache.num, A.ATTN_FP8_E4M3 if fp8 else A.ATTN_BF16, 0.25, 0.25)
        torch.cuda.synchronize()
        return q, cache.k[at[0], :, at[1]].clone(), cache.v[at[0], :, at[1]].clone()

    got, base = run(x), run(clean)
    assert _same(got[0][..., rot:], x[:, :Hq, rot:]) and _same(got[0][..., :rot], base[0][..., :rot])
    k, v = x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not fp8:
        assert _same(got[1][..., rot:], k[..., rot:]) and _same(got[1][..., :rot], base[1][..., :rot]) and _same(got[2], v)
        return
    assert torch.equal(got[1][..., :rot], base[1][..., :rot])
    for codes, want in ((got[1][..., rot:], k[..., rot:]), (got[2], v)):
        # (a quarter: quotients are exact, so that the code is torch's rounding of the clamped quotient)
        ref = (want.float() / 0.25).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        nan = want.isnan()
        assert bool(codes.view(torch.float8_e4m3fn).float()[nan].isnan().all()) and torch.equal(codes[~nan], ref.view(torch.uint8)[~nan])


# ---- the sums of kv_decode -----------------------------------------------------------------------


@pytest.mark.parametrize("Hq,Hkv,d,fp8", [(4, 2, 128, False), (4, 2, 64, False), (16, 1, 128, True), (5, 1, 64, True), (20, 1, 128, False), (24, 1, 64, True), (40, 1, 64, False),
                                          (70, 1, 128, True), (64, 1, 128, False)])
@pytest.mark.parametrize("copies", [1, 24])
def test_kv_decode_probabilities_keep_more_than_their_first_eight_bits(Hq, Hkv, d, fp8, copies):
    """Values of both signs, so that an output is small beside sum p |v| and what a probability loses shows.  The bound is decode_check's but for
    the probabilities: they are the sum of two bf16, the second of which (at most 2^-7 of the probability) is rounded and 2^-18 of it too large:
    (2^-15 + 2^-18) sum p |v|."""
    A = _A()
    lens = [2, 3, 17, 40, 129, 700] * copies
    gen = ku.generator(211 + Hq)
    cache = ku.Cache(gen, lens, Hkv, d, 32, fp8)
    B, scale = len(lens), d ** -0.5
    q = (torch.randn((B, Hq, d), generator=gen, device="cuda") * 0.25).bfloat16()
    o, lse = torch.empty_like(q), torch.empty((B, Hq), device="cuda")
    ws = torch.empty(A.kv_decode_workspace_bytes(B, Hq, Hkv, d) // 4, device="cuda")
    A.kv_decode(q, cache.k, cache.v, cache.pages, torch.tensor(lens, dtype=torch.int32, device="cuda"), o, lse, ws, B, Hq, Hkv, d, cache.width, 32, cache.num, scale,
                A.ATTN_FP8_E4M3 if fp8 else A.ATTN_BF16, *cache.descale)
    torch.cuda.synchronize()
    got, qd = f64(o), f64(q)
    for b in range(B):
        k, v = cache.visible(b)
        want, want_lse = orc.decode(qd[b], k, v, scale)
        kk, vv = np.repeat(k, Hq // Hkv, 0), np.repeat(v, Hq // Hkv, 0)
        p = np.exp(scale * np.einsum("hd,hnd->hn", qd[b], kk) - want_lse[:, None])
        a = scale * np.einsum("hd,hnd->hn", np.abs(qd[b]), np.abs(kk)).max(-1)
        rel = 2.0 ** -24 * (2 * (d + 8) * a + k.shape[1] / 16 + 32) + 2.0 ** -20
        pv = np.einsum("hn,hnd->hd", p, np.abs(vv))
        bound = (2.0 ** -15 + 2.0 ** -18 + rel[:, None]) * pv * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) + 1e-38
        off = np.abs(got[b] - want)
        assert (off <= bound).all(), (b, lens[b], float((off / bound).max()))


@pytest.mark.parametrize("Hq,d", [(4, 128), (4, 64), (20, 128), (40, 64)])
@pytest.mark.parametrize("value", [INF, -INF])
def test_kv_decode_infinite_values(Hq, d, value):
    """p times an infinite value is infinite for every p above zero, those that are bf16 numbers (equal scores: 1) among them, and reaches no other feature."""
    A = _A()
    lens = [1, 2, 33, 64, 300]
    gen = ku.generator(221 + Hq)
    cache = ku.Cache(gen, lens, 1, d, 16, False)
    q = (torch.randn((len(lens), Hq, d), generator=gen, device="cuda") * 0.5).bfloat16()
    q[:, 0] = 0.0  # equal scores
    lens_ = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def run():
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        ws = torch.empty(A.kv_decode_workspace_bytes(len(lens), Hq, 1, d) // 4, device="cuda")
        A.kv_decode(q, cache.k, cache.v, cache.pages, lens_, o, lse, ws, len(lens), Hq, 1, d, cache.width, 16, cache.num, 0.1, A.ATTN_BF16)
        torch.cuda.synchronize()
        return o, lse

    clean, clean_lse = run()
    for b, n in enumerate(lens):
        cache.v[cache.pages[b, n // 2 // 16].long(), 0, n // 2 % 16, 5 + b] = value
    o, lse = run()
    assert torch.equal(lse, clean_lse)
    for b in range(len(lens)):
        assert bool((o[b, :, 5 + b] == value).all())
        keep = [i for i in range(d) if i != 5 + b]
        assert torch.equal(o[b][:, keep], clean[b][:, keep])


# ---- captured calls ------------------------------------------------------------------------------


@pytest.mark.parametrize("norm", [False, True])
def test_captured_rope_and_its_backward_follow_their_inputs(norm):
    """rope_qkv and rope_qkv_bwd in one graph, replayed over other rows, positions, gradients and weights, with eager calls between."""
    A = _A()
    B, N, Hq, Hkv, d, npos = 2, 301, 6, 2, 128, 400
    gen = ku.generator(231)
    T, width, tab = B * N, (Hq + 2 * Hkv) * d, ku.table(npos, d)
    heads = (Hq, Hkv, Hkv)

    def buffers():
        dws = [torch.empty(d, device="cuda") if norm else None for _ in range(2)]
        ws = torch.full((A.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4,), NAN, device="cuda") if norm else None
        return [torch.empty((B, h, N, d), dtype=torch.bfloat16, device="cuda") for h in heads], torch.empty((T, width), dtype=torch.bfloat16, device="cuda"), dws, ws

    def inputs():
        return (ku.rows(gen, T, width, width), ku.weights(gen, d, norm), torch.randint(0, npos, (T,), generator=gen, device="cuda", dtype=torch.int32),
                [torch.randn((B, h, N, d), generator=gen, device="cuda").bfloat16() for h in heads])

    def call(inp, buf):
        (qkv, w, pos, grads), (outs, dqkv, dws, ws) = inp, buf
        A.rope_qkv(qkv, width, *w, 1e-5, tab, npos, d, False, pos, *outs, B, Hq, Hkv, N, d)
        A.rope_qkv_bwd(*grads, qkv, width, *w, 1e-5, tab, npos, d, False, pos, dqkv, width, *dws, ws, B, Hq, Hkv, N, d)

    flat = lambda x: [t for y in x for t in (y if isinstance(y, list) else [y]) if t is not None]
    held, got, eager = inputs(), buffers(), buffers()
    call(held, got)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(held, got)
    for _ in range(4):
        new = inputs()
        for dst, src in zip(flat(held), flat(new)):
            dst.copy_(src)
        for t in flat(got):
            t.fill_(7.0)
        graph.replay()
        call(new, eager)
        torch.cuda.synchronize()
        for x, y in zip(flat(got[:3]), flat(eager[:3])):
            assert torch.equal(x, y)
