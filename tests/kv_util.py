"""Helpers of the tests of include/kv.h: seeded inputs on the GPU, the oracle's answers, derived bounds."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv_ref as orc

NAN = float("nan")


def f64(t):
    if t.dtype == torch.uint8:
        t = t.view(torch.float8_e4m3fn)
    return t.float().cpu().numpy().astype(np.float64)


def table(npos, rot, base=500000.0):
    ang = torch.arange(npos, dtype=torch.float64)[:, None] * base ** (-2.0 * torch.arange(max(rot, 2) // 2, dtype=torch.float64) / max(rot, 2))
    return torch.stack((ang.cos(), ang.sin()), -1).float().contiguous().cuda()


def guarded(shape, dtype, fill=NAN, guard=128):
    """A tensor inside a longer buffer: (view, whether what lies around it is untouched)."""
    n = int(np.prod(shape))
    buf = torch.full((n + 2 * guard,), 7.0 if dtype.is_floating_point else 7, device="cuda").to(dtype)
    view = buf[guard:guard + n].view(shape)
    view.fill_(fill)
    return view, lambda: bool((buf[:guard].float() == 7).all()) and bool((buf[guard + n:].float() == 7).all())


def rows(gen, T, width, ld, sigma=1.0):
    """T rows of `width` bf16 features, ld apart; what lies between them is NaN."""
    buf = torch.full((T, ld), NAN, device="cuda", dtype=torch.bfloat16)
    buf[:, :width] = (torch.randn((T, width), generator=gen, device="cuda") * sigma).bfloat16()
    return buf[:, :width] if ld > width else buf


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def weights(gen, d, norm):
    return [(1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).bfloat16() if norm else None for _ in range(2)]


def arr(w):
    return None if w is None else f64(w)


def forward_bound(ref, size):
    """Of a rotated row: one rounding to bf16, half a step (2^-8 of the value); before it at most 16 roundings to 32 bits (mean
    square over d by a tree, root, quotient, two products, the rotation's three) of 2^-24 of the pair, which is at most 2 x
    the row's largest feature `size`: 32 * 2^-24 = 2^-19."""
    return 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + 2.0 ** -19 * size + 1e-38


def row_size(y):
    return np.abs(y).max(-1, keepdims=True)


class Cache:
    """Pages in no order, some that nobody has, every row NaN until it is written."""

    def __init__(self, gen, lens, Hkv, d, page, fp8, width=None, spare=2, fill=True):
        need = [-(-max(n, 0) // page) for n in lens]
        self.width = width or max(1, max(need))
        self.num, self.page, self.fp8, self.lens = sum(need) + spare, page, fp8, lens
        order = torch.randperm(self.num, generator=gen, device="cuda").cpu().tolist()
        table = [[-1] * self.width for _ in lens]
        for s, n in enumerate(need):
            for i in range(n):
                table[s][i] = order.pop()
        self.pages = torch.tensor(table, dtype=torch.int32, device="cuda")
        shape = (self.num, Hkv, page, d)
        self.k, self.v = (torch.full(shape, 0x7F, dtype=torch.uint8, device="cuda") if fp8 else torch.full(shape, NAN, dtype=torch.bfloat16, device="cuda")
                          for _ in range(2))
        self.descale = (0.013, 0.021) if fp8 else (1.0, 1.0)
        if fill:
            for cache, f in ((self.k, self.descale[0]), (self.v, self.descale[1])):
                x = torch.randn(shape, generator=gen, device="cuda")
                x = (x / f).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else x.bfloat16()
                for s, n in enumerate(lens):
                    for i in range(need[s]):
                        rows_ = min(page, n - i * page)
                        cache[table[s][i], :, :rows_] = x[table[s][i], :, :rows_]

    def visible(self, s):
        """Keys and values of sequence s in 64 bits, de-scaled."""
        pages = self.pages[s].cpu().tolist()
        out = []
        for cache, f in ((self.k, self.descale[0]), (self.v, self.descale[1])):
            n = min(max(self.lens[s], 0), self.width * self.page)
            used = pages[: -(-n // self.page)]
            ids = [p for p in used if 0 <= p < self.num]
            sub = f64(cache[torch.tensor(ids, device="cuda")]) if ids else np.zeros((0, *cache.shape[1:]))
            where = {p: i for i, p in enumerate(ids)}
            out.append(orc.gather(sub, [where.get(p, -1) for p in used], n, self.page) * f)
        return out


def decode_check(o, lse, q, cache, scale, label=""):
    """Every row against the oracle.  With p the probabilities, per element: the probabilities rounded to bf16 (half a step of each:
    2^-8 sum p |v|), the output rounded to bf16 (2^-8 |o|); scores: d + 8 roundings to 32 bits of sums of at most
    a = scale sum |q| |k| twice (the score and the reference maximum), the exponential and its argument (2^-20 holds both for
    arguments down to -16; below that p < 2^-16 of the largest), and sums over n keys by lanes and tiles (n / 16 + 32 roundings)."""
    got, got_lse = f64(o), lse.cpu().numpy().astype(np.float64)
    qd = f64(q)
    for b in range(q.shape[0]):
        k, v = cache.visible(b)
        want, want_lse = orc.decode(qd[b], k, v, scale)
        n, d, G = k.shape[1], q.shape[-1], q.shape[1] // k.shape[0]
        if n == 0:
            assert not got[b].any() and np.isneginf(got_lse[b]).all(), (label, b)
            continue
        kk, vv = np.repeat(k, G, 0), np.repeat(v, G, 0)
        s = scale * np.einsum("hd,hnd->hn", qd[b], kk)
        p = np.exp(s - want_lse[:, None])
        a = scale * np.einsum("hd,hnd->hn", np.abs(qd[b]), np.abs(kk)).max(-1)
        rel = 2.0 ** -24 * (2 * (d + 8) * a + n / 16 + 32) + 2.0 ** -20
        pv = np.einsum("hn,hnd->hd", p, np.abs(vv))
        bound = (2.0 ** -8 + rel[:, None]) * pv * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) + 1e-38
        off = np.abs(got[b] - want)
        assert np.isfinite(got[b]).all() and (off <= bound).all(), (label, b, n, float((off / bound).max()))
        assert (np.abs(got_lse[b] - want_lse) <= rel + 2.0 ** -22 * (1 + np.abs(want_lse))).all(), (label, b, n, got_lse[b], want_lse)
