"""Performance cases of the operators around attention in a transformer layer: what stands between the
projection (a GEMM) and attention in training, and the paged key-value cache of serving.

  rope      rope_qkv: the rows of a packed q|k|v projection are split into heads, q and k are RMS-normalised per
            head and rotated by their position, and all three are written in attention's [B, H, N, d] layout
  rope_bwd  rope_qkv_bwd: its gradients, from those of q, k, v to those of the projection and of the norms' weights
  append    kv_append: the same for new tokens of a serving batch; k and v go into a paged cache (bf16 or e4m3)
  decode    kv_decode: attention of one new token per sequence over the paged cache

listed() holds fixed cases, draw(rng) gives one more of the same ranges, prepare / run make the inputs of a case and
take ONE pass.  `own` False: run() computes the plain form in 32 bits; True: it calls the library.
A case is a dict of plain values:

  all       op, Hq, Hkv, d, norm (per-head RMS norm of q and k), rot (rotated leading dimensions), pairs ("halves":
            i and i + rot / 2, "adjacent": 2i and 2i + 1)
  rope      B, N; start (position of the first token)
  append    S sequences, new (most new tokens of one), context (most keys of one before), page, dtype of the cache
  decode    B, longest (most keys of a sequence), ragged (lengths spread over 1 .. longest), page, dtype
"""
import math

import torch

own = False

EPS = 1e-6
THETA = 500000.0


def _rope(name, op, B, N, Hq, Hkv, d, norm, rot, pairs, start=0):
    c = dict(op=op, B=B, N=N, Hq=Hq, Hkv=Hkv, d=d, norm=norm, rot=rot, pairs=pairs, start=start)
    return dict(name=name, **c) if name else c


def _append(name, S, new, context, Hq, Hkv, d, norm, rot, pairs, page, dtype):
    c = dict(op="append", S=S, new=new, context=context, Hq=Hq, Hkv=Hkv, d=d, norm=norm, rot=rot, pairs=pairs, page=page, dtype=dtype)
    return dict(name=name, **c) if name else c


def _decode(name, B, longest, ragged, Hq, Hkv, d, page, dtype):
    c = dict(op="decode", B=B, longest=longest, ragged=ragged, Hq=Hq, Hkv=Hkv, d=d, page=page, dtype=dtype)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a prompt of odd length in a grouped-query layer, half of each head rotated, no norm: far fewer bytes than the caches hold
        _rope("rope_prefill_1000", "rope", 1, 1000, 32, 8, 128, False, 64, "adjacent", start=70000),
        # a causal training batch of a grouped-query layer: bound by memory
        _rope("rope_train_gqa_4k", "rope", 4, 4096, 64, 8, 128, True, 128, "halves"),
        # the backward of a small batch of odd length at head dimension 64
        _rope("rope_bwd_777_d64", "rope_bwd", 2, 777, 12, 4, 64, True, 64, "halves"),
        # the backward of an ordinary training batch, as many key heads as query heads
        _rope("rope_bwd_train_2k", "rope_bwd", 4, 2048, 16, 16, 128, True, 128, "halves"),
        # one new token of one sequence: the smallest call, all latency
        _append("append_one_token", 1, 1, 900, 32, 8, 128, True, 128, "halves", 16, "bf16"),
        # one new token of each sequence of a serving batch
        _append("append_step_64", 64, 1, 4000, 64, 8, 128, True, 128, "halves", 64, "bf16"),
        # prompts of several lengths enter an e4m3 cache at once
        _append("append_prompts_fp8", 7, 2500, 0, 32, 8, 128, False, 128, "halves", 32, "fp8"),
        # one short sequence: latency
        _decode("decode_one_500", 1, 500, False, 32, 8, 128, 16, "bf16"),
        # as many key heads as query heads, head dimension 64, ragged
        _decode("decode_mha_d64", 24, 1500, True, 16, 16, 64, 16, "bf16"),
        # a serving batch with sequences of very different lengths
        _decode("decode_ragged_64", 64, 6000, True, 64, 8, 128, 64, "bf16"),
        # the same with an e4m3 cache
        _decode("decode_fp8_32", 32, 9000, True, 64, 8, 128, 32, "fp8"),
        # two very long contexts: few rows, the cache's length has to fill the chip
        _decode("decode_long_128k", 2, 131072, False, 64, 8, 128, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_CAP_BYTES = 6.0e8  # drawn cases stay below the largest listed ones


def draw(rng):
    while True:
        op = rng.choice(("rope", "rope_bwd", "append", "decode", "decode"))
        hkv, group, d = rng.choice((1, 2, 3, 4, 6, 8, 12, 16)), rng.choice((1, 2, 3, 4, 5, 7, 8, 16)), rng.choice((64, 128, 128))
        norm, rot, pairs = rng.random() < 0.6, rng.choice((d, d, d // 2, d - 32)), rng.choice(("halves", "halves", "adjacent"))
        page, dtype = rng.choice((16, 32, 64, 128, 256)), rng.choice(("bf16", "bf16", "fp8"))
        if op == "append":
            if rng.random() < 0.5:
                c = _append(None, _log_int(rng, 1, 512), 1, _log_int(rng, 1, 8000), hkv * group, hkv, d, norm, rot, pairs, page, dtype)
            else:
                c = _append(None, rng.randint(1, 12), _log_int(rng, 2, 4000), rng.choice((0, 0, 1000)), hkv * group, hkv, d, norm, rot, pairs, page, dtype)
            if _held(c) > _CAP_BYTES:
                continue
        elif op == "decode":
            c = _decode(None, _log_int(rng, 1, 256), _log_int(rng, 1, 100000), rng.random() < 0.6, hkv * group, hkv, d, page, dtype)
        else:
            c = _rope(None, op, rng.randint(1, 8), _log_int(rng, 1, 8192), hkv * group, hkv, d, norm, rot, pairs, rng.choice((0, 0, 100000)))
        if work(c)["bytes"] <= _CAP_BYTES:
            return c


def _spread(n, most, least=1):
    """n whole numbers of least .. most, the first of them `most`, the others spread evenly in no order."""
    return [most if i == 0 else least + int((most - least + 1) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _lengths(case):
    """append: (new tokens, keys before) of every sequence; decode: keys of every sequence."""
    if case["op"] == "append":
        return _spread(case["S"], case["new"]), _spread(case["S"], case["context"], 0)
    return _spread(case["B"], case["longest"]) if case["ragged"] else [case["longest"]] * case["B"]


def _cache_pages(case):
    """Pages of every sequence, with its new tokens."""
    if case["op"] == "append":
        return [-(-(a + b) // case["page"]) for a, b in zip(*_lengths(case))]
    return [-(-n // case["page"]) for n in _lengths(case)]


def _held(case):
    """Bytes of the cache."""
    return 2 * sum(_cache_pages(case)) * case["page"] * case["Hkv"] * case["d"] * (1 if case["dtype"] == "fp8" else 2)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c, st = case, dict(case)
    Hq, Hkv, d, op = c["Hq"], c["Hkv"], c["d"], c["op"]

    def normal(shape, sigma=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * sigma).to(dtype)

    def empty(shape, dtype=torch.bfloat16):
        return torch.empty(shape, device="cuda", dtype=dtype)

    def ints(values):
        return torch.tensor(values, device="cuda", dtype=torch.int32)

    if op in ("append", "decode"):
        # pages in no order, some that no sequence has; the page table is as wide as the longest sequence needs
        need, width = _cache_pages(c), max(_cache_pages(c))
        num = sum(need) + 3
        order = torch.randperm(num, generator=gen, device="cuda").to(torch.int32)
        pages = torch.full((len(need), width), -1, device="cuda", dtype=torch.int32)
        filled = torch.arange(width, device="cuda")[None, :] < ints(need)[:, None]
        pages[filled] = order[: sum(need)]
        fp8 = c["dtype"] == "fp8"
        for nm in ("k_cache", "v_cache"):
            x = normal((num, Hkv, c["page"], d), 100.0 if fp8 else 1.0)
            st[nm] = x.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else x
        # de-scales as a calibration leaves them: 448 codes for a little more than the largest value
        st.update(pages=pages, num=num, width=width, kd=0.0107 if fp8 else 1.0, vd=0.0113 if fp8 else 1.0)
    if op == "decode":
        B = c["B"]
        st.update(q=normal((B, Hq, d)), lens=ints(_lengths(c)), o=empty((B, Hq, d)), lse=empty((B, Hq), torch.float32), scale=1.0 / math.sqrt(d))
        if own:
            import paper_2605_10905_amd as A

            st["ws"] = empty((A.kv_decode_workspace_bytes(B, Hq, Hkv, d) // 4,), torch.float32)
        return st

    if op == "append":
        new, before = _lengths(c)
        T, npos = sum(new), max(a + b for a, b in zip(new, before))
        seq = torch.repeat_interleave(torch.arange(c["S"], device="cuda"), ints(new).long(), output_size=T)
        first = torch.cumsum(ints(new).long(), 0) - ints(new).long()
        pos = torch.arange(T, device="cuda") - first[seq] + ints(before).long()[seq]
        st.update(T=T, seq=seq.to(torch.int32), pos=pos.to(torch.int32), q=empty((T, Hq, d)))
    else:
        T, npos = c["B"] * c["N"], c["start"] + c["N"]
        st.update(T=T, pos=(torch.arange(c["N"], device="cuda", dtype=torch.int32) + c["start"]).repeat(c["B"]))
    # the angles of far positions need 64 bits, their cosines and sines do not
    freq = THETA ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) * 2.0 / c["rot"])
    angle = torch.arange(npos, device="cuda", dtype=torch.float64)[:, None] * freq
    st.update(npos=npos, table=torch.stack((angle.cos(), angle.sin()), -1).float().contiguous(), qkv=normal((T, (Hq + 2 * Hkv) * d)))
    for nm in ("wq", "wk"):
        st[nm] = (1.0 + normal((d,), 0.1, torch.float32)).bfloat16() if c["norm"] else None
    if op != "append":
        B, N = c["B"], c["N"]
        shapes = dict(q=(B, Hq, N, d), k=(B, Hkv, N, d), v=(B, Hkv, N, d))
        if op == "rope":
            st.update({nm: empty(s) for nm, s in shapes.items()})
        else:
            st.update({"d" + nm: normal(s) for nm, s in shapes.items()})
            st.update(dqkv=empty((T, (Hq + 2 * Hkv) * d)), ws=None)
            for nm in ("dwq", "dwk"):
                st[nm] = empty((d,), torch.float32) if c["norm"] else None
            if own and c["norm"]:
                import paper_2605_10905_amd as A

                st["ws"] = empty((A.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4,), torch.float32)
    return st


# ---- the plain forms -------------------------------------------------------------------------


def _rotate(x, table, pos, rot, pairs, back=False):
    """x [T, H, d] rotated by its positions (back: the transposed rotation)."""
    cs = table[pos.long()]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    if back:
        sin = -sin
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., : rot // 2], r[..., rot // 2:]) if pairs == "halves" else (r[..., 0::2], r[..., 1::2])
    u, w = a * cos - b * sin, b * cos + a * sin
    r = torch.cat((u, w), -1) if pairs == "halves" else torch.stack((u, w), -1).flatten(-2)
    return torch.cat((r, rest), -1)


def _normalise(x, weight):
    return x if weight is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()


def _heads(s):
    """The packed rows as q, k, v [T, heads, d] in 32 bits."""
    Hq, Hkv = s["Hq"], s["Hkv"]
    x = s["qkv"].view(s["T"], Hq + 2 * Hkv, s["d"]).float()
    return x[:, :Hq], x[:, Hq: Hq + Hkv], x[:, Hq + Hkv:]


def _plain_qkv(s):
    q, k, v = _heads(s)
    q, k = (_rotate(_normalise(x, w), s["table"], s["pos"], s["rot"], s["pairs"]) for x, w in ((q, s["wq"]), (k, s["wk"])))
    return q, k, v


def _plain_rope(s):
    return tuple(x.view(s["B"], s["N"], -1, s["d"]).transpose(1, 2).to(torch.bfloat16).contiguous() for x in _plain_qkv(s))


def _plain_rope_bwd(s):
    grads = [s["d" + nm].float().transpose(1, 2).reshape(s["T"], -1, s["d"]) for nm in ("q", "k", "v")]
    q, k, _ = _heads(s)

    def back(x, weight, g):
        g = _rotate(g, s["table"], s["pos"], s["rot"], s["pairs"], back=True)
        if weight is None:
            return g, None
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        hat, gw = x * r, g * weight.float()
        return r * (gw - hat * (gw * hat).mean(-1, keepdim=True)), (g * hat).sum((0, 1))

    (dq, dwq), (dk, dwk) = back(q, s["wq"], grads[0]), back(k, s["wk"], grads[1])
    return torch.cat((dq, dk, grads[2]), 1).to(torch.bfloat16).flatten(1), dwq, dwk


def _plain_append(s):
    q, k, v = _plain_qkv(s)
    seq, pos = s["seq"].long(), s["pos"].long()
    page, row = s["pages"][seq, pos // s["page"]].long(), pos % s["page"]
    for x, cache, descale in ((k, s["k_cache"], s["kd"]), (v, s["v_cache"], s["vd"])):
        if s["dtype"] == "fp8":
            x = (x / descale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        cache[page, :, row] = x.to(cache.dtype)
    return q.to(torch.bfloat16), s["k_cache"], s["v_cache"]


def _plain_decode(s):
    B, Hq, Hkv, d = s["B"], s["Hq"], s["Hkv"], s["d"]
    seen = torch.arange(s["width"] * s["page"], device="cuda")[None, :] < s["lens"][:, None]

    def gathered(cache, descale):
        x = cache.view(torch.float8_e4m3fn) if s["dtype"] == "fp8" else cache
        x = x.float()[s["pages"].clamp_min(0).long()].transpose(1, 2).reshape(B, Hkv, -1, d)
        return x * descale if s["dtype"] == "fp8" else x

    sc = torch.matmul(s["q"].float().view(B, Hkv, Hq // Hkv, d), gathered(s["k_cache"], s["kd"]).transpose(2, 3)) * s["scale"]
    sc = sc.masked_fill(~seen[:, None, None, :], -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = (sc - m).exp()
    total = p.sum(-1, keepdim=True)
    v = gathered(s["v_cache"], s["vd"]) * seen[:, None, :, None]
    o = torch.matmul(p / total, v)
    return o.view(B, Hq, d).to(torch.bfloat16), (m + total.log()).view(B, Hq)


# ---- one pass --------------------------------------------------------------------------------


def _whole(s, q, k, v):
    """What append returns; e4m3 codes as the values they stand for."""
    return (q, k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)) if s["dtype"] == "fp8" else (q, k, v)


def run(state):
    s = state
    if not own:
        if s["op"] == "append":
            return _whole(s, *_plain_append(s))
        return {"rope": _plain_rope, "rope_bwd": _plain_rope_bwd, "decode": _plain_decode}[s["op"]](s)
    import paper_2605_10905_amd as A

    if s["op"] == "decode":
        A.kv_decode(s["q"], s["k_cache"], s["v_cache"], s["pages"], s["lens"], s["o"], s["lse"], s["ws"], s["B"], s["Hq"], s["Hkv"], s["d"],
                    s["width"], s["page"], s["num"], s["scale"], A.ATTN_FP8_E4M3 if s["dtype"] == "fp8" else A.ATTN_BF16, s["kd"], s["vd"])
        return s["o"], s["lse"]
    rope = (s["wq"], s["wk"], EPS, s["table"], s["npos"], s["rot"], s["pairs"] == "adjacent", s["pos"])
    ld = (s["Hq"] + 2 * s["Hkv"]) * s["d"]
    if s["op"] == "append":
        A.kv_append(s["qkv"], ld, *rope, s["seq"], s["pages"], s["q"], s["k_cache"], s["v_cache"], s["T"], s["S"], s["Hq"], s["Hkv"], s["d"],
                    s["width"], s["page"], s["num"], A.ATTN_FP8_E4M3 if s["dtype"] == "fp8" else A.ATTN_BF16, s["kd"], s["vd"])
        return _whole(s, s["q"], s["k_cache"], s["v_cache"])
    sizes = (s["B"], s["Hq"], s["Hkv"], s["N"], s["d"])
    if s["op"] == "rope":
        A.rope_qkv(s["qkv"], ld, *rope, s["q"], s["k"], s["v"], *sizes)
        return s["q"], s["k"], s["v"]
    A.rope_qkv_bwd(s["dq"], s["dk"], s["dv"], s["qkv"], ld, *rope, s["dqkv"], ld, s["dwq"], s["dwk"], s["ws"], *sizes)
    return s["dqkv"], s["dwq"], s["dwk"]


def work(case):
    c = case
    Hq, Hkv, d, op = c["Hq"], c["Hkv"], c["d"], c["op"]
    if op == "decode":
        keys, es = sum(_lengths(c)), 1 if c["dtype"] == "fp8" else 2
        # q, o, lse, the page table's used entries, the lengths; keys and values once
        return {"bytes": 4 * c["B"] * Hq * d + 4 * c["B"] * Hq + 4 * sum(_cache_pages(c)) + 4 * c["B"] + 2 * keys * Hkv * d * es, "flops": 4 * keys * Hq * d}
    heads = Hq + 2 * Hkv
    small = 4 * d if c["norm"] else 0
    if op == "append":
        T, es = sum(_lengths(c)[0]), 1 if c["dtype"] == "fp8" else 2
        # the rows, their positions, sequences, angles and pages; q and the cache's rows
        most = min(T, max(a + b for a, b in zip(*_lengths(c))))
        return {"bytes": T * d * (2 * heads + 2 * Hq + 2 * es * Hkv) + 12 * T + 4 * c["rot"] * most + small, "flops": T * (Hq + Hkv) * (3 * c["rot"] + (4 * d if c["norm"] else 0))}
    T = c["B"] * c["N"]
    rest = 4 * T + 4 * c["rot"] * c["N"] + small
    if op == "rope":
        return {"bytes": 4 * T * heads * d + rest, "flops": T * (Hq + Hkv) * (3 * c["rot"] + (4 * d if c["norm"] else 0))}
    # the gradients read and written; the rows of q and k where their norm has to be gone back through
    return {"bytes": 4 * T * heads * d + (2 * T * (Hq + Hkv) * d + 8 * d if c["norm"] else 0) + rest, "flops": T * (Hq + Hkv) * (3 * c["rot"] + (12 * d if c["norm"] else 0))}


# ---- the definitions in 64 bits ----------------------------------------------------------------


def _turned(s, x, sign=1.0):
    """x [T, H, d] in 64 bits: complex numbers of the pairs times exp(i * sign * position * frequency)."""
    rot = s["rot"]
    freq = torch.exp(torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) * (-math.log(THETA) / rot))
    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), sign * s["pos"].double()[:, None] * freq)[:, None, :]
    r = x[..., :rot]
    r = r.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if s["pairs"] == "halves" else r.unflatten(-1, (rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(r.contiguous()) * turn)
    y = x.clone()
    y[..., :rot] = (z.transpose(-1, -2) if s["pairs"] == "halves" else z).flatten(-2)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, d = s["Hq"], s["Hkv"], s["d"]
    if s["op"] == "decode":
        o, lse = [], []
        kc, vc = (s[nm].view(torch.float8_e4m3fn) if s["dtype"] == "fp8" else s[nm] for nm in ("k_cache", "v_cache"))
        for b, n in enumerate(_lengths(case)):
            at = s["pages"][b, : -(-n // s["page"])].long()
            k, v = ((x.view(torch.uint8)[at].view(torch.float8_e4m3fn) if s["dtype"] == "fp8" else x[at]).double().transpose(0, 1).flatten(1, 2)[:, :n] * f
                    for x, f in ((kc, s["kd"]), (vc, s["vd"])))
            sc = (s["q"][b].double().view(Hkv, -1, d) @ k.transpose(1, 2)).flatten(0, 1) * s["scale"]
            lse.append(torch.logsumexp(sc, -1))
            o.append((torch.softmax(sc, -1).view(Hkv, Hq // Hkv, n) @ v).flatten(0, 1))
        return torch.stack(o), torch.stack(lse)

    x = s["qkv"].double().view(s["T"], Hq + 2 * Hkv, d)
    parts = torch.split(x, [Hq, Hkv, Hkv], 1)

    def unit(t):
        return t / (t.square().sum(-1, keepdim=True) / d + EPS).sqrt()

    if s["op"] == "rope_bwd":
        out, grads = [], []
        for t, w, nm in ((parts[0], s["wq"], "dq"), (parts[1], s["wk"], "dk"), (parts[2], None, "dv")):
            g = s[nm].double().movedim(1, 2).reshape(s["T"], -1, d)
            if nm != "dv":
                g = _turned(s, g, -1.0)
            if w is not None:
                # y_j = x_j w_j / n with n^2 = sum x^2 / d + eps:  dx_i = g_i w_i / n - x_i (sum_j g_j w_j x_j) / (d n^3)
                n = (t.square().sum(-1, keepdim=True) / d + EPS).sqrt()
                grads.append((g * t / n).flatten(0, 1).sum(0))
                g = g * w.double() / n - t * ((g * w.double() * t).sum(-1, keepdim=True) / (d * n ** 3))
            elif nm != "dv":
                grads.append(None)
            out.append(g)
        return torch.cat(out, 1).flatten(1), grads[0], grads[1]
    q, k, v = (parts[0] if s["wq"] is None else unit(parts[0]) * s["wq"].double()), (parts[1] if s["wk"] is None else unit(parts[1]) * s["wk"].double()), parts[2]
    q, k = _turned(s, q), _turned(s, k)
    if s["op"] == "rope":
        return tuple(t.unflatten(0, (s["B"], s["N"])).movedim(2, 1).contiguous() for t in (q, k, v))
    out = []
    for t, nm, f in ((k, "k_cache", s["kd"]), (v, "v_cache", s["vd"])):
        cache = (s[nm].view(torch.float8_e4m3fn) if s["dtype"] == "fp8" else s[nm]).double()
        seq, pos = s["seq"].long(), s["pos"].long()
        cache[s["pages"][seq, pos // s["page"]].long(), :, pos % s["page"]] = (t / f).clamp(-448.0, 448.0) if s["dtype"] == "fp8" else t
        out.append(cache)
    return q, out[0], out[1]
