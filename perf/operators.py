"""The operators that stand around the attention forward in a model, as measurable cases: the norms of
queries and keys with the position rotation (`rope.qk_norm_rope`, forward and backward), appending to a
paged cache of 4 bits and reading it back (`kv4.kv4_append`, `kv4.kv4_read`), and attention over that cache
(`kv4.kv4_attn`).  `own` chooses between the framework's kernels and the same operators in elementary torch
operations.

The cache is one tensor [pages, heads, page_size, d + d/16] of bytes.  The bytes of 16 consecutive tokens of
one head lie together: 8d bytes of key codes [token][channel / 2], 8d bytes of value codes
[token / 4][16 runs of d/16 channels][token % 4][channel of the run / 2] (a byte holds an even channel in its
low half and the next one in its high half), d/2 key scales [token][channel / 32] and d/2 value scales
[token / 4][channel / 32][token % 4].  A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; a scale byte b
stands for 2^(b - 127), 255 for NaN.
"""
import math
import random

import torch

own = False

_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-6


def _rope(name, B, N, H, Hkv, d, dtype, norm=True, interleaved=False, backward=False, head_major=True):
    return {"name": name, "op": "rope_bwd" if backward else "rope", "B": B, "N": N, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype,
            "norm": norm, "interleaved": interleaved, "head_major": head_major}


def _append(name, seqs, T, Hkv, d, dtype, page, interleaved=False, pad=0):
    return {"name": name, "op": "append", "seqs": seqs, "T": T, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page,
            "interleaved": interleaved, "pad": pad}


def _attn(name, B, L, nq, H, Hkv, d, dtype, page, causal=True, ragged=True):
    return {"name": name, "op": "attn", "B": B, "L": L, "nq": nq, "H": H, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page,
            "causal": causal, "ragged": ragged}


def listed():
    return [
        # one step of 8 requests: the projections' rows of one token each
        _rope("rope_step_bf16", 8, 1, 32, 8, 128, "bf16", head_major=False),
        # pre-training layer: two sequences, 32 query heads on 8 key heads
        _rope("rope_train_bf16", 2, 4096, 32, 8, 128, "bf16"),
        # its backward pass
        _rope("rope_bwd_train_bf16", 2, 4096, 32, 8, 128, "bf16", backward=True),
        # a small model's backward pass, a length that is no multiple of anything, rotation in neighbouring pairs
        _rope("rope_bwd_ragged_f16", 3, 1001, 12, 12, 64, "f16", interleaved=True, backward=True),
        # one step of 64 requests: one token each into pages of its own request
        _append("append_step_bf16", 64, 64, 8, 128, "bf16", 16),
        # prompts of four requests, padded to a common number of rows
        _append("append_prompts_f16", 4, 16384, 8, 64, "f16", 64, pad=900),
        # one request of a small batch answering its next token
        _attn("attn_step_short_bf16", 1, 1003, 1, 32, 8, 128, "bf16", 16, ragged=False),
        # a step of 64 requests of unequal lengths
        _attn("attn_step_batch_bf16", 64, 8192, 1, 32, 8, 128, "bf16", 16),
        # two very long documents
        _attn("attn_step_long_f16", 2, 131072, 1, 32, 4, 128, "f16", 256),
        # up to 5 guessed tokens checked at once, heads not shared
        _attn("attn_guesses_f16", 16, 4096, 5, 16, 16, 64, "f16", 32),
        # fresh prompts of several lengths, three query heads to a key head
        _attn("attn_prompts_f16", 6, 1500, 1500, 12, 4, 64, "f16", 64),
        # a chunk of a long prompt behind what the cache holds already
        _attn("attn_chunk_bf16", 1, 16384, 2048, 32, 8, 128, "bf16", 64, ragged=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: 1 to 16384 tokens through the norms and the append, 1 to 131072 keys and
    1 to 2048 queries of a sequence in the attention."""
    op = rng.choice(("rope", "rope_bwd", "append", "attn", "attn", "attn"))
    d, dtype, inter = rng.choice((64, 128)), rng.choice(("f16", "bf16")), rng.random() < 0.3
    Hkv = rng.choice((1, 2, 3, 4, 8, 12))
    H = Hkv * rng.choice([n for n in (1, 2, 3, 4, 5, 8) if Hkv * n <= 40])
    if op in ("rope", "rope_bwd"):
        while True:
            B, N = rng.choice((1, 2, 3, 8)), _log_uniform(rng, 1, 8192)
            c = _rope("", B, N, H, Hkv, d, dtype, rng.random() < 0.8, inter, op == "rope_bwd", rng.random() < 0.7)
            if B * N * (H + Hkv) * d <= 2 * 4096 * 40 * 128:
                break
    elif op == "append":
        T = _log_uniform(rng, 1, 16384)
        c = _append("", rng.randint(1, min(T, 8)), T, rng.choice((1, 2, 4, 8)), d, dtype, rng.choice((16, 32, 64, 128)), inter,
                    rng.choice((0, T // 10)))
    else:
        while True:
            B, L = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 131072)
            nq = rng.choice((1, 1, 2, 4, _log_uniform(rng, 1, 2048)))
            c = _attn("", B, L, nq, H, Hkv, d, dtype, rng.choice((16, 32, 64, 128)), rng.random() < 0.8, rng.random() < 0.7)
            w = work(c)
            if nq <= L and w["bytes"] <= 2.2e8 and w["flops"] <= 4e11 and B * nq * H * L <= 1.1e9:
                break
    del c["name"]
    return c


def _lengths(case):
    """Keys and queries of each sequence: a function of the case's sizes."""
    r = random.Random(case["B"] * 7919 + case["L"] * 31 + case["nq"])
    B, L, nq = case["B"], case["L"], case["nq"]
    if not case["ragged"]:
        return [L] * B, [nq] * B
    lens = [L] + [max(1, int(L * r.uniform(0.05, 1.0))) for _ in range(B - 1)]
    if nq == L:  # prompts: the cache holds nothing else
        return lens, list(lens)
    return lens, [min(n, nq if i == 0 else r.randint(1, nq)) for i, n in enumerate(lens)]


def _normal(g, shape, dtype, sigma=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(sigma).to(dtype)


def _tables(d, rows):
    """Cosines and sines of the angles, formed in 64 bits: a far position's angle has few exact bits in 32."""
    inv = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    a = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * inv
    return a.cos().float(), a.sin().float()


def _int(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = random.Random(seed)
    dt, d, Hkv = _DTYPES[case["dtype"]], case["d"], case["Hkv"]
    s = {k: case[k] for k in ("op", "d", "Hkv")}
    if case["op"] in ("rope", "rope_bwd"):
        B, N, H = case["B"], case["N"], case["H"]
        far = 0 if N > 1 else 8000  # single tokens stand anywhere in their sequences
        s["cos"], s["sin"] = _tables(d, N + far)
        s["positions"] = (torch.randint(0, far + 1, (B, 1), generator=g, device="cuda", dtype=torch.int32)
                          + torch.arange(N, device="cuda", dtype=torch.int32)).contiguous()
        qkv = _normal(g, (B, N, H + 2 * Hkv, d), dt)  # one projection's rows: queries, keys, values
        s["q"], s["k"] = qkv[:, :, :H], qkv[:, :, H:H + Hkv]
        s["qw"] = s["kw"] = None
        if case["norm"]:
            s["qw"], s["kw"] = (torch.rand(d, generator=g, device="cuda").add_(0.5).to(dt) for _ in range(2))

        def buffer(heads):
            if case["head_major"]:  # the attention forward's own layout
                return torch.empty((B, heads, N, d), device="cuda", dtype=dt).transpose(1, 2)
            return torch.empty((B, N, heads, d), device="cuda", dtype=dt)
        s["interleaved"] = case["interleaved"]
        if case["op"] == "rope":
            s["q_out"], s["k_out"] = buffer(H), buffer(Hkv)
        else:
            s["dq_out"], s["dk_out"] = buffer(H).copy_(_normal(g, (B, N, H, d), dt)), buffer(Hkv).copy_(_normal(g, (B, N, Hkv, d), dt))
            dqkv = torch.empty_like(qkv)
            s["dq"], s["dk"] = dqkv[:, :, :H], dqkv[:, :, H:H + Hkv]
            s["dqw"], s["dkw"] = ((torch.empty(d, device="cuda") for _ in range(2)) if case["norm"] else (None, None))
        return s
    page = case["page"]
    if case["op"] == "append":
        T, seqs = case["T"], case["seqs"]
        each = -(-T // seqs)  # tokens of a sequence, the last one's fewer
        first = [r.randrange(0, 5 * page) for _ in range(seqs)]  # tokens that each sequence holds already
        width = max(first) // page + -(-(max(first) % page + each) // page)
        pages = seqs * width + 1
        perm = list(range(pages - 1))
        r.shuffle(perm)
        t = torch.arange(T, device="cuda")
        b, at = t // each, _int(first)[t // each] + t % each
        slots = _int(perm).view(seqs, width)[b, at // page] * page + (at % page).int()
        if case["pad"]:  # rows behind the last token belong to nobody
            slots[T - case["pad"]:] = -1
        s["slots"], s["positions"] = slots.int().contiguous(), at.int().contiguous()
        s["cos"], s["sin"] = _tables(d, max(first) + each)
        kv = _normal(g, (T, 2 * Hkv, d), dt)
        kv[:, :Hkv, 5] *= 8  # a channel of large keys
        s["k"], s["v"] = kv[:, :Hkv], kv[:, Hkv:]
        s["cache"] = torch.zeros((pages, Hkv, page, d + d // 16), device="cuda", dtype=torch.uint8)
        s["k_out"], s["v_out"] = (torch.empty((T, Hkv, d), device="cuda", dtype=dt) for _ in range(2))
        s["interleaved"] = case["interleaved"]
        return s
    H = case["H"]
    lens, nqs = _lengths(case)
    order = list(range(case["B"]))
    r.shuffle(order)
    lens, nqs = [lens[i] for i in order], [nqs[i] for i in order]
    width = -(-max(lens) // page)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 1
    perm = list(range(pages - 1))
    r.shuffle(perm)
    rows, at = [], 0
    for n in need:
        rows.append(perm[at:at + n] + [-1] * (width - n))
        at += n
    s["tables"], s["lens"] = _int(rows), _int(lens)
    cu = [0]
    for n in nqs:
        cu.append(cu[-1] + n)
    s["cu_q"], s["max_q"], s["causal"], s["scale"] = _int(cu), max(nqs), case["causal"], d ** -0.5
    s["q"] = _normal(g, (cu[-1], H, d), dt, 1.5)
    s["cache"] = torch.empty((pages, Hkv, page, d + d // 16), device="cuda", dtype=torch.uint8)
    step = max(1, (1 << 26) // (Hkv * page * d))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        k, v = (_normal(g, (n * page, Hkv, d), torch.float32) for _ in range(2))
        k[:, :, 5] *= 8
        at = torch.arange(p * page, (p + n) * page, device="cuda")
        _put(s["cache"], at, _quantise(k), _quantise(v))
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((cu[-1], H), device="cuda")
    return s


# The plain forms.

def _pairs(x, interleaved):
    h = x.shape[-1] // 2
    return (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :h], x[..., h:])


def _join(a, b, interleaved):
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def _rotate(x, c, s, interleaved):
    a, b = _pairs(x, interleaved)
    return _join(a * c - b * s, b * c + a * s, interleaved)


def _norm_rope(x, w, c, s, interleaved):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + _EPS) * w.float()
    return _rotate(y, c, s, interleaved).to(x.dtype)


def _norm_rope_bwd(dy, x, w, c, s, interleaved):
    g = _rotate(dy.float(), c, -s, interleaved)
    if w is None:
        return g.to(x.dtype), None
    x32 = x.float()
    r = torch.rsqrt(x32.square().mean(-1, keepdim=True) + _EPS)
    n = x32 * r
    h = g * w.float()
    return (r * (h - n * (h * n).mean(-1, keepdim=True))).to(x.dtype), (g * n).sum((0, 1, 2))


def _quantise(x):
    """(codes, scale bytes) of [tokens, heads, d] in 32 bits.  The largest value of a block lies at most half a step over 6."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    byte = (((top.view(torch.int32) + 0x1fffff) >> 23) - 2).clamp(104, 140)
    y = x * ((254 - byte) << 23).view(torch.float32)
    m = y.abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    code = torch.where(torch.signbit(y), code | 8, code)
    finite = top < math.inf
    return torch.where(finite, code, 0).flatten(-2), torch.where(finite, byte, 255)[..., 0].to(torch.uint8)


def _regions(cache):
    """Views of the cache: key codes, value codes, key scales, value scales, all [pages, heads, groups of 16, ...]."""
    pages, heads, page, row = cache.shape
    d = row * 16 // 17
    c = cache.view(pages, heads, page // 16, 16 * row)
    return (c[..., :8 * d].unflatten(-1, (16, d // 2)), c[..., 8 * d:16 * d].unflatten(-1, (4, 16, 4, d // 32)),
            c[..., 16 * d:16 * d + d // 2].unflatten(-1, (16, d // 32)), c[..., 16 * d + d // 2:].unflatten(-1, (4, d // 32, 4)))


def _put(cache, slots, k, v):
    (kc, ks), (vc, vs) = k, v
    d, page = kc.shape[-1], cache.shape[2]
    p, a = slots // page, slots % page
    g, t, quad, one = a // 16, a % 16, a % 16 // 4, a % 4
    K, V, KS, VS = _regions(cache)
    K[p, :, g, t] = kc[..., 0::2] | (kc[..., 1::2] << 4)
    V[p, :, g, quad, :, one] = (vc[..., 0::2] | (vc[..., 1::2] << 4)).unflatten(-1, (16, d // 32))
    KS[p, :, g, t] = ks
    VS[p, :, g, quad, :, one] = vs


def _numbers(codes, scales, dtype):
    """What bytes of two codes and their scale bytes [..., d/2], [..., d/32] stand for."""
    one = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    one = torch.cat((one, -one))
    two = torch.stack((one.repeat(16), one.repeat_interleave(16)), -1)
    scale = torch.where(scales == 255, math.nan, (scales.int() << 23).view(torch.float32))
    return (two[codes.int()].flatten(-2).unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2).to(dtype)


def _get(cache, slots, dtype):
    page = cache.shape[2]
    p, a = slots // page, slots % page
    g, t, quad, one = a // 16, a % 16, a % 16 // 4, a % 4
    K, V, KS, VS = _regions(cache)
    return (_numbers(K[p, :, g, t], KS[p, :, g, t], dtype),
            _numbers(V[p, :, g, quad, :, one].flatten(-2), VS[p, :, g, quad, :, one], dtype))


def _plain_append(s):
    c, n = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    there = s["slots"] >= 0
    # rows without a place go to the cache's last page, which no sequence has
    slots = torch.where(there, s["slots"], s["cache"].shape[0] * s["cache"].shape[2] - 1).long()
    _put(s["cache"], slots, _quantise(_rotate(s["k"].float(), c, n, s["interleaved"])), _quantise(s["v"].float()))
    k, v = _get(s["cache"], slots, s["k"].dtype)
    there = there[:, None, None]
    return torch.where(there, k, 0), torch.where(there, v, 0)


def _plain_attn(s):
    q, cache, tables, lens, cu = s["q"], s["cache"], s["tables"], s["lens"], s["cu_q"]
    T, H, d = q.shape
    heads = cache.shape[1]
    B, n, group, L = lens.shape[0], s["max_q"], H // heads, tables.shape[1] * cache.shape[2]
    K, V, KS, VS = (x[tables.clamp(min=0).long()] for x in _regions(cache))  # [B, pages of a sequence, heads, groups, ...]
    V, VS = V.transpose(5, 6).flatten(6), VS.transpose(5, 6)
    k = _numbers(K, KS, torch.float32).permute(0, 2, 1, 3, 4, 5).reshape(B, heads, L, d)
    v = _numbers(V, VS, torch.float32).permute(0, 2, 1, 3, 4, 5, 6).reshape(B, heads, L, d)
    i, nq = torch.arange(n, device=q.device), cu[1:] - cu[:-1]
    rows = (cu[:-1, None] + i).clamp(max=T - 1).long()
    x = q[rows].float().unflatten(2, (heads, group)).permute(0, 2, 3, 1, 4).reshape(B, heads, group * n, d)
    x = (x @ k.transpose(2, 3) * s["scale"]).unflatten(2, (group, n))
    j = torch.arange(L, device=q.device)
    seen = j < lens[:, None, None]
    if s["causal"]:
        seen = seen & (j <= (lens - nq)[:, None, None] + i[:, None])
    seen = seen[:, None, None]
    x = x.masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0, m)
    p = x.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).unflatten(2, (group, n)) / torch.where(l == 0, 1, l)
    lse = (m + l.log())[..., 0]
    b = torch.searchsorted(cu, torch.arange(T, device=q.device, dtype=torch.int32), right=True) - 1
    at = torch.arange(T, device=q.device) - cu[b]
    return (o.permute(0, 3, 1, 2, 4).flatten(2, 3)[b, at].to(q.dtype), lse.permute(0, 3, 1, 2).flatten(2, 3)[b, at])


def run(s):
    if own:
        from paper_2403_16863_amd import kv4, rope
        if s["op"] == "rope":
            rope.qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["cos"], s["sin"], s["positions"], s["qw"], s["kw"], _EPS,
                              s["interleaved"])
            return s["q_out"], s["k_out"]
        if s["op"] == "rope_bwd":
            rope.qk_norm_rope_bwd(s["dq_out"], s["dk_out"], s["q"], s["k"], s["dq"], s["dk"], s["cos"], s["sin"], s["positions"],
                                  s["qw"], s["kw"], s["dqw"], s["dkw"], _EPS, s["interleaved"])
            return s["dq"], s["dk"], s["dqw"], s["dkw"]
        if s["op"] == "append":
            kv4.kv4_append(s["k"], s["v"], s["cache"], s["slots"], s["cos"], s["sin"], s["positions"], s["interleaved"])
            kv4.kv4_read(s["cache"], s["slots"], s["k_out"], s["v_out"])
            return s["k_out"], s["v_out"]
        kv4.kv4_attn(s["q"], s["cache"], s["tables"], s["lens"], s["out"], s["lse"], s["causal"], s["scale"], s["cu_q"], s["max_q"])
        return s["out"], s["lse"]
    if s["op"] in ("rope", "rope_bwd"):
        at = s["positions"].long()
        c, n, i = s["cos"][at][:, :, None], s["sin"][at][:, :, None], s["interleaved"]
        if s["op"] == "rope":
            return _norm_rope(s["q"], s["qw"], c, n, i), _norm_rope(s["k"], s["kw"], c, n, i)
        (dq, dqw), (dk, dkw) = _norm_rope_bwd(s["dq_out"], s["q"], s["qw"], c, n, i), _norm_rope_bwd(s["dk_out"], s["k"], s["kw"], c, n, i)
        return dq, dk, dqw, dkw
    return _plain_append(s) if s["op"] == "append" else _plain_attn(s)


def work(case):
    d, Hkv = case["d"], case["Hkv"]
    if case["op"] in ("rope", "rope_bwd"):
        B, N, H = case["B"], case["N"], case["H"]
        values, back = B * N * (H + Hkv) * d, case["op"] == "rope_bwd"
        tables = (N if N > 1 else B) * d * 4 + 4 * B * N
        moved = (3 if back and case["norm"] else 2) * 2 * values
        return {"bytes": moved + tables, "flops": (20 if back else 8) * values}
    if case["op"] == "append":
        T = case["T"]
        return {"bytes": T * (4 * Hkv * d * 2 + 2 * Hkv * (d + d // 16) + 4 * d + 8), "flops": 20 * T * Hkv * d}
    lens, nqs = _lengths(case)
    seen = sum(q * n - (q * (q - 1) // 2 if case["causal"] else 0) for n, q in zip(lens, nqs))  # (query, visible key)
    H = case["H"]
    return {"bytes": sum(lens) * Hkv * (d + d // 16) + sum(nqs) * H * (4 * d + 4), "flops": 4 * d * H * seen}


# The definitions once more, in 64 bits and from other steps than above.

def _exact_rope(x, w, c, s, interleaved):
    """With x as complex numbers (first, second of a pair), turned by c + i s."""
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + _EPS).sqrt() * w
    d = x.shape[-1]
    first = torch.arange(0, d, 2, device=x.device) if interleaved else torch.arange(d // 2, device=x.device)
    second = first + 1 if interleaved else first + d // 2
    z = torch.complex(x[..., first], x[..., second]) * torch.complex(c, s)
    y = torch.empty_like(x)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_4bit(x):
    """The values that a block of 32 is held as: whole multiples of the step of each value's binade."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))
    e = (e - 3 + (m > 0.875)).clamp(-23, 13)
    e = torch.where(m == 0, -23, e)
    y = torch.ldexp(b, -e)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return torch.ldexp((torch.round(y / step) * step).clamp(-6, 6), e).reshape(x.shape)


def _exact_cache(cache, d):
    """The values of all pages in 64 bits, [pages, heads, page_size, d] twice, byte by byte from the layout's words."""
    pages, heads, page, _ = cache.shape
    raw = cache.reshape(pages, heads, page // 16, -1)
    dev = cache.device
    t, c = torch.arange(16, device=dev)[:, None], torch.arange(d, device=dev)[None]
    run_, within = c // (d // 16), c % (d // 16)
    at = {"k": t * (d // 2) + c // 2, "v": 8 * d + t // 4 * (2 * d) + run_ * (d // 8) + t % 4 * (d // 32) + within // 2}
    at_scale = {"k": 16 * d + t * (d // 32) + c // 32, "v": 16 * d + d // 2 + t // 4 * (d // 8) + c // 32 * 4 + t % 4}
    found = []
    for x in ("k", "v"):
        code = (raw[..., at[x].flatten()].reshape(pages, heads, page // 16, 16, d) >> (c % 2 * 4).to(torch.uint8)) & 15
        e, m = (code >> 1 & 3).double(), (code & 1).double()
        value = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e - 1)) * (1 - 2 * (code >> 3).double())
        scale = raw[..., at_scale[x].flatten()].reshape(value.shape).double()
        found.append((value * torch.exp2(scale - 127)).reshape(pages, heads, page, d))
    return found


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rope", "rope_bwd"):
        at = s["positions"].long()
        c, n, i = s["cos"].double()[at][:, :, None], s["sin"].double()[at][:, :, None], case["interleaved"]
        found, weights = [], []
        for x, w, dy in ((s["q"], s["qw"], s.get("dq_out")), (s["k"], s["kw"], s.get("dk_out"))):
            x, w = x.double().requires_grad_(), None if w is None else w.double().requires_grad_()
            y = _exact_rope(x, w, c, n, i)
            if dy is None:
                found.append(y.detach())
                continue
            y.backward(dy.double())
            found.append(x.grad)
            weights.append(None if w is None else w.grad)
        return (*found, *weights)
    if case["op"] == "append":
        c, n = s["cos"].double(), s["sin"].double()
        at = s["positions"].long()
        there = (s["slots"] >= 0)[:, None, None]
        k = _exact_rope(s["k"].double(), None, c[at][:, None], n[at][:, None], case["interleaved"])
        return torch.where(there, _exact_4bit(k), 0), torch.where(there, _exact_4bit(s["v"].double()), 0)
    T, H, d = s["q"].shape
    group, page = H // case["Hkv"], case["page"]
    out, lse = torch.empty((T, H, d), device="cuda", dtype=torch.float64), torch.empty((T, H), device="cuda", dtype=torch.float64)
    cu, lens = s["cu_q"].tolist(), s["lens"].tolist()
    for b, n in enumerate(lens):
        mine = s["cache"][s["tables"][b, :-(-n // page)].long()]
        nq = cu[b + 1] - cu[b]
        for h in range(case["Hkv"]):
            k, v = (x.reshape(-1, d)[:n] for x in _exact_cache(mine[:, h:h + 1], d))
            for a in range(h * group, h * group + group):
                x = s["q"][cu[b]:cu[b + 1], a].double() @ k.T * s["scale"]
                if case["causal"]:
                    x = x + torch.full_like(x, -math.inf).triu(n - nq + 1)
                lse[cu[b]:cu[b + 1], a] = torch.logsumexp(x, 1)
                out[cu[b]:cu[b + 1], a] = torch.softmax(x, 1) @ v
    return out, lse
