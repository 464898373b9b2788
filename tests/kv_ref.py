"""Plain 64-bit forms of the paged key-value cache and of one token's attention over it, and the
tolerances of their tests.

The pages are taken apart byte by byte; codes and scales are exact, so that what a cache holds
is compared bit by bit. Tolerances of the attention (u = 2^-24), per channel d of an output
y_d = sum_t p_t v_td with p the softmax:
 * an error e_t of a score moves y by sum_t p_t e_t (v_td - y_d). A score is a sum of D terms in
   tensor-core steps of 16 that may truncate (2 u each; D / 16 <= 16 of them, twice or three times
   for a query in terms, and a few roundings beside them): 64 u of the sum of absolute terms,
   which for codes are those of the code with its offset. queries of 16 bits meet codes as subnormal numbers
   u 2^-24, whose products are lined up as if u were 1024: each step may cut off 2^-23 of 1024 times
   the head's largest |q|, in units of the code, 2^-13 |q| s. The exponent's difference from the
   reference and its exponential add 4 u of that sum (in absolute terms: |s| is below it) and 2^-21.
 * a weight enters as a sum of terms of 16 bits, each off by half a step of its type from what the terms
   before leave: eps of it, with eps = 2^-11 for one of fp16, (2^-8)^2 for two of bf16, (2^-11)^2 for two
   of fp16, (2^-8)^3 for three of bf16; in fp16 it also has no bits below 2^-25, where the largest of a warp's is 2^7 at least: 2^-32 of the largest (of the
   sum of all weights at most) for each token.
 * each warp adds up a fourth of the tokens or fewer, 16 at a time: 2 u for each of the n / 64
   steps, and some 64 u for the joins.
 * half a unit of y's type.
"""
import torch

U = 2.0 ** -24
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
KV_BF16, KV_F16, KV_INT8, KV_INT4 = range(4)
TYPE = {KV_BF16: torch.bfloat16, KV_F16: torch.float16}
BITS = {KV_BF16: 16, KV_F16: 16, KV_INT8: 8, KV_INT4: 4}


def encode(x, fmt):
    """Rows [..][D] of any type -> bytes [..][D bits / 8] and scales [..] fp16 (or None)."""
    bits = BITS[fmt]
    if bits == 16:
        return x.float().to(TYPE[fmt]).contiguous().view(torch.uint8), None
    q = 2 ** (bits - 1) - 1
    x = x.double()
    top = torch.where(x.isnan(), 0.0, x.abs()).amax(-1)
    s = (top / q).float().clamp(2.0 ** -14, 65504.0).half()
    u = torch.where(x.isnan(), 0.0, (x / s.double()[..., None]).float().round().clamp(-q, q)).to(torch.int16) + q + 1
    if bits == 4:
        u = u[..., 0::2] + 16 * u[..., 1::2]
    return u.to(torch.uint8), s


def split(pages, kv):
    """Views of the pages [n][L][heads]: bytes of K and V [..][tokens][row], scales [..][tokens]."""
    row, p = kv.head_dim * BITS[kv.format] // 8, kv.page_tokens
    seg = p * (2 * row + (4 if BITS[kv.format] < 16 else 0))
    t = pages.view(-1, kv.n_layers, kv.n_heads, seg)
    k, v = (t[..., i * p * row:(i + 1) * p * row].unflatten(-1, (p, row)) for i in range(2))
    if BITS[kv.format] == 16:
        return k, v, None, None
    return k, v, *(t[..., 2 * p * row + 2 * i * p:2 * p * row + 2 * (i + 1) * p].view(torch.float16) for i in range(2))


def decode(rows, s, fmt):
    """(values, |code with its offset| * scale) in 64 bits."""
    if BITS[fmt] == 16:
        x = rows.contiguous().view(TYPE[fmt]).double()
        return x, x.abs()
    if fmt == KV_INT4:
        rows = torch.stack([rows & 15, rows >> 4], -1).flatten(-2)
    half, s = 2.0 ** (BITS[fmt] - 1), s.double()[..., None]
    return (rows.double() - half) * s, (rows.double() + half) * s


def places(table, starts, lens, pt, seqs=None):
    """(page, place in it) of the tokens starts[b] .. of each sequence, packed."""
    page, at = [], []
    for b, (a, n) in enumerate(zip(starts, lens)):
        t = torch.arange(a, a + n, device=table.device)
        page.append(table[b][t // pt].long())
        at.append(t % pt)
    return torch.cat(page), torch.cat(at)


def append(pages, kv, layer, table, starts, lens, k, v):
    k_, v_, sk, sv = split(pages, kv)
    page, at = places(table, starts, lens, kv.page_tokens)
    for rows, scales, x in ((k_, sk, k), (v_, sv, v)):
        code, s = encode(x, kv.format)
        rows[page, layer, :, at] = code
        if s is not None:
            scales[page, layer, :, at] = s


def read(pages, kv, layer, table, starts, lens):
    """K, V [tokens][heads][D] in 64 bits, and their absolute values with the codes' offset."""
    k, v, sk, sv = split(pages, kv)
    page, at = places(table, starts, lens, kv.page_tokens)
    out = [decode(x[page, layer, :, at], None if s is None else s[page, layer, :, at], kv.format) for x, s in ((k, sk), (v, sv))]
    return out[0][0], out[1][0], out[0][1]


def eps_of(fmt, dtype):
    if fmt == KV_BF16:
        return 2.0 ** -24 if dtype is torch.float32 else 2.0 ** -16
    return 2.0 ** -11 if dtype is torch.bfloat16 else 2.0 ** -22


def attend(pages, kv, layer, table, lens, q, scale, window=0):
    """y [B][Hq][D] and lse [B][Hq] in 64 bits, and the bounds of both before y's own rounding."""
    B, Hq, D = q.shape
    y, tol = (torch.zeros((B, Hq, D), dtype=torch.float64, device=q.device) for _ in range(2))
    lse = torch.full((B, Hq), -torch.inf, dtype=torch.float64, device=q.device)
    ltol = torch.zeros_like(lse)
    eps = eps_of(kv.format, q.dtype)
    for b, n in enumerate(lens):
        lo = max(0, n - window) if window else 0
        if n <= lo:
            continue
        k, v, ka = read(pages, kv, layer, table[b:b + 1], [lo], [n - lo])
        qb = q[b].double().view(kv.n_heads, -1, D)
        s = scale * (qb @ k.permute(1, 2, 0))                                # [heads][G][tokens]
        p = torch.softmax(s, -1)
        e = abs(scale) * (qb.abs() @ ka.permute(1, 2, 0)) * 68 * U + 2.0 ** -21
        if BITS[kv.format] < 16 and q.dtype is not torch.float32:
            s_k = split(pages, kv)[2][places(table[b:b + 1], [lo], [n - lo], kv.page_tokens)[0], layer, :,
                                      places(table[b:b + 1], [lo], [n - lo], kv.page_tokens)[1]].double()
            e = e + abs(scale) * D / 16 * 2.0 ** -13 * qb.abs().amax(-1, keepdim=True) * s_k.t()[:, None, :]
        vh = v.transpose(0, 1)                                               # [heads][tokens][D]
        yb = p @ vh
        steps = (n - lo) / 64 * 2 + 64
        t = (p * e) @ vh.abs() + (p * e).sum(-1, keepdim=True) * yb.abs() + (eps + steps * U) * (p @ vh.abs())
        if kv.format != KV_BF16:
            t = t + 2.0 ** -32 * vh.abs().sum(1, keepdim=True)
        y[b], tol[b] = yb.reshape(Hq, D), t.reshape(Hq, D)
        lse[b] = torch.logsumexp(s, -1).reshape(Hq)
        ltol[b] = (e.amax(-1) + steps * U + lse[b].view(s.shape[:2]).abs() * 4 * U).reshape(Hq)
    return y, lse, tol, ltol


def rounded(tol, want, dtype):
    return tol + (want.abs() + tol) * HALF_UNIT[dtype] + TINY[dtype]


def assert_within(got, want, tol, what):
    d = (got.double() - want).abs()
    bad = ~((d <= tol) | (got.double() == want))
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((d / tol)[bad].max())} times, at {bad.nonzero()[0].tolist()}"
