"""Performance cases of the paged key-value cache: rows written to it in 16, 8 or 4 bits and
read back, and the attention of one new token a sequence over it.

attend  one token of `batch` sequences over their cached tokens (a window of them, or all)
chunk   a chunk of each sequence's prompt is written behind its prefix, then prefix and chunk
        are read back as dense rows, which the chunk's attention works on
read    cached prompts are read back as dense rows
step    one token of every sequence through `layers` layers: its key and value written, then
        its attention over the cache that holds them

`run` computes either the plain form (32-bit torch) or, with `own`, calls the library.
"""
import math
import random

import torch

own = False
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BITS = {"bf16": 16, "f16": 16, "int8": 8, "int4": 4}           # the cache's formats


def _attend(name, batch, tokens, hq, hk, D=128, fmt="bf16", dtype="bf16", page=16, ragged=False, window=0):
    """tokens: cached, all sequences together; ragged: lengths spread over a factor of about 50."""
    return {"name": name, "kind": "attend", "batch": batch, "tokens": tokens, "hq": hq, "hk": hk, "D": D, "fmt": fmt,
            "dtype": dtype, "page": page, "ragged": ragged, "window": window}


def _chunk(name, batch, tokens, prefix, hk, D=128, fmt="int8", dtype="bf16", page=16, ragged=False, fused=False):
    """tokens: written, all sequences together; prefix: cached before, of each sequence; fused:
    k and v are columns of one projection's rows."""
    return {"name": name, "kind": "chunk", "batch": batch, "tokens": tokens, "prefix": prefix, "hk": hk, "D": D,
            "fmt": fmt, "dtype": dtype, "page": page, "ragged": ragged, "fused": fused}


def _read(name, batch, tokens, hk, D=128, fmt="int8", dtype="bf16", page=16, ragged=False):
    return {"name": name, "kind": "read", "batch": batch, "tokens": tokens, "hk": hk, "D": D, "fmt": fmt,
            "dtype": dtype, "page": page, "ragged": ragged}


def _step(name, batch, tokens, hq, hk, layers, D=128, fmt="bf16", dtype="bf16", page=16, ragged=False):
    return {"name": name, "kind": "step", "batch": batch, "tokens": tokens, "hq": hq, "hk": hk, "layers": layers, "D": D,
            "fmt": fmt, "dtype": dtype, "page": page, "ragged": ragged}


def listed():
    return [
        # One request just begun on a small model: all latency.
        _attend("attend_tiny", 1, 37, 8, 2),
        # A serving batch of mixed lengths in bf16, four query heads to a key head.
        _attend("attend_batch", 64, 131072, 32, 8, ragged=True),
        # One long document: one sequence has to fill the GPU, wide heads.
        _attend("attend_long", 1, 200003, 16, 2, D=256),
        # A full batch in 8 bits.
        _attend("attend_int8", 128, 128 * 4096, 32, 8, fmt="int8"),
        # A large batch of long sequences in 4 bits, eight query heads to a key head.
        _attend("attend_int4", 256, 256 * 8191, 64, 8, fmt="int4", page=64),
        # Sliding-window layers without shared heads, fp32 vectors over fp16 pages.
        _attend("attend_window", 33, 33 * 3001, 10, 10, D=64, fmt="f16", dtype="f32", page=32, ragged=True, window=1000),
        # Four attention layers of a batch's token, as a hybrid stack has them among its others.
        _step("step_layers", 16, 16 * 1000, 32, 4, 4, fmt="f16", dtype="f16", page=64, ragged=True),
        # A few tokens of one request: all latency.
        _chunk("chunk_small", 1, 7, 50, 2),
        # A scheduler's batch of prompt chunks of odd lengths, columns of one projection, in 8 bits.
        _chunk("chunk_prompts", 24, 20011, 512, 8, ragged=True, fused=True),
        # fp32 rows of wide heads into 4 bits.
        _chunk("chunk_f32", 3, 4099, 0, 2, D=256, fmt="int4", dtype="f32", page=8),
        # One short cached prompt read back for a request that shares it.
        _read("read_small", 1, 333, 8),
        # The cached prompts of a batch out of 4 bits.
        _read("read_prompts", 32, 32 * 2000, 8, fmt="int4", page=64, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "chunk", "read", "step"])
    fmt, dtype = rng.choice(list(BITS)), rng.choice(["bf16", "bf16", "f16", "f32"])
    D, page = rng.choice([64, 128, 128, 256]), rng.choice([8, 16, 32, 64, 128])
    hk, G = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16])
    batch, ragged = _log(rng, 1, 256), rng.random() < 0.6
    row = hk * D * BITS[fmt] // 4                                # bytes of a token's K and V
    if kind in ("attend", "step"):
        layers = 1 if kind == "attend" else rng.choice([1, 2, 4])
        # no more cache, and no more products, than the largest listed case
        most = min(int(2.0e9 / (row * layers)), int(6e10 / (4 * hk * G * D * layers)), 1 << 20)
        tokens = max(batch, min(most, batch * _log(rng, 1, 32768)))
        if kind == "attend":
            window = _log(rng, 16, 4096) if rng.random() < 0.3 else 0
            c = _attend("", batch, tokens, hk * G, hk, D, fmt, dtype, page, ragged, window)
        else:
            c = _step("", batch, tokens, hk * G, hk, layers, D, fmt, dtype, page, ragged)
    else:
        most = int(1.5e8 / (hk * D * SIZE[dtype]))
        tokens = max(batch, min(most, _log(rng, 1, 65536)))
        if kind == "chunk":
            c = _chunk("", batch, tokens, min(_log(rng, 1, 2048) - 1, most // batch), hk, D, fmt, dtype, page, ragged,
                       rng.random() < 0.5)
        else:
            c = _read("", batch, tokens, hk, D, fmt, dtype, page, ragged)
    del c["name"]
    return c


def _lengths(c):
    """Tokens of each sequence, one at least, by the case's sizes alone."""
    B, n = c["batch"], c["tokens"]
    if not c["ragged"]:
        return [n // B + (i < n % B) for i in range(B)]
    r = random.Random(B * 1000003 + n)
    w = [math.exp(r.uniform(0, 4)) for _ in range(B)]
    cut = [round(sum(w[:i + 1]) / sum(w) * (n - B)) for i in range(B)]
    return [b - a + 1 for a, b in zip([0] + cut[:-1], cut)]


# ------------------------------------------------------------------ the pages
# A page holds, for each layer and key head, the rows of K of its tokens, those of V, and in
# 8 and 4 bits the fp16 scale of each row of K, then of V. Codes are offset binary, the lower
# channel of a byte of 4-bit codes in its lower half.
def _row_bytes(c):
    return c["D"] * BITS[c["fmt"]] // 8


def _segment_bytes(c):
    return c["page"] * (2 * _row_bytes(c) + (4 if BITS[c["fmt"]] < 16 else 0))


def _parts(c, seg):
    """Rows of K and V [..][page][bytes] and their scales [..][page] (or None), views of the
    segments seg [..][bytes]."""
    n, p = c["page"] * _row_bytes(c), c["page"]
    k, v = (seg[..., i * n:i * n + n].unflatten(-1, (p, _row_bytes(c))) for i in range(2))
    if BITS[c["fmt"]] == 16:
        return k, v, None, None
    return k, v, *(seg[..., 2 * n + 2 * i * p:2 * n + 2 * (i + 1) * p].view(torch.float16) for i in range(2))


def _encode(c, x):
    """Rows x [..][D] in 32 bits -> their bytes and scales."""
    bits = BITS[c["fmt"]]
    if bits == 16:
        return x.to(TYPES[c["fmt"]]).view(torch.uint8), None
    q = 2.0 ** (bits - 1) - 1
    top = x.abs().amax(-1)
    s = (top / torch.full_like(top, q)).clamp(2.0 ** -14, 65504.0).to(torch.float16)
    u = ((x / s.float()[..., None]).round().clamp(-q, q) + 2.0 ** (bits - 1)).to(torch.uint8)
    if bits == 4:
        u = u[..., 0::2] + 16 * u[..., 1::2]
    return u, s


def _decode(c, rows, s):
    """The values in 32 bits of rows' bytes and scales."""
    bits = BITS[c["fmt"]]
    if bits == 16:
        return rows.view(TYPES[c["fmt"]]).float()
    if bits == 4:
        rows = torch.stack([rows & 15, rows >> 4], -1).flatten(-2)
    return (rows.float() - 2.0 ** (bits - 1)) * s.float()[..., None]


# ------------------------------------------------------------------ preparation
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _keys(g, shape, loud):
    """Normal keys [..][D], some channels of a head five times as large."""
    return torch.randn(shape, generator=g, device="cuda").mul_(loud)


def _pool(g, c, n, loud):
    """n pages of cached tokens, all layers."""
    L, hk, p, D = c.get("layers", 1), c["hk"], c["page"], c["D"]
    pages = torch.empty((n, L, hk, _segment_bytes(c)), dtype=torch.uint8, device="cuda")
    at_once = max(1, (1 << 28) // (L * hk * p * D))
    for a in range(0, n, at_once):
        seg = pages[a:a + at_once]
        k, v, sk, sv = _parts(c, seg)
        for rows, scales, x in ((k, sk, _keys(g, (len(seg), L, hk, p, D), loud)),
                                (v, sv, torch.randn((len(seg), L, hk, p, D), generator=g, device="cuda"))):
            code, s = _encode(c, x)
            rows.copy_(code)
            if s is not None:
                scales.copy_(s)
    return pages


def _where(st, starts, lens):
    """Of packed rows, sequence b's tokens starts[b] .. starts[b] + lens[b] - 1: the page and the
    place in it, and the sequences' bounds."""
    n = torch.tensor(lens, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), n)
    cu = torch.cat([n.new_zeros(1), n.cumsum(0)])
    pos = torch.arange(int(sum(lens)), device="cuda") - cu[seq] + torch.tensor(starts, device="cuda")[seq]
    p = st["case"]["page"]
    return {"page": st["table"][seq, pos // p].long(), "at": pos % p, "cu": cu.to(torch.int32),
            "starts": torch.tensor(starts, dtype=torch.int32).cuda()}


def _groups(c, lens):
    """Sequences of like lengths, as many as gather into about 2 GB at a time, with the pages
    that hold their windows and which of the pages' tokens count."""
    p, W = c["page"], c["window"] if c.get("window") else 1 << 30
    spans = sorted(((n - max(0, n - W)) // p + 2, b) for b, n in enumerate(lens))
    out, i = [], 0
    while i < len(spans):
        j = i + 1
        while j < len(spans) and (j + 1 - i) * spans[j][0] * p * c["hk"] * c["D"] * 8 <= 2e9 and \
                spans[j][0] <= 2 * spans[i][0] + 8:
            j += 1
        rows = [b for _, b in spans[i:j]]
        n = torch.tensor([lens[b] for b in rows])[:, None]
        lo = (n - W).clamp_min(0)
        page = lo // p + torch.arange(int(((n - 1) // p - lo // p).max()) + 1)
        pos = (page[:, :, None] * p + torch.arange(p)).flatten(1)
        out.append({"rows": torch.tensor(rows).cuda(), "page": page.clamp(max=(max(lens) - 1) // p).cuda(),
                    "valid": ((pos >= lo) & (pos < n)).cuda()})
        i = j
    return out


def prepare(case, seed):
    c, g, dt = case, _gen(seed), TYPES[case["dtype"]]
    kind, B, hk, D, p, L = c["kind"], c["batch"], c["hk"], c["D"], c["page"], c.get("layers", 1)
    st = {"case": c}
    lens, before = _lengths(c), [c.get("prefix", 0)] * c["batch"]
    if kind == "step":
        before, lens = lens, [n + 1 for n in lens]
    ends = [a + n for a, n in zip(before, lens)] if kind == "chunk" else lens
    need = [-(-n // p) for n in ends]
    loud = torch.where(torch.rand(D, generator=g, device="cuda") < 1 / 16, 5.0, 1.0)
    # the pool holds other requests' pages too; a request's pages lie in any order
    ids = torch.randperm(sum(need) + 8 + sum(need) // 8, generator=g, device="cuda").to(torch.int32)
    st["pages"] = _pool(g, c, len(ids), loud)
    st["table"] = torch.zeros((B, max(need)), dtype=torch.int32, device="cuda")
    held = torch.arange(max(need), device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]
    st["table"][held] = ids[:sum(need)]
    if kind in ("attend", "step"):
        st["lens"], st["max_len"] = torch.tensor(lens, dtype=torch.int32).cuda(), max(lens)
        st["plan"] = _groups(c, lens)
        st["q"] = torch.randn((L, B, c["hq"], D), generator=g, device="cuda").to(dt)
        st["y"] = torch.empty_like(st["q"])
    if kind in ("chunk", "step"):
        n = sum(lens) if kind == "chunk" else B
        k, v = _keys(g, (L, n, hk, D), loud), torch.randn((L, n, hk, D), generator=g, device="cuda")
        if c.get("fused"):
            kv = torch.cat([k.flatten(2), v.flatten(2)], 2).to(dt)
            k, v = (t.unflatten(2, (hk, D)) for t in kv.split(hk * D, 2))
        st["k"], st["v"] = k.to(dt), v.to(dt)
        st["new"] = _where(st, before, lens if kind == "chunk" else [1] * B)
        if kind == "step" and BITS[c["fmt"]] < 16:
            st["kept"] = [torch.empty((L, B, hk, D), device="cuda") for _ in range(2)]
    if kind in ("chunk", "read"):
        st["all"] = _where(st, [0] * B, ends)
        st["out"] = [torch.empty((sum(ends), hk, D), dtype=dt, device="cuda") for _ in range(2)]
    return st


# ------------------------------------------------------------------ the library's calls
def _run_own(st):
    import paper_2609_38169_gb300 as P
    c = st["case"]
    kv = P.KvConfig(n_layers=c.get("layers", 1), n_heads=c["hk"], head_dim=c["D"], page_tokens=c["page"],
                    format={"bf16": P.KV_BF16, "f16": P.KV_F16, "int8": P.KV_INT8, "int4": P.KV_INT4}[c["fmt"]])
    pages, table = st["pages"], st["table"]
    if c["kind"] in ("attend", "step"):
        if "ws" not in st:
            n = P.stepq_kv_workspace_bytes(kv, c["hq"], c["batch"], st["max_len"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        for layer in range(c.get("layers", 1)):
            if c["kind"] == "step":
                P.stepq_kv_append(kv, layer, pages, table, st["new"]["starts"], st["k"][layer], st["v"][layer])
            P.stepq_kv_attend(kv, layer, pages, table, st["lens"], st["q"][layer], st["y"][layer],
                              window=c.get("window", 0), max_len=st["max_len"], workspace=st["ws"])
            if "kept" in st:
                P.stepq_kv_read(kv, layer, pages, table, st["new"]["starts"], st["kept"][0][layer], st["kept"][1][layer])
        return _attended(st)
    if c["kind"] == "chunk":
        w = st["new"]
        P.stepq_kv_append(kv, 0, pages, table, w["starts"], st["k"][0], st["v"][0], cu_seqlens=w["cu"])
    w = st["all"]
    P.stepq_kv_read(kv, 0, pages, table, w["starts"], *st["out"], cu_seqlens=w["cu"])
    return {"k": st["out"][0], "v": st["out"][1]}


def _attended(st):
    """What a step leaves: the outputs, and the pages that it wrote to, or the values that its
    codes in them stand for."""
    c = st["case"]
    if c["kind"] == "attend":
        return {"y": st["y"]}
    if "kept" in st:
        return {"y": st["y"], "k": st["kept"][0], "v": st["kept"][1]}
    return {"y": st["y"], "pages": st["pages"].view(TYPES[c["fmt"]])}


# ------------------------------------------------------------------ the plain forms
def _plain_append(st, layer):
    c, w = st["case"], st["new"]
    k, v, sk, sv = _parts(c, st["pages"][:, layer])
    for rows, scales, x in ((k, sk, st["k"][layer]), (v, sv, st["v"][layer])):
        code, s = _encode(c, x.float())
        rows[w["page"], :, w["at"]] = code
        if s is not None:
            scales[w["page"], :, w["at"]] = s


def _plain_read(st, layer, w, outs):
    c = st["case"]
    k, v, sk, sv = _parts(c, st["pages"][:, layer])
    for rows, scales, out in ((k, sk, outs[0]), (v, sv, outs[1])):
        out.copy_(_decode(c, rows[w["page"], :, w["at"]], None if scales is None else scales[w["page"], :, w["at"]]))


def _plain_attend(st, layer):
    c = st["case"]
    for grp in st["plan"]:
        rows = grp["rows"]
        k, v, sk, sv = _parts(c, st["pages"][st["table"][rows[:, None], grp["page"]].long(), layer])
        k, v = (_decode(c, x, s).transpose(1, 2).flatten(2, 3) for x, s in ((k, sk), (v, sv)))   # [rows][hk][tokens][D]
        q = st["q"][layer, rows].float().unflatten(1, (c["hk"], -1))
        s = (q @ k.transpose(-1, -2)) * c["D"] ** -0.5
        s = torch.where(grp["valid"][:, None, None], s, -math.inf)
        e = torch.exp(s - s.amax(-1, keepdim=True))
        st["y"][layer, rows] = ((e @ v) / e.sum(-1, keepdim=True)).flatten(1, 2).to(TYPES[c["dtype"]])


def run(state):
    st, c = state, state["case"]
    if own:
        return _run_own(st)
    if c["kind"] in ("attend", "step"):
        for layer in range(c.get("layers", 1)):
            if c["kind"] == "step":
                _plain_append(st, layer)
            _plain_attend(st, layer)
            if "kept" in st:
                _plain_read(st, layer, st["new"], [t[layer] for t in st["kept"]])
        return _attended(st)
    if c["kind"] == "chunk":
        _plain_append(st, 0)
    _plain_read(st, 0, st["all"], st["out"])
    return {"k": st["out"][0], "v": st["out"][1]}


# ------------------------------------------------------------------ floors
def work(case):
    c, e, lens = case, SIZE[case["dtype"]], _lengths(case)
    hk, D = c["hk"], c["D"]
    held = hk * (2 * _row_bytes(c) + (4 if BITS[c["fmt"]] < 16 else 0))        # a token in the cache
    rows = 2 * hk * D * e                                                      # a token's K and V
    if c["kind"] == "read":
        return {"bytes": c["tokens"] * (held + rows), "flops": 2.0 * c["tokens"] * hk * D}
    if c["kind"] == "chunk":
        # rows in, codes out; the prefix's codes in; all rows out
        n, old = c["tokens"], c["prefix"] * c["batch"]
        return {"bytes": n * (rows + held) + old * held + (n + old) * rows, "flops": 8.0 * n * hk * D}
    L, step = c.get("layers", 1), c["kind"] == "step"
    used = sum(min(n + step, c.get("window") or n + step) for n in lens)
    vec = c["batch"] * (2 * c["hq"] * D * e + step * (rows + held))
    return {"bytes": L * (used * held + vec), "flops": 4.0 * L * used * c["hq"] * D}


# ------------------------------------------------------------------ 64 bits
def _quantised(c, x):
    """What the cache holds of rows x, in 64 bits."""
    x, bits = x.double(), BITS[c["fmt"]]
    if bits == 16:
        return x.to(TYPES[c["fmt"]]).double()
    q = 2 ** (bits - 1) - 1
    s = torch.clip(x.abs().max(-1).values / q, 2.0 ** -14, 65504.0).half().double()[..., None]
    return torch.clip(torch.round((x / s).float().double()), -q, q) * s


def _held(st, layer, b, lo, hi):
    """K and V [tokens][hk][D] of sequence b's tokens lo .. hi - 1 in 64 bits, from the bytes."""
    c = st["case"]
    p, hk, D, bits, seg = c["page"], c["hk"], c["D"], BITS[c["fmt"]], _segment_bytes(c)
    t = torch.arange(lo, hi, device="cuda")
    base = (st["table"][b, t // p].long() * c.get("layers", 1) + layer)[:, None] * hk + torch.arange(hk, device="cuda")
    base = base * seg                                            # [tokens][hk], the segment's first byte
    raw, out = st["pages"].view(-1), []
    for part in range(2):
        row = base + (part * p + t % p)[:, None] * (D * bits // 8)
        byte = raw[row[..., None] + torch.arange(D * bits // 8, device="cuda")]
        if bits == 16:
            out.append(byte.view(TYPES[c["fmt"]]).double())
            continue
        place = base + 2 * p * (D * bits // 8) + 2 * (part * p + t % p)[:, None]
        s = raw[place[..., None] + torch.arange(2, device="cuda")].view(torch.float16).double()
        if bits == 4:
            u = torch.empty((*byte.shape[:-1], D), dtype=torch.float64, device="cuda")
            u[..., 0::2], u[..., 1::2] = byte % 16, byte // 16
            out.append((u - 8) * s)
        else:
            out.append((byte.double() - 128) * s)
    return out


def exact(case, seed):
    c, st = case, prepare(case, seed)
    lens, B, hk, D, L = _lengths(c), c["batch"], c["hk"], c["D"], c.get("layers", 1)
    if c["kind"] in ("chunk", "read"):
        out, at, prefix, new = [[], []], 0, c.get("prefix", 0), [None, None]
        if c["kind"] == "chunk":
            new = [_quantised(c, st[n][0]) for n in "kv"]
        for b, n in enumerate(lens):
            held = _held(st, 0, b, 0, prefix if c["kind"] == "chunk" else n)
            for i in range(2):
                out[i] += [held[i]] if new[i] is None else [held[i], new[i][at:at + n]]
            at += n
        return {"k": torch.cat(out[0]), "v": torch.cat(out[1])}
    step = c["kind"] == "step"
    y = torch.empty(st["y"].shape, dtype=torch.float64, device="cuda")
    new = [_quantised(c, st[n]) for n in "kv"] if step else None
    for layer in range(L):
        for b, n in enumerate(lens):
            k, v = _held(st, layer, b, max(0, n - c["window"]) if c.get("window") else 0, n)
            if step:
                k, v = torch.cat([k, new[0][layer, b:b + 1]]), torch.cat([v, new[1][layer, b:b + 1]])
            q = st["q"][layer, b].double().view(hk, -1, D)
            s = torch.einsum("hgd,thd->hgt", q, k) / math.sqrt(D)
            w = torch.softmax(s, -1)
            y[layer, b] = torch.einsum("hgt,thd->hgd", w, v).reshape(-1, D)
    if not step:
        return {"y": y}
    if BITS[c["fmt"]] < 16:
        return {"y": y, "k": new[0], "v": new[1]}
    pages = st["pages"].view(TYPES[c["fmt"]]).double()
    both = pages.view(len(pages), L, hk, 2, c["page"], D)
    for layer in range(L):
        for i in range(2):
            both[st["new"]["page"], layer, :, i, st["new"]["at"]] = new[i][layer]
    return {"y": y, "pages": pages}
