"""Performance cases of the linear-attention operators and the group norm that follows
them, over the sizes a serving program calls them at.

  prefill  prompts through one layer: S_t = g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t from
           each sequence's slot (or from zero), packed ragged sequences
  decode   one token of `batch` slots through `layers` layers
  norm     group norm of rows of channels with an activation or a gate

With `norm` set, prefill and decode return act-gated, per-head normalised readouts.
`run` computes either the plain form (32-bit torch) or, with `own`, calls the library.
"""
import math
import random

import torch

own = False
D = 128
CHUNK = 64                     # tokens per chunk of the plain form
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _prefill(name, batch, tokens, hk, hv, dtype="bf16", ragged=False, resume=1.0, resets=False, norm="", fused=False):
    """tokens: all sequences together; ragged: their lengths are spread over a factor of
    about 50; resume: the share of sequences that continue from their slot's state."""
    return {"name": name, "kind": "prefill", "batch": batch, "tokens": tokens, "hk": hk, "hv": hv, "dtype": dtype,
            "ragged": ragged, "resume": resume, "resets": resets, "norm": norm, "fused": fused}


def _decode(name, batch, hk, hv, layers=1, dtype="bf16", slots=0, norm="", fused=False):
    """slots: the pool's, in which the batch's are spread; fused: q, k, v (and z) are
    columns of one projection's rows."""
    return {"name": name, "kind": "decode", "batch": batch, "hk": hk, "hv": hv, "layers": layers, "dtype": dtype,
            "slots": slots or batch, "norm": norm, "fused": fused}


def _norm(name, rows, groups, width, dtype="bf16", center=True, act="silu", gated=True, affine="channel", pad=0):
    """width: channels of a group; affine: none, or weights per channel or shared by the
    groups; pad: elements between the rows of x (a slice of wider rows)."""
    return {"name": name, "kind": "norm", "rows": rows, "groups": groups, "width": width, "dtype": dtype,
            "center": center, "act": act, "gated": gated, "affine": affine, "pad": pad}


def listed():
    return [
        # A short prompt of one request on a small model: the smallest call, all latency.
        _prefill("prefill_tiny", 1, 7, 4, 4, resume=0.0),
        # Prompts of 512 tokens for a full batch of new requests on the GQA layer.
        _prefill("prefill_gqa", 128, 128 * 512, 16, 32, resume=0.0),
        # One long prompt: fewer heads than the GPU has multiprocessors.
        _prefill("prefill_long", 1, 16384, 16, 32, resume=0.0),
        # What a scheduler packs: prompts of very different, odd lengths, some continued from
        # their slots, several documents in one (decays of zero between them), q, k, v and
        # the gate z as columns of one projection, normalised and gated readouts.
        _prefill("prefill_ragged", 24, 20011, 16, 32, ragged=True, resume=0.5, resets=True, norm="group", fused=True),
        # A few prompts of an odd length in the fp32 that the Delta-rule calls take.
        _prefill("prefill_f32", 3, 999, 32, 32, dtype="f32"),
        # One request, one token on a small model, fp32 vectors.
        _decode("decode_tiny", 1, 4, 4, dtype="f32"),
        # One token of a GQA batch through four layers, readouts normalised and gated.
        _decode("decode_layers", 16, 16, 32, layers=4, norm="group", fused=True),
        # An odd batch of a GQA layer, RMS-normalised readouts.
        _decode("decode_gqa", 67, 16, 32, slots=96, norm="rms"),
        # The serving pool: 1024 slots in random order.
        _decode("decode_pool", 1024, 32, 32),
        # Readouts of a decode batch: 64 rows of 32 heads, all latency.
        _norm("norm_decode", 64, 32, 128),
        # Readouts of a prompt batch: 65536 tokens of 32 heads.
        _norm("norm_prompt", 65536, 32, 128, center=False, affine="shared"),
        # Groups of an odd width in fp32, an activation in place of a gate, padded rows.
        _norm("norm_odd", 4099, 12, 75, dtype="f32", gated=False, pad=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prefill", "prefill", "prefill", "decode", "decode", "norm"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32", "f16"])
    hv = rng.choice([4, 7, 10, 16, 20, 32])
    hk = hv // rng.choice([g for g in (1, 2, 4) if hv % (4 * g if g == 4 else g) == 0 and (hv, g) != (16, 4)])
    norm = rng.choice(["", "", "group", "rms"])
    if kind == "prefill":
        tokens = _log(rng, 1, 32768)
        tokens = min(tokens, (65536 if dtype == "bf16" else 16384) * 32 // hv)
        batch = min(tokens, _log(rng, 1, 128))
        c = _prefill("", batch, tokens, hk, hv, dtype, rng.random() < 0.6, rng.choice([0.0, 0.5, 1.0]),
                     rng.random() < 0.3, norm, rng.random() < 0.5)
    elif kind == "decode":
        batch, layers = _log(rng, 1, 1024), rng.choice([1, 1, 2, 4])
        batch = min(batch, 1024 * 32 // (hv * layers))
        c = _decode("", batch, hk, hv, layers, dtype, batch + rng.choice([0, rng.randint(1, 64)]), norm,
                    rng.random() < 0.5)
    else:
        width = rng.choice([128, 128, 64, 256, rng.randint(1, 640)])
        groups = rng.choice([1, 4, 7, 16, 32])
        width += width * groups == 24 * D                        # not a multiple of a vector either
        rows = min(_log(rng, 1, 65536), 65536 * 4096 * 2 // (width * groups * SIZE[dtype]))
        c = _norm("", rows, groups, width, dtype, rng.random() < 0.5, rng.choice(["silu", "sigmoid", "none"]),
                  rng.random() < 0.7, rng.choice(["none", "channel", "shared"]), rng.choice([0, 0, 8, 3]))
    del c["name"]
    return c


def _lengths(c):
    """Lengths of the sequences of a prefill, by its sizes alone."""
    B, n = c["batch"], c["tokens"]
    if not c["ragged"]:
        return [n // B + (i < n % B) for i in range(B)]
    r = random.Random(B * 1000003 + n)
    w = [math.exp(r.uniform(0, 4)) for _ in range(B)]
    cut = [round(sum(w[:i + 1]) / sum(w) * n) for i in range(B)]
    return [b - a for a, b in zip([0] + cut[:-1], cut)]          # zero for some where they are many


# ------------------------------------------------------------------ preparation
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(g, n, widths, dt, fused):
    """Normal rows [n][w] for each of `widths`, either tensors of their own or columns of one."""
    if fused:
        return list(torch.randn((n, sum(widths)), generator=g, device="cuda").to(dt).split(widths, dim=1))
    return [torch.randn((n, w), generator=g, device="cuda").to(dt) for w in widths]


def _affine(g, c, channels):
    if c.get("affine", "channel") == "none":
        return None, None
    n = c["width"] if c.get("affine") == "shared" else channels
    return 1 + 0.1 * torch.randn(n, generator=g, device="cuda"), 0.1 * torch.randn(n, generator=g, device="cuda")


def _gates(g, n, hv):
    """Decays in (0.9, 0.999), a quarter of the heads long-lived."""
    long_lived = torch.rand(hv, generator=g, device="cuda") < 0.25
    u = torch.rand((n, hv), generator=g, device="cuda")
    return torch.where(long_lived, 0.998 + 0.001 * u, 0.9 + 0.099 * u)


def _token_inputs(g, n, c, dt):
    """q, k, v, z [n][heads][128] and the decays [n][hv]: normal q, v and z, unit keys."""
    hk, hv = c["hk"], c["hv"]
    widths = [hk * D, hk * D, hv * D] + ([hv * D] if c["norm"] else [])
    x = [r.unflatten(1, (-1, D)) for r in _rows(g, n, widths, dt, c["fused"])]
    k = x[1].float()
    x[1].copy_(k / torch.linalg.vector_norm(k, dim=-1, keepdim=True))
    return dict(zip("qkvz", x)) | {"gate": _gates(g, n, hv)}


def _states(g, n, layers, hv):
    s = torch.randn((n, layers, hv, D, D), generator=g, device="cuda")
    return s.mul_(0.3)


def prepare(case, seed):
    c, g, dt = case, _gen(seed), TYPES[case["dtype"]]
    st = {"case": c}
    if c["kind"] == "norm":
        C = c["groups"] * c["width"]
        wide = torch.randn((c["rows"], C + c["pad"]), generator=g, device="cuda").mul_(1.5).add_(0.2).to(dt)
        st["x"] = wide[:, :C]
        st["z"] = torch.randn((c["rows"], C), generator=g, device="cuda").to(dt) if c["gated"] else None
        st["w"], st["b"] = _affine(g, c, C)
        st["out"] = torch.empty((c["rows"], C), device="cuda", dtype=dt)
        return st
    hv, B, layers = c["hv"], c["batch"], c.get("layers", 1)
    slots = c.get("slots", B + B // 4)
    st["pool"] = _states(g, slots, layers, hv)
    st["slots"] = torch.randperm(slots, generator=g, device="cuda")[:B].to(torch.int32)
    if c["norm"]:
        st["w"], st["b"] = _affine(g, {}, hv * D)
        if c["norm"] == "rms":
            st["b"] = None
    if c["kind"] == "decode":
        st["in"] = [_token_inputs(g, B, c, dt) for _ in range(layers)]
        st["y"] = torch.empty((layers, B, hv, D), device="cuda", dtype=dt)
        return st
    n, lens = c["tokens"], _lengths(c)
    st["in"] = _token_inputs(g, n, c, dt)
    if c["resets"]:                                              # a document ends about every 300 tokens
        at = torch.rand(n, generator=g, device="cuda") < 1 / 300
        st["in"]["gate"].masked_fill_(at[:, None], 0.0)
    st["resume"] = (torch.rand(B, generator=g, device="cuda") < c["resume"]).to(torch.uint8)
    st["y"] = torch.empty((n, hv, D), device="cuda", dtype=dt)
    starts = [sum(lens[:i]) for i in range(B + 1)]
    st["cu"] = torch.tensor(starts, dtype=torch.int32).cuda()
    st["max_len"] = max(lens)
    # The batch cut into chunks, as a scheduler that knows the lengths lays it out: each
    # chunk's tokens, sequence, and whether it is its sequence's first.
    chunks = [(b, a) for b in range(B) for a in range(starts[b], starts[b + 1], CHUNK)]
    seq = torch.tensor([b for b, _ in chunks])
    pos = torch.tensor([a for _, a in chunks])[:, None] + torch.arange(CHUNK)
    valid = pos < torch.tensor(starts)[1:][seq][:, None]
    first = torch.tensor([i == 0 or chunks[i - 1][0] != b for i, (b, _) in enumerate(chunks)])
    last = torch.tensor([i + 1 == len(chunks) or chunks[i + 1][0] != b for i, (b, _) in enumerate(chunks)])
    st["plan"] = {"tok": pos.clamp(max=n - 1).cuda(), "valid": valid.cuda(), "seq": seq.cuda(), "first": first.cuda(),
                  "last": last.nonzero()[:, 0].cuda(), "flat": valid.reshape(-1).nonzero()[:, 0].cuda(),
                  "longest": -(-max(lens) // CHUNK)}
    return st


def _config(c):
    import paper_2609_38169_gb300 as P
    return P.Config(n_layers=c.get("layers", 1), n_key_heads=c["hk"], n_value_heads=c["hv"])


def _norm_arg(P, st, z):
    kind = st["case"]["norm"]
    return P.Norm(weight=st["w"], bias=st["b"], z=z, act=P.ACT_SILU, center=kind == "group") if kind else None


def _run_own(st):
    import paper_2609_38169_gb300 as P
    c = st["case"]
    if c["kind"] == "norm":
        act = {"silu": P.ACT_SILU, "sigmoid": P.ACT_SIGMOID, "none": P.ACT_NONE}[c["act"]]
        P.stepq_group_norm(st["x"], c["groups"], st["out"],
                           P.Norm(weight=st["w"], bias=st["b"], z=st["z"], act=act, center=c["center"],
                                  shared=c["affine"] == "shared"))
        return st["out"]
    cfg = _config(c)
    if c["kind"] == "decode":
        for layer, x in enumerate(st["in"]):
            P.stepq_linattn_decode_step(cfg, layer, st["pool"], st["slots"], x["q"], x["k"], x["v"], x["gate"],
                                        st["y"][layer], norm=_norm_arg(P, st, x.get("z")))
    else:
        x = st["in"]
        P.stepq_linattn_prefill(cfg, 0, st["pool"], st["slots"], x["q"], x["k"], x["v"], x["gate"], st["y"],
                                cu_seqlens=st["cu"], max_len=st["max_len"], resume=st["resume"],
                                norm=_norm_arg(P, st, x.get("z")))
    return {"y": st["y"], "state": st["pool"]}


# ------------------------------------------------------------------ the plain forms
def _act(x, act):
    return x * torch.sigmoid(x) if act == "silu" else torch.sigmoid(x) if act == "sigmoid" else x


def _plain_norm(x, z, w, b, center, act, eps=1e-5):
    """x [rows][groups][n] in 32 bits; w, b [groups][n] or [n]; z as x, or None."""
    if center:
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        x = x * w
    if b is not None:
        x = x + b
    return x * _act(z.float(), act) if z is not None else _act(x, act)


def _emit(st, y, z):
    """Readouts [rows][hv][128] in 32 bits, normalised if the case asks for it, in its type."""
    c = st["case"]
    if c["norm"]:
        w, b = (None if t is None else t.unflatten(0, (-1, D)) for t in (st["w"], st["b"]))
        y = _plain_norm(y, z, w, b, c["norm"] == "group", "silu")
    return y.to(TYPES[c["dtype"]])


def _plain_decode(st, layer, x):
    c, slots = st["case"], st["slots"].long()
    grp = c["hv"] // c["hk"]
    q, k = (x[n].float().repeat_interleave(grp, 1) for n in "qk")
    S = st["pool"][slots, layer]
    S.mul_(x["gate"][..., None, None]).add_(k[..., :, None] * x["v"].float()[..., None, :])
    st["pool"][slots, layer] = S
    st["y"][layer] = _emit(st, torch.matmul(q[..., None, :], S)[..., 0, :], x.get("z"))


def _plain_prefill(st):
    c, x, p = st["case"], st["in"], st["plan"]
    grp, slots = c["hv"] // c["hk"], st["slots"].long()
    keep = p["valid"][..., None, None]

    def chunked(t, rep):                                         # [chunks][hv][CHUNK][128]
        return (t[p["tok"]].float() * keep).transpose(1, 2).repeat_interleave(rep, 1)

    q, k, v = chunked(x["q"], grp), chunked(x["k"], grp), chunked(x["v"], 1)
    g = torch.where(p["valid"][..., None], x["gate"][p["tok"]], 1.0).transpose(1, 2)
    lg = torch.log(g.clamp_min(1e-36)).cumsum(-1)                # a decay of zero: exp(-83)
    diff = lg[..., :, None] - lg[..., None, :]
    lower = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device=q.device).tril()
    P = (q @ k.transpose(-1, -2)) * torch.exp(torch.where(lower, diff, -math.inf))
    total = lg[..., -1:]
    U = (k * torch.exp(total - lg)[..., None]).transpose(-1, -2) @ v     # each chunk's own part of the state
    A = torch.exp(total)[..., None]                              # what a chunk keeps of the state before it
    S0 = st["pool"][slots, 0] * st["resume"].to(torch.float32)[:, None, None, None]
    first = p["first"][:, None, None, None]
    U += torch.where(first, A * S0[p["seq"]], 0.0)
    A = torch.where(first, 0.0, A)
    S_in = torch.where(first, S0[p["seq"]], 0.0)
    d = 1
    while d < p["longest"]:                                      # scan of S -> A S + U over a sequence's chunks
        U = torch.cat([U[:d], U[d:] + A[d:] * U[:-d]])
        A = torch.cat([A[:d], A[d:] * A[:-d]])
        d *= 2
    S_in[1:] += torch.where(first[1:], 0.0, U[:-1])
    y = P @ v + torch.exp(lg)[..., None] * (q @ S_in)
    st["pool"][slots[p["seq"][p["last"]]], 0] = U[p["last"]]
    y = y.transpose(1, 2).reshape(-1, c["hv"], D)[p["flat"]]
    st["y"].copy_(_emit(st, y, x.get("z")))


def run(state):
    st, c = state, state["case"]
    if own:
        return _run_own(st)
    if c["kind"] == "norm":
        by = lambda t, n: None if t is None else t.unflatten(n, (-1, c["width"]))  # noqa: E731
        y = _plain_norm(by(st["x"], 1).float(), by(st["z"], 1), by(st["w"], 0), by(st["b"], 0), c["center"], c["act"])
        return y.reshape(c["rows"], -1).to(TYPES[c["dtype"]])
    if c["kind"] == "decode":
        for layer, x in enumerate(st["in"]):
            _plain_decode(st, layer, x)
    else:
        _plain_prefill(st)
    return {"y": st["y"], "state": st["pool"]}


# ------------------------------------------------------------------ floors
def work(case):
    c, e = case, SIZE[case["dtype"]]
    if c["kind"] == "norm":
        n = c["rows"] * c["groups"] * c["width"]
        return {"bytes": n * e * (3 if c["gated"] else 2), "flops": 8.0 * n}
    hk, hv, N = c["hk"], c["hv"], D * D
    vec = e * D * (2 * hk + (3 if c["norm"] else 2) * hv) + 4 * hv      # q, k, v, y, z and the decays of a token
    if c["kind"] == "decode":
        n = c["batch"] * c["layers"]
        return {"bytes": n * (vec + 8 * N * hv), "flops": n * hv * 5.0 * N}
    used = sum(length > 0 for length in _lengths(c))
    return {"bytes": c["tokens"] * vec + used * hv * 4 * N * (1 + c["resume"]), "flops": c["tokens"] * hv * 5.0 * N}


# ------------------------------------------------------------------ 64 bits
def _exact_norm(x, z, w, b, center, act):
    m = x.mean(-1, keepdim=True) if center else torch.zeros_like(x[..., :1])
    var = ((x - m) ** 2).mean(-1, keepdim=True)
    u = (x - m) / torch.sqrt(var + 1e-5)
    u = u if w is None else u * w.double()
    u = u if b is None else u + b.double()
    t = u if z is None else z.double()
    a = t if act == "none" else 1 / (1 + torch.exp(-t)) * (t if act == "silu" else 1)
    return a if z is None else u * a


def exact(case, seed):
    """The recurrences token by token."""
    c, st = case, prepare(case, seed)
    if c["kind"] == "norm":
        shape = (c["rows"], c["groups"], c["width"])
        by = lambda t: None if t is None else t.reshape(-1, c["width"])  # noqa: E731
        z = None if st["z"] is None else st["z"].reshape(shape)
        return _exact_norm(st["x"].double().reshape(shape), z, by(st["w"]), by(st["b"]), c["center"],
                           c["act"]).reshape(c["rows"], -1)
    hv, grp, slots, B = c["hv"], c["hv"] // c["hk"], st["slots"].long(), c["batch"]
    pool = st["pool"].double()
    head = torch.arange(hv, device="cuda") // grp

    def step(S, x, at):
        """One token of the rows `at` of the inputs on the states S [n][hv][128][128]."""
        q, k, v, g = (x[n][at].double() for n in ("q", "k", "v", "gate"))
        S *= g[..., None, None]
        S += k[:, head, :, None] * v[:, :, None, :]
        return torch.einsum("nhij,nhi->nhj", S, q[:, head])

    def emit(y, z):
        if not c["norm"]:
            return y
        w, b = (None if t is None else t.reshape(hv, D) for t in (st["w"], st["b"]))
        return _exact_norm(y, z, w, b, c["norm"] == "group", "silu")

    if c["kind"] == "decode":
        y = torch.empty(st["y"].shape, dtype=torch.float64, device="cuda")
        every = torch.arange(B, device="cuda")
        for layer, x in enumerate(st["in"]):
            S = pool[slots, layer]
            y[layer] = emit(step(S, x, every), x.get("z"))
            pool[slots, layer] = S
        return {"y": y, "state": pool}
    lens = _lengths(c)
    by_length = sorted(range(B), key=lambda b: -lens[b])
    order = torch.tensor(by_length, device="cuda")
    start = st["cu"].long()[order]
    S = pool[slots[order], 0] * st["resume"][order].double()[:, None, None, None]
    y = torch.empty(st["y"].shape, dtype=torch.float64, device="cuda")
    active = sum(length > 0 for length in lens)
    for t in range(max(lens)):
        while lens[by_length[active - 1]] <= t:
            active -= 1
        at = start[:active] + t
        y[at] = step(S[:active], st["in"], at)
    used = sum(length > 0 for length in lens)
    pool[slots[order[:used]], 0] = S[:used]
    return {"y": emit(y, st["in"].get("z")), "state": pool}
