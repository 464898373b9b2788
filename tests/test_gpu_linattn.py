"""Decayed linear attention against the 64-bit recurrence (tolerances: linattn_ref)."""
import pytest

from paper_2609_38169_gb300 import api as A

import linattn_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
D = 128
TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAMES = ["f32", "bf16", "f16"]


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert A.stepq_device_error() == 0


def rows(g, n, heads, dt, wide):
    """[n][heads][128]: rows of their own, or a slice of wider rows."""
    x = torch.randn((n, heads + (3 if wide else 0), D), generator=g, device="cuda").to(dt)
    return x[:, 1:1 + heads] if wide else x


def inputs(g, n, hk, hv, dt, wide=False):
    q, k, v, z = (rows(g, n, h, dt, wide) for h in (hk, hk, hv, hv))
    k.mul_(0.09)
    u = torch.rand((n, hv), generator=g, device="cuda")
    long_lived = torch.arange(hv, device="cuda") % 3 == 0
    return q, k, v, z, torch.where(long_lived, 0.99 + 0.0099 * u, 0.7 + 0.29 * u)


def norm_of(kind, hv, z, g):
    """The library's norm and the reference's arguments."""
    if kind is None:
        return None, None
    w, b = 1 + 0.2 * torch.randn((2, hv * D), generator=g, device="cuda")
    args = {"group": dict(w=w, b=b - 1, z=z, kind=1, center=True),
            "rms": dict(w=w[:D].contiguous(), z=z, kind=2, center=False, shared=True),
            "silu": dict(kind=1, center=True), "plain": dict(b=b, z=z, kind=0, center=False)}[kind]
    return A.Norm(weight=args.get("w"), bias=args.get("b"), z=args.get("z"), act=args["kind"],
                  center=args["center"], shared=args.get("shared", False)), args


def check_y(got, y, ya, dt, args, rows_):
    """One sequence's outputs [T][hv][128] against y, with the norm's arguments if any."""
    hv = y.shape[1]
    e = R.y_bound(y, ya, dt)
    if args is None:
        want, tol = y, e
    else:
        args = dict(args)
        if args.get("z") is not None:
            args["z"] = args["z"][rows_].flatten(1)
        want, gain, part = R.norm(y.flatten(1), hv, **args)
        tol = R.norm_bound(e.flatten(1), gain, part, hv)
        want, tol = want.view_as(y), tol.view_as(y)
    R.assert_within(got, want, R.rounded(tol, want, dt), "y")


def run_prefill(lens, hk, hv, dt, norm=None, wide=False, resume=None, layers=1, seed=0, edit=None, extra=0,
                max_len=None, per_head=False, stream=None):
    """A packed batch through the library and the reference; checks every output."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, n = len(lens), sum(lens)
    q, k, v, z, gate = inputs(g, n + extra, hk, hv, dt, wide)
    if per_head:
        gate = gate[0].contiguous()
    if edit:
        edit(q, k, v, gate)
    pool = torch.randn((B + 2, layers, hv, D, D), generator=g, device="cuda")
    slots = torch.randperm(B + 2, generator=g, device="cuda")[:B].to(torch.int32)
    flags = None if resume is None else torch.tensor([resume(b) for b in range(B)], dtype=torch.uint8, device="cuda")
    before = pool.clone()
    if flags is not None:                                    # a new sequence's slot may hold anything
        for b in range(B):
            if not flags[b] and lens[b]:
                pool[slots[b].long()] = torch.nan
        kept = pool.clone()
    cfg = A.Config(n_layers=layers, n_key_heads=hk, n_value_heads=hv)
    lib_norm, args = norm_of(norm, hv, z, g)
    y = torch.full((n + extra, hv, D), 7.0, dtype=dt, device="cuda")
    cu = torch.tensor([sum(lens[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    layer = layers - 1
    torch.cuda.synchronize()
    A.stepq_linattn_prefill(cfg, layer, pool, slots, q, k, v, gate, y, cu_seqlens=cu,
                            max_len=max(lens, default=0) if max_len is None else max_len, resume=flags, norm=lib_norm,
                            stream=stream)
    torch.cuda.synchronize()
    at = 0
    for b, T in enumerate(lens):
        s, r = int(slots[b]), slice(at, at + T)
        if T:
            S = before[s, layer].double() if flags is None or flags[b] else torch.zeros((hv, D, D), dtype=torch.float64, device="cuda")
            yr, ya, Sa = R.linattn(S, q[r], k[r], v[r], gate if per_head else gate[r])
            check_y(y[r], yr, ya, dt, args, r)
            R.assert_within(pool[s, layer], S, 64 * R.U * Sa + 1e-37, f"state of sequence {b}")
            before[s, layer] = pool[s, layer]
            if flags is not None and not flags[b] and layers > 1:
                assert bool(pool[s, :layer].isnan().all())
                before[s, :layer] = 0
                pool[s, :layer] = 0
        at += T
    assert torch.equal(pool, before)                         # nothing else in the pool moved
    assert bool((y[n:] == 7.0).all())
    return y, pool


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("lens", [[1], [2], [7], [31], [63], [64], [65], [127], [128], [129], [200], [515]], ids=str)
def test_lengths(lens, dt):
    run_prefill(lens, 2, 4, dt, seed=lens[0])


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("hk,hv", [(1, 1), (1, 4), (3, 3), (7, 14)])
def test_ragged_batches_and_heads(hk, hv, dt):
    run_prefill([5, 0, 130, 64, 1, 0, 77, 193, 0], hk, hv, dt, resume=lambda b: b % 2, layers=2, seed=hv, extra=9)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("norm", ["group", "rms", "silu", "plain"])
def test_norm_of_readouts_and_strided_rows(norm, dt):
    run_prefill([70, 3, 129], 2, 4, dt, norm=norm, wide=True, seed=5, resume=lambda b: b != 1)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("kind", ["resets", "reset runs", "tiny", "ones", "zeros", "small", "per head"])
def test_decays(kind, dt):
    """Zeros (alone, in runs, at a chunk's ends, everywhere), decays whose products leave
    fp32's range, no decay at all, and one decay per head for all tokens."""
    def edit(q, k, v, gate):
        if kind == "resets":
            gate[[0, 13, 63, 64, 100, 127, 128, 255]] = 0.0
        elif kind == "reset runs":
            gate[60:70] = 0.0
            gate[190:, 0] = 0.0
        elif kind == "tiny":
            gate[::3] = 1e-20
            gate[1::3] = 1e-30
        elif kind == "ones":
            gate.fill_(1.0)
        elif kind == "zeros":
            gate.zero_()
        elif kind == "small":
            gate.mul_(0.05)
    run_prefill([260], 1, 3, dt, edit=edit, per_head=kind == "per head", seed=11)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("lens", [[4096], [3000, 40, 5, 2049], [900] * 3], ids=str)
def test_long_sequences_on_few_heads(lens, dt):
    run_prefill(lens, 1, 2, dt, seed=3, resume=lambda b: b % 2 == 0, norm="group")


@pytest.mark.parametrize("max_len", [0, 1, 10 ** 6])
def test_the_longest_length_is_only_a_hint(max_len):
    run_prefill([1500, 3, 700], 1, 2, torch.bfloat16, max_len=max_len, seed=4)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
def test_values_over_a_wide_range(dt):
    """Keys and values over the type's exponents (states far above fp16's range)."""
    def edit(q, k, v, gate):
        s = torch.exp2(torch.randint(-10, 11, (v.shape[0], 1, 1), device="cuda").float())
        v.mul_(s.to(dt))
        k.mul_(torch.exp2(torch.randint(-4, 11, (k.shape[0], 1, 1), device="cuda").float()).to(dt))
        q.mul_(1e-4)
    run_prefill([150, 90], 2, 2, dt, edit=edit, seed=8)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_sequence_with_bad_values_leaves_the_others_alone(dt, bad):
    """Non-finite q, k, v and decays right beside a sequence's rows, in a full and a ragged
    chunk: its outputs and state are the ones it has without them."""
    lens, hk, hv = [70, 65, 64, 3], 1, 2
    g = torch.Generator(device="cuda").manual_seed(2)
    n = sum(lens)
    q, k, v, z, gate = inputs(g, n, hk, hv, dt)
    cfg = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv)
    slots = torch.arange(4, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 70, 135, 199, 202], dtype=torch.int32, device="cuda")
    got = []
    for spoil in (False, True):
        if spoil:
            for x in (q, k, v):
                x[70:135] = bad
            gate[70:135] = bad
        pool = torch.zeros((4, 1, hv, D, D), device="cuda")
        y = torch.zeros((n, hv, D), dtype=dt, device="cuda")
        A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, cu_seqlens=cu, max_len=70)
        got.append((torch.cat([y[:70], y[135:]]), pool[[0, 2, 3]]))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_equal_lengths_without_offsets():
    g = torch.Generator(device="cuda").manual_seed(6)
    q, k, v, z, gate = inputs(g, 3 * 50, 2, 4, torch.bfloat16)
    cfg, slots = A.Config(n_layers=1, n_key_heads=2, n_value_heads=4), torch.arange(3, dtype=torch.int32, device="cuda")
    out = []
    for cu in (None, torch.tensor([0, 50, 100, 150], dtype=torch.int32, device="cuda")):
        pool = torch.ones((3, 1, 4, D, D), device="cuda")
        y = torch.zeros((150, 4, D), dtype=torch.bfloat16, device="cuda")
        A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, cu_seqlens=cu, max_len=50)
        out.append((y, pool))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


# ------------------------------------------------------------------ single tokens
@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("norm", [None, "group", "rms", "silu"])
@pytest.mark.parametrize("B,hk,hv", [(1, 1, 1), (1, 4, 4), (3, 2, 4), (41, 16, 32), (130, 7, 7)])
def test_decode(B, hk, hv, norm, dt):
    g = torch.Generator(device="cuda").manual_seed(B + hv)
    q, k, v, z, gate = inputs(g, B, hk, hv, dt, wide=B % 2 == 1)
    gate[0, 0] = 0.0
    layers, layer = 2, 1
    pool = torch.randn((B + 3, layers, hv, D, D), generator=g, device="cuda")
    slots = torch.randperm(B + 3, generator=g, device="cuda")[:B].to(torch.int32)
    before = pool.clone()
    lib_norm, args = norm_of(norm, hv, z, g)
    y = torch.zeros((B, hv, D), dtype=dt, device="cuda")
    A.stepq_linattn_decode_step(A.Config(n_layers=layers, n_key_heads=hk, n_value_heads=hv), layer, pool, slots, q, k, v,
                                gate, y, norm=lib_norm)
    for b in range(B):
        s, r = int(slots[b]), slice(b, b + 1)
        S = before[s, layer].double()
        yr, ya, Sa = R.linattn(S, q[r], k[r], v[r], gate[r])
        check_y(y[r], yr, ya, dt, args, r)
        R.assert_within(pool[s, layer], S, 4 * R.U * Sa, "state")     # two roundings
        before[s, layer] = pool[s, layer]
    assert torch.equal(pool, before)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
def test_decode_continues_a_prompt(dt):
    """A prompt, then tokens one by one: the recurrence over all of them."""
    g = torch.Generator(device="cuda").manual_seed(1)
    hk, hv, T, more = 2, 4, 133, 5
    q, k, v, z, gate = inputs(g, T + more, hk, hv, dt)
    cfg, slots = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv), torch.zeros(1, dtype=torch.int32, device="cuda")
    pool = torch.full((1, 1, hv, D, D), torch.nan, device="cuda")
    y = torch.empty((T + more, hv, D), dtype=dt, device="cuda")
    fresh = torch.zeros(1, dtype=torch.uint8, device="cuda")
    A.stepq_linattn_prefill(cfg, 0, pool, slots, q[:T], k[:T], v[:T], gate[:T], y[:T], max_len=T, resume=fresh)
    for t in range(T, T + more):
        r = slice(t, t + 1)
        A.stepq_linattn_decode_step(cfg, 0, pool, slots, q[r], k[r], v[r], gate[r], y[r])
    S = torch.zeros((hv, D, D), dtype=torch.float64, device="cuda")
    yr, ya, Sa = R.linattn(S, q, k, v, gate)
    check_y(y, yr, ya, dt, None, None)
    R.assert_within(pool[0, 0], S, 64 * R.U * Sa, "state")


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens", [0, 9, 100])
def test_infinite_gates(tokens, dt):
    """A sigmoid gate of plus infinity passes the normalised readout, of minus infinity stops it
    (0 tokens: one a sequence, by the decode step)."""
    hk, hv, n = 2, 4, tokens or 3
    g = torch.Generator(device="cuda").manual_seed(tokens)
    q, k, v, z, gate = inputs(g, n, hk, hv, dt)
    cfg, got = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv), []
    for act, fill in ((A.ACT_NONE, 1.0), (A.ACT_SIGMOID, torch.inf), (A.ACT_SIGMOID, -torch.inf)):
        pool = torch.ones((n, 1, hv, D, D), device="cuda")
        y, norm = torch.empty((n, hv, D), dtype=dt, device="cuda"), A.Norm(z=torch.full_like(z, fill), act=act)
        slots = torch.arange(n if not tokens else 1, dtype=torch.int32, device="cuda")
        if tokens:
            A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, max_len=n, norm=norm)
        else:
            A.stepq_linattn_decode_step(cfg, 0, pool, slots, q, k, v, gate, y, norm=norm)
        got.append(y)
    assert torch.equal(got[1], got[0]) and bool((got[2] == 0).all())


# ------------------------------------------------------------------ streams, graphs, errors
def test_side_stream_and_graph():
    """Captured on a side stream, a prompt and two tokens replay to the bytes of the calls
    made one by one."""
    g = torch.Generator(device="cuda").manual_seed(7)
    hk, hv, lens = 2, 4, [300, 40]
    n, B = sum(lens), 2
    q, k, v, z, gate = inputs(g, n, hk, hv, torch.bfloat16)
    cfg, slots = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv), torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 300, 340], dtype=torch.int32, device="cuda")
    pool, y = torch.empty((2, 1, hv, D, D), device="cuda"), torch.empty((n, hv, D), dtype=torch.bfloat16, device="cuda")
    yd = torch.empty((B, hv, D), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(max(256, A.stepq_linattn_workspace_bytes(cfg, B, n, 300)), dtype=torch.uint8, device="cuda")
    norm = A.Norm(z=z, act=A.ACT_SILU)

    def chain(between=lambda: None):
        pool.fill_(0.5); between()
        A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, cu_seqlens=cu, max_len=300, norm=norm, workspace=work)
        between()
        for _ in range(2):
            A.stepq_linattn_decode_step(cfg, 0, pool, slots, q[:B], k[:B], y[:B], gate[:B], yd); between()
            A.stepq_group_norm(yd.flatten(1), hv, yd.flatten(1), A.Norm(act=A.ACT_SILU)); between()

    chain(torch.cuda.synchronize)
    want = [t.clone() for t in (pool, y, yd)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (pool, y, yd)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(3):
        for t in (pool, y, yd):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (pool, y, yd)))


def test_device_errors():
    """Slots and bounds out of range are skipped and reported; the others are served."""
    g = torch.Generator(device="cuda").manual_seed(9)
    hk, hv = 1, 2
    q, k, v, z, gate = inputs(g, 90, hk, hv, torch.bfloat16)
    cfg = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def prefill(slots, cu):
        pool, y = torch.ones((3, 1, hv, D, D), device="cuda"), torch.zeros((90, hv, D), dtype=torch.bfloat16, device="cuda")
        A.stepq_linattn_prefill(cfg, 0, pool, i32(*slots), q, k, v, gate, y, cu_seqlens=i32(*cu), max_len=90)
        return pool, y, A.stepq_device_error()

    want, wy, err = prefill((0, 1, 2), (0, 30, 60, 90))
    assert err == 0
    for bad in (3, -1):
        pool, y, err = prefill((0, bad, 2), (0, 30, 60, 90))
        assert err == 2 and torch.equal(pool[[0, 2]], want[[0, 2]]) and bool((pool[1] == 1).all())
        assert torch.equal(y[:30], wy[:30]) and bool((y[30:60] == 0).all()) and torch.equal(y[60:], wy[60:])
    for cu in ((0, 30, 20, 90), (-1, 30, 60, 90), (0, 30, 60, 91), (0, 2 ** 31 - 1, 60, 90)):
        pool, y, err = prefill((0, 1, 2), cu)
        assert err == 1
    pool = torch.ones((3, 1, hv, D, D), device="cuda")
    y = torch.zeros((3, hv, D), dtype=torch.bfloat16, device="cuda")
    for slots, code in (((0, 5, 1), 2), ((2, 0, 2), 3)):
        A.stepq_linattn_decode_step(cfg, 0, pool, i32(*slots), q[:3], k[:3], v[:3], gate[:3], y)
        assert A.stepq_device_error() == code


@pytest.mark.parametrize("norm", [False, True])
def test_a_stalled_prompt_reports_a_timeout(norm):
    """Copies that never start: every wait gives up within its bound, the launch ends and
    reports it, and the next one is whole."""
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v, z, gate = inputs(g, 4 * 200, 1, 2, torch.bfloat16)
    cfg, slots = A.Config(n_layers=1, n_key_heads=1, n_value_heads=2), torch.arange(4, dtype=torch.int32, device="cuda")

    def call():
        pool, y = torch.ones((4, 1, 2, D, D), device="cuda"), torch.zeros((800, 2, D), dtype=torch.bfloat16, device="cuda")
        A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, max_len=200, norm=A.Norm(z=z) if norm else None)
        return pool, y, A.stepq_device_error()

    want = call()
    assert want[2] == 0
    try:
        A.stepq_debug_stall(2_000_000, 3)
        assert call()[2] == 8
    finally:
        A.stepq_debug_stall()
    got = call()
    assert got[2] == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("T", [5, 40, 1500])
def test_rows_given_once_for_all_tokens(T, dt):
    """q and k of one row, broadcast over the tokens by a stride of zero."""
    hk, hv = 1, 2
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k, v, z, gate = inputs(g, T, hk, hv, dt)
    q, k = q[:1].expand(T, hk, D), k[:1].expand(T, hk, D)
    cfg = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv)
    pool, y = torch.randn((1, 1, hv, D, D), generator=g, device="cuda"), torch.empty((T, hv, D), dtype=dt, device="cuda")
    S = pool[0, 0].double()
    A.stepq_linattn_prefill(cfg, 0, pool, torch.zeros(1, dtype=torch.int32, device="cuda"), q, k, v, gate, y, max_len=T)
    yr, ya, Sa = R.linattn(S, q, k, v, gate)
    check_y(y, yr, ya, dt, None, None)
    R.assert_within(pool[0, 0], S, 64 * R.U * Sa + 1e-37, "state")


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("hk,hv,tokens", [(1, 2, 4096), (16, 32, 1000)])
def test_split_sequences_that_share_rows_are_refused(hk, hv, tokens, dt):
    """Bounds that go back and forth make three sequences of all the rows. Their segments would be
    more than the workspace has room for: the call is reported and writes nothing, and the next
    one with the same workspace is whole."""
    g = torch.Generator(device="cuda").manual_seed(hv)
    q, k, v, z, gate = inputs(g, tokens, hk, hv, dt)
    cfg, B = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv), 5
    need = A.stepq_linattn_workspace_bytes(cfg, B, tokens, tokens)
    assert need > A.stepq_linattn_workspace_bytes(cfg, B, tokens, 256)      # split
    work = torch.full((need + (1 << 24),), 0x5A, dtype=torch.uint8, device="cuda")
    slots = torch.arange(B, dtype=torch.int32, device="cuda")

    def call(*cu):
        pool, y = torch.ones((B, 1, hv, D, D), device="cuda"), torch.full((tokens, hv, D), 7.0, dtype=dt, device="cuda")
        A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, max_len=tokens, workspace=work[:need],
                                cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        return pool, y, A.stepq_device_error()

    pool, y, err = call(0, tokens, 0, tokens, 0, tokens)
    assert err == 1 and bool((pool == 1).all()) and bool((y == 7.0).all()) and bool((work[need:] == 0x5A).all())
    pool, y, err = call(0, 0, tokens - 7, tokens, tokens, tokens)
    assert err == 0 and bool((pool[[0, 3, 4]] == 1).all()) and bool((work[need:] == 0x5A).all())
    S = torch.ones((hv, D, D), dtype=torch.float64, device="cuda")
    r = slice(0, tokens - 7)
    yr, ya, Sa = R.linattn(S, q[r], k[r], v[r], gate[r])
    check_y(y[r], yr, ya, dt, None, r)
    R.assert_within(pool[1, 0], S, 64 * R.U * Sa + 1e-37, "state")


def test_a_workspace_belongs_to_the_stream_of_its_call(monkeypatch):
    """Blocks of another stream may still be in use there: what a call on a given stream takes from
    torch is a block of that stream."""
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v, z, gate = inputs(g, 1500, 1, 2, torch.bfloat16)
    cfg, slots = A.Config(n_layers=1, n_key_heads=1, n_value_heads=2), torch.zeros(1, dtype=torch.int32, device="cuda")
    pool, y = torch.ones((1, 1, 2, D, D), device="cuda"), torch.empty((1500, 2, D), dtype=torch.bfloat16, device="cuda")
    side, seen, empty = torch.cuda.Stream(), [], torch.empty
    torch.cuda.synchronize()

    def watched(*a, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **kw)

    monkeypatch.setattr(torch, "empty", watched)
    for stream in (side, None, side):
        A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, max_len=1500, stream=stream)
        torch.cuda.synchronize()
    here = torch.cuda.current_stream().cuda_stream
    assert seen == [side.cuda_stream, here, side.cuda_stream]


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
def test_unrelated_prompts_on_two_streams(dt):
    """Split prompts on the current and on a given stream, nothing ordering them and each with a
    workspace of its own from torch, give the bytes of the calls made one by one."""
    T, n, hk, hv = 3000, 4, 2, 4
    g = torch.Generator(device="cuda").manual_seed(12)
    cfg, slots = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv), torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = [inputs(g, T - 100 * i, hk, hv, dt) for i in range(n)]
    pools = [torch.empty((1, 1, hv, D, D), device="cuda") for _ in calls]
    ys = [torch.empty((T - 100 * i, hv, D), dtype=dt, device="cuda") for i in range(n)]
    side = torch.cuda.Stream()

    def serve(i, stream):
        q, k, v, z, gate = calls[i]
        A.stepq_linattn_prefill(cfg, 0, pools[i], slots, q, k, v, gate, ys[i], max_len=T - 100 * i, stream=stream)

    def round_(between, streams):
        for p in pools:
            p.fill_(0.5)
        torch.cuda.synchronize()
        for i in range(n):
            serve(i, streams[i % 2])
            between()
        torch.cuda.synchronize()
        return [t.clone() for t in pools + ys]

    want = round_(torch.cuda.synchronize, (None, None))
    for _ in range(5):
        got = round_(lambda: None, (None, side))
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("lens", [[1] * 30 + [1500] + [3] * 20 + [1000, 0, 17], [700, 699, 1, 641, 640, 639]], ids=["one beside many", "close"])
def test_split_sequences_beside_others(lens, dt):
    """Sequences that are split, some just, between sequences of a few tokens."""
    run_prefill(lens, 1, 2, dt, seed=len(lens), resume=lambda b: b % 3 > 0, layers=2)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("lens,max_len", [([5, 3, 7], 7), ([40, 30, 50], 50), ([70, 700, 90], 700), ([9] * 2500, 9), ([65] * 2500, 65)],
                         ids=["few", "blocks", "split", "many few", "many"])
def test_slots_given_twice(lens, max_len, dt):
    """Two sequences with one slot are reported, wherever they stand; one without tokens shares a slot
    with nobody."""
    B, n = len(lens), sum(lens)
    g = torch.Generator(device="cuda").manual_seed(B)
    q, k, v, z, gate = inputs(g, n, 1, 1, dt)
    cfg, pool = A.Config(n_layers=1, n_key_heads=1, n_value_heads=1), torch.zeros((B, 1, 1, D, D), device="cuda")
    y = torch.empty((n, 1, D), dtype=dt, device="cuda")
    ends = torch.tensor(lens).cumsum(0)

    def call(twice=None, empty=False):
        slots, cu = torch.randperm(B, generator=g, device="cuda").to(torch.int32), torch.cat([torch.zeros(1, dtype=torch.int64), ends])
        if twice:
            slots[twice[1]] = slots[twice[0]]
        if empty:                                                # its rows go to the one after it
            cu[twice[0] + 1] = cu[twice[0]]
        A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, gate, y, cu_seqlens=cu.to("cuda", torch.int32), max_len=max_len)
        return A.stepq_device_error()

    assert call() == 0
    for twice in ((0, B - 1), (0, 1), (B - 2, B - 1), (B // 2, B - 1)):
        assert call(twice) == 3
    assert call((0, 2), empty=True) == 0


# ------------------------------------------------------------------ split sequences: streams, graphs, errors
def split_batch(lens, hk, hv, dt, norm, seed):
    """Inputs of a packed batch on a layer with few heads, whose long sequences are split."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, B = sum(lens), len(lens)
    q, k, v, z, gate = inputs(g, n, hk, hv, dt)
    cfg = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv)
    need = A.stepq_linattn_workspace_bytes(cfg, B, n, max(lens))
    assert need > A.stepq_linattn_workspace_bytes(cfg, B, n, 64)          # room for states: split
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    cu = torch.tensor([sum(lens[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    slots = torch.randperm(B, generator=g, device="cuda").to(torch.int32)
    pool, y = torch.empty((B, 1, hv, D, D), device="cuda"), torch.empty((n, hv, D), dtype=dt, device="cuda")
    lib_norm = A.Norm(z=z, act=A.ACT_SILU) if norm else None

    def call(**kw):
        args = dict(slots=slots, cu_seqlens=cu, max_len=max(lens), norm=lib_norm, workspace=work)
        args.update(kw)
        A.stepq_linattn_prefill(cfg, 0, pool, args.pop("slots"), q, k, v, gate, y, **args)
    return call, pool, y, cu, slots


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("norm", [False, True])
def test_split_prompts_on_side_streams_and_in_graphs(norm, dt):
    """The plan, both passes and the scan between them, captured and replayed, and in calls in a row
    through one workspace: the bytes of a call by itself."""
    call, pool, y, _, _ = split_batch([2049, 40, 900], 2, 4, dt, norm, 5)

    def chain():
        pool.fill_(0.5)
        call()
        call()

    chain()
    torch.cuda.synchronize()
    want = pool.clone(), y.clone()
    pool.fill_(0.5)
    for _ in range(2):                                       # the same, each call by itself
        torch.cuda.synchronize()
        call()
    torch.cuda.synchronize()
    assert torch.equal(want[0], pool) and torch.equal(want[1], y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pool.zero_(), y.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    side.synchronize()
    assert torch.equal(want[0], pool) and torch.equal(want[1], y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(3):
        pool.zero_(), y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0], pool) and torch.equal(want[1], y)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
def test_device_errors_between_split_sequences(dt):
    """Slots and bounds out of range beside sequences that are split: skipped and reported, the others
    served."""
    lens = [1500, 700, 1000, 40]
    call, pool, y, cu, slots = split_batch(lens, 1, 2, dt, False, 6)
    pool.fill_(1.0), y.fill_(7.0)
    call()
    want, wy = pool.clone(), y.clone()
    assert A.stepq_device_error() == 0
    at = cu.tolist()
    for b, value in ((0, -1), (1, len(lens)), (2, 10 ** 6), (3, -5)):
        bad = slots.clone()
        bad[b] = value
        pool.fill_(1.0), y.fill_(7.0)
        call(slots=bad)
        assert A.stepq_device_error() == 2
        for c in range(len(lens)):
            s, rows_ = int(slots[c]), slice(at[c], at[c + 1])
            if c == b:
                assert bool((pool[s] == 1.0).all()) and bool((y[rows_] == 7.0).all())
            else:
                assert torch.equal(pool[s], want[s]) and torch.equal(y[rows_], wy[rows_])
    for edge, value in ((0, -1), (4, at[4] + 1), (4, at[3] - 1)):             # the first's, the last's
        bad = cu.clone()
        bad[edge] = value
        pool.fill_(1.0), y.fill_(7.0)
        call(cu_seqlens=bad)
        assert A.stepq_device_error() == 1
        for c in range(len(lens)):
            s, rows_ = int(slots[c]), slice(at[c], at[c + 1])
            if c == min(edge, 3):
                assert bool((pool[s] == 1.0).all()) and bool((y[rows_] == 7.0).all())
            else:
                assert torch.equal(pool[s], want[s]) and torch.equal(y[rows_], wy[rows_])


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("item", [0, 3, 8, 13])
def test_a_stalled_split_prompt_reports_a_timeout(item, norm):
    """Copies that never start in the pass for the segments' parts, or in the one for the outputs: every
    wait gives up within its bound, both passes end, and the next call is whole."""
    call, pool, y, _, _ = split_batch([1500, 40, 900], 1, 2, torch.bfloat16, norm, 7)
    pool.fill_(0.5)
    call()
    assert A.stepq_device_error() == 0
    want = pool.clone(), y.clone()
    try:
        A.stepq_debug_stall(2_000_000, item)
        pool.fill_(0.5)
        call()
        assert A.stepq_device_error() == 8
    finally:
        A.stepq_debug_stall()
    pool.fill_(0.5)
    call()
    assert A.stepq_device_error() == 0 and torch.equal(want[0], pool) and torch.equal(want[1], y)


def test_a_wait_bound_beyond_the_clock_still_holds():
    """A bound above what the kernel's 32-bit clock counts is cut to what it can see: the stalled call
    ends after about a second."""
    call, pool, y, _, _ = split_batch([1500, 40, 900], 1, 2, torch.bfloat16, False, 8)
    pool.fill_(0.5)
    call()
    assert A.stepq_device_error() == 0
    want = pool.clone(), y.clone()
    try:
        A.stepq_debug_stall(5_000_000_000, 3)
        pool.fill_(0.5)
        call()
        assert A.stepq_device_error() == 8
    finally:
        A.stepq_debug_stall()
    pool.fill_(0.5)
    call()
    assert A.stepq_device_error() == 0 and torch.equal(want[0], pool) and torch.equal(want[1], y)


# ------------------------------------------------------------------ readouts that cancel
# 1 + r for two r's of which a rest of 8 bits after a truncated head loses 2^-16, with either sign;
# head and rest rounded to nearest hold both exactly, and any value to 2^-17.
UP, DOWN = 1 + 2.0 ** -7 - 2.0 ** -16, 1 + 2.0 ** -7 - 3 * 2.0 ** -16


def check_cancelled(y, terms, dt):
    """y against the sum of `terms` over the last axis: 2^-17 of each term's value, 64 u for the
    sums, and half a unit."""
    want, size = terms.sum(-1), terms.abs().sum(-1)
    R.assert_within(y, want, R.rounded((2.0 ** -17 + 64 * R.U) * size, want, dt), "y")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("T", [9, 70])
def test_readouts_of_a_state_that_cancel(T, dt):
    """Half of a state's rows against the other half."""
    cfg, slots = A.Config(n_layers=1, n_key_heads=1, n_value_heads=1), torch.zeros(1, dtype=torch.int32, device="cuda")
    sign = torch.ones(D, device="cuda")
    sign[1::2] = -1
    pool = torch.where(sign > 0, UP, DOWN).float()[:, None].expand(D, D).contiguous().view(1, 1, 1, D, D)
    q, zero = sign.to(dt).expand(T, 1, D).contiguous(), torch.zeros((T, 1, D), dtype=dt, device="cuda")
    y, gate = torch.empty((T, 1, D), dtype=dt, device="cuda"), torch.ones((T, 1), device="cuda")
    A.stepq_linattn_prefill(cfg, 0, pool, slots, q, zero, zero, gate, y, max_len=T)
    check_cancelled(y, (pool[0, 0, 0].double() * sign[:, None]).t().expand(T, 1, D, D), dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("T", [8, 64])
def test_readouts_of_scores_that_cancel(T, dt):
    """Half of a prompt's tokens against the other half."""
    cfg, slots = A.Config(n_layers=1, n_key_heads=1, n_value_heads=1), torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((T, 1, D), dtype=dt, device="cuda") for _ in range(3))
    q[..., :3], k[..., 0], k[..., 1] = 1, 1, 2.0 ** -7
    k[::2, :, 2], k[1::2, :, 2] = -2.0 ** -16, -3 * 2.0 ** -16
    v[::2], v[1::2] = 1, -1
    pool, y = torch.zeros((1, 1, 1, D, D), device="cuda"), torch.empty((T, 1, D), dtype=dt, device="cuda")
    A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, torch.ones((T, 1), device="cuda"), y, max_len=T)
    scores = (q[:, 0].double() @ k[:, 0].double().t()).tril()
    check_cancelled(y, scores[:, None, None, :] * v[:, 0].double().t()[None, None], dt)


# fp16 factors of two terms each, 1 and 2^-8: products of the small ones are 2^-16 of the whole.
TWO, ABOVE, BELOW = 1 + 2.0 ** -8, 1 + 2.0 ** -8 - 2.0 ** -16, 1 + 2.0 ** -8 + 2.0 ** -16


@pytest.mark.parametrize("T", [9, 70])
def test_readouts_of_two_terms_and_a_state_that_cancel(T):
    cfg, slots = A.Config(n_layers=1, n_key_heads=1, n_value_heads=1), torch.zeros(1, dtype=torch.int32, device="cuda")
    sign = torch.ones(D, device="cuda")
    sign[1::2] = -1
    pool = torch.where(sign > 0, ABOVE, BELOW).float()[:, None].expand(D, D).contiguous().view(1, 1, 1, D, D)
    q, zero = (sign * TWO).half().expand(T, 1, D).contiguous(), torch.zeros((T, 1, D), dtype=torch.float16, device="cuda")
    y = torch.empty_like(q)
    A.stepq_linattn_prefill(cfg, 0, pool, slots, q, zero, zero, torch.ones((T, 1), device="cuda"), y, max_len=T)
    check_cancelled(y, (pool[0, 0, 0].double() * q[0, 0].double()[:, None]).t().expand(T, 1, D, D), torch.float16)


@pytest.mark.parametrize("T", [8, 64])
@pytest.mark.parametrize("of", ["scores", "values"])
def test_readouts_of_two_terms_and_scores_that_cancel(of, T):
    """Scores of two terms by two, or values of two terms weighed by such scores."""
    cfg, slots = A.Config(n_layers=1, n_key_heads=1, n_value_heads=1), torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((T, 1, D), dtype=torch.float16, device="cuda") for _ in range(3))
    if of == "scores":
        q[:], k[::2], k[1::2] = TWO, TWO, TWO + 2.0 ** -10
        v[::2], v[1::2] = 1, -1
    else:
        q[..., :3], k[..., 0], k[..., 1] = 1, 1, 2.0 ** -8
        k[::2, :, 2], k[1::2, :, 2] = -2.0 ** -16, 2.0 ** -16
        v[::2], v[1::2] = TWO, -TWO
    pool, y = torch.zeros((1, 1, 1, D, D), device="cuda"), torch.empty((T, 1, D), dtype=torch.float16, device="cuda")
    A.stepq_linattn_prefill(cfg, 0, pool, slots, q, k, v, torch.ones((T, 1), device="cuda"), y, max_len=T)
    scores = (q[:, 0].double() @ k[:, 0].double().t()).tril()
    check_cancelled(y, scores[:, None, None, :] * v[:, 0].double().t()[None, None], torch.float16)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("T", [9, 150])
def test_the_largest_finite_values_stay_where_they_are_kept_out(T, dt):
    """The type's largest and lowest values in tokens whose key is zero, and fp32's in rows of the state
    that no query reads and no key writes: they add nothing, neither NaN."""
    hk, hv = 1, 2
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k, v, z, gate = inputs(g, T, hk, hv, dt)
    f, lim = torch.finfo(torch.float32), torch.finfo(dt)
    k[[3, T - 1]] = 0
    v[3], v[T - 1] = lim.min, lim.max
    q[:, :, [7, 90]] = 0
    k[:, :, [7, 90]] = 0
    pool = torch.randn((1, 1, hv, D, D), generator=g, device="cuda")
    pool[..., 7, :], pool[..., 90, :] = f.max, f.min
    S = pool[0, 0].double()
    y = torch.empty((T, hv, D), dtype=dt, device="cuda")
    cfg = A.Config(n_layers=1, n_key_heads=hk, n_value_heads=hv)
    A.stepq_linattn_prefill(cfg, 0, pool, torch.zeros(1, dtype=torch.int32, device="cuda"), q, k, v, gate, y, max_len=T)
    yr, ya, Sa = R.linattn(S, q, k, v, gate)
    check_y(y, yr, ya, dt, None, None)
    R.assert_within(pool[0, 0], S, 64 * R.U * Sa + 1e-37, "state")
