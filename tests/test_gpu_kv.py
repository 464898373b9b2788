"""The paged key-value cache against its 64-bit forms: pages byte for byte, rows read back bit
for bit, and one token's attention within the bounds that kv_ref derives."""
import math

import pytest

from paper_2609_38169_gb300 import api as A

import kv_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = [torch.float32, torch.bfloat16, torch.float16]
FORMATS = [A.KV_BF16, A.KV_F16, A.KV_INT8, A.KV_INT4]
type_ids = lambda t: str(t).split(".")[1] if isinstance(t, torch.dtype) else None  # noqa: E731
fmt_ids = ["bf16", "f16", "int8", "int4"]


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert A.stepq_device_error() == 0


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def tables(g, kv, most, spare=3):
    """A page table for sequences of up to most[b] tokens, pages in random order, and their number;
    entries that hold nothing are out of range."""
    need = [-(-n // kv.page_tokens) for n in most]
    ids = torch.randperm(sum(need) + spare, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(most), max(max(need), 1) + 1), -7, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, len(ids)


def normal_pages(g, kv, n):
    """Pages of normal keys and values."""
    pages = A.alloc_pages(kv, n)
    k, v, sk, sv = R.split(pages, kv)
    for rows, s in ((k, sk), (v, sv)):
        code, scale = R.encode(torch.randn((*rows.shape[:-1], kv.head_dim), generator=g, device="cuda"), kv.format)
        rows.copy_(code)
        if s is not None:
            s.copy_(scale)
    return pages


# ------------------------------------------------------------------ rows in and out
@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
@pytest.mark.parametrize("D,heads,pt", [(64, 3, 8), (128, 8, 16), (256, 1, 64), (128, 1, 256), (64, 17, 32)])
def test_append_and_read(D, heads, pt, fmt, dt):
    """Ragged sequences, some without tokens, that start inside a page, one of two layers, k and v
    columns of one projection; the rest of the pages stays as it was."""
    g = gen(D + heads)
    kv = A.KvConfig(2, heads, D, pt, fmt)
    lens, starts = [5, 0, 1, pt, 2 * pt + 3, 0, 77], [0, 3, pt - 1, 1, pt // 2, 0, 130]
    table, n = tables(g, kv, [a + m for a, m in zip(starts, lens)])
    pages = torch.randint(0, 256, (n * A.stepq_kv_page_bytes(kv),), generator=g, device="cuda", dtype=torch.uint8)
    rows = torch.randn((sum(lens) + 9, 2 * heads * D + 8), generator=g, device="cuda").to(dt)
    k, v = rows[:, :heads * D].unflatten(1, (heads, D)), rows[:, heads * D + 8:].unflatten(1, (heads, D))
    cu = i32([sum(lens[:b]) for b in range(len(lens) + 1)])
    want = pages.clone()
    R.append(want, kv, 1, table, starts, lens, k[:sum(lens)], v[:sum(lens)])
    A.stepq_kv_append(kv, 1, pages, table, i32(starts), k, v, cu_seqlens=cu)
    assert torch.equal(pages, want)
    out = torch.full((2, len(rows), heads, D), 7.0, dtype=dt, device="cuda")
    A.stepq_kv_read(kv, 1, pages, table, i32(starts), *out, cu_seqlens=cu)
    wk, wv, _ = R.read(pages, kv, 1, table, starts, lens)
    for o, w in zip(out, (wk, wv)):
        assert torch.equal(o[:sum(lens)], w.float().to(dt)) and bool((o[sum(lens):] == 7).all())


@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_rows_at_the_edges(fmt, dt):
    """Zeros, one value, the smallest and largest scales, borders between codes, infinities, NaN."""
    kv = A.KvConfig(1, 1, 128, 16, fmt)
    big = torch.finfo(dt).max
    x = torch.zeros((12, 1, 128), device="cuda")
    x[1] = 3.0
    x[2, 0, 5] = -1e-6
    x[3] = torch.arange(-64, 64, device="cuda") * 2.0 ** -14
    x[4] = torch.arange(-64, 64, device="cuda") * 0.5 + 0.25
    x[4, 0, 0] = 127.0                                      # scale 1: borders at every half
    x[5] = torch.randn(128, device="cuda") * min(big, 1e30) / 8
    x[6, 0, ::2], x[6, 0, 1::2] = big, -big
    x[7, 0, 3], x[7, 0, 9] = math.inf, 5.0
    x[8, 0, 3], x[8, 0, 9] = math.nan, 5.0
    x[9, 0, :], x[9, 0, 0] = -math.inf, math.nan
    x[10] = torch.arange(-64, 64, device="cuda") * 0.25
    x[10, 0, 0] = 7.0                                       # scale 1 in 4 bits
    x[11] = math.nan
    x = x.to(dt)
    table, starts, lens = i32([[2]]), [1], [12]
    pages = torch.zeros(3 * A.stepq_kv_page_bytes(kv), dtype=torch.uint8, device="cuda")
    want = pages.clone()
    R.append(want, kv, 0, table, starts, lens, x, -x)
    A.stepq_kv_append(kv, 0, pages, table, i32(starts), x, -x)
    out = torch.zeros((2, 12, 1, 128), dtype=dt, device="cuda")
    A.stepq_kv_read(kv, 0, pages, table, i32(starts), *out)
    if R.BITS[fmt] == 16:                                   # NaN's bits are open
        y = x.float().to(R.TYPE[fmt]).float().to(dt)
        assert torch.equal(out[0].nan_to_num(1.25), y.nan_to_num(1.25)) and torch.equal(out[0].isnan(), y.isnan())
        return
    assert torch.equal(pages, want)
    wk, wv, _ = R.read(pages, kv, 0, table, starts, lens)
    assert torch.equal(out[0], wk.float().to(dt)) and torch.equal(out[1], wv.float().to(dt))


@pytest.mark.parametrize("fmt", [A.KV_INT8, A.KV_INT4], ids=["int8", "int4"])
@pytest.mark.parametrize("exponent", [-13, -3, 0, 9])
def test_borders_between_codes(fmt, exponent):
    """fp32 values on the border of two codes, and next to it on both sides, for every scale of 11 bits."""
    kv, q = A.KvConfig(1, 1, 128, 64, fmt), 127 if fmt == A.KV_INT8 else 7
    g = gen(20)
    s = (1 + torch.arange(1024, device="cuda").double() / 1024) * 2.0 ** exponent
    k = torch.randint(-q, q, (1024, 128), generator=g, device="cuda").double() + 0.5
    x = (k * s[:, None]).float()
    x = torch.where(torch.arange(128, device="cuda") % 3 == 1, x.nextafter(torch.tensor(1e30, device="cuda")), x)
    x = torch.where(torch.arange(128, device="cuda") % 3 == 2, x.nextafter(torch.tensor(-1e30, device="cuda")), x)
    x[:, 0] = (q * s).float()                               # the row's largest: its scale is s
    table = torch.arange(16, device="cuda", dtype=torch.int32)[None]
    pages = torch.zeros(16 * A.stepq_kv_page_bytes(kv), dtype=torch.uint8, device="cuda")
    want = pages.clone()
    x = x[:, None]
    R.append(want, kv, 0, table, [0], [1024], x, -x)
    A.stepq_kv_append(kv, 0, pages, table, i32([0]), x, -x)
    assert torch.equal(pages, want)
    assert torch.equal(R.split(pages, kv)[2].reshape(-1).double(), s)


@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_equal_lengths_and_many_sequences(fmt):
    """No cu_seqlens: one token each of 1,500 sequences, then three each; 1,500 ragged ones."""
    g, kv = gen(1), A.KvConfig(1, 2, 64, 8, fmt)
    B = 1500
    starts = torch.randint(0, 60, (B,), generator=g, device="cuda").tolist()
    table, n = tables(g, kv, [a + 9 for a in starts])
    pages = normal_pages(g, kv, n)
    ragged = torch.randint(0, 9, (B,), generator=g, device="cuda").tolist()
    for lens in ([1] * B, [3] * B, ragged):
        cu = None if lens is not ragged else i32([0] + torch.tensor(lens).cumsum(0).tolist())
        k, v = torch.randn((2, sum(lens), 2, 64), generator=g, device="cuda").bfloat16()
        want = pages.clone()
        R.append(want, kv, 0, table, starts, lens, k, v)
        A.stepq_kv_append(kv, 0, pages, table, i32(starts), k, v, cu_seqlens=cu)
        assert torch.equal(pages, want)


@pytest.mark.parametrize("fmt,dt", [(A.KV_BF16, torch.float32), (A.KV_INT8, torch.float16), (A.KV_INT4, torch.bfloat16)],
                         ids=["bf16", "int8", "int4"])
@pytest.mark.parametrize("D,heads", [(64, 1), (64, 2), (128, 1)])
def test_long_prompts_of_few_heads(D, heads, fmt, dt):
    """More than 8,192 tokens, several a warp: odd lengths, empty sequences in a row, bad places among them."""
    g, kv = gen(4), A.KvConfig(1, heads, D, 8, fmt)
    lens = [3001, 0, 0, 1, 2, 0, 4997, 3, 0, 700, 1, 1, 1, 513]
    starts = torch.randint(0, 30, (len(lens),), generator=g, device="cuda").tolist()
    table, n = tables(g, kv, [a + m for a, m in zip(starts, lens)])
    pages = normal_pages(g, kv, n)
    k, v = torch.randn((2, sum(lens) + 5, heads, D), generator=g, device="cuda").to(dt)
    cu = i32([sum(lens[:b]) for b in range(len(lens) + 1)])
    want = pages.clone()
    R.append(want, kv, 0, table, starts, lens, k[:sum(lens)], v[:sum(lens)])
    A.stepq_kv_append(kv, 0, pages, table, i32(starts), k, v, cu_seqlens=cu)
    assert torch.equal(pages, want)
    out = torch.full((2, len(k), heads, D), 7.0, dtype=dt, device="cuda")
    A.stepq_kv_read(kv, 0, pages, table, i32(starts), *out, cu_seqlens=cu)
    wk, wv, _ = R.read(pages, kv, 0, table, starts, lens)
    for o, w in zip(out, (wk, wv)):
        assert torch.equal(o[:sum(lens)], w.float().to(dt)) and bool((o[sum(lens):] == 7).all())
    # a page out of range, a negative start: their tokens are skipped
    t, s = table.clone(), list(starts)
    t[6, 100], s[9] = n, -5
    got = torch.full_like(out, 7.0)
    A.stepq_kv_read(kv, 0, pages, t, i32(s), *got, cu_seqlens=cu)
    assert A.stepq_device_error() == 2
    skip = torch.zeros(len(k), dtype=torch.bool, device="cuda")
    first = sum(lens[:6]) + 800 - starts[6]
    skip[first:first + 8] = True
    skip[sum(lens[:9]):sum(lens[:10])] = True
    assert torch.equal(got[:, ~skip], out[:, ~skip]) and bool((got[:, skip] == 7).all())
    # equal lengths
    A.stepq_kv_read(kv, 0, pages, table[6:7], i32([2]), *out[:, :4990].unbind(0))
    A.stepq_kv_read(kv, 0, pages, table[[0, 6, 6]], i32([0, 0, 3]), *(x := torch.empty((2, 9000, heads, D), dtype=dt, device="cuda")))
    wk, wv, _ = R.read(pages, kv, 0, table[[0, 6, 6]], [0, 0, 3], [3000] * 3)
    assert torch.equal(x[0], wk.float().to(dt)) and torch.equal(x[1], wv.float().to(dt))


@pytest.mark.parametrize("fmt", [A.KV_BF16, A.KV_INT4], ids=["bf16", "int4"])
def test_bad_places_are_reported_and_skipped(fmt):
    g, kv = gen(2), A.KvConfig(1, 2, 64, 16, fmt)
    pages = normal_pages(g, kv, 4)
    k, v = torch.randn((2, 6, 2, 64), generator=g, device="cuda").bfloat16()
    good = i32([[0, 1], [2, 3], [1, 1]])

    def both(table, starts, skip, code, cu=None):
        want, p = pages.clone(), pages.clone()
        keep = [b for b in range(3) if b not in skip]
        R.append(want, kv, 0, good[keep], [starts[b] for b in keep], [2] * len(keep),
                 torch.cat([k[2 * b:2 * b + 2] for b in keep]), torch.cat([v[2 * b:2 * b + 2] for b in keep]))
        A.stepq_kv_append(kv, 0, p, table, i32(starts), k, v, cu_seqlens=cu)
        assert torch.equal(p, want) and A.stepq_device_error() == code
        out = torch.full((2, 6, 2, 64), 7.0, device="cuda")
        A.stepq_kv_read(kv, 0, p, table, i32(starts), *out, cu_seqlens=cu)
        assert A.stepq_device_error() == code
        for b in range(3):
            assert bool((out[:, 2 * b:2 * b + 2] == 7).all()) == (b in skip)

    both(good, [0, 5, -1], [2], 2)
    both(good, [3, 32, 7], [1], 2)
    both(i32([[0, 1], [4, 3], [1, 1]]), [3, 5, 20], [1], 2)
    both(i32([[-1, 1], [2, 3], [1, 1]]), [3, 5, 20], [0], 2)
    both(good, [2147483647, 5, 20], [0], 2)
    # rows 2 and 3 between the bounds' ends, and in no sequence
    p, out = pages.clone(), torch.full((2, 6, 2, 64), 7.0, device="cuda")
    A.stepq_kv_read(kv, 0, p, good, i32([0, 0, 0]), *out, cu_seqlens=i32([0, 6, 2, 6]))
    assert A.stepq_device_error() in (0, 1)


def test_rows_outside_the_bounds_stay():
    g, kv = gen(3), A.KvConfig(1, 1, 128, 16, A.KV_INT8)
    pages = normal_pages(g, kv, 2)
    out = torch.full((2, 20, 1, 128), 7.0, device="cuda")
    A.stepq_kv_read(kv, 0, pages, i32([[1]]), i32([2]), *out, cu_seqlens=i32([4, 9]))
    wk, wv, _ = R.read(pages, kv, 0, i32([[1]]), [2], [5])
    assert torch.equal(out[0][4:9], wk.float()) and torch.equal(out[1][4:9], wv.float())
    assert bool((out[:, :4] == 7).all()) and bool((out[:, 9:] == 7).all())


# ------------------------------------------------------------------ attention
def check(kv, pages, table, lens, q, layer=0, scale=None, window=0, max_len=None, want=None, **kw):
    y = torch.full_like(q, 9.0)
    lse = torch.full(q.shape[:2], 9.0, device="cuda")
    A.stepq_kv_attend(kv, layer, pages, table, i32(lens), q, y, scale=scale, window=window, lse=lse,
                      max_len=max(lens) if max_len is None else max_len, **kw)
    wy, wl, tol, ltol = R.attend(pages, kv, layer, table, lens, q, kv.head_dim ** -0.5 if scale is None else scale, window)
    R.assert_within(lse, wl, ltol, "lse")
    R.assert_within(y, wy, R.rounded(tol, wy, q.dtype), "y")
    return y


LENS = [1, 2, 7, 8, 9, 15, 16, 17, 0, 31, 33, 63, 64, 65, 127, 128, 129, 300, 513, 1000]


@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
@pytest.mark.parametrize("D,heads,G,pt", [(64, 2, 1, 8), (64, 1, 16, 32), (128, 2, 4, 16), (128, 1, 8, 64), (128, 1, 12, 8),
                                          (128, 1, 33, 128), (256, 2, 8, 16), (256, 1, 9, 256)])
def test_lengths(D, heads, G, pt, fmt, dt):
    g, kv = gen(D + G), A.KvConfig(2, heads, D, pt, fmt)
    table, n = tables(g, kv, LENS)
    pages = normal_pages(g, kv, n)
    q = torch.randn((len(LENS), heads * G, D), generator=g, device="cuda").to(dt)
    check(kv, pages, table, LENS, q, layer=1)
    few = [x for x in LENS if x <= 65]                      # short ones alone: no CTA shares a sequence
    check(kv, pages, table[[LENS.index(x) for x in few]], few, q[:len(few)])


@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_one_long_sequence_fills_the_gpu(fmt, dt):
    g, kv = gen(5), A.KvConfig(1, 2, 128, 16, fmt)
    table, n = tables(g, kv, [70001])
    pages = normal_pages(g, kv, n)
    q = torch.randn((1, 8, 128), generator=g, device="cuda").to(dt)
    for length in (70001, 69999, 4097, 1):
        check(kv, pages, table, [length], q)
    check(kv, pages, table, [70001], q, max_len=0)
    check(kv, pages, table, [70001], q, max_len=5)          # a wrong hint: only slower


@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
@pytest.mark.parametrize("window", [1, 5, 16, 100, 257, 5000])
def test_windows(fmt, window):
    g, kv = gen(6), A.KvConfig(1, 2, 128, 8, fmt)
    table, n = tables(g, kv, LENS)
    q = torch.randn((len(LENS), 6, 128), generator=g, device="cuda").bfloat16()
    check(kv, normal_pages(g, kv, n), table, LENS, q, window=window)


@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
@pytest.mark.parametrize("D,heads,G,pt,dt", [(64, 4, 2, 16, torch.float16), (128, 3, 4, 8, torch.bfloat16), (128, 2, 1, 64, torch.float32),
                                             (64, 2, 9, 32, torch.bfloat16), (128, 1, 16, 16, torch.bfloat16), (256, 2, 3, 32, torch.bfloat16)],
                         ids=["64", "128", "128-f32", "64-9", "128-16", "256"])
def test_many_rows_of_mixed_lengths(D, heads, G, pt, dt, fmt):
    """More (sequence, head) pairs than CTAs, shares that hold many sequences and parts of others."""
    g, kv = gen(7), A.KvConfig(1, heads, D, pt, fmt)
    lens = (torch.rand(700, generator=g, device="cuda") ** 6 * 3000).int().tolist()
    table, n = tables(g, kv, lens)
    q = torch.randn((700, heads * G, D), generator=g, device="cuda").to(dt)
    pages = normal_pages(g, kv, n)
    check(kv, pages, table, lens, q)
    check(kv, pages, table, lens, q, window=200)


@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
@pytest.mark.parametrize("D,heads,G", [(128, 4, 16), (64, 8, 12), (256, 2, 20), (128, 5, 3)])
def test_long_rows_among_short_ones(D, heads, G, fmt, dt):
    """Two sequences of most tokens, whose parts are many, among some of two parts and of one; and both alone."""
    g, kv = gen(17), A.KvConfig(1, heads, D, 32, fmt)
    lens = [20011 // heads, 9001 // heads] + [(7 * i) % 400 + 1 for i in range(38)]
    table, n = tables(g, kv, lens)
    pages = normal_pages(g, kv, n)
    q = torch.randn((len(lens), heads * G, D), generator=g, device="cuda").to(dt)
    check(kv, pages, table, lens, q)
    check(kv, pages, table[:2], lens[:2], q[:2])


@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_a_window_beyond_every_length(fmt):
    g, kv = gen(18), A.KvConfig(1, 2, 64, 16, fmt)
    lens = [5000, 3, 0, 700]
    table, n = tables(g, kv, lens)
    pages = normal_pages(g, kv, n)
    q = torch.randn((4, 4, 64), generator=g, device="cuda").bfloat16()
    want = check(kv, pages, table, lens, q)
    for window in (5000, 2 ** 30, 2 ** 31 - 64, 2 ** 31 - 1):
        assert torch.equal(check(kv, pages, table, lens, q, window=window), want)


@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_values_that_are_no_tokens(fmt, dt):
    """Every byte that is no token's set to all ones (NaN, or the largest code and a NaN scale),
    tokens before a window among them, and table entries behind the tokens out of range."""
    g, kv = gen(8), A.KvConfig(2, 2, 128, 16, fmt)
    lens = [1, 5, 16, 40, 100, 333, 1500, 0]
    table, n = tables(g, kv, lens)
    full = normal_pages(g, kv, n)
    q = torch.randn((len(lens), 8, 128), generator=g, device="cuda").to(dt)
    for window in (0, 21):
        pages = torch.full_like(full, 255)
        lo = [max(0, m - window) if window else 0 for m in lens]
        page, at = R.places(table, lo, [m - a for m, a in zip(lens, lo)], 16)
        for src, dst in zip(R.split(full, kv), R.split(pages, kv)):
            if src is not None:
                dst[page, 1, :, at] = src[page, 1, :, at]
        t = table.clone()
        for b, a in enumerate(lo):
            t[b, :a // 16] = 1 << 30
        y = torch.empty_like(q)
        A.stepq_kv_attend(kv, 1, pages, t, i32(lens), q, y, window=window)
        wy, _, tol, _ = R.attend(full, kv, 1, table, lens, q, 128 ** -0.5, window)
        R.assert_within(y, wy, R.rounded(tol, wy, dt), "y")


@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
@pytest.mark.parametrize("scale", [0.0, 1e-3, 3.0, -0.5])
def test_scores_flat_and_steep(scale, fmt, dt):
    g, kv = gen(9), A.KvConfig(1, 1, 64, 16, fmt)
    lens = [500, 90]
    table, n = tables(g, kv, lens)
    q = torch.randn((2, 4, 64), generator=g, device="cuda").to(dt)
    check(kv, normal_pages(g, kv, n), table, lens, q, scale=scale)


@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_scores_that_rise_along_the_sequence(fmt):
    """The largest score comes last, far above the rest: every reference is replaced late; and
    values of very different size, whose scales take the weights' range."""
    g, kv = gen(10), A.KvConfig(1, 1, 128, 16, fmt)
    n = 3000
    table, pages_n = tables(g, kv, [n])
    pages = A.alloc_pages(kv, pages_n)
    q = torch.randn((1, 8, 128), generator=g, device="cuda")
    k = q[0, :1] * torch.linspace(-3, 3, n, device="cuda")[:, None] + 0.1 * torch.randn((n, 128), generator=g, device="cuda")
    v = torch.randn((n, 128), generator=g, device="cuda") * torch.logspace(-3, 3, n, device="cuda").flip(0)[:, None]
    for dt in TYPES:
        A.stepq_kv_append(kv, 0, pages, table, i32([0]), k[:, None].to(dt), v[:, None].to(dt))
        check(kv, pages, table, [n], q.to(dt))
        A.stepq_kv_append(kv, 0, pages, table, i32([0]), k[:, None].to(dt), v.flip(0)[:, None].to(dt))
        check(kv, pages, table, [n], q.to(dt), scale=0.02)


@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_queries_of_any_size(fmt):
    """Queries from 2^-30 to 2^30 times the usual, keys the other way round (as far as fp16 goes)."""
    g, kv = gen(11), A.KvConfig(1, 1, 128, 16, fmt)
    table, n = tables(g, kv, [200, 200, 200, 200])
    pages = normal_pages(g, kv, n)
    q = torch.randn((4, 8, 128), generator=g, device="cuda")
    q[1] *= 2.0 ** -30
    q[2] *= 2.0 ** -14
    q[3, :, 1:] *= 2.0 ** -20                               # one channel far above the others
    check(kv, pages, table, [200] * 4, q, scale=1.0)
    check(kv, pages, table, [200] * 4, (q * 2.0 ** 30), scale=2.0 ** -31)
    check(kv, pages, table, [200] * 4, q.bfloat16() * 2.0 ** 30, scale=2.0 ** -31)


@pytest.mark.parametrize("fmt", [A.KV_BF16, A.KV_F16], ids=["bf16", "f16"])
def test_values_that_are_not_finite_stay_in_their_sequence_and_head(fmt):
    g, kv = gen(12), A.KvConfig(1, 2, 64, 16, fmt)
    lens = [50, 2000, 50]
    table, n = tables(g, kv, lens)
    pages = normal_pages(g, kv, n)
    q = torch.randn((3, 8, 64), generator=g, device="cuda").bfloat16()
    good = check(kv, pages, table, lens, q)
    k, v, _, _ = R.split(pages, kv)
    page, at = int(table[1, 100]), 3
    k.view(R.TYPE[fmt])[page, 0, 0, at, 5] = math.nan
    v.view(R.TYPE[fmt])[page, 0, 1, at, 7] = math.inf
    y = torch.empty_like(q)
    A.stepq_kv_attend(kv, 0, pages, table, i32(lens), q, y)
    assert torch.equal(y[[0, 2]], good[[0, 2]]) and bool(y[1, :4].isnan().all())
    ok = [i for i in range(64) if i != 7]
    assert torch.equal(y[1, 4:][:, ok], good[1, 4:][:, ok]) and not bool(y[1, 4:, 7].isfinite().any())
    # a key of minus infinity that every query meets with a positive channel: weight zero
    pages = normal_pages(gen(12), kv, n)
    k, v, _, _ = R.split(pages, kv)
    q = q.abs()
    k.view(R.TYPE[fmt])[page, 0, 0, at, 5] = -math.inf
    A.stepq_kv_attend(kv, 0, pages, table, i32(lens), q, y)
    assert bool(y.isfinite().all())


def test_nothing_to_do():
    """No sequences; sequences without tokens over a table without entries."""
    kv = A.KvConfig(1, 2, 64, 16, A.KV_INT8)
    pages, z = A.alloc_pages(kv, 2), lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    for B, W in ((0, 3), (0, 0), (3, 0), (3, 2)):
        t, n, y = torch.zeros((B, W), dtype=torch.int32, device="cuda"), i32([0] * B), z(B, 4, 64) + 5
        A.stepq_kv_attend(kv, 0, pages, t, n, z(B, 4, 64), y)
        assert not bool(y.any())
        A.stepq_kv_append(kv, 0, pages, t, n, z(0, 2, 64), z(0, 2, 64))
        A.stepq_kv_read(kv, 0, pages, t, n, z(0, 2, 64), z(0, 2, 64), cu_seqlens=i32([0] * (B + 1)))


def test_calls_stay_within_their_buffers():
    """Nothing outside pages, rows, outputs and workspace is written."""
    g, kv = gen(18), A.KvConfig(1, 2, 128, 16, A.KV_INT4)
    lens = [3000, 17, 0, 900]
    table, n = tables(g, kv, lens)
    each, guard = A.stepq_kv_page_bytes(kv), 4096

    def guarded(nbytes):
        whole = torch.full((nbytes + 2 * guard,), 0x5A, dtype=torch.uint8, device="cuda")
        return whole, whole[guard:guard + nbytes]
    held = []
    whole, pages = guarded(n * each)
    held.append((whole, n * each))
    pages.copy_(normal_pages(g, kv, n))
    q = torch.randn((4, 8, 128), generator=g, device="cuda").bfloat16()
    for max_len in (3000, 100):
        bytes_y, bytes_l, bytes_w = 4 * 8 * 128 * 2, 4 * 8 * 4, A.stepq_kv_workspace_bytes(kv, 8, 4, 3000)
        (wy, y), (wl, l), (ww, ws) = guarded(bytes_y), guarded(bytes_l), guarded(bytes_w)
        held += [(wy, bytes_y), (wl, bytes_l), (ww, bytes_w)]
        A.stepq_kv_attend(kv, 0, pages, table, i32(lens), q, y.view(torch.bfloat16).view(4, 8, 128), lse=l.view(torch.float32),
                          max_len=max_len, workspace=ws)
    bytes_k = sum(lens) * 2 * 128 * 2
    rows = [guarded(bytes_k) for _ in range(2)]
    held += [(w, bytes_k) for w, _ in rows]
    k, v = (x.view(torch.bfloat16).view(-1, 2, 128) for _, x in rows)
    cu = i32([sum(lens[:b]) for b in range(5)])
    A.stepq_kv_read(kv, 0, pages, table, i32([0] * 4), k, v, cu_seqlens=cu)
    A.stepq_kv_append(kv, 0, pages, table, i32([0] * 4), k, v, cu_seqlens=cu)
    for whole, nbytes in held:
        assert bool((whole[:guard] == 0x5A).all()) and bool((whole[guard + nbytes:] == 0x5A).all())


def test_bad_lengths_and_pages_are_reported():
    g, kv = gen(13), A.KvConfig(1, 2, 64, 16, A.KV_INT8)
    lens = [40, 40, 40]
    table, n = tables(g, kv, lens)
    pages, y = normal_pages(g, kv, n), torch.empty((3, 4, 64), device="cuda")
    q = torch.randn((3, 4, 64), generator=g, device="cuda")
    good = check(kv, pages, table, lens, q)
    A.stepq_kv_attend(kv, 0, pages, table, i32([40, -3, 40]), q, y)
    assert A.stepq_device_error() == 1 and torch.equal(y[[0, 2]], good[[0, 2]]) and not bool(y[1].any())
    t = table[:, :3].contiguous()
    A.stepq_kv_attend(kv, 0, pages, t, i32([40, 49, 40]), q, y)
    assert A.stepq_device_error() == 2
    wy, _, tol, _ = R.attend(pages, kv, 0, t, [40, 48, 40], q, 0.125)
    R.assert_within(y, wy, R.rounded(tol, wy, q.dtype), "y")
    t[1, 1] = n
    A.stepq_kv_attend(kv, 0, pages, t, i32([40, 40, 40]), q, y)
    assert A.stepq_device_error() == 2 and torch.equal(y[[0, 2]], good[[0, 2]]) and bool(y.isfinite().all())


@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_offsets_above_32_bits(fmt):
    """Pages more than 4 GB into the pool, and a stride of rows that passes 2^31 elements."""
    kv = A.KvConfig(4, 8, 256, 256, fmt)
    n = 5 * 2 ** 30 // A.stepq_kv_page_bytes(kv) + 2
    pages = torch.empty(n * A.stepq_kv_page_bytes(kv), dtype=torch.uint8, device="cuda")
    g, lens = gen(14), [600, 3]
    table = i32([[n - 1, 0, n - 2], [n - 3, -1, -1]])
    k, v = torch.randn((2, 603, 8, 256), generator=g, device="cuda").bfloat16()
    A.stepq_kv_append(kv, 3, pages, table, i32([0, 0]), k, v, cu_seqlens=i32([0, 600, 603]))
    out = torch.empty_like(k), torch.empty_like(v)
    A.stepq_kv_read(kv, 3, pages, table, i32([0, 0]), *out, cu_seqlens=i32([0, 600, 603]))
    wk, wv, _ = R.read(pages, kv, 3, table, [0, 0], lens)
    assert torch.equal(out[0], wk.float().bfloat16()) and torch.equal(out[1], wv.float().bfloat16())
    wide = torch.empty(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    q = wide.as_strided((2, 16, 256), (2 ** 31, 256, 1))
    q.copy_(torch.randn((2, 16, 256), generator=g, device="cuda"))
    check(kv, pages, table, lens, q, layer=3)


@pytest.mark.parametrize("dt", TYPES, ids=type_ids)
def test_strided_rows_and_outputs_in_place(dt):
    g, kv = gen(15), A.KvConfig(1, 2, 128, 32, A.KV_INT8)
    lens = [33, 700, 2]
    table, n = tables(g, kv, lens)
    pages = normal_pages(g, kv, n)
    wide = torch.randn((3, 4 * 128 + 256), generator=g, device="cuda").to(dt)
    q = wide[:, 128:128 + 512].unflatten(1, (4, 128))
    want = check(kv, pages, table, lens, q.contiguous())
    before = wide.clone()
    A.stepq_kv_attend(kv, 0, pages, table, i32(lens), q, q)
    assert torch.equal(q, want)
    assert torch.equal(wide[:, :128], before[:, :128]) and torch.equal(wide[:, 640:], before[:, 640:])
    # one query for every sequence, flat rows, a table that every sequence shares
    one = torch.randn((1, 512), generator=g, device="cuda").to(dt)
    y = torch.empty((3, 512), dtype=dt, device="cuda")
    A.stepq_kv_attend(kv, 0, pages, table[1:2].expand(3, -1), i32(lens), one.expand(3, -1), y)
    wy, _, tol, _ = R.attend(pages, kv, 0, table[1:2].expand(3, -1), lens, one.view(1, 4, 128).expand(3, -1, -1), 128 ** -0.5)
    R.assert_within(y.view(3, 4, 128), wy, R.rounded(tol, wy, dt), "y")


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("fmt", FORMATS, ids=fmt_ids)
def test_prompts_then_tokens(fmt):
    """As a server uses them: prompts in two chunks, then tokens one at a time in every layer, on a
    side stream, the whole step also captured once and replayed for all tokens."""
    g, kv = gen(16), A.KvConfig(3, 2, 128, 16, fmt)
    prompts, new, L, Hq = [37, 5, 90], 20, 3, 6
    most = [n + new for n in prompts]
    table, n = tables(g, kv, most)
    k, v = torch.randn((2, L, sum(most), 2, 128), generator=g, device="cuda").bfloat16()
    q = torch.randn((new, L, 3, Hq, 128), generator=g, device="cuda").bfloat16()
    first = [sum(most[:b]) for b in range(3)]
    side = torch.cuda.Stream()
    pages = A.alloc_pages(kv, n)

    def fill():
        pages.zero_()
        for at, size in ((0, 4), (4, None)):
            part = [(4 if size else m - 4) for m in prompts]
            rows = torch.cat([torch.arange(f + at, f + at + m, device="cuda") for f, m in zip(first, part)])
            cu = i32([sum(part[:b]) for b in range(4)])
            for i in range(L):
                A.stepq_kv_append(kv, i, pages, table, i32([at] * 3), k[i, rows], v[i, rows], cu_seqlens=cu)

    kt, vt, qt = torch.empty((L, 3, 2, 128), dtype=k.dtype, device="cuda"), torch.empty((L, 3, 2, 128), dtype=k.dtype, device="cuda"), \
        torch.empty_like(q[0])
    y = torch.empty_like(qt)
    lens = i32(prompts)
    ws = torch.empty(A.stepq_kv_workspace_bytes(kv, Hq, 3, 4096), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        for i in range(L):
            A.stepq_kv_append(kv, i, pages, table, lens, kt[i], vt[i], stream=stream)
            A.stepq_kv_attend(kv, i, pages, table, lens + 1, qt[i], y[i], max_len=4096, workspace=ws, stream=stream)

    def inputs(t):
        rows = torch.tensor([f + p + t for f, p in zip(first, prompts)], device="cuda")
        kt.copy_(k[:, rows])
        vt.copy_(v[:, rows])
        qt.copy_(q[t])

    fill()
    got = []
    for t in range(new):
        inputs(t)
        step()
        got.append(y.clone())
        lens += 1
    after = pages.clone()
    for t in (0, new - 1):
        for i in range(L):
            wy, _, tol, _ = R.attend(pages, kv, i, table, [p + t + 1 for p in prompts], q[t, i], 128 ** -0.5)
            R.assert_within(got[t][i], wy, R.rounded(tol, wy, q.dtype), f"layer {i}, token {t}")
    # the same on a side stream, and by replays of one captured step
    lens.copy_(i32(prompts))
    fill()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        inputs(0)
        step()
        assert torch.equal(y, got[0])
    side.synchronize()
    lens.copy_(i32(prompts))
    fill()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        lens += 1
    for t in range(new):
        inputs(t)
        graph.replay()
        assert torch.equal(y, got[t]), t
    assert torch.equal(pages, after)
    # everything read back is what was written
    out = torch.empty((2, sum(most), 2, 128), dtype=k.dtype, device="cuda")
    for i in range(L):
        A.stepq_kv_read(kv, i, pages, table, i32([0] * 3), *out, cu_seqlens=i32(first + [sum(most)]))
        for o, x in zip(out, (k[i], v[i])):
            code, s = R.encode(x, fmt)
            assert torch.equal(o, R.decode(code, s, fmt)[0].float().to(o.dtype))


def test_graphs_that_share_a_workspace_and_calls_on_two_streams():
    g, kv = gen(17), A.KvConfig(1, 4, 128, 16, A.KV_INT8)
    lens = [5000, 300]
    table, n = tables(g, kv, lens)
    pages = normal_pages(g, kv, n)
    qs = torch.randn((2, 2, 16, 128), generator=g, device="cuda").bfloat16()
    want = [check(kv, pages, table, lens, q) for q in qs]
    ws = torch.empty(A.stepq_kv_workspace_bytes(kv, 16, 2, 5000), dtype=torch.uint8, device="cuda")
    ys, graphs, ln = [torch.empty_like(q) for q in qs], [], i32(lens)
    for q, y in zip(qs, ys):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            for _ in range(3):
                A.stepq_kv_attend(kv, 0, pages, table, ln, q, y, max_len=5000, workspace=ws)
        graphs.append(gr)
    for _ in range(5):
        for gr, y in zip(graphs, ys):
            y.zero_()
            gr.replay()
    assert all(torch.equal(y, w) for y, w in zip(ys, want))
    # two streams at once, workspaces from torch on each
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, q, y in zip(streams, qs, ys):
            A.stepq_kv_attend(kv, 0, pages, table, ln, q, y, max_len=5000, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for y, w in zip(ys, want))


def test_binding_refuses_layouts():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    kv = A.KvConfig(1, 2, 128, 16)
    pages, table, n, k, q = A.alloc_pages(kv, 4), z(3, 2, dt=torch.int32), z(3, dt=torch.int32), z(3, 2, 128), z(3, 4, 128)
    append = lambda **kw: A.stepq_kv_append(**{**dict(kv=kv, layer=0, pages=pages, table=table, starts=n, k=k, v=k), **kw})  # noqa: E731
    attend = lambda **kw: A.stepq_kv_attend(**{**dict(kv=kv, layer=0, pages=pages, table=table, lens=n, q=q, y=q.clone()), **kw})  # noqa: E731
    append()
    attend()
    for call, kw, say in ((append, dict(v=k.float()), "v: expected BFloat16"), (append, dict(k=k.cpu()), "k: expected a CUDA"),
                          (append, dict(k=z(3, 2, 64)), "k: expected"), (append, dict(k=z(3, 2, 256)[:, :, ::2]), "k: expected"),
                          (append, dict(v=z(4, 2, 128)), "v: expected"), (append, dict(k=z(3, 2, 128, dt=torch.float64), v=z(3, 2, 128, dt=torch.float64)), "float32, bfloat16"),
                          (append, dict(table=table.long()), "table"), (append, dict(table=z(3, 4, dt=torch.int32)[:, ::2]), "table"),
                          (append, dict(table=z(2, 2, dt=torch.int32)), "table: expected 3"), (append, dict(starts=n.long()), "starts: expected contiguous int32"), (attend, dict(workspace=pages[::2]), "workspace"),
                          (append, dict(pages=pages[::2]), "contiguous"), (attend, dict(y=q.float()), "y: expected"),
                          (attend, dict(y=z(3, 2, 128)), "y: expected"), (attend, dict(q=z(2, 4, 128)), "q: expected"),
                          (attend, dict(lse=z(3, 4)), "float32"), (attend, dict(lse=z(3, 2, dt=torch.float32)), "lse: expected 12")):
        with pytest.raises(ValueError, match=say):
            call(**kw)
    with pytest.raises(RuntimeError, match="status 1"):
        attend(q=z(3, 3, 128), y=z(3, 3, 128))              # 3 query heads, 2 key heads
