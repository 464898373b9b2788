"""One token's attention over the paged cache at the ends of its range: what lies in places that hold no
token, the largest values and scores, scales of zero, and scores that need more than a few bits."""
import math

import pytest

from paper_2609_38169_gb300 import api as A

import kv_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = [torch.float32, torch.bfloat16, torch.float16]
FORMATS = [A.KV_BF16, A.KV_F16, A.KV_INT8, A.KV_INT4]
CODES = [A.KV_INT8, A.KV_INT4]
NAMES = {A.KV_BF16: "bf16", A.KV_F16: "f16", A.KV_INT8: "int8", A.KV_INT4: "int4"}
ids = lambda x: str(x).split(".")[1] if isinstance(x, torch.dtype) else NAMES.get(x)  # noqa: E731
# head channels, key heads, query heads of each, tokens of a page
SHAPES = [(64, 2, 12, 8), (128, 2, 4, 16), (256, 1, 3, 64)]


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


def tables(g, kv, lens):
    """A page table in random order for sequences of lens[b] tokens, and the pages' number."""
    need = [-(-n // kv.page_tokens) for n in lens]
    page = torch.randperm(sum(need), generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(need)), -7, dtype=torch.int32, device="cuda")
    for b, n in enumerate(need):
        table[b, :n] = page[sum(need[:b]):sum(need[:b]) + n]
    return table, len(page)


def attend(kv, pages, table, lens, q, scale=None, window=0, max_len=None):
    y, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
    A.stepq_kv_attend(kv, 0, pages, table, i32(lens), q, y, scale=scale, window=window, lse=lse,
                      max_len=max(lens) if max_len is None else max_len)
    return y, lse


def check(kv, pages, table, lens, q, scale=None, window=0, max_len=None):
    y, lse = attend(kv, pages, table, lens, q, scale, window, max_len)
    wy, wl, tol, ltol = R.attend(pages, kv, 0, table, lens, q, kv.head_dim ** -0.5 if scale is None else scale, window)
    R.assert_within(lse, wl, ltol, "lse")
    R.assert_within(y, wy, R.rounded(tol, wy, q.dtype), "y")


def filled(g, kv, lens, k=None, v=None, size=1.0):
    """Pages of rows k, v [tokens][heads][D] (or normal ones) and their table."""
    table, n = tables(g, kv, lens)
    pages = A.alloc_pages(kv, n)
    shape = (sum(lens), kv.n_heads, kv.head_dim)
    k, v = (torch.randn(shape, generator=g, device="cuda") * size if x is None else x for x in (k, v))
    R.append(pages, kv, 0, table, [0] * len(lens), lens, k, v)
    return pages, table


# 16-bit words that fill what is no token: the infinities and the largest value of either type, NaN, a subnormal
@pytest.mark.parametrize("word", [0x7C00, 0xFC00, 0x7BFF, 0x7F80, 0xFF80, 0x7FC0, 0x0001],
                         ids=lambda w: f"{w:04x}")
@pytest.mark.parametrize("dt", TYPES, ids=ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=ids)
def test_what_lies_outside_the_tokens_reaches_nothing(fmt, dt, word):
    for D, heads, G, pt in SHAPES:
        g, kv = gen(D), A.KvConfig(1, heads, D, pt, fmt)
        lens = [1, 5, 16, 41, 100, 333, 1500, 0]
        full, table = filled(g, kv, lens)
        q = torch.randn((len(lens), heads * G, D), generator=g, device="cuda").to(dt)
        for window in (0, 21):
            lo = [max(0, n - window) if window else 0 for n in lens]
            page, at = R.places(table, lo, [n - a for n, a in zip(lens, lo)], pt)
            pages = torch.full((full.numel() // 2,), word - (word >> 15 << 16), dtype=torch.int16, device="cuda").view(torch.uint8)
            for src, dst in zip(R.split(full, kv), R.split(pages, kv)):
                if src is not None:
                    dst[page, 0, :, at] = src[page, 0, :, at]
            y, lse = attend(kv, pages, table, lens, q, window=window)
            wy, wl, tol, ltol = R.attend(full, kv, 0, table, lens, q, D ** -0.5, window)
            R.assert_within(lse, wl, ltol, "lse")
            R.assert_within(y, wy, R.rounded(tol, wy, dt), "y")


# ------------------------------------------------------------------ values
LARGEST = torch.finfo(torch.bfloat16).max


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=ids)
@pytest.mark.parametrize("D,heads,G,pt", SHAPES)
@pytest.mark.parametrize("lens", [[1, 2, 9, 100], [3000, 700], [40001]], ids=["short", "some", "long"])
def test_values_up_to_the_largest_of_bf16(lens, D, heads, G, pt, dt):
    """An output lies between the values that it weighs, so it is finite where they are: all of the largest
    magnitude, of either sign, one among small ones, and sizes whose largest scores come last."""
    g, kv = gen(3), A.KvConfig(1, heads, D, pt, A.KV_BF16)
    n, shape = sum(lens), (sum(lens), heads, D)
    q = torch.randn((len(lens), heads * G, D), generator=g, device="cuda").to(dt)
    normal = torch.randn(shape, generator=g, device="cuda")
    rising = torch.linspace(-4, 4, n, device="cuda")[:, None, None]
    lone = normal.clone()
    lone[n // 2] = LARGEST
    for v in (torch.full(shape, LARGEST, device="cuda"), LARGEST * normal.sign(), lone, normal * 2.0 ** 113, normal.clamp(-1, 1) * 2.0 ** 124):
        for k in (None, q[:1, ::G].float() * rising):
            pages, table = filled(g, kv, lens, k, v)
            check(kv, pages, table, lens, q)
            check(kv, pages, table, lens, q, window=50)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=ids)
def test_small_values_of_bf16(dt):
    """Values of 2^-60, whose weighted sums stay far above the least number."""
    g, kv = gen(4), A.KvConfig(1, 2, 128, 16, A.KV_BF16)
    lens = [1, 3000]
    v = torch.randn((3001, 2, 128), generator=g, device="cuda") * 2.0 ** -60
    pages, table = filled(g, kv, lens, None, v)
    check(kv, pages, table, lens, torch.randn((2, 8, 128), generator=g, device="cuda").to(dt))


# ------------------------------------------------------------------ scales of codes
@pytest.mark.parametrize("dt", TYPES, ids=ids)
@pytest.mark.parametrize("D,heads,G,pt", SHAPES)
@pytest.mark.parametrize("fmt", CODES, ids=ids)
def test_scales_of_zero_stand_for_zeros(fmt, D, heads, G, pt, dt):
    """Tokens of a page that nothing was written to count as zeros, as stepq_kv_read gives them: all of
    a sequence, some of one; and scales below those that an append writes."""
    g, kv = gen(5), A.KvConfig(1, heads, D, pt, fmt)
    lens = [40, 700, 3000, 2 * pt + 3]
    q = torch.randn((4, heads * G, D), generator=g, device="cuda").to(dt)
    pages, table = filled(g, kv, lens)
    blank = torch.zeros_like(pages)
    y, _ = attend(kv, blank, table, lens, q)
    assert not bool(y.any())
    check(kv, blank, table, lens, q)
    _, _, sk, sv = R.split(pages, kv)
    some = torch.rand(sv.shape, generator=g, device="cuda")
    sv[some < 0.3] = 0
    sk[(some > 0.2) & (some < 0.4)] = 0
    sv[(some > 0.5) & (some < 0.6)] = 2.0 ** -24
    check(kv, pages, table, lens, q)
    sv.copy_(torch.where(some < 0.5, 2.0 ** -24, 2.0 ** -20))
    check(kv, pages, table, lens, q)


@pytest.mark.parametrize("dt", TYPES, ids=ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=ids)
@pytest.mark.parametrize("D,heads,G,pt", SHAPES)
def test_pages_outside_the_pool_count_as_zeros(D, heads, G, pt, fmt, dt):
    g, kv = gen(6), A.KvConfig(1, heads, D, pt, fmt)
    lens = [5 * pt + 3, 700, 3000]
    pages, table = filled(g, kv, lens)
    n = pages.numel() // A.stepq_kv_page_bytes(kv)
    q = torch.randn((3, heads * G, D), generator=g, device="cuda").to(dt)
    bad, zero = table.clone(), table.clone()
    for b, at in ((0, 0), (0, 5), (1, 3), (2, 1), (2, 3000 // pt - 1)):
        bad[b, at], zero[b, at] = (n, -1, 1 << 30)[at % 3], n
    y, lse = attend(kv, pages, bad, lens, q)
    assert A.stepq_device_error() == 2
    more = torch.cat([pages, torch.zeros(A.stepq_kv_page_bytes(kv), dtype=torch.uint8, device="cuda")])
    wy, wl, tol, ltol = R.attend(more, kv, 0, zero, lens, q, D ** -0.5)
    R.assert_within(lse, wl, ltol, "lse")
    R.assert_within(y, wy, R.rounded(tol, wy, dt), "y")


# ------------------------------------------------------------------ scores
def one_token(kv, fmt, dt, k, v, lens, win, q, scale, ltol):
    """Where one token's score is so far above that the others weigh nothing (or `rest`), an output is its
    value. Its weight comes in terms (eps) of which those in fp16 end at 2^-25, for a weight of 2^-6 at least."""
    g = gen(7)
    pages, table = filled(g, kv, lens, k, v)
    wk, wv, _ = R.read(pages, kv, 0, table, [0] * len(lens), lens)
    G = q.shape[1] // kv.n_heads
    y, lse = attend(kv, pages, table, lens, q.to(dt), scale=scale)
    want = wv[win].repeat_interleave(G, 1)
    tol = want.abs() * (R.eps_of(fmt, dt) + 2.0 ** -18) + 2.0 ** -15
    R.assert_within(y, want, R.rounded(tol, want, dt), "y")
    score = (wk[win].repeat_interleave(G, 1) * q.double()).sum(-1) * scale
    R.assert_within(lse, score, score.abs() * ltol + 2.0 ** -14, "lse")


@pytest.mark.parametrize("e", [0, 10, 20, 24, 26, 28, 29, 30, 31, 32, 34, 40, 48])
@pytest.mark.parametrize("dt", TYPES, ids=ids)
@pytest.mark.parametrize("fmt", FORMATS, ids=ids)
def test_one_score_far_above_the_others(fmt, dt, e):
    """Scores of 2^6 to 2^55, of which one is above the others by a fourth of itself (the others' weights are
    3,100 times e^-20 at most, 2^-17). Beyond 2^29 they are so far apart that no exponent lies between."""
    for D, heads, G, pt in SHAPES:
        g, kv = gen(D), A.KvConfig(1, heads, D, pt, fmt)
        for lens in ([1, 3, 100], [3000, 700]):
            n = sum(lens)
            v = torch.randn((n, heads, D), generator=g, device="cuda").clamp(-4, 4)
            k = torch.zeros((n, heads, D), device="cuda")
            k[:, :, 0] = torch.randint(1, 6, (n, heads), generator=g, device="cuda").float()
            k[:, :, 1] = 7.0                                # of every row the largest: the scales are equal
            win = [sum(lens[:b]) + m * 3 // 4 for b, m in enumerate(lens)]
            k[win, :, 0] = 7.0
            q = torch.zeros((len(lens), heads * G, D), device="cuda")
            q[:, :, 0] = 1.375 * 2.0 ** (min(e, 12) if dt is torch.float16 else e // 2)
            # 16-bit queries over codes: each of D / 16 products cuts off 2^-13 q s, of a score of 7 q
            ltol = 2.0 ** -20 if dt is torch.float32 or R.BITS[fmt] == 16 else 2.0 ** -11
            one_token(kv, fmt, dt, k, v, lens, win, q, 8 * 1.375 * 2.0 ** e / float(q[0, 0, 0]), ltol)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=ids)
@pytest.mark.parametrize("fmt", [A.KV_F16] + CODES, ids=ids)
@pytest.mark.parametrize("e", [100, 118, 122, 126])
def test_queries_up_to_the_largest(e, fmt, dt):
    """Queries of up to 2^126 over keys of 7 / 1024 and less: products and scores below 2^120."""
    g, kv, lens = gen(8), A.KvConfig(1, 1, 128, 16, fmt), [1, 40, 700]
    k = torch.zeros((741, 1, 128), device="cuda")
    k[:, :, 0] = torch.randint(-5, 6, (741, 1), generator=g, device="cuda").float()
    k[:, :, 1] = 7.0
    win = [0, 31, 541]
    k[win, :, 0] = 7.0
    q = torch.zeros((3, 4, 128), device="cuda")
    q[:, :, 0] = 2.0 ** e
    v = torch.randn((741, 1, 128), generator=g, device="cuda").clamp(-4, 4)
    one_token(kv, fmt, dt, k / 1024, v, lens, win, q, 0.25, 2.0 ** -11)


@pytest.mark.parametrize("D,heads,G,pt", SHAPES)
@pytest.mark.parametrize("fmt,dt", [(A.KV_INT8, torch.float32), (A.KV_INT4, torch.float32), (A.KV_INT8, torch.float16),
                                    (A.KV_INT4, torch.float16), (A.KV_INT8, torch.bfloat16)], ids=ids)
def test_small_channels_beside_a_large_one(fmt, dt, D, heads, G, pt):
    """A query whose largest channel meets zeros of K only: a score is the sum of the small ones, held as in
    fp32, so that it is off by 68 u of their absolute terms at most (u = 2^-24, as in kv_ref). bf16 vectors
    over 4 bits are the exception: there the largest channel's offset takes part in the sum."""
    g, kv, lens = gen(9), A.KvConfig(1, heads, D, pt, fmt), [40, 900]
    k = torch.randint(-7, 8, (940, heads, D), generator=g, device="cuda").float()
    k[:, :, 0], k[:, :, 1] = 0, 7
    pages, table = filled(g, kv, lens, k)
    q = torch.randint(-15, 16, (2, heads * G, D), generator=g, device="cuda") / 64
    q[:, :, 0] = 1024
    y, lse = attend(kv, pages, table, lens, q.to(dt), scale=0.25)
    for b, n in enumerate(lens):
        rk, rv, _ = R.read(pages, kv, 0, table[b:b + 1], [0], [n])
        qb = q[b].double().view(heads, G, D)
        s = 0.25 * (qb @ rk.permute(1, 2, 0))
        e = 0.25 * (qb.abs() @ rk.abs().permute(1, 2, 0)) * 68 * R.U + 2.0 ** -21
        p, steps, vh = torch.softmax(s, -1), n / 64 * 2 + 64, rv.transpose(0, 1)
        want = torch.logsumexp(s, -1)
        R.assert_within(lse[b].view(heads, G), want, e.amax(-1) + steps * R.U + want.abs() * 4 * R.U, "lse")
        want = p @ vh
        tol = (p * e) @ vh.abs() + (p * e).sum(-1, keepdim=True) * want.abs() \
            + (R.eps_of(fmt, dt) + steps * R.U) * (p @ vh.abs()) + 2.0 ** -32 * vh.abs().sum(1, keepdim=True)
        R.assert_within(y[b].view(heads, G, D), want, R.rounded(tol, want, dt), "y")
