"""Bounds of packed rows that are not ascending: reported, and every row goes to a sequence that holds it or nowhere."""
import pytest

from paper_2609_38169_gb300 import api as A

import kv_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
I32 = torch.iinfo(torch.int32)


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert A.stepq_device_error() == 0


def ascending(lens):
    return [sum(lens[:b]) for b in range(len(lens) + 1)]


CASES = {  # name -> (bounds, rows)
    "overlap": ([0, 6, 2, 6], 6),
    "negative": ([-3, 2, 6], 6),
    "least": ([I32.min, 4, 6], 6),
    "greatest": ([0, I32.max, 6], 6),
    "beyond": ([0, 3, 9], 6),
    "all beyond": ([7, 9], 6),
    "reversed": (list(range(120, -1, -3)), 120),
    "one of many, least": (lambda c: c[:7] + [I32.min] + c[8:], 40),
    "one of many, greatest": (lambda c: c[:8] + [I32.max] + c[9:], 40),
    "many of many": (lambda c: [x if b % 5 else (7 * b) % 120 for b, x in enumerate(c)], 40),
    "more than a warp looks at": (lambda c: c[:-3] + [c[-2], c[-3], c[-1]], 3000),
    "long, least": (lambda c: c[:3] + [I32.min] + c[4:], [3000, 0, 1500, 4000, 700]),
    "long, overlap": (lambda c: c[:3] + [1000] + c[4:], [3000, 0, 1500, 4000, 700]),
    "long, beyond": (lambda c: c[:-1] + [c[-1] + 9], [3000, 0, 1500, 4000, 700]),
}


@pytest.mark.parametrize("fmt,dt", [(A.KV_F16, torch.float32), (A.KV_INT8, torch.bfloat16)], ids=["f16", "int8"])
@pytest.mark.parametrize("name", list(CASES))
def test_bounds_out_of_order(name, fmt, dt):
    bounds, rows = CASES[name]
    if callable(bounds):
        c = ascending(rows if isinstance(rows, list) else [3] * rows)
        bounds, rows = bounds(c), c[-1]
    B = len(bounds) - 1
    g, kv = torch.Generator(device="cuda").manual_seed(len(name)), A.KvConfig(1, 1, 64, 8, fmt)
    # where a row may go
    holders = [[] for _ in range(rows)]
    for b, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        if 0 <= lo and hi <= rows:
            for i in range(lo, hi):
                holders[i].append((b, b % 5 + i - lo))
    each = max((pos for h in holders for _, pos in h), default=0) // 8 + 1
    table = torch.randperm(B * each, generator=g, device="cuda").to(torch.int32).view(B, each)
    pages = torch.randint(0, 100, (B * each * A.stepq_kv_page_bytes(kv),), generator=g, device="cuda").to(torch.uint8)
    k, v = torch.randn((2, rows, 1, 64), generator=g, device="cuda").to(dt)
    starts, cu = torch.arange(B, device="cuda").int() % 5, torch.tensor(bounds, dtype=torch.int32, device="cuda")
    out = torch.full((2, rows, 1, 64), 7.0, dtype=dt, device="cuda")
    A.stepq_kv_read(kv, 0, pages, table, starts, *out, cu_seqlens=cu)
    assert A.stepq_device_error() == 1
    used = [False] * rows
    for n in range(max(map(len, holders), default=0)):
        at = [i for i in range(rows) if len(holders[i]) > n]
        b, pos = (torch.tensor(x, device="cuda") for x in zip(*(holders[i][n] for i in at)))
        wk, wv, sk, sv = R.split(pages, kv)
        place = table[b, pos // 8].long(), 0, slice(None), pos % 8
        want = [R.decode(w[place], None if s is None else s[place], fmt)[0].float().to(dt) for w, s in ((wk, sk), (wv, sv))]
        same = (out[0, at] == want[0]).flatten(1).all(1) & (out[1, at] == want[1]).flatten(1).all(1)
        for i, x in zip(at, same.tolist()):
            used[i] |= x
    left = (out == 7).flatten(2).all(2).all(0).tolist()
    assert all(u or x for u, x in zip(used, left))
    if B <= 3 and name != "overlap":                        # sequences apart from the bad bounds are read
        assert used == [len(h) > 0 for h in holders]
    # and written: only places that rows may go to change
    before = pages.clone()
    A.stepq_kv_append(kv, 0, pages, table, starts, k, v, cu_seqlens=cu)
    assert A.stepq_device_error() == 1
    may = torch.zeros((B * each, 8), dtype=torch.bool, device="cuda")
    for h in holders:
        for b, pos in h:
            may[table[b, pos // 8].long(), pos % 8] = True
    for x, y in zip(R.split(pages, kv), R.split(before, kv)):
        if x is not None:
            same = (x == y).view(B * each, 8, -1) if x.dim() == 5 else (x.view(torch.int16) == y.view(torch.int16)).view(B * each, 8, 1)
            assert bool((same.all(2) | may).all())


def test_good_bounds_raise_nothing():
    """Ascending ones, with empty sequences, rows before the first and behind the last."""
    kv, B = A.KvConfig(1, 1, 64, 8, A.KV_INT8), 3000
    g = torch.Generator(device="cuda").manual_seed(1)
    lens = torch.randint(0, 3, (B,), generator=g, device="cuda")
    cu = torch.cat([torch.zeros(1, device="cuda"), lens.cumsum(0)]).int() + 5
    rows = int(cu[-1]) + 4
    k = torch.randn((rows, 1, 64), generator=g, device="cuda")
    pages, table = A.alloc_pages(kv, B), torch.arange(B, device="cuda").int()[:, None].contiguous()
    starts = torch.zeros(B, dtype=torch.int32, device="cuda")
    A.stepq_kv_append(kv, 0, pages, table, starts, k, k, cu_seqlens=cu)
    out = torch.full((2, rows, 1, 64), 7.0, device="cuda")
    A.stepq_kv_read(kv, 0, pages, table, starts, *out, cu_seqlens=cu)
    code, s = R.encode(k, kv.format)
    want = R.decode(code, s, kv.format)[0].float()
    assert torch.equal(out[0, 5:-4], want[5:-4]) and torch.equal(out[1, 5:-4], want[5:-4])
    assert bool((out[:, :5] == 7).all()) and bool((out[:, -4:] == 7).all())
