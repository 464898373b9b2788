"""Group norm with an activation or a gate against its 64-bit form. x is exact in fp32, so
the bound is that of fp32 statistics (a mean and a centred sum of squares, each within a
few u times sqrt(n), far below 2^-17 of the largest centred value) and of the type."""
import pytest

from paper_2609_38169_gb300 import api as A

import linattn_ref as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAMES = ["f32", "bf16", "f16"]


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert A.stepq_device_error() == 0


def check(x, groups, out, norm, x0=None):
    """Runs the library on x and compares with the reference on x0 (x as it was)."""
    x0 = x.clone() if x0 is None else x0
    A.stepq_group_norm(x, groups, out, norm)
    want, gain, part = R.norm(x0, groups, norm.weight, norm.bias, norm.z, norm.act, norm.center, norm.shared, norm.eps)
    e = 4 * R.U * x0.double().abs()                              # the mean's and the difference's roundings
    tol = R.norm_bound(e, gain, part, groups)
    R.assert_within(out, want, R.rounded(tol, want, x.dtype), "out")


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("groups,width", [(4, 1), (3, 2), (1, 7), (12, 75), (4, 128), (32, 128), (5, 256), (2, 640),
                                          (3, 1000), (1, 1024), (2, 4096), (1, 5003)])
@pytest.mark.parametrize("form", ["gate", "self", "rms"])
def test_widths(groups, width, dt, form):
    g = torch.Generator(device="cuda").manual_seed(width)
    rows, C = 37, groups * width
    x = (torch.randn((rows, C), generator=g, device="cuda") * 2 + 0.5).to(dt)
    w, b = torch.randn((2, C), generator=g, device="cuda")
    z = torch.randn((rows, C), generator=g, device="cuda").to(dt) * 3
    norm = {"gate": A.Norm(weight=w, bias=b, z=z, act=A.ACT_SILU),
            "self": A.Norm(bias=b[:width].contiguous(), act=A.ACT_SIGMOID, shared=True),
            "rms": A.Norm(weight=w, z=z, act=A.ACT_NONE, center=False, eps=1e-6)}[form]
    check(x, groups, torch.empty_like(x), norm)


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 8), (1, 5)])
def test_strides_and_alignment(dt, pad, shift):
    """Rows that start anywhere their type allows, wider than the channels."""
    g = torch.Generator(device="cuda").manual_seed(pad)
    rows, groups, width = 50, 3, 128
    C = groups * width

    def at(k):
        buf = torch.randn(shift + rows * (C + k), generator=g, device="cuda").to(dt)
        return buf[shift:].view(rows, C + k)[:, :C]
    x, z, out = at(pad), at(pad), at(2 * pad)
    check(x, groups, out, A.Norm(z=z))
    check(at(pad), groups, torch.empty((rows, C), dtype=dt, device="cuda"), A.Norm(z=at(0)))


@pytest.mark.parametrize("width", [64, 75, 1500])
def test_in_place(width):
    x = torch.randn((9, 4 * width), device="cuda")
    check(x, 4, x, A.Norm(act=A.ACT_SILU), x.clone())


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
def test_rows_without_spread_and_far_from_zero(dt):
    """Constant groups (variance 0), zeros, a large common offset, and large values."""
    x = torch.ones((6, 2 * 128), device="cuda")
    x[1], x[2, :128], x[3] = 0.0, -7.5, 1000.0
    x[4] = 900 + torch.randn(256, device="cuda") * 8
    x[5] = torch.randn(256, device="cuda") * 3e4 if dt is not torch.float16 else torch.randn(256, device="cuda") * 1e4
    x = x.to(dt)
    check(x, 2, torch.empty_like(x), A.Norm(act=A.ACT_NONE))
    check(x, 2, torch.empty_like(x), A.Norm(act=A.ACT_SILU, center=False))


def test_a_bad_value_stays_in_its_group():
    x = torch.randn((4, 3 * 128), device="cuda", dtype=torch.bfloat16)
    want, got = torch.empty_like(x), torch.empty_like(x)
    A.stepq_group_norm(x, 3, want, A.Norm())
    x[1, 130], x[2, 5] = torch.nan, torch.inf
    A.stepq_group_norm(x, 3, got, A.Norm())
    same = torch.ones((4, 3), dtype=torch.bool, device="cuda")
    same[1, 1] = same[2, 0] = False
    for r in range(4):
        for c in range(3):
            s = slice(128 * c, 128 * c + 128)
            assert torch.equal(got[r, s], want[r, s]) if same[r, c] else bool(got[r, s].isnan().any())


def test_gates_that_saturate():
    """Large gates of either sign: silu and sigmoid reach their limits without NaN."""
    x = torch.randn((2, 128), device="cuda")
    z = torch.full((2, 128), 200.0, device="cuda")
    z[1] = -200.0
    for act in (A.ACT_SILU, A.ACT_SIGMOID):
        for dt in TYPES:
            out = torch.empty((2, 128), device="cuda", dtype=dt)
            check(x.to(dt), 1, out, A.Norm(z=z.to(dt), act=act))


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("rows,groups,width", [(5000, 5, 64), (9000, 32, 8), (700, 97, 24), (60, 1009, 16), (9001, 3, 75),
                                               (1500, 7, 333), (3001, 3, 600), (2000, 1, 2048), (700, 2, 1003),
                                               (4000, 3, 360), (3000, 1, 7168), (300, 1, 16384)])
def test_many_rows(rows, groups, width, dt):
    """More groups than the GPU holds at once: a team's later groups, of one column or another."""
    g = torch.Generator(device="cuda").manual_seed(width)
    C = groups * width
    x, z = torch.randn((2, rows, C), generator=g, device="cuda").to(dt)
    w, b = torch.randn((2, C), generator=g, device="cuda")
    check(x, groups, torch.empty_like(x), A.Norm(weight=w, bias=b, z=z, act=A.ACT_SILU))
    check(x, groups, torch.empty_like(x), A.Norm(weight=w[:width].contiguous(), act=A.ACT_NONE, center=False, shared=True))


@pytest.mark.parametrize("dt", TYPES, ids=NAMES)
@pytest.mark.parametrize("width", [128, 75])
def test_infinite_gates(width, dt):
    """A sigmoid gate of plus infinity passes the value, of minus infinity stops it."""
    x = torch.randn((5, 2 * width), device="cuda").to(dt)
    z = torch.zeros_like(x)
    z[:, ::2], z[:, 1::2] = torch.inf, -torch.inf
    got, want = torch.empty_like(x), torch.empty_like(x)
    A.stepq_group_norm(x, 2, got, A.Norm(z=z, act=A.ACT_SIGMOID))
    A.stepq_group_norm(x, 2, want, A.Norm(act=A.ACT_NONE))
    assert torch.equal(got[:, ::2], want[:, ::2]) and bool((got[:, 1::2] == 0).all())
