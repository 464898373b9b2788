"""Refusals of the decayed linear-attention calls and the group norm, before anything is
launched, and their launches against a CUDA runtime without a GPU."""
import ctypes as C
import os
import subprocess
import sys

import pytest

from paper_2609_38169_gb300 import _lib, api as A, build_ext

HERE = os.path.dirname(os.path.abspath(__file__))
OK, ARG, ALIGN, UNSUPPORTED = 0, 1, 4, 7
P = 1 << 20                                        # aligned, never dereferenced


def io(**kw):
    base = dict(dtype=1, q=P, k=P, v=P, gate=P, y=P, q_stride=256, k_stride=256, v_stride=512, gate_stride=4, y_stride=512)
    return _lib.StepqLinattnIo(**{**base, **kw})


def norm(**kw):
    return _lib.StepqNorm(**{**dict(act=1, center=1, shared=0, eps=1e-5), **kw})


def decode(cfg=None, layer=0, pool=P, pool_slots=4, slots=P, B=2, i=None, n=None):
    c = (cfg or A.Config(n_layers=2, n_key_heads=2, n_value_heads=4)).c()
    return _lib.lib().stepq_linattn_decode_step(C.byref(c), layer, pool, pool_slots, slots, B,
                                                C.byref(i or io()), C.byref(n) if n else None, None)


def prefill(cfg=None, layer=0, pool=P, pool_slots=4, slots=P, resume=None, cu=P, B=2, tokens=10, max_len=0, i=None,
            n=None, ws=None, nbytes=0):
    c = (cfg or A.Config(n_layers=2, n_key_heads=2, n_value_heads=4)).c()
    return _lib.lib().stepq_linattn_prefill(C.byref(c), layer, pool, pool_slots, slots, resume, cu, B, tokens, max_len,
                                            C.byref(i or io()), C.byref(n) if n else None, ws, nbytes, None)


BAD_IO = [(dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(q=0), ARG), (dict(k=0), ARG), (dict(v=0), ARG),
          (dict(gate=0), ARG), (dict(y=0), ARG), (dict(q=P + 8), ALIGN), (dict(k=P + 2), ALIGN), (dict(v=P + 4), ALIGN),
          (dict(y=P + 8), ALIGN), (dict(gate=P + 2), ALIGN), (dict(q_stride=-256), ARG), (dict(y_stride=511), ARG),
          (dict(y_stride=504), ARG), (dict(gate_stride=-1), ARG), (dict(k_stride=260), ALIGN), (dict(v_stride=513), ALIGN),
          (dict(y_stride=516), ALIGN), (dict(dtype=0, k_stride=258), ALIGN)]
BAD_NORM = [(dict(act=3), ARG), (dict(act=-1), ARG), (dict(center=2), ARG), (dict(shared=-1), ARG), (dict(eps=-1e-5), ARG),
            (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(weight=P + 2), ALIGN), (dict(bias=P + 1), ALIGN),
            (dict(z=P + 8, z_stride=512), ALIGN), (dict(z=P, z_stride=-512), ARG), (dict(z=P, z_stride=514), ALIGN)]


@pytest.mark.parametrize("call", [decode, prefill])
def test_refusals(call):
    for kw, code in BAD_IO:
        assert call(i=io(**kw)) == code, kw
    for kw, code in BAD_NORM:
        assert call(n=norm(**kw)) == code, kw
    two = dict(n_layers=2, n_key_heads=2, n_value_heads=4)
    assert call(cfg=A.Config(**two, gate_kind=A.GATE_CHANNEL)) == UNSUPPORTED
    assert call(cfg=A.Config(**two, dk=64)) == UNSUPPORTED
    assert call(cfg=A.Config(2, 3, 4)) == ARG
    for kw in (dict(layer=2), dict(layer=-1), dict(pool=None), dict(pool_slots=0), dict(slots=None), dict(B=-1),
               dict(B=1 << 30)):
        assert call(**kw) == ARG, kw
    for kw in (dict(pool=P + 8), dict(slots=P + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(B=0) == OK


def test_prefill_refusals():
    assert prefill(tokens=-1) == ARG and prefill(max_len=-1) == ARG
    assert prefill(cu=None, B=3, tokens=10) == ARG           # not equal lengths
    assert prefill(cu=P + 2) == ALIGN
    assert prefill(tokens=0) == OK


def test_workspace():
    cfg = A.Config(n_layers=1, n_key_heads=1, n_value_heads=2)
    for args in ((0, 100, 100), (2, 0, 0), (-1, 5, 5), (1, -5, 0), (1, 5, -1), (1 << 30, 1 << 30, 0)):
        assert A.stepq_linattn_workspace_bytes(cfg, *args) == 0
    bad = A.Config(n_layers=1, n_key_heads=2, n_value_heads=3)
    assert A.stepq_linattn_workspace_bytes(bad, 1, 100000, 100000) == 0
    need = A.stepq_linattn_workspace_bytes(cfg, 1, 1 << 20, 1 << 20)
    if need:
        kw = dict(cfg=cfg, B=1, tokens=1 << 20, max_len=1 << 20, i=io(q_stride=128, k_stride=128, v_stride=256, y_stride=256,
                                                                     gate_stride=2))
        assert prefill(**kw) == ARG                            # no workspace
        assert prefill(**kw, ws=P, nbytes=need - 1) == ARG
        assert prefill(**kw, ws=P + 128, nbytes=need) == ALIGN


@pytest.mark.parametrize("hv", [1, 2, 7, 16, 32, 64, 90])
@pytest.mark.parametrize("longest", [600, 8192, 100000, 1 << 22])
@pytest.mark.parametrize("others", [0, 512, 5000])
def test_the_workspace_holds_the_states_of_split_sequences_only(hv, longest, others):
    """One long sequence beside others of one token. Split, it makes segments of a third of a
    multiprocessor's share of the work (152 of them) at least, so about 456 over all heads that
    have one after them, and no more than twice as many states of 64 KiB; a sequence adds its
    places in two tables (40 bytes)."""
    cfg = A.Config(n_layers=1, n_key_heads=hv, n_value_heads=hv)
    need = A.stepq_linattn_workspace_bytes(cfg, 1 + others, longest + others, longest)
    assert need <= 2 * 456 * (65536 + 4) + 40 * others + 32768


def group(dtype=1, rows=3, groups=2, width=5, x=P, xs=10, out=P, os_=10, n=None):
    return _lib.lib().stepq_group_norm(dtype, rows, groups, width, x, xs, out, os_, C.byref(n or norm()), None)


def test_group_norm_refusals():
    for kw, code in BAD_NORM[:9] + [(dict(z=P + 1, z_stride=10), ALIGN), (dict(z=P, z_stride=-1), ARG)]:
        assert group(n=norm(**kw)) == code, kw
    for kw in (dict(dtype=3), dict(rows=-1), dict(groups=0), dict(width=0), dict(x=None), dict(out=None), dict(xs=-1),
               dict(os_=9), dict(groups=1 << 20, width=1 << 20, os_=1 << 40), dict(rows=1 << 41)):
        assert group(**kw) == ARG, kw
    assert group(x=P + 1) == ALIGN and group(dtype=0, out=P + 2) == ALIGN
    assert _lib.lib().stepq_group_norm(1, 3, 2, 5, P, 10, P, 10, None, None) == ARG
    assert group(rows=0) == OK


def test_group_norm_in_place_keeps_the_rows():
    """out may be x or z only where their rows lie alike."""
    far = P << 10
    assert group(x=P, xs=12, out=P, os_=10) == ARG and group(x=P, xs=0, out=P, os_=10) == ARG
    assert group(x=P, xs=10, out=far, os_=12, n=norm(z=far, z_stride=10)) == ARG
    assert group(rows=0, x=P, xs=12, out=P, os_=10) == OK


def test_binding_refuses_shapes_and_types():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 128)
    cfg = A.Config(1, 4, 4)
    with pytest.raises(ValueError, match="expected a CUDA tensor"):
        A.stepq_linattn_decode_step(cfg, 0, x, torch.zeros(2, dtype=torch.int32), x, x, x, x, x)
    with pytest.raises(ValueError, match="expected 3 rows"):
        A.stepq_linattn_decode_step(cfg, 0, x, torch.zeros(3, dtype=torch.int32), x, x, x, x, x)
    with pytest.raises(ValueError, match="cu_seqlens"):
        A.stepq_linattn_prefill(cfg, 0, x, torch.zeros(3, dtype=torch.int32), x, x, x, x, x,
                                cu_seqlens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="do not make"):
        A.stepq_group_norm(torch.zeros(2, 10), 3, torch.zeros(2, 10), A.Norm())


@pytest.mark.gpu
def test_binding_refuses_layouts():
    torch = pytest.importorskip("torch")
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    cfg, slots = A.Config(1, 2, 4), z(3, dt=torch.int32)
    pool, q, v, g = z(3, 1, 4, 128, 128, dt=torch.float32), z(3, 2, 128), z(3, 4, 128), z(3, 4, dt=torch.float32)
    call = lambda **kw: A.stepq_linattn_decode_step(**{**dict(  # noqa: E731
        cfg=cfg, layer=0, pool=pool, slots=slots, q=q, k=q, v=v, gate=g, y=v.clone()), **kw})
    for kw, say in ((dict(k=q.float()), "expected torch.bfloat16"), (dict(q=q.double()), "bfloat16 or float16|expected"),
                    (dict(v=z(3, 4, 256)[:, :, ::2]), "v: expected"), (dict(v=z(3, 128, 4).transpose(1, 2)), "v: expected"),
                    (dict(v=z(2, 4, 128)), "v: expected"), (dict(gate=g.bfloat16()), "float32"), (dict(gate=g[:, :3]), "gate"),
                    (dict(pool=pool.bfloat16()), "float32"),
                    (dict(norm=A.Norm(weight=z(128, dt=torch.float32))), "weight: expected 512"),
                    (dict(norm=A.Norm(weight=z(512, dt=torch.float32), shared=True)), "weight: expected 128"),
                    (dict(norm=A.Norm(z=z(3, 4, 64))), "z: expected")):
        with pytest.raises(ValueError, match=say):
            call(**kw)


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    build_ext.build()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(build_ext.nvcc())))
    fake = str(tmp_path_factory.mktemp("fake") / "libfake.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-Wall", "-I", os.path.join(cuda, "include"),
                    os.path.join(HERE, "fake_cudart.c"), os.path.join(HERE, "fake_tensormap.c"), "-o", fake], check=True)

    def child(code):
        r = subprocess.run([sys.executable, "-c", CALLS + code], cwd=os.path.dirname(HERE), capture_output=True,
                           text=True, env={**os.environ, "LD_PRELOAD": fake, "PYTHONPATH": HERE}, timeout=120)
        assert r.returncode == 0, r.stderr
    return child


CALLS = """
import ctypes as C
import test_linattn_cpu as T
from paper_2609_38169_gb300 import api as A, _lib
fake = C.CDLL(None)
L, P = _lib.lib(), T.P
wide = A.Config(n_layers=1, n_key_heads=1, n_value_heads=2)
io = lambda dt: T.io(dtype=dt, q_stride=128, k_stride=128, v_stride=256, y_stride=256, gate_stride=2)
calls = {}
for dt in (0, 1, 2):
    for name, n in (("", None), ("norm", T.norm()), ("gate", T.norm(z=P, z_stride=512))):
        calls["decode", dt, name] = lambda dt=dt, n=n: T.decode(i=T.io(dtype=dt), n=n)
        for tokens in (1, 40, 5000, 200000):
            ws = A.stepq_linattn_workspace_bytes(wide, 2, tokens, 0)
            calls["prefill", dt, name, tokens] = lambda dt=dt, n=n, t=tokens, ws=ws: T.prefill(
                cfg=wide, tokens=t, i=io(dt), n=n, ws=P, nbytes=ws)
    for width in (1, 5, 128, 600, 5000):
        calls["norm", dt, width] = lambda dt=dt, w=width: T.group(dt, 3, 2, w, P, 2 * w, P, 2 * w)
"""
LAUNCH, SET_ATTRIBUTE, GET_ATTRIBUTES = range(3)


@pytest.mark.parametrize("kind", [LAUNCH, SET_ATTRIBUTE, GET_ATTRIBUTES])
def test_a_refused_launch_leaves_no_error(run, kind):
    """Every variant launches; one that the runtime refuses returns STEPQ_ERR_CUDA (or, where
    the refused query was not needed, runs) and leaves no error behind."""
    run(f"""
for name, call in calls.items():
    fake.fake_refuse({kind}, 1)
    before, status = fake.fake_launches(), call()
    fake.fake_refuse({kind}, 0)
    assert status == (0 if fake.fake_launches() > before else 5), (name, status)
    assert fake.fake_pending_error() == 0, name
    assert call() == 0 and fake.fake_launches() > before, name
""")


def test_packed_structures_are_the_declared_ones():
    """The binding's packed arguments, byte for byte the ctypes structures'."""
    io = _lib.StepqLinattnIo(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11)
    assert bytes(io) == A._pack_io(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11)
    norm = _lib.StepqNorm(2, 1, 0, 0.5, 4, 5, 6, 7)
    assert bytes(norm) == A._pack_norm(2, True, False, 0.5, 4, 5, 6, 7)


def test_kept_configurations_follow_the_fields():
    """A changed field reaches the library although the structure is kept."""
    cfg = A.Config(n_layers=1, n_key_heads=2, n_value_heads=4)
    before = A.stepq_linattn_workspace_bytes(cfg, 2, 4096, 4000)
    cfg.n_value_heads = 8
    after = A.stepq_linattn_workspace_bytes(cfg, 2, 4096, 4000)
    assert before and after and before != after
    cfg.n_value_heads = 4
    assert A.stepq_linattn_workspace_bytes(cfg, 2, 4096, 4000) == before
