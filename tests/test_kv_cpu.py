"""Refusals of the paged cache's calls before anything is launched, sizes, and their launches
against a CUDA runtime without a GPU."""
import ctypes as C
import os
import subprocess
import sys

import pytest

from paper_2609_38169_gb300 import _lib, api as A, build_ext

HERE = os.path.dirname(os.path.abspath(__file__))
OK, ARG, ALIGN, UNSUPPORTED = 0, 1, 4, 7
P = 1 << 20                                        # aligned, never dereferenced


def config(**kw):
    return C.byref(_lib.StepqKvConfig(**{**dict(n_layers=2, n_heads=4, head_dim=128, page_tokens=16, format=2), **kw}))


def pages(**kw):
    return C.byref(_lib.StepqKvPages(**{**dict(pages=P, n_pages=9, table_width=8, table=P, table_stride=8), **kw}))


def rows(**kw):
    return C.byref(_lib.StepqKvRows(**{**dict(dtype=1, k=P, v=P, k_stride=512, v_stride=512), **kw}))


def query(**kw):
    base = dict(dtype=1, n_heads=8, q=P, y=P << 4, lse=None, q_stride=1024, y_stride=1024, scale=0.1, window=0, max_len=100)
    return C.byref(_lib.StepqKvQuery(**{**base, **kw}))


def move(name, c=None, layer=0, p=None, starts=P, cu=None, B=2, tokens=6, r=None):
    return getattr(_lib.lib(), name)(c or config(), layer, p or pages(), starts, cu, B, tokens, r or rows(), None)


def attend(c=None, layer=0, p=None, lens=P, B=2, q=None, ws=P, nbytes=1 << 30):
    return _lib.lib().stepq_kv_attend(c or config(), layer, p or pages(), lens, B, q or query(), ws, nbytes, None)


BAD_CONFIG = [(dict(n_layers=0), ARG), (dict(n_heads=0), ARG), (dict(format=4), ARG), (dict(format=-1), ARG),
              (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED), (dict(page_tokens=4), UNSUPPORTED),
              (dict(page_tokens=24), UNSUPPORTED), (dict(page_tokens=512), UNSUPPORTED), (dict(n_heads=1 << 20), ARG),
              (dict(n_layers=1 << 12, n_heads=1 << 9), UNSUPPORTED)]
BAD_PAGES = [(dict(pages=None), ARG), (dict(n_pages=0), ARG), (dict(table_width=-1), ARG), (dict(table_stride=-1), ARG),
             (dict(table=None), ARG), (dict(table_width=(1 << 26) + 1), ARG), (dict(pages=P + 8), ALIGN), (dict(table=P + 2), ALIGN)]


@pytest.mark.parametrize("call", [lambda **kw: move("stepq_kv_append", **kw), lambda **kw: move("stepq_kv_read", **kw), attend],
                         ids=["append", "read", "attend"])
def test_refusals_in_common(call):
    for kw, code in BAD_CONFIG:
        assert call(c=config(**kw)) == code, kw
    for kw, code in BAD_PAGES:
        assert call(p=pages(**kw)) == code, kw
    for kw in (dict(layer=-1), dict(layer=2), dict(B=-1)):
        assert call(**kw) == ARG, kw
    assert call(B=0) == OK and call(B=0, p=pages(table=None)) == OK and call(B=0, p=pages(table=None, table_width=0)) == OK


@pytest.mark.parametrize("name", ["stepq_kv_append", "stepq_kv_read"])
def test_rows_refusals(name):
    for kw, code in [(dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(k=None), ARG), (dict(v=None), ARG), (dict(k_stride=-8), ARG),
                     (dict(k=P + 8), ALIGN), (dict(v=P + 2), ALIGN), (dict(k_stride=516), ALIGN), (dict(v_stride=514), ALIGN)]:
        assert move(name, r=rows(**kw)) == code, kw
    assert move(name, tokens=-1) == ARG and move(name, tokens=(1 << 30) + 2) == ARG and move(name, starts=None) == ARG and move(name, tokens=5) == ARG
    assert move(name, starts=P + 1) == ALIGN and move(name, cu=P + 2, tokens=5) == ALIGN
    assert move(name, tokens=0) == OK and move(name, tokens=0, starts=None) == OK


def test_read_into_rows_that_overlap():
    assert move("stepq_kv_read", r=rows(k_stride=504)) == ARG and move("stepq_kv_read", r=rows(v_stride=0)) == ARG


def test_attend_refusals():
    for kw, code in [(dict(dtype=3), ARG), (dict(n_heads=0), ARG), (dict(n_heads=6), ARG), (dict(n_heads=-4), ARG), (dict(q=None), ARG),
                     (dict(y=None), ARG), (dict(q_stride=-8), ARG), (dict(y_stride=1016), ARG), (dict(scale=float("inf")), ARG),
                     (dict(scale=float("nan")), ARG), (dict(window=-1), ARG), (dict(max_len=-1), ARG), (dict(q=P + 8), ALIGN),
                     (dict(y=P + 4), ALIGN), (dict(lse=P + 2), ALIGN), (dict(q_stride=1028), ALIGN), (dict(y=P, q_stride=2048), ARG)]:
        assert attend(q=query(**kw)) == code, kw
    assert attend(lens=None) == ARG and attend(lens=P + 1) == ALIGN and attend(B=1 << 28) == ARG


def test_workspace():
    bytes_of = lambda c=None, hq=8, B=2, n=100000: _lib.lib().stepq_kv_workspace_bytes(c or config(), hq, B, n)  # noqa: E731
    for kw, _ in BAD_CONFIG:
        assert bytes_of(config(**kw)) == 0
    for kw in (dict(hq=6), dict(hq=0), dict(B=0), dict(B=-1), dict(n=-1), dict(B=1 << 29)):
        assert bytes_of(**kw) == 0
    sizes = [bytes_of(n=n) for n in (1, 100, 513, 5000, 100000, 1 << 30)]
    assert sizes[0] == 0 and sizes[2] > 0 and sizes == sorted(sizes) and bytes_of(n=0) == sizes[-1]
    wide = pages(table_width=1 << 16)
    q = query(max_len=100000)
    assert attend(p=wide, q=q, ws=None) == ARG and attend(p=wide, q=q, nbytes=bytes_of() - 1) == ARG
    assert attend(p=wide, q=q, ws=P + 128) == ALIGN


def test_page_bytes():
    n = lambda **kw: _lib.lib().stepq_kv_page_bytes(config(**kw))  # noqa: E731
    assert n(format=0) == n(format=1) == 2 * 4 * 16 * 512 and n() == 2 * 4 * 16 * 260 and n(format=3) == 2 * 4 * 16 * 132
    assert n(head_dim=64, format=3, page_tokens=8, n_layers=1, n_heads=1) == 8 * 68
    assert all(n(**kw) == 0 for kw, _ in BAD_CONFIG)


def test_configurations_follow_the_fields():
    kv = A.KvConfig(1, 2)
    before = A.stepq_kv_page_bytes(kv)
    kv.n_layers = 3
    assert A.stepq_kv_page_bytes(kv) == 3 * before
    kv.page_tokens = 5
    assert A.stepq_kv_page_bytes(kv) == 0


def test_binding_refuses_cpu_tensors_and_shapes():
    torch = pytest.importorskip("torch")
    kv, pg, t = A.KvConfig(1, 4), torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(2, 8, dtype=torch.int32)
    n, x = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, 128)
    with pytest.raises(ValueError, match="table: expected a CUDA tensor"):
        A.stepq_kv_append(kv, 0, pg, t, n, x, x)
    with pytest.raises(ValueError, match="table: expected 3 rows"):
        A.stepq_kv_attend(kv, 0, pg, t, torch.zeros(3, dtype=torch.int32), x, x)
    with pytest.raises(ValueError, match="cu_seqlens: expected 3"):
        A.stepq_kv_read(kv, 0, pg, t, n, x, x, cu_seqlens=n)
    with pytest.raises(ValueError, match="starts: expected a tensor"):
        A.stepq_kv_read(kv, 0, pg, t, [0, 0], x, x)
    with pytest.raises(ValueError, match="n_layers: .* does not fit"):
        A.stepq_kv_read(A.KvConfig(1 << 40, 4), 0, pg, t, n, x, x)
    with pytest.raises(TypeError):
        A.stepq_kv_read(A.KvConfig("1", 4), 0, pg, t, n, x, x)
    with pytest.raises(AttributeError):
        A.stepq_kv_read(None, 0, pg, t, n, x, x)


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
import test_kv_cpu as T
fake = C.CDLL(None)
calls = {}
for fmt in range(4):
    for D in (64, 128, 256):
        c = T.config(format=fmt, head_dim=D)
        for dt in (0, 1, 2):
            for name in ("stepq_kv_append", "stepq_kv_read"):
                calls[name, fmt, D, dt] = lambda n=name, c=c, dt=dt: T.move(n, c, r=T.rows(dtype=dt, k_stride=1024, v_stride=1024))
            for hq in (4, 48):
                for n in (10, 100000):
                    calls["attend", fmt, D, dt, hq, n] = lambda c=c, dt=dt, hq=hq, n=n: T.attend(
                        c, p=T.pages(table_width=1 << 16),
                        q=T.query(dtype=dt, n_heads=hq, max_len=n, q_stride=1 << 14, y_stride=1 << 14))
"""
LAUNCH, SET_ATTRIBUTE = range(2)


@pytest.mark.parametrize("kind", [LAUNCH, SET_ATTRIBUTE])
def test_a_refused_launch_leaves_no_error(run, kind):
    """Every variant launches; one that the runtime refuses returns STEPQ_ERR_CUDA and leaves no
    error behind."""
    run(f"""
for name, call in calls.items():
    fake.fake_refuse({kind}, 1)
    before, status = fake.fake_launches(), call()
    fake.fake_refuse({kind}, 0)
    assert status == (0 if fake.fake_launches() > before else 5), (name, status)
    assert fake.fake_pending_error() == 0, name
    assert call() == 0 and fake.fake_launches() > before, name
""")
