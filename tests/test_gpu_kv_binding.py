"""What the paged cache's compiled binding does beside the calls: it lets other Python threads run, and writes to no
tensor but the ones that it is given."""
import ctypes as C
import subprocess
import threading

import pytest

from paper_2609_38169_gb300 import _lib, api as A

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
KV = A.KvConfig(1, 2, 128, 16, A.KV_INT8)

WAITS = """
#include <time.h>
volatile int flag;
/* 0 once the flag is set, 5 after five seconds without it */
int wait_for_flag(void) {
    struct timespec ms = {0, 1000000};
    for (int i = 0; i < 5000 && !flag; i++) nanosleep(&ms, 0);
    return flag ? 0 : 5;
}
"""


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def z(*shape, dt=torch.bfloat16):
    return torch.zeros(shape, dtype=dt, device="cuda")


def calls(pages, table, n, k, v, q, y):
    return [lambda: A.stepq_kv_append(KV, 0, pages, table, n, k, v), lambda: A.stepq_kv_read(KV, 0, pages, table, n, k, v),
            lambda: A.stepq_kv_attend(KV, 0, pages, table, n, q, y)]


@pytest.mark.parametrize("call", range(3), ids=["append", "read", "attend"])
def test_other_threads_run_while_a_call_waits(call, tmp_path):
    """The library's call is replaced by one that waits for another Python thread."""
    (tmp_path / "waits.c").write_text(WAITS)
    so = str(tmp_path / "waits.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", str(tmp_path / "waits.c"), "-o", so], check=True)
    waits = C.CDLL(so)
    address, flag = C.cast(waits.wait_for_flag, C.c_void_p).value, C.c_int.in_dll(waits, "flag")
    do = calls(A.alloc_pages(KV, 4), z(3, 2, dt=torch.int32), z(3, dt=torch.int32), z(3, 2, 128), z(3, 2, 128), z(3, 4, 128), z(3, 4, 128))[call]
    do()
    real = [C.cast(getattr(_lib.lib(), "stepq_kv_" + f), C.c_void_p).value for f in ("append", "read", "attend", "page_bytes")]
    go = threading.Event()

    def set_flag():
        go.wait()
        flag.value = 1

    other = threading.Thread(target=set_flag)
    other.start()
    _lib.bind().use(address, address, address, real[3])
    try:
        go.set()
        do()
    finally:
        _lib.bind().use(*real)
        other.join()


def test_tensors_that_share_memory_until_one_is_written():
    """torch's lazy clones: what a call writes reaches no other owner of the memory."""
    g = torch.Generator(device="cuda").manual_seed(1)
    pages, table, n = A.alloc_pages(KV, 6), torch.randperm(6, generator=g, device="cuda").int().view(3, 2), torch.full((3,), 5, dtype=torch.int32, device="cuda")
    k, v = torch.randn((2, 3, 2, 128), generator=g, device="cuda").bfloat16()
    q = torch.randn((3, 4, 128), generator=g, device="cuda").bfloat16()

    def lazy(t):
        t = torch._lazy_clone(t)
        assert torch._C._is_cow_tensor(t)
        return t

    A.stepq_kv_append(KV, 0, lazy(pages), table, n, k, v)
    assert not bool(pages.any())
    own, rows = lazy(pages), (lazy(k), lazy(v))
    A.stepq_kv_append(KV, 0, own, table, n, *rows)              # rows are only read
    assert torch.equal(k, rows[0]) and torch._C._is_cow_tensor(rows[0]) and bool(own.any())
    zk = z(3, 2, 128)
    a, b = lazy(zk), lazy(zk)
    A.stepq_kv_read(KV, 0, own, table, n, a, b)
    assert not bool(zk.any()) and bool(a.any()) and bool(b.any())
    y, lse, ws = z(3, 4, 128), z(3, 4, dt=torch.float32), torch.zeros(A.stepq_kv_workspace_bytes(KV, 4, 3, 1 << 20), dtype=torch.uint8, device="cuda")
    ly, ll, lw = lazy(y), lazy(lse), lazy(ws)
    A.stepq_kv_attend(KV, 0, own, table, n + 1, q, ly, lse=ll, max_len=1 << 20, workspace=lw)
    assert not bool(y.any()) and not bool(lse.any()) and not bool(ws.any()) and bool(ly.any()) and bool(ll.any())
    both = lazy(q)                                              # outputs in place of the queries
    A.stepq_kv_attend(KV, 0, own, table, n + 1, both, both)
    assert torch.equal(both, ly) and not torch.equal(both, q)
    assert A.stepq_device_error() == 0
