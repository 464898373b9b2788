"""What the paged cache's compiled binding does beside the calls: it lets other Python threads run."""
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
