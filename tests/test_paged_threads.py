"""The paged cache's calls let other Python threads run while the library has them: a launch may wait for the GPU to take
it, and what the GPU waits for may be a host function in Python."""
import ctypes
import subprocess
import threading
import time

import pytest

from test_paged_binding import AT, I32, T, append, attend, calls, rows, table  # noqa: F401

SLOW = r"""
#include <unistd.h>
static volatile int inside, go;
int called(void) { return inside; }
void let_go(void) { go = 1; }
void again(void) { inside = go = 0; }
/* waits until somebody lets it go, three seconds at most */
int slow(void) {
  inside = 1;
  for (int i = 0; i < 3000 && !go; ++i) usleep(1000);
  return go ? 7 : 9;
}
"""


@pytest.fixture(scope="module")
def slow(tmp_path_factory):
    d = tmp_path_factory.mktemp("slow")
    (d / "slow.c").write_text(SLOW)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(d / "slow.so"), str(d / "slow.c")], check=True)
    return ctypes.CDLL(str(d / "slow.so"))


@pytest.mark.parametrize("which", ["append", "attend", "read"])
def test_other_threads_run_during_a_call(calls, slow, which):  # noqa: F811
    m = calls[0]
    import torch
    at = ctypes.cast(slow.slow, ctypes.c_void_p).value
    m.init(at, at, at, torch.int32, torch.float32, torch.bfloat16)
    slow.again()

    def other():
        while not slow.called():
            time.sleep(0.001)
        slow.let_go()

    t = threading.Thread(target=other)
    t.start()
    try:
        rc = {"append": lambda: append(m), "attend": lambda: attend(m),
              "read": lambda: m.read(*AT, table(), T((2,), I32), rows(), rows(), None, None, 0)}[which]()
    finally:
        slow.let_go()
        t.join()
    assert rc == 7
