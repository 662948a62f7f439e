"""A call into the library leaves the interpreter to other threads while it
waits: a stand-in for the runtime holds the call until another Python thread has
let it go on, for two seconds at most."""
import ctypes
import os
import subprocess
import sys
import threading
import time

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)

WAITS = """
#include <unistd.h>
volatile int armed, inside, go, missed;
int hipGetDevice(int *d) {
  *d = 0;
  if (!armed) return 0;
  inside = 1;
  for (int i = 0; i < 2000 && !go; ++i) usleep(1000);
  if (!go) missed = 1;
  armed = 0;
  return 0;
}
"""


@pytest.mark.parametrize("call", ["attention", "read back"])
def test_other_threads_run_beside_a_call(call, tmp_path):
    from operator_launches import recorder
    from store_calls import _standins
    src, lib = tmp_path / "waits.c", tmp_path / "libwaits.so"
    src.write_text(WAITS)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(lib), str(src)],
                   check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), call,
                        str(lib), recorder(), _standins()], cwd=ROOT,
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-3000:]
    assert r.stdout.splitlines()[-1] == "inside 1 missed 0"


def _child(call, *libraries):
    waits = [ctypes.CDLL(p, mode=ctypes.RTLD_GLOBAL) for p in libraries][0]
    word = {n: ctypes.c_int.in_dll(waits, n)
            for n in ("armed", "inside", "go", "missed")}
    sys.path.insert(0, ROOT)
    import numpy as np
    import torch
    import paper_2609_03311_amd as D
    desc, _keep = D._desc(1, 2, 128, np.array([40], np.int32))
    h = ctypes.c_void_p(0)
    assert D.lib().dopr_store_create_as(ctypes.byref(desc), 1, 1 << 20,
                                        1 << 60, None, ctypes.byref(h)) == 0

    class Store:
        handle, n_kv_heads, head_dim = h.value, 2, 128

    class Stream:
        cuda_stream = 0

    ids = torch.zeros(1, dtype=torch.int32)
    cu = torch.tensor([0, 3], dtype=torch.int32)
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    ws = torch.zeros((1 << 20) + 256, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:][:1 << 20]

    def let_go():
        while not word["inside"].value:
            time.sleep(0.001)
        word["go"].value = 1

    other = threading.Thread(target=let_go, daemon=True)
    other.start()
    word["armed"].value = 1
    if call == "attention":
        D.dopr_prefix_attn(Store, 0, ids, cu, x, x, x, None, None, x, ws,
                           max_tokens=3, stream=Stream())
    else:
        D.dopr_gather_prefix(Store, 0, ids, torch.tensor([0, 40]), x, x,
                             stream=Stream())
    print("inside", word["inside"].value, "missed", word["missed"].value)
    sys.stdout.flush()
    os._exit(0)


if __name__ == "__main__":
    _child(*sys.argv[1:])
