"""Calls on a prefix store made without a GPU: a child process loads
launch_recorder.c and a few more stand-ins ahead of the library, creates the
store in a pool that nothing reads, and makes the calls.

``store_calls(store, calls)``: store is (layers, kv heads, head dim, doc_len,
format); a call is (function, structure or None, fields) and becomes
``function(handle, [layer,] structure, NULL)``.  Gives status, error text and
launches of each."""
import ctypes
import functools
import json
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)

STANDINS = """
#include <stddef.h>
int hipMemsetAsync(void *p, int v, size_t n, void *s) { return 0; }
int hipMemcpyAsync(void *a, const void *b, size_t n, int k, void *s) {
  return 0;
}
int hipStreamSynchronize(void *s) { return 0; }
int hipDeviceGetAttribute(int *v, int what, int dev) { *v = 256; return 0; }
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int *n, const void *f, int b,
                                                 size_t lds) {
  *n = 2;
  return 0;
}
int hipModuleOccupancyMaxActiveBlocksPerMultiprocessor(int *n, void *f, int b,
                                                       size_t lds) {
  *n = 2;
  return 0;
}
"""


@functools.lru_cache(maxsize=None)
def _standins():
    folder = tempfile.mkdtemp(prefix="store_")
    src = os.path.join(folder, "standins.c")
    with open(src, "w") as f:
        f.write(STANDINS)
    out = os.path.join(folder, "libstandins.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", out, src], check=True)
    return out


def store_calls(store, calls):
    from operator_launches import demangled, recorder
    r = subprocess.run([sys.executable, os.path.abspath(__file__), recorder(),
                        _standins()], input=json.dumps([store, calls]),
                       cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    out = json.loads(r.stdout.splitlines()[-1])
    for call in out:
        lines = [x.split() for x in call.pop("record").splitlines()]
        call["launches"] = [
            dict(zip(("gx", "gy", "gz", "bx", "by", "bz", "lds"),
                     map(int, f[1:8])), kernel=demangled(f[8]))
            for f in lines if f[0] == "launch"]
    return out


def _child(*libraries):
    loaded = [ctypes.CDLL(p, mode=ctypes.RTLD_GLOBAL) for p in libraries]
    R = loaded[0]
    R.record_take.restype = ctypes.c_char_p
    sys.path.insert(0, ROOT)
    import numpy as np
    import paper_2609_03311_amd as D
    L = D.lib()
    (layers, hkv, d, doc_len, fmt), calls = json.load(sys.stdin)
    lens = np.asarray(doc_len, np.int32)
    desc, _keep = D._desc(layers, hkv, d, lens)
    h = ctypes.c_void_p(0)
    status = L.dopr_store_create_as(ctypes.byref(desc), fmt, 1 << 20, 1 << 60,
                                    None, ctypes.byref(h))
    assert status == 0, L.dopr_last_error()
    out = []
    for name, struct, fields in calls:
        R.record_take()
        fn = getattr(L, name)
        if struct is None:
            status = fn(h, *fields, None)
        else:
            a = getattr(D, struct)()
            layer = fields.pop("_layer", None)
            for k, v in fields.items():
                setattr(a, k, v)
            args = [h] + ([] if layer is None else [layer])
            status = fn(*args, ctypes.byref(a), None)
        out.append({"status": status,
                    "error": L.dopr_last_error().decode() if status else "",
                    "record": R.record_take().decode()})
    print(json.dumps(out))


if __name__ == "__main__":
    _child(*sys.argv[1:])
