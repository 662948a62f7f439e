"""What the operators' calls launch, found out without a GPU: a child process
loads launch_recorder.c ahead of the library and makes the calls with addresses
that nothing reads.

``launches(calls)`` takes (function, argument structure, fields) triples and
gives, for each call, its status, its error text, the kernels it launches and
the limits of dynamic LDS it raises.  A fourth item of a call is a dict: the
device it is made on, and whether raising a limit is refused there."""
import ctypes
import functools
import json
import os
import re
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@functools.lru_cache(maxsize=None)
def recorder():
    folder = tempfile.mkdtemp(prefix="recorder_")
    out = os.path.join(folder, "librecorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", out,
                    os.path.join(HERE, "launch_recorder.c")], check=True)
    return out


@functools.lru_cache(maxsize=None)
def demangled(name):
    """A kernel's name with its template's arguments."""
    text = subprocess.run(["c++filt", name], capture_output=True, text=True,
                          check=True).stdout.strip()
    m = re.search(r"(k_\w+)(<.*?>)?\(", text)
    short = m.group(1) + (m.group(2) or "") if m else text
    return re.sub(r"dopr::|\(anonymous namespace\)::", "", short)


def _run(calls):
    r = subprocess.run([sys.executable, os.path.abspath(__file__),
                        recorder()], input=json.dumps(calls), cwd=ROOT,
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.splitlines()[-1])


def kernels():
    """The names of the library's kernels."""
    return {demangled(name) for name in _run(None).split() if "dopr" in name}


def launches(calls):
    out = _run(calls)
    for call in out:
        lines = [line.split() for line in call.pop("record").splitlines()]
        call["launches"] = [
            dict(zip(("gx", "gy", "gz", "bx", "by", "bz", "lds"),
                     map(int, f[1:8])), kernel=demangled(f[8]))
            for f in lines if f[0] == "launch"]
        call["limits"] = [(int(f[1]), int(f[2]), demangled(f[3]))
                          for f in lines if f[0] == "limit"]
    return out


def _child(path):
    R = ctypes.CDLL(path, mode=ctypes.RTLD_GLOBAL)
    R.record_take.restype = ctypes.c_char_p
    sys.path.insert(0, ROOT)
    import paper_2609_03311_amd as D
    L = D.lib()
    R.record_kernels.restype = ctypes.c_char_p
    calls, out = json.load(sys.stdin), []
    if calls is None:
        print(json.dumps(R.record_kernels().decode()))
        return
    for name, struct, fields, *more in calls:
        env = more[0] if more else {}
        R.record_device(env.get("device", 0))
        R.record_refuse(int(env.get("refuse", False)))
        a = getattr(D, struct)()
        for k, v in fields.items():
            setattr(a, k, v)
        status = getattr(L, name)(ctypes.byref(a), None)
        out.append({"status": status,
                    "error": L.dopr_last_error().decode() if status else "",
                    "record": R.record_take().decode()})
    print(json.dumps(out))


if __name__ == "__main__":
    _child(sys.argv[1])
