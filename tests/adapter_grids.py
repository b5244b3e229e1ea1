"""The kernels that adapters calls launch and their grids, on the CPU (run as a script for its child
process): group_launches.py gives the names alone."""
import ctypes
import json
import os
import re
import subprocess
import sys
import tempfile

import launches as L
from block_launches import RECORDER


def adapter_grids(cases):
    """For each case (backward, T, adapters, r, n, d): [(kernel, (x, y, z))] of one call without base."""
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "recorder.so")
        subprocess.run(["gcc", f"-DCUS={L.CUS}", "-shared", "-fPIC", "-O1", "-x", "c", "-", "-o", so],
                       input=RECORDER, text=True, check=True)
        res = subprocess.run([sys.executable, os.path.abspath(__file__)], text=True, check=True,
                             input=json.dumps(dict(so=so, lib=L.LIB, cases=cases)),
                             stdout=subprocess.PIPE)
    out = json.loads(res.stdout)
    names = sorted({n for one in out for n, _ in one})
    short = {n: re.sub(r"\([^()]*\)", "", s) for n, s in zip(names, L.short_names(names))}
    return [[(short[n], tuple(g)) for n, g in one] for one in out]


def _child():
    import types
    request = json.load(sys.stdin)
    rec = ctypes.CDLL(request["so"], mode=ctypes.RTLD_GLOBAL)   # ahead of the HIP runtime
    rec.recorder_text.restype = ctypes.c_char_p
    sys.modules["torch"] = types.ModuleType("torch")            # the binding's types only
    sys.path.insert(0, os.path.join(L.ROOT, "paper_2602_07265_amd"))
    import xshare as X
    X.LIB_PATH = request["lib"]
    lib, fake, far, out = X.lib(), ctypes.c_void_p(1 << 20), ctypes.c_void_p(1 << 50), []
    for backward, T, N, r, n, d in request["cases"]:
        rec.recorder_clear()
        a = X.AdaptersArgs(struct_size=ctypes.sizeof(X.AdaptersArgs), T=T, n_adapters=N, rank=r, n=n,
                           d=d, ldx=d, ld_out=d if backward else n, lddy=n, ws_bytes=1 << 44)
        for name in ("x", "a", "b", "ids", "out", "dy", "da", "db", "ws"):
            setattr(a, name, far if name == "out" else fake)
        status = (lib.xshare_adapters_backward if backward else lib.xshare_adapters)(ctypes.byref(a))
        if status != 0:
            raise RuntimeError(f"status {status} for {backward, T, N, r, n, d}")
        rows = [line.split() for line in rec.recorder_text().decode().splitlines()]
        out.append([(one[0], [int(v) for v in one[1:4]]) for one in rows])
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _child()
