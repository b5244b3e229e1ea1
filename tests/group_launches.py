"""The kernels that calls on groups of rows and adapters launch, on the CPU (as launches.py has them for
the layer's calls; run as a script for its child process)."""
import json
import os
import re
import subprocess
import sys
import tempfile

import launches as L
from block_launches import RECORDER


def group_launches(cases):
    """For each case, ("linear" | "x" | "w", P, E, n, k), ("adapters" | "backward", T, L, r, n, d),
    ("order", T, k, E) or ("beside", P, n, k, ld, apart), the names of the kernels of one call, for instance
    tile_kernel<0, 64, 32, 4, 1, 4, 64>."""
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "recorder.so")
        subprocess.run(["gcc", f"-DCUS={L.CUS}", "-shared", "-fPIC", "-O1", "-x", "c", "-", "-o", so],
                       input=RECORDER, text=True, check=True)
        res = subprocess.run([sys.executable, os.path.abspath(__file__)], text=True, check=True,
                             input=json.dumps(dict(so=so, lib=L.LIB, cases=cases)),
                             stdout=subprocess.PIPE)
    out = json.loads(res.stdout)
    names = sorted({n for one in out for n in one})
    short = {n: re.sub(r"\([^()]*\)", "", s) for n, s in zip(names, L.short_names(names))}
    return [[short[n] for n in one] for one in out]


def _child():
    import ctypes
    import types
    request = json.load(sys.stdin)
    rec = ctypes.CDLL(request["so"], mode=ctypes.RTLD_GLOBAL)   # ahead of the HIP runtime
    rec.recorder_text.restype = ctypes.c_char_p
    sys.modules["torch"] = types.ModuleType("torch")            # the binding's types only
    sys.path.insert(0, os.path.join(L.ROOT, "paper_2602_07265_amd"))
    import xshare as X
    X.LIB_PATH = request["lib"]
    lib, fake, far, big = X.lib(), ctypes.c_void_p(1 << 20), ctypes.c_void_p(1 << 50), 1 << 44
    out = []
    for what, *c in request["cases"]:
        rec.recorder_clear()
        if what == "order":
            T, k, E = c
            status = lib.xshare_expert_order(fake, T, k, E, fake, fake, fake, fake, big, None)
        elif what == "beside":
            P, n, k, ld, apart = c                     # y lies `apart` elements from x, in rows of ld
            status = lib.xshare_grouped_linear(fake, ld, fake, fake, P, 2, n, k,
                                               ctypes.c_void_p(fake.value + 2 * apart), ld, fake, big,
                                               None)
        elif what in ("adapters", "backward"):
            T, N, r, n, d = c
            cols = n if what == "adapters" else d
            a = X.AdaptersArgs(struct_size=ctypes.sizeof(X.AdaptersArgs), T=T, n_adapters=N, rank=r,
                               n=n, d=d, ldx=d, ld_out=cols, lddy=n, ws_bytes=big)
            for name in ("x", "a", "b", "ids", "out", "dy", "da", "db", "ws"):
                setattr(a, name, far if name == "out" else fake)
            call = lib.xshare_adapters if what == "adapters" else lib.xshare_adapters_backward
            status = call(ctypes.byref(a))
        else:
            P, E, n, k = c
            if what == "linear":
                status = lib.xshare_grouped_linear(fake, k, fake, fake, P, E, n, k, far, n, fake,
                                                   big, None)
            elif what == "x":
                status = lib.xshare_grouped_linear_backward_x(fake, n, fake, fake, P, E, n, k, far,
                                                              k, fake, big, None)
            else:
                status = lib.xshare_grouped_linear_backward_w(fake, n, fake, k, fake, P, E, n, k,
                                                              fake, 0, 0, fake, big, None)
        if status != 0:
            raise RuntimeError(f"status {status} for {what} {c}")
        out.append([r.split()[0] for r in rec.recorder_text().decode().splitlines()])
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _child()
