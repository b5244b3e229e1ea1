"""The kernels that block_linear and block_experts calls launch, on the CPU (as launches.py has them
for the layer's calls; run as a script for its child process)."""
import json
import os
import re
import subprocess
import sys
import tempfile

import launches as L

RECORDER = L.RECORDER + """
int hipFuncSetAttribute(const void* fn, int attr, int value) {
  (void)fn; (void)attr; (void)value;
  return 0;
}
"""


def block_launches(cases):
    """For each case, ("linear", T, n, k, quantised) or ("experts", T, E, k, d, f), the names of the
    kernels of one call, for instance tile_kernel<0, 64, 32, 2, 2, 4, false>."""
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "recorder.so")
        subprocess.run(["gcc", f"-DCUS={L.CUS}", "-shared", "-fPIC", "-O1", "-x", "c", "-", "-o", so],
                       input=RECORDER, text=True, check=True)
        res = subprocess.run([sys.executable, os.path.abspath(__file__)], text=True, check=True,
                             input=json.dumps(dict(so=so, lib=L.LIB, cases=cases)),
                             stdout=subprocess.PIPE)
    out = json.loads(res.stdout)
    names = sorted({n for one in out for n in one})
    # (what stays of the types of template and function arguments)
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
    lib, fake, big = X.lib(), ctypes.c_void_p(1 << 20), 1 << 44
    out = []
    for c in request["cases"]:
        rec.recorder_clear()
        if c[0] == "linear":
            T, n, k, quantised = c[1:]
            x = (None, k, fake, fake) if quantised else (fake, k, None, None)
            status = lib.xshare_block_linear(*x, T, n, k, fake, fake, fake, n, fake, big, None)
        else:
            T, E, k, d, f = c[1:]
            a = X.BlockExpertsArgs(struct_size=ctypes.sizeof(X.BlockExpertsArgs), T=T, top_k=k,
                                   n_experts=E, d=d, f=f, ldx=d, ldy=d, ws_bytes=big)
            for name, kind in a._fields_:
                if kind is ctypes.c_void_p and name != "stream":
                    setattr(a, name, fake)
            status = lib.xshare_block_experts(ctypes.byref(a))
        if status != 0:
            raise RuntimeError(f"status {status} for {c}")
        out.append([r.split()[0] for r in rec.recorder_text().decode().splitlines()])
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _child()
