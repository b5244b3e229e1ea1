"""Which matrices of rows count as overlapping, on the host: one of a single row has no distance between
rows, whatever a call is given for it.  Launches are recorded, pointers never followed."""
import ctypes
import json
import os
import subprocess
import sys
import tempfile

import launches as L
from block_launches import RECORDER

AT = 1 << 20


def _statuses(cases):
    """Each case's status: ("dispatch", T, k, d, x, ldx, out, ldo), ("linear", P, n, k, x, ldx, y, ldy),
    ("base", T, n, base, ld_base, out, ld_out); addresses in elements from one place on."""
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "recorder.so")
        subprocess.run(["gcc", f"-DCUS={L.CUS}", "-shared", "-fPIC", "-O1", "-x", "c", "-", "-o", so],
                       input=RECORDER, text=True, check=True)
        res = subprocess.run([sys.executable, os.path.abspath(__file__)], text=True, check=True,
                             input=json.dumps(dict(so=so, lib=L.LIB, cases=cases)),
                             stdout=subprocess.PIPE)
    return json.loads(res.stdout)


def _child():
    import types
    request = json.load(sys.stdin)
    ctypes.CDLL(request["so"], mode=ctypes.RTLD_GLOBAL)         # ahead of the HIP runtime
    sys.modules["torch"] = types.ModuleType("torch")            # the binding's types only
    sys.path.insert(0, os.path.join(L.ROOT, "paper_2602_07265_amd"))
    import xshare as X
    X.LIB_PATH = request["lib"]
    lib, fake, far, big, out = X.lib(), ctypes.c_void_p(AT), ctypes.c_void_p(1 << 50), 1 << 44, []
    at = lambda elements: ctypes.c_void_p(AT + 2 * elements)  # noqa: E731
    for what, *c in request["cases"]:
        if what == "dispatch":
            T, k, d, x, ldx, o, ldo = c
            status = lib.xshare_dispatch(at(x), ldx, 1, T, k, d, far, at(o), ldo, None)
        elif what == "linear":
            P, n, k, x, ldx, y, ldy = c
            status = lib.xshare_grouped_linear(at(x), ldx, far, far, P, 1, n, k, at(y), ldy, far, big,
                                               None)
        else:
            T, n, base, ld_base, o, ld_out = c
            a = X.AdaptersArgs(struct_size=ctypes.sizeof(X.AdaptersArgs), T=T, n_adapters=2, rank=16,
                               n=n, d=64, ldx=64, ld_base=ld_base, ld_out=ld_out, ws_bytes=big,
                               base=at(base), out=at(o))
            for name in ("x", "a", "b", "ids", "ws"):
                setattr(a, name, far)
            status = lib.xshare_adapters(ctypes.byref(a))
        out.append(status)
    json.dump(out, sys.stdout)


OK, EINVAL = 0, 1
CASES = [
    # one token beside the rows that it goes to, in one buffer of rows of 128
    (("dispatch", 1, 4, 64, 128 + 64, 64, 0, 128), OK), (("dispatch", 1, 4, 64, 0, 64, 64, 128), OK),
    (("dispatch", 1, 4, 64, 128 + 64, 4096, 0, 128), OK),
    (("dispatch", 1, 4, 64, 128, 64, 0, 128), EINVAL), (("dispatch", 1, 4, 64, 63, 64, 64, 128), EINVAL),
    (("dispatch", 1, 4, 64, 128 + 63, 64, 0, 128), EINVAL),
    (("dispatch", 1, 4, 64, 128 + 65, 64, 0, 128), EINVAL),
    # past the last row's end, and a single row on either side
    (("dispatch", 1, 4, 64, 3 * 128 + 64, 64, 0, 128), OK), (("dispatch", 1, 1, 64, 64, 64, 0, 128), OK),
    (("dispatch", 1, 1, 64, 63, 64, 0, 128), EINVAL),
    (("linear", 1, 40, 64, 0, 64, 64, 104), OK), (("linear", 1, 40, 64, 0, 104, 56, 40), EINVAL),
    # more rows, differently far apart, in the same memory
    (("dispatch", 2, 2, 64, 64, 256, 0, 128), EINVAL),
    # a single row in place
    (("base", 1, 40, 0, 48, 0, 40), OK), (("base", 1, 40, 0, 40, 0, 4096), OK),
    (("base", 1, 40, 8, 40, 0, 48), EINVAL), (("base", 2, 40, 0, 48, 0, 40), EINVAL)]


def test_a_single_row_overlaps_what_it_shares_memory_with():
    got = _statuses([c for c, _ in CASES])
    assert got == [want for _, want in CASES], \
        [(c, s) for (c, want), s in zip(CASES, got) if s != want]


if __name__ == "__main__":
    _child()
