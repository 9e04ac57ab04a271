"""Failed launches of the residual norms, token log probabilities and distillation are reported, whichever launch of a call it is
(no GPU: the runtime's launch call is a stand-in, as in test_launch_status.py)."""
import os
import subprocess
import sys

import pytest

from paper_2410_06511_amd import f8
from test_launch_status import stand_in  # noqa: F401 (the fixture)

CALLS = r"""
import ctypes as C, sys
stand_in = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
l = C.CDLL(sys.argv[2])
top = 1 << 32
def at(nbytes=1 << 30):     # addresses apart from each other
    global top
    top += 2 * nbytes
    return C.c_void_p(top)
i, f, size = C.c_int64, C.c_float, C.c_size_t
def ws(n=1 << 30): return [at(), size(n)]
def res(M, D, G, amax):
    return l.f8_residual_norm(at(), i(D), at(), i(D), i(M), i(D), at(), at() if G else None, i(G), at(), f(1), f(1), f(1e-5), at(), i(D), at(), i(D), at(), at(), at() if amax else None, *ws(), None)
def bwd(M, D, G, sums, amax):
    g = lambda: at() if sums else None
    return l.f8_residual_norm_bwd(at(), i(D), at(), i(D), at(), i(D), at(), i(D), i(M), i(D), at(), at() if G else None, i(G), at(), at(), at(), f(1), f(1), at(), i(D), at(), i(D), g(), g() if G else None, g(), at() if amax else None, *ws(), None)
def logp(M, V, k): return l.f8_token_logprobs(at(), i(V), i(M), i(V), f(1), at(), at(), at(), at(), i(k), at(), at(), *ws(), None)
def logp_bwd(M, V, amax): return l.f8_token_logprobs_bwd(at(), i(V), i(M), i(V), f(1), at(), at(), at(), at(), at(), at(), i(V), i(V), at() if amax else None, *ws(), None)
def kd(M, V): return l.f8_distill(at(), i(V), i(M), i(V), f(1), at(), at(), i(16), 1, f(1), at(), at(), at(), at(), *ws(), None)
def kd_bwd(M, V, amax): return l.f8_distill_bwd(at(), i(V), i(M), i(V), f(1), at(), at(), i(16), 1, f(1), at(), at(), at(), at(), at(), i(V), i(V), at() if amax else None, *ws(), None)
call = eval("lambda: " + sys.argv[3])
stand_in.f8_test_reset(-1)
status, n = call(), stand_in.f8_test_launches()
seen = []
for k in range(n):
    stand_in.f8_test_reset(k)
    seen.append(call())
print(status, n, *seen)
"""

# call -> launches: the gains' sums and the maxima take one of their own, rows that blocks share are joined by one
LAUNCHES = {
    "res(64, 4096, 0, 0)": 1, "res(64, 4096, 2, 1)": 2, "res(64, 512, 64, 1)": 2, "res(0, 512, 0, 1)": 1, "res(0, 512, 0, 0)": 0,
    "bwd(64, 4096, 0, 0, 0)": 1, "bwd(64, 4096, 0, 1, 0)": 2, "bwd(64, 4096, 4, 1, 1)": 2, "bwd(64, 4096, 64, 0, 1)": 2, "bwd(2000, 1024, 2000, 1, 1)": 2,
    "bwd(0, 4096, 4, 1, 1)": 2,
    "logp(1, 131072, 20)": 2, "logp(600, 32768, 20)": 1, "logp(600, 131080, 0)": 2, "logp(0, 32768, 20)": 0,
    "logp_bwd(64, 32768, 0)": 1, "logp_bwd(5000, 32768, 1)": 2, "logp_bwd(0, 32768, 1)": 1,
    "kd(1, 131072)": 2, "kd(600, 32768)": 1, "kd_bwd(64, 32768, 1)": 2,
}


@pytest.mark.parametrize("call", LAUNCHES)
def test_a_failed_launch_is_reported(stand_in, call):  # noqa: F811
    r = subprocess.run([sys.executable, "-c", CALLS, stand_in, os.path.abspath(f8.LIB_PATH), call], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    status, n, *seen = map(int, r.stdout.split())
    assert (status, n) == (0, LAUNCHES[call])
    assert seen == [6] * n  # F8_ERR_LAUNCH
