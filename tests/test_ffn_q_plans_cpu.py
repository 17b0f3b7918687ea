"""The plan queries of the 8-bit products, and that the GPU tests' cases are every plan there is."""
import ctypes as C
import os

import pytest

import qplans

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2510_11331_amd", "libsd.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libsd.so not built (run __graft_entry__.build())")

ROWS = [1, 5, 16, 17, 32, 33, 40, 48, 49, 64, 65, 70, 80, 96, 100, 128, 129, 160, 192, 200, 256, 257, 320, 384, 400, 512, 520, 640, 769,
        1000, 1024, 1200, 1500, 1537, 2048, 2100, 3000, 4096, 4200, 8192, 20000, 1 << 22]
COLS = [1, 16, 48, 130, 300, 512, 520, 700, 1000, 1024, 1040, 1500, 2048, 2100, 2800, 3000, 4096, 4100, 4200, 5000, 5120, 6000, 8192, 8200,
        11008, 12000, 13824, 16130, 16400, 18000, 22016, 27648, 32000, 60000]
DEPTHS = [1, 130, 140, 300, 700, 1100, 1300, 1500, 2048, 2100, 2560, 2816, 3200, 4096, 4200, 5130, 6000, 8192, 8400, 10000, 10300, 11008, 13824,
          16384, 16500, 28672, 40000, 262144]


@needs_lib
def test_cases_are_the_plans_they_name():
    for kind, cases in (("linear", qplans.LINEAR), ("gate_up", qplans.GATE_UP)):
        for fast, rows, cols, ranges, M, N, K in cases:
            assert qplans.plan(kind, M, N, K, fast) == qplans.expected(fast, rows, cols, ranges, M), (kind, M, N, K)
            blocks, width = -(-K // 128), N if kind == "linear" else 2 * N
            assert K % 128 and blocks >= 5 * ranges and (ranges > 1 or blocks >= 9)
            if M > 64:
                assert M > rows and M % rows and width > cols and width % cols


@needs_lib
def test_cases_cover_every_plan():
    """No plan of any of these sizes is missing among the cases."""
    known = {"linear": set(), "gate_up": set()}
    for kind, cases in (("linear", qplans.LINEAR), ("gate_up", qplans.GATE_UP)):
        for fast, rows, cols, ranges, M, _, _ in cases:
            known[kind].add(qplans.expected(fast, rows, cols, ranges, M))
    for M in ROWS:
        for N in COLS:
            for K in DEPTHS:
                for fast in (0, 1):
                    assert qplans.plan("linear", M, N, K, fast) in known["linear"], (M, N, K, fast)
                    if N >= 16:
                        assert qplans.plan("gate_up", M, N // 16 * 16, K, fast) in known["gate_up"], (M, N, K, fast)


@needs_lib
def test_plan_queries():
    """Up to 64 rows every plan is exact, whatever K is; sizes that the calls refuse; the K ranges' sums fit the workspace."""
    from paper_2510_11331_amd import _lib
    L, p = _lib.lib(), _lib.LinearQPlan()
    for M in ROWS:
        for K in DEPTHS:
            for fast in (0, 1):
                few = qplans.plan("linear", M, 4096, K, fast), qplans.plan("gate_up", M, 4096, K, fast)
                assert all(x[1] == (fast and M > 64) and x[0] == (M <= 64 and K <= 16384) for x in few)
                assert L.sd_linear_q_workspace_bytes(M, 4096, K) >= (few[0][4] > 1) * few[0][4] * M * 4096 * 4
    for M, N, K in ((0, 16, 1), (-1, 16, 1), ((1 << 22) + 1, 16, 1), (1, 0, 1), (1, 16, 0), (1, 16, (1 << 18) + 1)):
        assert L.sd_plan_linear_q(M, N, K, 0, C.byref(p)) == L.sd_plan_gate_up_q(M, N, K, 0, C.byref(p)) == _lib.SD_EINVAL
    assert L.sd_plan_gate_up_q(1, 24, 1, 0, C.byref(p)) == _lib.SD_EINVAL
    assert L.sd_plan_linear_q(1, 16, 1, 0, None) == L.sd_plan_gate_up_q(1, 16, 1, 0, None) == _lib.SD_EINVAL


@needs_lib
def test_fast_calls_refuse():
    """What the plain calls refuse.  The pointers are never dereferenced."""
    from paper_2510_11331_amd import _lib
    L, E, A = _lib.lib(), _lib.SD_EINVAL, 1 << 20
    n = L.sd_linear_q_workspace_bytes(100, 64, 11008)
    ln = dict(M=100, N=64, K=11008, q=A, exps=A, w=A, add=A, out=A, ldo=64, dtype=_lib.SD_DTYPE_F32, ws=A, n=n)
    for bad in (dict(M=-1), dict(N=0), dict(K=(1 << 18) + 1), dict(q=None), dict(out=None), dict(ldo=63), dict(dtype=2), dict(w=A + 8),
                dict(add=A + 2), dict(ws=None), dict(n=n - 1), dict(exps=A + 2)):
        assert L.sd_linear_q_fast(*{**ln, **bad}.values(), None) == E, bad
    assert L.sd_linear_q_fast(*{**ln, "M": 0, "out": None}.values(), None) == _lib.SD_OK
    n = L.sd_gate_up_q_workspace_bytes(2, 64, 64)
    gu = dict(M=2, F=64, K=64, q=A, exps=A, w=A, q_out=A, exps_out=A, ws=A, n=n)
    for bad in (dict(M=-1), dict(F=72), dict(K=0), dict(w=None), dict(exps_out=None), dict(ws=None), dict(n=n - 1), dict(q_out=A + 8)):
        assert L.sd_gate_up_q_fast(*{**gu, **bad}.values(), None) == E, bad
    assert L.sd_gate_up_q_fast(*{**gu, "M": 0, "q": None}.values(), None) == _lib.SD_OK
