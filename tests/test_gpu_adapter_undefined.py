"""Infinite and undefined values in the adapters' calls, at sizes that reach every kernel: what they enter is what 64-bit arithmetic makes of
them (infinite of the same sign, or undefined), everything else keeps its bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1
# rows, d_in, d_out, rank, adapters, order: a workgroup a row and sixteen columns a workgroup; tiles with few adapters among 32 rows and
# with many, of whole pieces and of odd widths
SIZES = [(96, 48, 80, 8, 5, "mixed"), (4200, 520, 520, 16, 6, "grouped"), (4200, 520, 520, 16, 40, "mixed"), (6000, 515, 523, 12, 6, "grouped"),
         (6000, 515, 523, 12, 40, "mixed"), (4200, 520, 520, 32, 3, "mixed")]
SUMS = ("dw0", "dbias", "dA", "dB")


def results(dims, d):
    from test_gpu_adapter import run_bwd, run_fwd
    out = {"y": run_fwd(dims, d)}
    out.update(run_bwd(dims, d))
    return {k: v.clone() for k, v in out.items()}


def in_64_bits(ref, P):
    x, w0, A, B, dy, index = (ref[k] for k in ("x", "w0", "A", "B", "dy", "index"))
    with np.errstate(all="ignore"):
        y, dx, dA, dB = x @ w0.T + ref["bias"], dy @ w0, np.zeros_like(A), np.zeros_like(B)
        for p in range(P):
            m = index == p
            u, v = x[m] @ B[p].T, dy[m] @ A[p]
            y[m] += u @ A[p].T
            dx[m] += v @ B[p]
            dA[p], dB[p] = dy[m].T @ u, v.T @ x[m]
        return {"y": y, "dx": dx, "dw0": dy.T @ x, "dbias": dy.sum(0), "dA": dA, "dB": dB}


def rows_of(ref, p):
    return np.nonzero(ref["index"] == p)[0]


def where_they_go(M, I, O, r, P, mix, value, dtype, outputs):
    import torch
    from test_gpu_adapter import problem
    dims, d, ref = problem(M, I, O, r, P, dtype, mix, seed=M + r)
    clean = results(dims, d)
    row = int(rows_of(ref, 2)[len(rows_of(ref, 2)) // 2])
    for name, where in (("A", (2, 7, 3)), ("B", (2, 3, 5)), ("x", (row, 11)), ("dy", (row, 13))):
        keep = d[name][where].clone()
        d[name][where] = value
        spoilt = dict(ref)
        spoilt[name] = ref[name].copy()
        spoilt[name][where] = value
        got, want = results(dims, d), in_64_bits(spoilt, P)
        d[name][where] = keep
        for k in outputs:
            w = torch.from_numpy(want[k]).cuda()
            fine = torch.isfinite(w)
            assert torch.equal(got[k][fine], clean[k][fine]), (name, k)
            if value == value:
                assert torch.equal(got[k][~fine].double().nan_to_num(nan=2.0, posinf=1.0, neginf=-1.0), w[~fine].nan_to_num(nan=2.0, posinf=1.0, neginf=-1.0)), (name, k)
            else:
                assert torch.isnan(got[k][~fine]).all(), (name, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,I,O,r,P,mix", SIZES)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_in_sums_over_the_rows(M, I, O, r, P, mix, value, dtype):
    where_they_go(M, I, O, r, P, mix, value, dtype, SUMS)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,I,O,r,P,mix", SIZES)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_in_rows(M, I, O, r, P, mix, value, dtype):
    where_they_go(M, I, O, r, P, mix, value, dtype, ("y", "dx"))
