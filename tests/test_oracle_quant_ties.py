"""INT8 codes by float32 arithmetic are nearest codes: bf16 values have 8 bits, so that 127 x / a
is either halfway between two codes or at least 1 / (2 * 255) of its step's parts away from
there, which two float32 roundings do not bridge.  Halfway, either neighbour may come out."""
import numpy as np

from oracle import cache_ops as co


def test_int8_codes_are_nearest():
    m = np.arange(128, 256)
    halfway = off_even = 0
    for j in range(0, 10):                                   # x = X 2^-j, a = A
        X, A = np.meshgrid(m, m)
        X, A = X.ravel(), A.ravel()
        keep = X <= A * 2 ** j
        X, A = X[keep], A[keep]
        rows = np.stack([A, X * 2.0 ** -j], axis=1)[:, :, None].transpose(0, 2, 1).reshape(len(A), 1, 2)
        codes, _ = co.quantise(rows, "int8")
        c = codes.view(np.int8)[:, 0, 1].astype(np.int64)
        miss = 2 * np.abs(c * A * 2 ** j - 127 * X)          # twice the distance, times a 2^j
        assert np.all(miss <= A * 2 ** j)
        tie = miss == A * 2 ** j
        halfway += int(tie.sum())
        off_even += int((tie & (c % 2 != 0)).sum())
    assert halfway > 0 and off_even > 0                      # (the stated arithmetic, not ties to even of the quotient)
