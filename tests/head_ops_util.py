"""Error bounds of the LM-head operators' GPU tests, from the arithmetic of the kernels.

u = 2^-24 is half a step of binary32 relative to the value, e = 2^-8 half a step of bfloat16.
  logits   an fp32 sum of d exact (bf16) or rounded (fp32) products.  Taken 16 terms at a time or one by one, each addition is off
           by at most 2 u (rounding or truncation) of the running sum, which sum |h w| bounds:
           tol_z = 2 u (n_adds + 8) max sum |h w|, n_adds = d / 16 + 5 for bf16, d for fp32.
  sums     of V positive exponentials (each off by 4 u for exp, and by the error of its fp32 argument,
           at most 2 u times the largest distance from the maximum): tol_l = u (2 V / 32 + 64 + 4 range), relative.
  lse      tol_z + tol_l + 4 u |lse|.
  entropy  sum p |d entropy / dz| <= 2 log V, and log l - u / l carries the sums' errors with weights up to 1 + log V:
           4 (1 + log V) (tol_z + tol_l).
"""
import numpy as np

U = 2.0 ** -24
E_BF16 = 2.0 ** -8


def tolerances(H, W, on, z, bf16):
    """tol_z, tol_l of a problem (float64 arrays; rows off are left out)."""
    d = H.shape[1]
    Hc = np.abs(np.where(on[:, None], H, 0.0))
    big = float((Hc @ np.abs(W).T).max()) if on.any() else 0.0
    adds = d / 16 + 5 if bf16 else d
    tol_z = 2 * U * (adds + 8) * big
    spread = float((z.max(axis=1) - z.min(axis=1)).max())
    tol_l = U * (2 * z.shape[1] / 32 + 64 + 4 * spread)
    return tol_z, tol_l


TWO_TERM_ROWS = 128      # batches of up to this many rows form dz as two bf16 terms


def check_grads(got_H, got_W, want, W, H, tol, bf16, dW_bf16=None):
    """Elementwise: dz off by its rounding (bf16) and by `tol` of its terms (exponentials of logits that are off), plus `tol` itself times
    the factor of a difference of logarithms (want[3]: that difference may be 0, as for one token, while its two sides are off
    by tol); the fp32 sum of the contraction by 2 u per addition, the result by its own rounding; and, for the whole, relative L2
    within twice a rounding where no such difference is left out.  dz in two terms is off by half a step of the second: 2^-16."""
    dH, dW, terms = want[:3]
    coef = want[3] if len(want) > 3 else np.zeros_like(terms)
    dW_bf16 = bf16 if dW_bf16 is None else dW_bf16
    two = bf16 and H.shape[0] <= TWO_TERM_ROWS
    e = 0.0 if not bf16 else 2.0 ** -16 if two else E_BF16
    for got, ref, mag, dif, n, rounded in ((got_H, dH, terms @ np.abs(W), coef @ np.abs(W), terms.shape[1], bf16),
                                           (got_W, dW, terms.T @ np.abs(H), coef.T @ np.abs(H), terms.shape[0], dW_bf16)):
        rel = e + 1.01 * tol + 2 * U * (n + 8)
        off = rel * mag + 1.02 * tol * dif
        bound = off + (E_BF16 if rounded else U) * (np.abs(ref) + off) + 2.0 ** -126
        err = np.abs(got - ref)
        assert np.all(err <= bound), (float((err / bound).max()), np.unravel_index(int((err / bound).argmax()), err.shape))
        norm = np.linalg.norm(ref)
        if bf16 and norm > 0:
            allowed = (1.01 * tol + e) * np.linalg.norm(mag) + E_BF16 * norm if two else 2 * E_BF16 * norm
            assert np.linalg.norm(got - ref) <= allowed + 1.02 * tol * np.linalg.norm(dif)
