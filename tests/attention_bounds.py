"""How far the attention kernels' outputs may be from the 64-bit ones, by counting roundings (test-side only).

A kernel forms scores s = scale q . k in fp32, weights w = exp(s - top) rounded to fp16, sums w v and w in fp32, and rounds the
quotient to fp16.  With u = 2^-24 (half a step of fp32) and h = 2^-11 (half a step of fp16), per output element

  weights      h sum_t p_t |v_t|, and 2^-25 of the largest weight for each one that is subnormal in fp16.  Where the denominator
               is the sum of the rounded weights, o moves by sum (w_t - p_t) (v_t - o) / sum w_t: h sum_t p_t (|v_t| + |o|)
  scores       a score is a sum of d products and a factor, each rounded: (d + 4) u scale sum |q| |k|; for 4-bit keys |k| is the
               size of what is subtracted, (code + |zero|) times the step.  The exponent's argument is rounded at the size of the
               score twice more, 4 u |s|; where it carries the logarithm of a value's step (up to 30 in size), that and the
               exponential are good to 2^-18.  A weight that is off by the factor 1 + e moves the output by at most
               e sum_t p_t (|v_t| + |o|).
  sums         n + 64 roundings of fp32 over n tokens at the size of what is summed: sum_t p_t |v_t|, for 4-bit values
               sum_t p_t (code + |zero|) step
  output       h |o|, or half a subnormal step, 2^-25

The 64-bit side's own error is negligible; products of these terms are inside the factor 1.02.
"""
import numpy as np

U, H = 2.0 ** -24, 2.0 ** -11


def attention_bound(q, k_size, v, v_size, o, p, s, scale, rounded_total=False):
    """q [n, d], k_size, v, v_size [m, d] (sizes as above), o [n, d], p [n, m], s [n, m] -> [n, d]."""
    n_keys, d = k_size.shape
    ds = (d + 4) * U * scale * (np.abs(q) @ k_size.T) + 4 * U * np.abs(s) + 2.0 ** -18
    e = np.where(p > 0, ds, 0).max(-1, initial=0)[:, None]
    v = np.abs(v)
    pv = p @ v
    subnormal = n_keys * 2.0 ** -25 * np.where((p > 0).any(-1)[:, None], v.max(0, initial=0)[None, :], 0)
    return 1.02 * (H * (pv + np.abs(o) * rounded_total) + e * (pv + np.abs(o)) + (n_keys + 64) * U * (p @ v_size) + subnormal + H * np.abs(o)) + 2.0 ** -25


def check_attention(got, o, bound, what=""):
    got = np.asarray(got, np.float64)
    assert got.shape == o.shape, (got.shape, o.shape)
    assert np.isfinite(got).all(), what + ": not finite"
    off = np.abs(got - o)
    worst = float((off / bound).max(initial=0))
    assert (off <= bound).all(), "%s: %.3g times the bound (off %.3g, largest value %.3g)" % (what, worst, off.max(), np.abs(o).max())
    return worst
