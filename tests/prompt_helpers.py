"""Bounds shared by the tests of the attention entry points of moeflow_prompt.h."""
import numpy as np

from paper_2410_17954_amd import synth


def values(a):
    return synth.values(a) if a.dtype == np.uint16 else a.astype(np.float64)


def draw(g, dtype, *shape, std=1.0):
    a = (std * g.standard_normal(shape)).astype(np.float32)
    return synth.bf16_bits(a) if dtype == "bf16" else a


def check_row(out, lse, ref, ref_lse, q, k, v, scale, dtype):
    """One query q [D] over k, v [n, D] (float64 of the exact inputs). With weights w_i:
    * a score is a float32 sum of D products (3 D of float32 queries whose three
      bf16 parts are multiplied), times scale log2 e: off by at most e_i =
      2 (3 D + 1) 2^-24 |scale| sum |q k| + 3 2^-24 |s_i| (the factor 2: the additions of
      the matrix cores may round either way), the exponential of the difference to
      the running maximum by (|s_i - max| + 3) 2^-23 more: eps_i, relative to w_i;
    * numerators are rounded to bf16 for the second product of bf16 inputs (u = 2^-8);
    * sums of n terms in any order, and some rescales and joins: c = (n + 40) 2^-23
      (3 n for the parts of float32 numerators);
    * out is rounded once: u |out| (2^-24 float32).
    |d out| <= sum w_i |v_i| (u + eps_i + c) + |out| (sum w_i eps_i + c) + u |out|,
    |d lse| <= sum w_i eps_i + c + 2^-22 |lse|."""
    if len(k) == 0:
        assert (out == 0).all() and lse == -np.inf
        return
    D = len(q)
    s = scale * (k @ q)
    e = 2 * (3 * D + 1) * 2.0 ** -24 * abs(scale) * (np.abs(k) @ np.abs(q))
    eps = e + 3 * 2.0 ** -24 * np.abs(s) + (s.max() - s + 3) * 2.0 ** -23
    w = np.exp(s - ref_lse)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    un = u if dtype == "bf16" else 0.0
    c = ((1 if dtype == "bf16" else 3) * len(k) + 40) * 2.0 ** -23
    we = w @ eps + c
    bound = (w * (un + eps + c)) @ np.abs(v) + np.abs(ref) * (we + u) + 1e-37
    bound *= 1 + u
    err = np.abs(out - ref)
    assert (err <= bound).all(), (err / bound).max()
    assert abs(lse - ref_lse) <= we + 2.0 ** -22 * abs(ref_lse), (lse, ref_lse)
