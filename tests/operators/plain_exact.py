"""Bounds for kernels that multiply with the weights themselves: what is added up is s (q - z) x, and a weight of 0 adds nothing."""
import numpy as np

import plain


def int4_product(x, values, scale_bits, zero, group, act):
    """x [tokens, cols] -> result float64, and a bound on the error of an fp32 evaluation: q - z is exact in bf16 and so is each product in fp32, which leaves
    the roundings of the sums, of a scale's product and of the join (plain.int4_steps), each of at most 2^-24 of the absolute terms."""
    w, _ = plain.int4_matrix(values, scale_bits, zero, group)
    return plain.activate(x @ w.T, plain.int4_steps(values.shape[1], group) * plain.U32 * (np.abs(x) @ np.abs(w).T), act)
