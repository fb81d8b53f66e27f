"""Long sequences, checked so that a lost or repeated stretch of them shows: inputs whose result says which slots went into it, and a bound of the error
by the depth of the sums that are formed, not by the number of slots."""
import torch


def counted_values(n, dh):
    """V of n slots: each group of 16 has a one in a channel of the first half and one in a channel of the second, and no two groups the same two
    channels.  Under equal weights a channel's result counts the slots of its groups."""
    group, half = torch.arange(n) // 16, dh // 2
    assert (n - 1) // 16 < half * half
    v = torch.zeros(n, dh)
    v[torch.arange(n), group % half] = 1
    v[torch.arange(n), half + group // half] = 1
    return v


def counted_tolerance(ref, half):
    """All weights are 1, all sums whole numbers below 2^24: exact.  Left are the reciprocal of their sum, its product with the count, and the rounding to
    the output's type."""
    return (half + 2.0 ** -22) * ref.abs()


CHUNKS = 16             # chunks of 64 slots in a run at most, in the cases below


def tolerance(out, magnitude, size, dh, half):
    """Of an output, given sum_j p_j |v_j| and the largest sum |q||k|, for runs of at most CHUNKS chunks.

    A softmax weight's relative error: the score's dh products and their sum, each step off by at most 2^-23 (the tensor pipe truncates) of the sum of
    magnitudes `size`; log2 e, the maximum (or the log of the sum) three roundings of the score; exp2 2 ulp.
    The sum of weights: four steps a chunk and lane, two over lanes, the four warps, at most 32 parts (74 if the bound on parts is not there), each with a factor.
    The product with V: two multiplications of 16 products and what was there a chunk (fp32: 16 steps), then warps and parts as before.
    bf16 weights enter it as two numbers: half a step of half a step is left."""
    weight = 2.0 ** -23 * ((dh + 3) * size + 4)
    joins = 2 * (4 + 74) + 2
    sums = 2.0 ** -23 * (4 * CHUNKS + joins)
    product = 2.0 ** -23 * (2 * 17 * CHUNKS + joins) + (half ** 2 if half > 2.0 ** -20 else 0.0)
    return half * out.abs() + (2 * weight + sums + product) * magnitude * (1 + half)


def reference(q, k, v, scale):
    """Rows q [r, dh] over k, v [n, dh] in 64 bits: out, sum_j p_j |v_j|, lse, the largest sum |q||k|, the weights."""
    q, k, v = q.double(), k.double(), v.double()
    s = scale * (q @ k.T)
    z = torch.logsumexp(s, 1)
    p = torch.exp(s - z[:, None])
    return p @ v, p @ v.abs(), z, float((scale * (q.abs() @ k.abs().T)).max()), p
