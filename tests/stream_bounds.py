"""Bounds of attention over streams of tokens that tell the kernels' ways of multiplying apart, in 64 bits.

As in streams_reference.attend, with u = eps / 2 of a type and u32 = 2^-24, but with every rounding named by the caller:
  terms     products of a score that are not zero (a zero adds no error): the sum is off by (2 terms + 6) u32 of its magnitude, with
            the scaling, accumulators that cut included
  products  what a product loses: 0 of bf16 operands or fp32 multiply-adds.  tf32 halves: x = hi + lo, |lo| <= 2^-11 |x|; lo lo is left
            out (2^-22), and of the 12 bits that each lo has the last is cut (2^-23 each): 2^-21 of the product
  weights   what a weight loses next to the values: 2^-8 as bf16; as two bf16 parts 2^-16 (the upper one is cut, the rest below 2^-7
            of the weight's binade, so below 2^-8 of it after its leading bit, and rounded by 2^-8 of itself)
so that  E = ((2 terms + 6) u32 + products) sum |q k| s + 2^-22 + 2 reach u32  is what a logit and its exponential are off, and
  |o - o64| <= (2 E + 4 n u32 + weights + products) (weighted mean of |v|) (1 + E) + u_out |o64| + least
with least = n 2^-148 for terms below the normal range (each is off by 2^-150 at most, and the sum is divided by at least the
largest weight) and half the storage type's smallest number."""
import math

import torch

U32 = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}

# kernel -> (products, weights): bf16 and fp32 windows, the CUDA-core kernel for either storage, the caches
WINDOW = {("bf16", 0): (0.0, 2.0 ** -8), ("fp32", 0): (2.0 ** -21, 0.0), ("bf16", 2): (0.0, 0.0), ("fp32", 2): (0.0, 0.0)}
CACHE = {"bf16": (0.0, 2.0 ** -16 + 2.0 ** -24), "fp32": (0.0, 0.0)}


def attend(q, k, v, visible, scale, storage, terms, products, weights):
    """q [r, d], k and v [n, d] float64, visible [r, n] (a key for every row).  Result, log-sum-exp and their bounds."""
    s = (q @ k.T) * scale
    s = torch.where(visible, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, dim=1)
    w = torch.exp(s - lse.unsqueeze(1))
    o, mean = w @ v, w @ v.abs()
    n = int(visible.sum(1).max())
    top = torch.where(visible, (q.abs() @ k.abs().T) * scale, torch.zeros_like(s)).amax(1)
    reach = 2 * top / math.log(2.0)
    E = ((2 * terms + 6) * U32 + products) * top + 2.0 ** -22 + 2 * reach * U32
    bound = (2 * E + 4 * n * U32 + weights + products).unsqueeze(1) * mean * (1 + E).unsqueeze(1)
    bound = bound + U[storage] * (o.abs() + bound) + n * 2.0 ** -148 + LEAST[storage]
    return o, lse, bound, E + 4 * n * U32 + 4 * U32 * (1 + lse.abs())
