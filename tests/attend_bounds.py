"""Inputs whose outputs show every single row of V, and the bound that holds
them.

Row j of V is zero but for coordinate j % D, so that a coordinate of the output
is the sum of the weights of N / D tokens (one at most where N <= D), times
values between 1/2 and 3/2.  All terms are positive: every error of the bound in
attend_ref.check is relative to the output itself, below 2^-7 for a bf16 cache
through matrix products in bf16 (the weights' rounding and the result's, 2^-8
each), and 2^-8 where the weights go in as two terms.  A row lost or misplaced
changes its coordinate by about D / N."""
import torch

import attend_ref


def spread_rows(V, first=0, seed=0):
    """V [..., tokens, D] overwritten in place, token j taken as number first + j."""
    n, D = V.shape[-2:]
    j = torch.arange(n)
    g = torch.Generator().manual_seed(seed + n)
    v = torch.zeros(n, D)
    v[j, (first + j) % D] = 0.5 + torch.rand(n, generator=g)
    V.copy_(v.to(V.dtype).expand(V.shape))
    return V


def two_terms(d, T, tiled_prefix=False):
    """Whether a call's weights keep more bits than the cache's type: fp32
    caches, and up to 32 rows (queries times heads) of a bf16 one."""
    return d.dtype != 1 or (d.G * T <= 32 and not tiled_prefix)


def check(d, T, ref, out, lse, mass, before, N, tiled_prefix=False):
    return attend_ref.check(ref, out, lse, mass, before, N, weights_in_type=not two_terms(d, T, tiled_prefix))
