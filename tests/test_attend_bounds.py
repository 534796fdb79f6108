"""The bound of the attention tests refuses what it is there for: on the CPU,
outputs as a right kernel rounds them pass, and the same with a row of V lost,
two rows swapped or fewer bits of the weights do not."""
import pytest
import torch

import attend_bounds
import attend_ref
import paper_2609_04971_amd as bkv

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def attend(q, K, V, causal, bits16):
    """[1, Hq, T, D] outputs from logits, weights and sums in 32 bits; the weights in bf16 where bits16."""
    Hq, T, D = q.shape[1:]
    Hkv, N = K.shape[1], K.shape[2]
    out, lse = torch.empty(1, Hq, T, D), torch.empty(1, Hq, T)
    for hq in range(Hq):
        h = hq * Hkv // Hq
        l = torch.matmul(q[0, hq].float(), K[0, h].float().T.contiguous()) / D ** 0.5
        if causal:
            l = l.masked_fill(torch.arange(N) > N - T + torch.arange(T).unsqueeze(1), float("-inf"))
        m = l.amax(-1, keepdim=True)
        e = torch.exp(l - m)
        z = e.sum(-1, keepdim=True)
        out[0, hq] = torch.matmul(e.bfloat16().float() if bits16 else e, V[0, h].float()) / z
        lse[0, hq] = (m + torch.log(z)).squeeze(-1)
    return out.to(q.dtype), lse


def case(dtype, T, N, D, G=4, causal=True):
    g = torch.Generator().manual_seed(N + T)
    r = lambda *s: torch.randn(*s, generator=g).to(DT[dtype])  # noqa: E731
    q, K, V = r(1, 2 * G, T, D), r(1, 2, N, D), torch.empty(1, 2, N, D, dtype=DT[dtype])
    attend_bounds.spread_rows(V)
    d = bkv.dims(B=1, Hq=2 * G, Hkv=2, D=D, N=N, W=0, C=0, budget=1, dtype=dtype)
    ref = attend_ref.reference(q, K, V, N, causal=causal)
    return d, q, K, V, lambda out, lse: attend_bounds.check(d, T, ref, out, lse, None, None, N)


SIZES = [(1, 700, 64), (1, 700, 128), (3, 4097, 128), (1, 5000, 128), (9, 1111, 64), (100, 1111, 128), (40, 4097, 128), (300, 1111, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N,D", SIZES)
def test_a_row_lost_or_misplaced_is_seen(dtype, T, N, D):
    d, q, K, V, check = case(dtype, T, N, D)
    bits16 = not attend_bounds.two_terms(d, T)
    check(*attend(q, K, V, True, bits16))
    unseen = 0
    for j in (0, 31, 32, 63, 64, N // 2, N - T, N - T - 1 if N > T else 0):  # the tokens that every query sees
        bad = V.clone()
        bad[:, 0, j] = 0
        with pytest.raises(AssertionError):
            check(*attend(q, K, bad, True, bits16))
        bad = V.clone()
        at = (j, j + 1) if j + 1 < N else (j - 1, j)
        bad[:, 0, list(at)] = V[:, 0, list(at)[::-1]]
        try:
            check(*attend(q, K, bad, True, bits16))
            unseen += 1
        except AssertionError:
            pass
    assert unseen == 0, f"{unseen} swaps of 8 unseen"
    bad = V.clone()
    bad[:, 0, N - 1] = 0  # seen by the last query only
    with pytest.raises(AssertionError):
        check(*attend(q, K, bad, True, bits16))


@pytest.mark.parametrize("T,N", [(1, 100), (1, 128), (4, 300), (8, 700)])
def test_fewer_bits_of_the_weights_are_seen(T, N):
    # up to 32 rows the weights have two bf16 terms: one alone is outside the bound
    d, q, K, V, check = case("bf16", T, N, 128)
    assert attend_bounds.two_terms(d, T)
    check(*attend(q, K, V, True, False))
    with pytest.raises(AssertionError):
        check(*attend(q, K, V, True, True))
