"""pbsa_cross_attention_fwd on both sides of the rule that shares a call out by rows or by states, against the plain form in 64 bits."""
import math

import pytest
import torch

from tests import layer_reference as ref
from tests.test_gpu_cross import B, DEV, H16, forward, made
from tests.test_gpu_rotary import guarded, untouched

pytestmark = pytest.mark.gpu

# n, T, Nk, Hq, Hk, d, dtype, major, lengths (None: all), share of states that the mask keeps (None: no mask)
CASES = [
    (1, 300, 512, 12, 12, 128, B, "token", None, None),      # by rows, below a round of workgroups
    (1, 40, 3000, 4, 2, 128, H16, "token", None, 0.5),       # by states, shared out, some masked
    (2, 100, 2500, 2, 2, 64, B, "head", (2500, 0), 0.3),
    (1, 100, 130, 2, 2, 64, B, "head", (65,), 0.3),          # by rows, a list of states
    (1, 6, 9000, 2, 1, 128, B, "token", (8999,), None),
    (3, 700, 65, 2, 1, 128, H16, "head", (64, 1, 65), 0.9),
]


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    n, T, Nk, Hq, Hk, d, dtype, major, _, _ = case
    q, k, v, k_len, k_mask, _ = made(case, seed=6)
    whole, o = guarded(n, Hq, T, d, dtype, major)
    lse = torch.full((n, Hq, T), math.nan, device=DEV)
    forward(q, k, v, k_len, k_mask, o, lse)
    r = ref.Cross(q, k, v, d ** -0.5, k_len, k_mask)
    assert ref.worst(o, r.o, r.o_tol) <= 1
    assert ref.worst(lse, r.lse, r.lse_tol) <= 1
    untouched(whole)


@pytest.mark.parametrize("n_k", [128, 129])
def test_masked_states_far_apart_in_memory(n_k):
    """Few states, so far apart that a list's offsets fill 32 bits: the 128th lies at 0.99 of 2^32 bytes, the 129th at 2^32, which the
    kernel that counts by tiles takes; K and V in the same memory."""
    step = 1 << 24                                           # elements between two states
    mem = torch.empty((n_k - 1) * step + 256, dtype=B, device=DEV)
    k, v = (mem[at:].as_strided((1, 1, n_k, 128), (0, 0, step, 1)) for at in (0, 128))
    g = torch.Generator(device=DEV).manual_seed(22)
    k.copy_(torch.randn(1, 1, n_k, 128, generator=g, device=DEV))
    v.copy_(torch.randn(1, 1, n_k, 128, generator=g, device=DEV))
    mask = (torch.rand(1, n_k, generator=g, device=DEV) < 0.6).to(torch.uint8)
    mask[0, -1] = 1
    for T in (3, 70, 40000):
        q = torch.randn(1, 1, T, 128, generator=g, device=DEV).to(B)
        o, lse = torch.empty_like(q), torch.empty(1, 1, T, device=DEV)
        forward(q, k, v, None, mask, o, lse)
        r = ref.Cross(q, k.contiguous(), v.contiguous(), 128 ** -0.5, None, mask)
        assert ref.worst(o, r.o, r.o_tol) <= 1 and ref.worst(lse, r.lse, r.lse_tol) <= 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [3, 40, 2100])
@pytest.mark.parametrize("Nk,lens,keep", [(90, None, None), (90, (90, 33), None), (130, None, 0.5), (200, (150, 1), 0.7), (64, None, None), (1, None, None)])
def test_infinite_values_are_the_rows_results(Nk, lens, keep, T, d):
    """An infinity in V of an attended state, the first or the last one too, is an infinity of the outputs in its place."""
    case = (2, T, Nk, 16, 16, d, B, "token", lens, keep)
    q, k, v, k_len, k_mask, _ = made(case, seed=7)
    at = ref.attended(2, Nk, k_len, k_mask, DEV)
    for b in range(2):
        own = at[b].nonzero().flatten()
        if len(own):
            v[b, 3, own[-1], 9], v[b, 5, own[0], 10] = math.inf, -math.inf
    o, lse = torch.empty_like(q), torch.empty(2, 16, T, device=DEV)
    forward(q, k, v, k_len, k_mask, o, lse)
    r = ref.Cross(q, k, v, d ** -0.5, k_len, k_mask)
    assert int(torch.isinf(r.o).sum()) == 2 * T * int(at.any(1).sum())
    assert ref.worst(o, r.o, r.o_tol) <= 1 and ref.worst(lse, r.lse, r.lse_tol) <= 1


@pytest.mark.parametrize("first", [30, 40, 64, 100])
@pytest.mark.parametrize("T", [3, 40, 2100])
@pytest.mark.parametrize("far", [0.0, 40.0])
def test_scores_of_minus_infinity_count_for_nothing(T, first, far):
    """Attended states whose keys are -infinite draw nothing from rows of positive queries, wherever the other scores lie."""
    g = torch.Generator(device=DEV).manual_seed(8)
    q, k, v = (torch.randn(1, 16, t, 64, generator=g, device=DEV) for t in (T, 200, 200))
    q, k, v = (0.1 + q.abs()).to(B), (k / 8 - far).to(B), v.to(B)
    k[:, :, :first] = -math.inf
    o, lse = torch.empty_like(q), torch.empty(1, 16, T, device=DEV)
    forward(q, k, v, None, None, o, lse)
    r = ref.Cross(q, k[:, :, first:], v[:, :, first:], 0.125)
    assert ref.worst(o, r.o, r.o_tol) <= 1 and ref.worst(lse, r.lse, r.lse_tol) <= 1
