"""include/pbsa_layer.h with more sequences than a launch holds workgroups for: against the same calls in two halves, bit for bit."""
import pytest
import torch

from paper_2604_21221_amd import layer
from tests.test_gpu_cross import B, DEV, backward, forward

pytestmark = pytest.mark.gpu


def test_a_mask_of_more_sequences_than_a_launch_of_lists_takes():
    n, T = (1 << 22) + 3, 5
    g = torch.Generator(device=DEV).manual_seed(61)
    q = torch.randn(n, 1, T, 64, generator=g, dtype=B, device=DEV)
    k, v = (torch.randn(1, 1, 2, 64, generator=g, device=DEV).to(B).expand(n, -1, -1, -1) for _ in range(2))
    mask = (torch.rand(n, 2, generator=g, device=DEV) < 0.6).to(torch.uint8)
    o, lse = torch.empty_like(q), torch.empty(n, 1, T, device=DEV)
    grads = [torch.empty_like(q), *(torch.empty(n, 1, 2, 64, dtype=B, device=DEV) for _ in range(2))]
    forward(q, k, v, None, mask, o, lse)
    assert ((o == 0).flatten(1).all(1) == (mask == 0).all(1)).all()
    backward(q, k, v, None, mask, o, q, lse, *grads)
    for part in (slice(0, n // 2), slice(n // 2, n)):
        x = [y[part] for y in (q, k, v)]
        o2, lse2 = torch.empty_like(o[part]), torch.empty_like(lse[part])
        again = [torch.empty_like(y[part]) for y in grads]
        forward(*x, None, mask[part], o2, lse2)
        backward(*x, None, mask[part], o2, x[0], lse2, *again)
        assert torch.equal(o2, o[part]) and torch.equal(lse2, lse[part])
        assert all(torch.equal(a, b[part]) for a, b in zip(again, grads))


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("n,T", [((1 << 24) + 5, 1), (1, (1 << 28) + 40)])
def test_more_tokens_than_a_launch_of_the_rotation_takes(n, T, norm):
    g = torch.Generator(device=DEV).manual_seed(62)
    q = torch.randn(n, 1, T, 16, generator=g, dtype=B, device=DEV)
    pos = torch.arange(n * T, device=DEV).view(n, T, 1)
    freq, _ = layer.rotary_frequencies((8,), device=DEV)

    def call(x, at):
        y = torch.empty_like(x)
        p = layer.make_rotary(x, None, y, None)
        if norm:
            layer.pbsa_norm_rotate_fwd(p, x, None, None, None, at, freq, y, None)
        else:
            layer.pbsa_rotate(p, x, None, at, freq, y, None)
        return y

    y = call(q, pos)
    for i in range(3):                                       # in parts that a launch takes
        if n > 1:
            part = slice(i * n // 3, (i + 1) * n // 3)
            assert torch.equal(call(q[part], pos[part]), y[part])
        else:
            part = slice(i * T // 3, (i + 1) * T // 3)
            assert torch.equal(call(q[:, :, part], pos[:, part]), y[:, :, part])
