"""harness/layer.py: a layer's operators run together, against their plain forms and against the cache fed in the plain way."""
import pytest
import torch

from harness import layer as example
from paper_2604_21221_amd.cache import PbsaCache
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GEOMETRY = (3, 64, 64, 200, 2, 2, 3, 77)                     # H, d, B, Nq (a ragged last block), window, C, k, prompt


def made(seed=0, **kw):
    return example.random_layer(*GEOMETRY, seed=seed, **kw)


def test_a_rollout_is_its_parts():
    H, d, B, Nq, w, C, k, _ = GEOMETRY
    one, g = made(prompt_len=torch.tensor([70], dtype=torch.int32, device=DEV))
    plain = PbsaCache(H, d, B, Nq, w, C, k, d ** -0.5, device=DEV)
    for i in range(w + 3):
        q, kk, v, qc = example.random_chunk(one, g)
        pos = example.frame_positions(Nq, (5, 8), i, DEV)
        o, cross = one.step(q, kk, v, qc, pos, i)
        # the cache holds the keys that an append of the rotated keys would have stored
        at = (one.cache.n_appended - 1) % one.cache.ring * one.cache.nqb
        keys = one.cache.Kl[:, at:at + one.cache.nqb].reshape(H, -1, d)
        assert (keys[:, Nq:] == 0).all()
        want = plain.step(one.q, keys[:, :Nq].contiguous(), v.transpose(0, 1).contiguous(), i)
        assert torch.equal(o, want.transpose(0, 1))
        t = lambda x: x[None].transpose(1, 2)  # noqa: E731
        r = ref.Cross(t(qc), one.prompt_k, one.prompt_v, d ** -0.5, one.prompt_len)
        assert ref.worst(t(cross), r.o, r.o_tol) <= 1
    assert torch.equal(one.cache.p_id, plain.p_id)


def test_gradients_of_the_first_chunk():
    """Where the chunk sees nothing but itself, in full, the layer is softmax attention: its gradients against autograd's in 64 bits,
    to the steps of bf16 that pass through two operators (norms of the differences)."""
    H, d, B, Nq, w, C, k, n_prompt = GEOMETRY
    cache = PbsaCache(H, d, B, Nq, w, C, 4, d ** -0.5, causal=0, device=DEV)     # four blocks of the chunk's four
    one, g = made(seed=3)
    one = example.LayerAttention(cache, one.wq, one.wk, one.prompt_k, one.prompt_v)
    x = example.random_chunk(one, g)
    pos = example.frame_positions(Nq, (5, 8), 0, DEV)
    do, dcross = (torch.randn(Nq, H, d, generator=g, device=DEV).bfloat16() for _ in range(2))
    (o, cross), got = one.train(*x, pos, 0, lambda *_: (do, dcross))

    leaves = dict(zip(("q", "k", "v", "qc"), x), wq=one.wq, wk=one.wk, prompt_k=one.prompt_k, prompt_v=one.prompt_v)
    leaves = {n: y.detach().double().requires_grad_() for n, y in leaves.items()}
    axis = torch.tensor([i for i, m in enumerate(one.sections) for _ in range(m)], device=DEV)
    angle = (pos[0].double()[:, axis] * one.freq)[:, None]

    def rotated(y, weight):
        y = y * (y.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight
        a, b, co, si = y[..., ::2], y[..., 1::2], angle.cos(), angle.sin()
        return torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2)

    def attend(a, b, c):                                     # [tokens, H, d]
        a, b, c = (y.transpose(0, 1) for y in (a, b, c))
        return (torch.softmax(a @ b.transpose(1, 2) * d ** -0.5, -1) @ c).transpose(0, 1)

    with torch.enable_grad():
        want_o = attend(rotated(leaves["q"], leaves["wq"]), rotated(leaves["k"], leaves["wk"]), leaves["v"])
        want_c = attend(leaves["qc"], leaves["prompt_k"][0].transpose(0, 1), leaves["prompt_v"][0].transpose(0, 1))
        ((want_o * do.double()).sum() + (want_c * dcross.double()).sum()).backward()
    off = lambda a, b: float((a.double() - b.detach()).norm() / b.detach().norm())  # noqa: E731
    # random roundings of 2^-9 (rms 2^-9 / sqrt 3 of a value): the rotated q and k, P or dS, the gradient between the operators
    # and the one that comes out add up to less than 2^-7 of the whole in quadrature
    assert off(o, want_o) < 2.0 ** -7 and off(cross, want_c) < 2.0 ** -7
    for n, y in leaves.items():
        assert off(got[n], y.grad) < 2.0 ** -6, n


def test_a_backward_that_saved_the_ring_notices_a_step():
    """As with an append of the cache's own: what autograd saved of the keys or the values is known to have changed."""
    H, d, B, Nq, w, C, k, _ = GEOMETRY
    for name in ("Kl", "Vl"):
        one, g = made()
        ring = getattr(one.cache, name)
        x = torch.ones(d, device=DEV, requires_grad=True)
        with torch.enable_grad():
            y = (ring.float() * 1).mul(x).sum() + (ring * x.bfloat16()).float().sum()      # saves the ring itself
        q, kk, v, qc = example.random_chunk(one, g)
        one.step(q, kk, v, qc, example.frame_positions(Nq, (5, 8), 0, DEV), 0)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
