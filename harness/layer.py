"""One layer's attention over a roll-out, as a model would run it: norm and rotation of the chunk's queries and keys, the keys
straight into the cache's ring, block-sparse attention over the cache, cross attention to the prompt; and its backward.

    python -m harness.layer [chunks]      a roll-out of 12 heads of 128 on three frames of 30 x 52 patches, with times
"""
from __future__ import annotations

import sys

import torch

from paper_2604_21221_amd import layer
from paper_2604_21221_amd.cache import PbsaCache


def frame_positions(Nq, grid, chunk_id, device):
    """(frame, row, column) of a chunk's tokens, [1, Nq, 3]; grid: rows and columns of a frame."""
    rows, cols = grid
    t = torch.arange(chunk_id * Nq, (chunk_id + 1) * Nq, device=device)
    return torch.stack([t // (rows * cols), t // cols % rows, t % cols], dim=-1)[None]


class LayerAttention:
    """Projections come in and go out as [tokens, H, d], the memory order of a linear layer's output."""

    def __init__(self, cache: PbsaCache, wq, wk, prompt_k, prompt_v, prompt_len=None, prompt_mask=None, sections=None, **scaling):
        self.cache, self.wq, self.wk = cache, wq, wk
        self.prompt_k, self.prompt_v, self.prompt_len, self.prompt_mask = prompt_k, prompt_v, prompt_len, prompt_mask
        d = cache.d
        self.sections = sections or (d // 2 - 2 * (d // 6), d // 6, d // 6)
        self.freq, self.mscale = layer.rotary_frequencies(self.sections, device=cache.dev, **scaling)
        H, Nq = cache.H, cache.Nq
        e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device=cache.dev)  # noqa: E731
        self.q, self.o, self.cross = e(H, Nq, d), e(H, Nq, d), e(1, Nq, H, d).transpose(1, 2)
        self.lse, self.cross_lse = e(H, Nq, dt=torch.float32), e(1, H, Nq, dt=torch.float32)
        self._ws = {}

    def _scratch(self, name, size):
        if size and (name not in self._ws or self._ws[name].numel() < size):
            self._ws[name] = torch.empty(size, dtype=torch.uint8, device=self.cache.dev)
        return self._ws[name] if size else None

    def _append(self, q, k, v, pos, chunk_id):
        """Norm and rotation; the keys are appended to the cache as they are made."""
        c = self.cache
        at = c.n_appended % c.ring
        slots = c.Kl[:, at * c.nqb:(at + 1) * c.nqb].view(c.H, c.nqb * c.B, c.d)[None, :, :c.Nq]
        qt, kt = q[None].transpose(1, 2), k[None].transpose(1, 2)
        p = layer.make_rotary(qt, kt, self.q[None], slots, sections=self.sections, mscale=self.mscale)
        torch.autograd.graph.increment_version([c.Kl])         # as an append would, so that a backward which saved the ring notices
        layer.pbsa_norm_rotate_fwd(p, qt, kt, self.wq, self.wk, pos, self.freq, self.q[None], slots)
        c.adopt_chunk(chunk_id)
        c.rewrite_chunk(V=v.transpose(0, 1))

    def _attend_prompt(self, qc):
        qt = qc[None].transpose(1, 2)
        p = layer.make_cross(qt, self.prompt_k, self.prompt_v, self.cross)
        layer.pbsa_cross_attention_fwd(p, qt, self.prompt_k, self.prompt_v, self.prompt_len, self.prompt_mask, self.cross, self.cross_lse,
                                       self._scratch("cross", layer.pbsa_cross_workspace_bytes(p)))

    def step(self, q, k, v, qc, pos, chunk_id):
        """A decoding step: (attention over the cache, attention to the prompt), [Nq, H, d] views; the window slides."""
        c = self.cache
        self._append(q, k, v, pos, chunk_id)
        c.select(self.q)
        c.attention(self.q, self.o)
        c.update()
        self._attend_prompt(qc)
        return self.o.transpose(0, 1), self.cross[0].transpose(0, 1)

    def train(self, q, k, v, qc, pos, chunk_id, gradient):
        """A step with gradients; gradient(o, cross) gives those of the two outputs.  Returns the outputs and the gradients of q, k,
        v, qc, the norms' weights and the prompt's states.  They end at the chunk: what its attention owes to the keys and values of
        earlier ones, in the window, the slots or the summary, is left out."""
        c = self.cache
        self._append(q, k, v, pos, chunk_id)
        c.select(self.q)
        c.attention(self.q, self.o, self.lse)
        self._attend_prompt(qc)
        out = self.o.transpose(0, 1), self.cross[0].transpose(0, 1)
        do, dcross = gradient(*out)
        own = c.attention_bwd(self.q, self.o, do.transpose(0, 1).contiguous(), self.lse)      # (laid out as o)
        at = c.chunk_pos[-1]
        newest = lambda x: x[:, at * c.nqb:(at + 1) * c.nqb].reshape(c.H, c.nqb * c.B, c.d)[:, :c.Nq]  # noqa: E731
        dq_in, dk_in = own["dQ"].bfloat16()[None], newest(own["dKl"]).bfloat16()[None]
        g = dict(q=torch.empty_like(q), k=torch.empty_like(k), qc=torch.empty_like(qc), v=newest(own["dVl"]).transpose(0, 1).bfloat16(),
                 wq=torch.empty_like(self.wq), wk=torch.empty_like(self.wk), prompt_k=torch.empty_like(self.prompt_k),
                 prompt_v=torch.empty_like(self.prompt_v))
        t = lambda x: x[None].transpose(1, 2)  # noqa: E731
        p = layer.make_rotary(t(q), t(k), dq_in, dk_in, sections=self.sections, mscale=self.mscale, dq=t(g["q"]), dk=t(g["k"]))
        layer.pbsa_norm_rotate_bwd(p, t(q), t(k), self.wq, self.wk, pos, self.freq, dq_in, dk_in, t(g["q"]), t(g["k"]), g["wq"], g["wk"],
                                   self._scratch("norm", layer.pbsa_norm_rotate_workspace_bytes(p)))
        p = layer.make_cross(t(qc), self.prompt_k, self.prompt_v, self.cross, do=t(dcross), dq=t(g["qc"]), dk=g["prompt_k"], dv=g["prompt_v"])
        layer.pbsa_cross_attention_bwd(p, t(qc), self.prompt_k, self.prompt_v, self.prompt_len, self.prompt_mask, self.cross, t(dcross),
                                       self.cross_lse, t(g["qc"]), g["prompt_k"], g["prompt_v"],
                                       self._scratch("cross_bwd", layer.pbsa_cross_bwd_workspace_bytes(p)))
        c.update()
        return out, g


def random_layer(H, d, B, Nq, window, C, k, n_prompt, device="cuda:0", seed=0, **kw):
    """A layer of random weights and a random prompt, and a generator for its inputs."""
    g = torch.Generator(device=device).manual_seed(seed)
    cache = PbsaCache(H, d, B, Nq, window, C, k, d ** -0.5, device=device)
    w = [1 + 0.2 * torch.randn(d, generator=g, device=device) for _ in range(2)]
    prompt = [torch.randn(1, n_prompt, H, d, generator=g, device=device).bfloat16().transpose(1, 2) for _ in range(2)]
    return LayerAttention(cache, *w, *prompt, **kw), g


def random_chunk(one: LayerAttention, g):
    c = one.cache
    return [torch.randn(c.Nq, c.H, c.d, generator=g, device=c.dev).bfloat16() for _ in range(4)]


def main(chunks=6):
    H, d, B, Nq, grid = 12, 128, 64, 4680, (30, 52)
    one, g = random_layer(H, d, B, Nq, 3, 32, 48, 512, theta=1e4)
    for i in range(chunks):
        x, pos = random_chunk(one, g), frame_positions(Nq, grid, i, one.cache.dev)
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        o, cross = one.step(*x, pos, i)
        b.record()
        torch.cuda.synchronize()
        print(f"chunk {i}: {a.elapsed_time(b) * 1e3:.0f} us, rms of the outputs {o.float().square().mean().sqrt():.4f} "
              f"{cross.float().square().mean().sqrt():.4f}", flush=True)


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:]))
