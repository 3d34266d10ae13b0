"""What layer.py makes of the arguments that a description does not describe, on the CPU: a tensor of the right type and size is only
refused for not being on the GPU (TypeError), any other one for what it is (ValueError)."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2604_21221_amd import pbsa  # noqa: E402
from tests.test_layer_abi import cross, cross_bwd, cross_fwd, norm_bwd, norm_fwd, rotary, rotate  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(pbsa.LIB_PATH) or not os.path.exists(os.path.join(os.path.dirname(pbsa.LIB_PATH), "_pbsa_host.so")):
        from paper_2604_21221_amd import build
        build.build()


def t(*shape, dtype):
    return torch.zeros(shape, dtype=dtype)


def fits(call, p, **kw):
    with pytest.raises(TypeError, match="GPU|contiguous"):
        call(p, stream=0, **kw)


def refused(call, p, name, **kw):
    with pytest.raises(ValueError, match=name):
        call(p, stream=0, **kw)


I64, I32, U8, F32, F64, BF = torch.int64, torch.int32, torch.uint8, torch.float32, torch.float64, torch.bfloat16


@pytest.mark.parametrize("call", [rotate, norm_fwd, norm_bwd])
def test_positions_and_frequencies(call):
    p = rotary(n=2, T=10, n_axes=2, pairs=(20, 12), pos_stride_b=20)          # d = 64
    fits(call, p, pos=t(2, 10, 2, dtype=I64))
    fits(call, p, pos=t(40, dtype=I64))
    fits(call, p, pos=t(5, 10, 2, dtype=I64))
    fits(call, p, freq=t(32, dtype=F64))
    for bad in (t(2, 10, 2, dtype=I32), t(2, 10, 2, dtype=F64), t(1, 10, 2, dtype=I64), t(39, dtype=I64), t(2, 10, 4, dtype=I64)[..., ::2],
                t(2, 2, 10, dtype=I64).transpose(1, 2), t(1, 10, 2, dtype=I64).expand(2, 10, 2), t(4, 10, 2, dtype=I64)[::2]):
        refused(call, p, "pos", pos=bad)
    for bad in (t(32, dtype=F32), t(31, dtype=F64), t(64, dtype=F64)[::2]):
        refused(call, p, "freq", freq=bad)
    shared = rotary(n=2, T=10, n_axes=2, pairs=(20, 12), pos_stride_b=0)
    for good in (t(1, 10, 2, dtype=I64), t(10, 2, dtype=I64), t(1, 10, 2, dtype=I64).expand(2, 10, 2)):
        fits(call, shared, pos=good)
    fits(call, rotary(n=2, T=10, n_axes=2, pairs=(20, 12), pos_stride_b=40), pos=t(4, 10, 2, dtype=I64)[::2])


def test_norm_weights_and_their_gradients():
    for call in (norm_fwd, norm_bwd):
        for name in ("wq", "wk"):
            fits(call, rotary(), **{name: t(64, dtype=F32)})
            fits(call, rotary(), **{name: torch.nn.Parameter(t(64, dtype=F32))})
            for bad in (t(64, dtype=BF), t(64, dtype=torch.float16), t(64, dtype=F64), t(63, dtype=F32), t(128, dtype=F32)[::2],
                        torch.nn.Parameter(t(64, dtype=BF))):
                refused(call, rotary(), "norm weights", **{name: bad})
    for name in ("dwq", "dwk"):
        fits(norm_bwd, rotary(), **{name: t(64, dtype=F32)})
        for bad in (t(64, dtype=BF), t(32, dtype=F32), t(128, dtype=F32)[::2]):
            refused(norm_bwd, rotary(), "gradients of the norm weights", **{name: bad})


@pytest.mark.parametrize("call", [cross_fwd, cross_bwd])
def test_lengths_masks_and_lse(call):
    p = cross()                              # 2 sequences, 10 tokens of 4 heads, 20 states
    fits(call, p, k_len=t(2, dtype=I32))
    for bad in (t(2, dtype=I64), t(1, dtype=I32), t(4, dtype=I32)[::2], t(2, dtype=F32)):
        refused(call, p, "k_len", k_len=bad)
    for good in (U8, torch.bool, torch.int8):
        fits(call, p, k_mask=t(2, 20, dtype=good))
    for bad in (t(2, 20, dtype=I32), t(2, 20, dtype=F32), t(1, 20, dtype=U8), t(2, 19, dtype=U8), t(2, 40, dtype=U8)[:, ::2]):
        refused(call, p, "k_mask", k_mask=bad)
    fits(call, cross(mask_stride_b=0), k_mask=t(1, 20, dtype=U8))
    fits(call, cross(mask_stride_b=32), k_mask=t(2, 32, dtype=U8))
    fits(call, p, lse=t(2, 4, 10, dtype=F32))
    for bad in (t(2, 4, 10, dtype=BF), t(2, 4, 10, dtype=F64), t(2, 4, 9, dtype=F32), t(2, 10, 4, dtype=F32).transpose(1, 2)):
        refused(call, p, "lse", lse=bad)


def test_what_is_not_looked_at_is_not_refused():
    for call in (rotate, norm_fwd, norm_bwd):
        fits(call, rotary(T=0), pos=t(2, 0, 1, dtype=I64))
    fits(cross_fwd, cross(T=0), k_len=t(2, dtype=I32), k_mask=t(2, 20, dtype=U8), lse=t(2, 4, 0, dtype=F32))
    refused(cross_fwd, cross(T=0), "k_len", k_len=t(2, dtype=I64))
