"""pbsa_rotate, pbsa_norm_rotate_fwd and _bwd against the plain forms in 64 bits, within what their roundings allow."""
import math

import pytest
import torch

from paper_2604_21221_amd import layer, pbsa
from tests import layer_reference as ref
from tests.layer_reference import F

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GUARD = 64               # elements on either side of an output that have to stay as they are


def tensor(n, H, T, d, dtype, major, g, pad=0):
    """[n, H, T, d] normal values in the memory order named, `pad` more elements between rows (a multiple of 8)"""
    shape = (n, T, H, d + pad) if major == "token" else (n, H, T, d + pad)
    x = torch.randn(shape, generator=g, device=DEV).to(dtype)[..., :d]
    return x.transpose(1, 2) if major == "token" else x


def guarded(n, H, T, d, dtype, major):
    shape = (n, T, H, d) if major == "token" else (n, H, T, d)
    whole = torch.full((2 * GUARD + n * H * T * d,), 7.0, dtype=dtype, device=DEV)
    x = whole[GUARD:GUARD + n * H * T * d].view(shape)
    return whole, x.transpose(1, 2) if major == "token" else x


def untouched(*wholes):
    for w in wholes:
        assert (w[:GUARD] == 7).all() and (w[-GUARD:] == 7).all(), "written outside the output"


def positions(n, T, axes, far, g):
    return far + torch.randint(-50, 5000, (n, T, axes), generator=g, device=DEV)


CASES = [
    # n, T, Hq, Hk, d, rot, half, sections, dtype, major in, major out, far, mscale, pad
    (1, 1, 1, 0, 16, 16, False, (8,), torch.bfloat16, "token", "token", 0, 1.0, 0),
    (16, 1, 12, 12, 128, 128, True, (64,), torch.bfloat16, "token", "token", 1 << 20, 1.2, 0),
    (3, 1, 5, 1, 64, 64, False, (32,), torch.float16, "head", "head", 1 << 31, 1.0, 8),
    (2, 7, 3, 3, 64, 32, True, (16,), torch.float32, "token", "head", 100, 0.5, 0),
    (1, 33, 12, 4, 128, 128, False, (22, 21, 21), torch.bfloat16, "token", "head", 0, 1.0, 0),
    (1, 1000, 2, 5, 80, 48, False, (10, 7, 7), torch.float16, "head", "token", 1 << 40, 1.0, 16),
    (2, 129, 17, 2, 96, 96, True, (40, 8), torch.bfloat16, "head", "head", 7, 1.0, 0),
    (1, 40, 2, 2, 256, 16, True, (8,), torch.float32, "token", "token", 1 << 20, 1.0, 0),
    (1, 40, 2, 2, 256, 240, False, (120,), torch.bfloat16, "token", "token", 0, 1.0, 0),
    (1, 50, 3, 3, 48, 0, False, (0,), torch.bfloat16, "token", "token", 0, 2.0, 0),
    (1, 2600, 4, 4, 32, 32, True, (16,), torch.bfloat16, "token", "token", 0, 1.0, 0),
    (1, 9000, 2, 1, 64, 64, False, (32,), torch.bfloat16, "token", "head", 0, 1.0, 0),      # many groups of tokens
]


def made(case, seed=0):
    n, T, Hq, Hk, d, rot, half, sections, dtype, mi, mo, far, mscale, pad = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = tensor(n, Hq, T, d, dtype, mi, g, pad)
    k = tensor(n, Hk, T, d, dtype, mi, g, pad) if Hk else None
    freq, _ = layer.rotary_frequencies(sections, device=DEV)
    return g, q, k, positions(n, T, len(sections), far, g), freq


def outputs(case, majors=None):
    n, T, Hq, Hk, d, _, _, _, dtype, _, mo, _, _, _ = case
    a = guarded(n, Hq, T, d, dtype, majors or mo)
    b = guarded(n, Hk, T, d, dtype, majors or mo) if Hk else (torch.full((2 * GUARD,), 7.0, device=DEV), None)
    return a, b


def allowed(y, mag, dtype, ops=32):
    u, floor = ref.unit(dtype)
    return u * y.abs() + ops * F * mag + floor


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_rotate(case, inverse):
    n, T, Hq, Hk, d, rot, half, sections, dtype, _, _, _, mscale, _ = case
    g, q, k, pos, freq = made(case)
    (wq, qo), (wk, ko) = outputs(case)
    p = layer.make_rotary(q, k, qo, ko, sections=sections, half=half, mscale=mscale)
    layer.pbsa_rotate(p, q, k, pos, freq, qo, ko, inverse=inverse)
    angle = ref.angles(pos, freq, sections)
    for x, y in ((q, qo), (k, ko)):
        if x is None:
            continue
        want = ref.rotate(x.double(), angle, rot, half, mscale, inverse)
        mag = ref.rotate(x.double(), angle, rot, half, mscale, inverse, magnitude=True)
        assert ref.worst(y, want, allowed(want, mag, dtype)) <= 1
        assert torch.equal(y[..., rot:], x[..., rot:])     # what is not rotated passes bit for bit
    untouched(wq, wk)
    # in place
    a = q.contiguous()
    b = k.contiguous() if k is not None else None
    p = layer.make_rotary(a, b, a, b, sections=sections, half=half, mscale=mscale)
    layer.pbsa_rotate(p, a, b, pos, freq, a, b, inverse=inverse)
    assert torch.equal(a, qo) and (b is None or torch.equal(b, ko))


def test_rotation_back_gives_the_input():
    g = torch.Generator(device=DEV).manual_seed(3)
    q = torch.randn(2, 3, 50, 64, generator=g, device=DEV)
    freq, _ = layer.rotary_frequencies((32,), device=DEV)
    pos = positions(2, 50, 1, 1 << 30, g)
    p = layer.make_rotary(q, None, q, None)
    y, z = torch.empty_like(q), torch.empty_like(q)
    layer.pbsa_rotate(p, q, None, pos, freq, y, None)
    layer.pbsa_rotate(p, y, None, pos, freq, z, None, inverse=True)
    assert float((z - q).abs().max()) <= 16 * F * 2 * float(q.abs().max())


@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("case", CASES)
def test_norm_rotate(case, weights):
    n, T, Hq, Hk, d, rot, half, sections, dtype, _, _, _, mscale, _ = case
    eps = 1e-5
    g, q, k, pos, freq = made(case, 1)
    w = [1 + 0.3 * torch.randn(d, generator=g, device=DEV) if weights else None for _ in range(2)]
    (gq, qo), (gk, ko) = outputs(case)
    p = layer.make_rotary(q, k, qo, ko, sections=sections, half=half, mscale=mscale, eps=eps)
    layer.pbsa_norm_rotate_fwd(p, q, k, w[0], w[1], pos, freq, qo, ko)
    angle = ref.angles(pos, freq, sections)
    for x, y, v in ((q, qo, w[0]), (k, ko, w[1])):
        if x is None:
            continue
        nx = ref.norm(x.double(), v, eps)
        want = ref.rotate(nx, angle, rot, half, mscale)
        mag = ref.rotate(nx, angle, rot, half, mscale, magnitude=True)
        assert ref.worst(y, want, allowed(want, mag, dtype, 64)) <= 1
    untouched(gq, gk)
    a = q.contiguous()
    b = k.contiguous() if k is not None else None
    p = layer.make_rotary(a, b, a, b, sections=sections, half=half, mscale=mscale, eps=eps)
    layer.pbsa_norm_rotate_fwd(p, a, b, w[0], w[1], pos, freq, a, b)
    assert torch.equal(a, qo) and (b is None or torch.equal(b, ko))


def backward(p, q, k, w, pos, freq, dqo, dko, dq, dk, dw, ws=None):
    if ws is None:
        ws = torch.empty(layer.pbsa_norm_rotate_workspace_bytes(p), dtype=torch.uint8, device=DEV).fill_(255)
    layer.pbsa_norm_rotate_bwd(p, q, k, w[0], w[1], pos, freq, dqo, dko, dq, dk, dw[0], dw[1], ws)


@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("case", CASES)
def test_norm_rotate_gradient(case, weights):
    n, T, Hq, Hk, d, rot, half, sections, dtype, mi, mo, _, mscale, _ = case
    eps = 1e-5
    g, q, k, pos, freq = made(case, 2)
    w = [1 + 0.3 * torch.randn(d, generator=g, device=DEV) if weights else None for _ in range(2)]
    dqo = tensor(n, Hq, T, d, dtype, mo, g)
    dko = tensor(n, Hk, T, d, dtype, mo, g) if Hk else None
    (gq, dq), (gk, dk) = outputs(case, mi)
    dw = torch.full((2, d), math.nan, device=DEV)
    p = layer.make_rotary(q, k, dqo, dko, sections=sections, half=half, mscale=mscale, eps=eps, dq=dq, dk=dk)
    backward(p, q, k, w, pos, freq, dqo, dko, dq, dk, dw)
    angle = ref.angles(pos, freq, sections)
    for i, (x, dy, dx, v) in enumerate(((q, dqo, dq, w[0]), (k, dko, dk, w[1]))):
        if x is None:
            assert (dw[i] == 0).all()
            continue
        gr = ref.rotate(dy.double(), angle, rot, half, mscale, inverse=True)
        gm = ref.rotate(dy.double(), angle, rot, half, mscale, inverse=True, magnitude=True)
        want, want_w, size, size_w = ref.norm_grad(x.double(), v, gr, eps)
        assert ref.worst(dx, want, allowed(want, size(gm), dtype, 96)) <= 1
        assert ref.worst(dw[i], want_w, 160 * F * size_w(gm)) <= 1
    untouched(gq, gk)
    again = torch.empty_like(dw)
    d2q, d2k = torch.empty_like(dq), torch.empty_like(dk) if dk is not None else None
    p2 = layer.make_rotary(q, k, dqo, dko, sections=sections, half=half, mscale=mscale, eps=eps, dq=d2q, dk=d2k)
    backward(p2, q, k, w, pos, freq, dqo, dko, d2q, d2k, again)
    assert torch.equal(again, dw) and torch.equal(d2q, dq) and (dk is None or torch.equal(d2k, dk))
    only = torch.empty(d, device=DEV)                      # the weights' gradients are asked for or not
    backward(p2, q, k, w, pos, freq, dqo, dko, d2q, d2k, (only, None))
    assert torch.equal(only, dw[0]) and torch.equal(d2q, dq)
    if mi == mo and dqo.is_contiguous() and (dko is None or dko.is_contiguous()):
        p3 = layer.make_rotary(q, k, dqo, dko, sections=sections, half=half, mscale=mscale, eps=eps, dq=dqo, dk=dko)
        backward(p3, q, k, w, pos, freq, dqo, dko, dqo, dko, (None, None))   # over the gradients that came in
        assert torch.equal(dqo, dq) and (dk is None or torch.equal(dko, dk))


def test_gradient_against_differences():
    """sum(y * c) of the forward call in binary32, moved along the gradient: a central difference."""
    g = torch.Generator(device=DEV).manual_seed(5)
    q = torch.randn(1, 3, 20, 64, generator=g, device=DEV)
    w = 1 + 0.2 * torch.randn(64, generator=g, device=DEV)
    c = torch.randn(q.shape, generator=g, device=DEV)
    freq, _ = layer.rotary_frequencies((16,), device=DEV)
    pos = positions(1, 20, 1, 0, g)
    dq, dw = torch.empty_like(q), torch.empty(64, device=DEV)
    p = layer.make_rotary(q, None, c, None, sections=(16,), half=True, dq=dq)
    backward(p, q, None, (w, None), pos, freq, c, None, dq, None, (dw, None))

    def value(x, v):
        y = torch.empty_like(x)
        layer.pbsa_norm_rotate_fwd(layer.make_rotary(x, None, y, None, sections=(16,), half=True), x, None, v, None, pos, freq, y, None)
        return float((y.double() * c.double()).sum())

    # the value, of 3840 terms of size 1, is known to 1e-7 of each; curvature over a step of 1e-2 is 1e-4 of the slope
    for of, grad in ((q, dq), (w, dw)):
        way = grad / grad.norm()
        h = 1e-2
        slope = (value(*((q + h * way, w) if of is q else (q, w + h * way))) -
                 value(*((q - h * way, w) if of is q else (q, w - h * way)))) / (2 * h)
        assert abs(slope - float(grad.norm())) <= 2e-3 * float(grad.norm())


def test_infinities_and_nan_stay_in_their_rows():
    q = torch.randn(1, 2, 9, 64, device=DEV).to(torch.bfloat16)
    q[0, 1, 3, 40] = math.inf
    q[0, 0, 5, 3] = math.nan
    y = torch.empty_like(q)
    freq, _ = layer.rotary_frequencies((16,), device=DEV)
    pos = torch.arange(9, device=DEV).view(1, 9, 1) + 1
    p = layer.make_rotary(q, None, y, None, sections=(16,))
    layer.pbsa_rotate(p, q, None, pos, freq, y, None)
    bad = ~torch.isfinite(y)
    assert bad.sum() == 3 and bad[0, 1, 3, 40] and bad[0, 0, 5, 2:4].all()
    layer.pbsa_norm_rotate_fwd(p, q, None, None, None, pos, freq, y, None)
    assert not torch.isfinite(y[0, 0, 5]).any()
    rows = torch.isfinite(y).all(-1)
    assert rows.sum() == 16 and not rows[0, 0, 5] and not rows[0, 1, 3]


def test_shared_positions_and_broadcast_inputs():
    g = torch.Generator(device=DEV).manual_seed(6)
    one = torch.randn(1, 3, 20, 64, generator=g, device=DEV).to(torch.bfloat16)
    q = one.expand(4, 3, 20, 64)                           # all sequences the same memory
    pos = positions(1, 20, 1, 0, g)
    freq, _ = layer.rotary_frequencies((32,), device=DEV)
    y, z = torch.empty(4, 3, 20, 64, dtype=torch.bfloat16, device=DEV), torch.empty_like(one)
    layer.pbsa_rotate(layer.make_rotary(q, None, y, None, pos_stride_b=0), q, None, pos, freq, y, None)
    layer.pbsa_rotate(layer.make_rotary(one, None, z, None), one, None, pos, freq, z, None)
    assert torch.equal(y, z.expand_as(y))


def test_keys_go_straight_into_a_cache():
    """Ko may be the ring slots of a cache: what an append of the rotated keys stores."""
    from paper_2604_21221_amd.cache import PbsaCache
    H, d, B, Nq = 3, 64, 64, 200
    g = torch.Generator(device=DEV).manual_seed(7)
    c = PbsaCache(H, d, B, Nq, 2, 2, 3, 0.125)
    q, k = (torch.randn(1, H, Nq, d, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(Nq, device=DEV).view(1, Nq, 1)
    freq, _ = layer.rotary_frequencies((32,), device=DEV)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    layer.pbsa_norm_rotate_fwd(layer.make_rotary(q, k, qo, ko), q, k, None, None, pos, freq, qo, ko)
    slots = c.Kl[:, c.nqb:2 * c.nqb].view(H, c.nqb * B, d)[None, :, :Nq]      # the second ring position
    layer.pbsa_norm_rotate_fwd(layer.make_rotary(q, k, qo, slots), q, k, None, None, pos, freq, qo, slots)
    assert torch.equal(c.Kl[:, c.nqb:2 * c.nqb].reshape(H, c.nqb * B, d)[:, :Nq], ko[0])
    assert (c.Kl[:, :c.nqb] == 0).all() and (c.Kl[:, 2 * c.nqb:] == 0).all()
    assert (c.Kl[:, c.nqb:2 * c.nqb].reshape(H, c.nqb * B, d)[:, Nq:] == 0).all()


def test_another_stream_and_a_graph():
    case = (2, 300, 4, 2, 64, 64, False, (32,), torch.bfloat16, "token", "head", 0, 1.0, 0)
    g, q, k, pos, freq = made(case, 8)
    w = [torch.rand(64, generator=g, device=DEV) + 0.5 for _ in range(2)]
    (_, qo), (_, ko) = outputs(case)
    dq, dk, dw = torch.empty_like(q), torch.empty_like(k), torch.empty(2, 64, device=DEV)
    p = layer.make_rotary(q, k, qo, ko, dq=dq, dk=dk)
    ws = torch.empty(layer.pbsa_norm_rotate_workspace_bytes(p), dtype=torch.uint8, device=DEV)

    def both():
        layer.pbsa_norm_rotate_fwd(p, q, k, w[0], w[1], pos, freq, qo, ko)
        backward(p, q, k, w, pos, freq, qo, ko, dq, dk, dw, ws)

    both()
    want = [x.clone() for x in (qo, ko, dq, dk, dw)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for x in (qo, ko, dq, dk, dw):
            x.zero_()
        both()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip((qo, ko, dq, dk, dw), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(3):
        q.mul_(1.5)
        k.neg_()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (qo, ko, dq, dk, dw)]
        both()
        assert all(torch.equal(x, y) for x, y in zip((qo, ko, dq, dk, dw), got))


def test_empty_gradients_are_zero():
    q = torch.empty(2, 3, 0, 64, device=DEV)
    dw = torch.full((2, 64), math.nan, device=DEV)
    p = layer.make_rotary(q, q, q, q, dq=q, dk=q)
    backward(p, q, q, (None, None), torch.empty(2, 0, 1, dtype=torch.int64, device=DEV), torch.empty(32, dtype=torch.float64, device=DEV),
             q, q, q, q, dw)
    assert (dw == 0).all()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_an_infinite_gradient_reaches_its_own_weight_alone(half, dtype):
    """An infinity in an element that is not rotated: its weight's gradient is infinite, the other ones are as they are, and of the
    row's own gradient nothing is NaN but what the formula makes so."""
    g = torch.Generator(device=DEV).manual_seed(9)
    q, dy = (torch.randn(1, 2, 9, 64, generator=g, device=DEV).to(dtype) for _ in range(2))
    q[0, 1, 3, 40] = 0.5
    dy[0, 1, 3, 40] = math.inf
    dq, dw = torch.empty_like(q), torch.empty(64, device=DEV)
    freq, _ = layer.rotary_frequencies((16,), device=DEV)
    pos = torch.arange(9, device=DEV).view(1, 9, 1) + 1
    p = layer.make_rotary(q, None, dy, None, sections=(16,), half=half, dq=dq)
    backward(p, q, None, (None, None), pos, freq, dy, None, dq, None, (dw, None))
    gr = ref.rotate(dy.double(), ref.angles(pos, freq, (16,)), 32, half, 1.0, inverse=True)
    want, want_w, _, size_w = ref.norm_grad(q.double(), None, gr, 1e-6)
    assert torch.isinf(want_w).sum() == 1 and torch.isnan(want).sum() == 1
    fine = torch.isfinite(want_w)
    assert torch.equal(dw[~fine], want_w[~fine].float())
    gm = torch.where(torch.isinf(gr), 0.0, ref.rotate(dy.double(), ref.angles(pos, freq, (16,)), 32, half, 1.0, inverse=True, magnitude=True))
    assert ref.worst(dw[fine], want_w[fine], 160 * F * size_w(gm)[fine]) <= 1
    assert torch.equal(torch.isnan(dq), torch.isnan(want)) and torch.equal(torch.isinf(dq), torch.isinf(want))
