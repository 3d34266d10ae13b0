"""include/pbsa_layer.h at the ends of its ranges, without a GPU: which kernel a masked forward call goes to where its states' offsets
reach the end of 32 bits, seen by the scratch that it asks for."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2604_21221_amd import layer, pbsa  # noqa: E402
from tests.test_layer_abi import A, ESHAPE, EWS, cross, cross_fwd, refused  # noqa: E402

LOAD = 240 + 3 * 1024    # bytes that a load of the list kernel adds to its state's offset: a chunk of the row, its place among four


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(pbsa.LIB_PATH):
        from paper_2604_21221_amd import build
        build.build()


def by_list(d, Nk, step):
    """Whether a masked call of many rows, states `step` elements apart, goes to the kernel that walks a list of states: it needs room
    for the list (the other kernel, with so many rows, and a call without a mask need none)."""
    p = cross(n=1, T=40000, Nk=Nk, Hq=1, Hk=1, d=d, k=(0, 0, step), v=(0, 0, d))
    q = cross(n=1, T=40000, Nk=Nk, Hq=1, Hk=1, d=d, k=(0, 0, d), v=(0, 0, step))
    size = layer.pbsa_cross_workspace_bytes(p)
    assert size == layer.pbsa_cross_workspace_bytes(q) and size in (0, 4 * (64 + Nk))
    return size > 0


@pytest.mark.parametrize("d,step", [(64, 64), (64, 1 << 20), (128, 128), (128, 136), (128, 256), (128, 512), (128, 768), (128, 1 << 12),
                                    (128, 1 << 24)])
def test_offsets_of_listed_states_stay_within_32_bits(d, step):
    most = min(layer.PBSA_CROSS_MAX_NK, (1 << 32) // (2 * step) + 3)
    for Nk in range(most, max(most - 40, 0), -1):
        if by_list(d, Nk, step):
            assert (Nk - 1) * 2 * step + LOAD + 16 <= 1 << 32, Nk
    far = (1 << 32) // (2 * step) // 2                       # halfway there is nothing to be careful about
    assert by_list(d, far, step)


def test_more_rows_than_a_launch_takes_are_refused():
    """Masked states that lie too far apart for a list go by units of 32 rows, 256 threads to each."""
    for T, Hq in ((1 << 30, 1), ((1 << 29) + 32, 1), (1 << 22, 256)):
        refused(ESHAPE, cross_fwd, cross(n=1, T=T, Nk=129, Hq=Hq, Hk=1, d=64, k=(0, 0, 1 << 24), q=(0, 0, 0), o=(0, 64 * T, 64)), k_mask=A)
    # half as many go on to the next check
    refused(EWS, cross_fwd, cross(n=1, T=40, Nk=1 << 14, Hq=1, Hk=1, d=64, k=(0, 0, 1 << 24)), k_mask=A, ws=None)
