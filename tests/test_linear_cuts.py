"""Which cuts the layer products can be asked for (runs without a GPU)."""
import threading

import pytest

import paper_2605_29843_b200 as harp
from paper_2605_29843_b200 import build as harp_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    harp_build.build()
    yield
    harp.harp_linear_set_cut(0)


@pytest.mark.parametrize("cut", [(256, 1, 0), (32, 1, 0), (32, 1, 1), (32, 2, 0), (32, 4, 0), (64, 1, 0), (64, 1, 1), (64, 2, 0), (64, 2, 1), (64, 4, 0),
                                 (64, 4, 1), (0, 1, 0), (0, 0, 0)])
def test_cuts(cut):
    assert harp.lib().harp_linear_set_cut(*cut) == 0


@pytest.mark.parametrize("cut", [(256, 2, 0), (256, 1, 1), (128, 1, 0), (32, 3, 0), (32, 0, 0), (32, 8, 0), (32, 2, 1), (32, 4, 1), (64, 1, 2), (64, -1, 0),
                                 (-1, 1, 0), (33, 1, 0)])
def test_refusals(cut):
    assert harp.lib().harp_linear_set_cut(*cut) == 2
    if cut[2] in (0, 1):
        with pytest.raises(harp.HarpError):
            harp.harp_linear_set_cut(*cut)


def test_no_product_yet():
    """A thread's own: what another one asked for or took is not seen."""
    harp.harp_linear_set_cut(64, 2)
    seen = []
    t = threading.Thread(target=lambda: seen.append(harp.harp_linear_last_cut()))
    t.start()
    t.join()
    assert seen == [(0, 1, False)]
