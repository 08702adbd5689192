"""The scratch size of layer norm's backward pass over the sizes that its arguments can have (no GPU needed)."""
import ctypes

import pytest

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb

MOST, MOST_FEATURES = 1 << 27, 1 << 24


@pytest.fixture(scope="module")
def work():
    darb_build.build()
    L = darb.lib()

    def call(layout, steps, tokens, features):
        need = ctypes.c_int64(-7)
        return L.darb_layer_norm_grad_work(layout, steps, tokens, features, ctypes.byref(need)), need.value
    return call


@pytest.mark.parametrize("layout,steps,tokens,features", [
    (1, MOST, MOST, MOST_FEATURES), (1, MOST, MOST, 1), (1, MOST, MOST, 64), (1, MOST, 1, MOST_FEATURES), (1, 1, MOST, MOST_FEATURES),
    (0, 1, MOST, MOST_FEATURES), (1, 1 << 25, 1 << 20, 1 << 3 | 1), (1, MOST, 1 << 21, 2)])
def test_activations_of_more_elements_than_a_call_takes_are_unsupported(work, layout, steps, tokens, features):
    assert steps * tokens * features > 1 << 48
    assert work(layout, steps, tokens, features) == (darb.ERR_UNSUPPORTED, -7)


@pytest.mark.parametrize("layout,steps,tokens,features", [
    (1, MOST, 1 << 21, 1), (1, 1 << 24, 1, MOST_FEATURES), (1, 1, 1 << 24, MOST_FEATURES), (0, 1, 1 << 24, MOST_FEATURES), (1, MOST, 3, 1 << 19),
    (0, 1, MOST, 1), (1, 1, MOST, 1)])
def test_the_largest_that_it_takes(work, layout, steps, tokens, features):
    st, need = work(layout, steps, tokens, features)
    # a partial result of features and up to 14 more in fp32, twice, for 4 tokens at least (a step of fewer, a row); all in 64 bits
    partials = steps * -(-tokens // 4)
    assert st == darb.OK and 0 < need <= 64 * max(partials, 1 << 16) * (features + 14)


def test_no_tokens(work):
    assert work(0, 1, 0, 100)[0] == darb.OK and work(1, 0, 5, 100)[0] == darb.OK and work(1, 5, 0, 100)[0] == darb.OK
