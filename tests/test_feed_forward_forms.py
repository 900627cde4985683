"""Which form of the feed-forward half a size takes (csrc/linear_plan.h, compiled for the host): the GPU tests' sizes take the forms that they name, and
no form that one of 40000 drawn sizes takes is without a test.  A change of the costs that the choice goes by shows here."""
import math
import random

import pytest

from tests import plans
from tests import test_gpu_feed_forward as general
from tests import test_gpu_padding_tiles as padding
from tests.test_gpu_feed_forward_forms import BACKWARD, FORWARD


def test_forward_sizes_take_the_named_forms():
    for B, N, E, F, codes, form in FORWARD:
        assert plans.forward(B * N, E, F, codes) == form, (B, N, E, F, codes)
    for B, N, E, F, form in padding.FORWARD:
        assert plans.forward(B * N, E, F, True) == form, (B, N, E, F)


def test_backward_sizes_take_the_named_forms():
    for B, N, E, F, form, how in BACKWARD:
        assert plans.backward(B * N, E, F) == (form, how), (B, N, E, F)
    for B, N, E, F, form in padding.BACKWARD:
        assert plans.backward(B * N, E, F)[0] == form, (B, N, E, F)


def sizes():
    """Tokens and widths over the whole range, each with its neighbours' shapes: one to 70000 tokens, 8 to 65536 wide."""
    rng = random.Random(0)
    log = lambda top: int(math.exp(rng.uniform(0, math.log(top))))
    for _ in range(40000):
        yield log(70000), 8 * log(8192), 8 * log(8192)


def test_every_form_is_tested():
    forward = {codes: {form for *_, c, form in FORWARD if c == codes} for codes in (0, 1)}
    # a tile, a split and their number of ranges are the same kernel whether results are kept in 8 bits, few tokens' forms are not
    anywhere = forward[0] | forward[1]
    # dw's kernel and whether several ranges of it are added, dx's tiles and its number of ranges: each, and the two that one launch has together
    part = lambda form: {form.split(", dx")[0].replace("ranges 9", "ranges 2"), form.split(", ")[0] + form.split(",")[-1]}
    backward = set().union(*(part(form) for *_, form, _ in BACKWARD))
    both = {tuple(sorted(part(form))) + (how,) for *_, form, how in BACKWARD if form.startswith("one")}
    assert {how for *_, how in BACKWARD} == {"direct", "copied"} and len(both) > 20
    for T, E, F in sizes():
        for codes in (0, 1):
            form = plans.forward(T, E, F, codes)
            assert form in (forward[codes] if form.startswith("few") else anywhere), (T, E, F, codes, form)
        form, _ = plans.backward(T, E, F)
        dw, dx = form.split(", dx")[0], form.split(", ")[0] + form.split(",")[-1]
        if dw.startswith("two") and "ranges 1" not in dw:   # (added behind the product, however many there are)
            dw = dw[:dw.index("ranges")] + "ranges 2" + (" listed apart" if "listed" in dw else "")
        assert dw in backward, (T, E, F, form)
        assert dx in backward, (T, E, F, form)


@pytest.mark.parametrize("B,N,E,F", general.SPLITS)
def test_sizes_of_the_split_tests_are_split_with_results_in_8_bits(B, N, E, F):
    assert plans.forward(B * N, E, F, True).startswith("split")
