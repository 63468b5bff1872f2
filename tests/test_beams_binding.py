"""A beam search's rule refuses numbers of beams and picks that no call takes, ahead of any arithmetic with them."""

import pytest

from paper_2605_05819_amd import cl
from tests.test_layer_refusals import _raises


@pytest.mark.parametrize("beams,picks", [(0, None), (0, 4), (-3, None), (65, None), (4, 0), (4, -1), (4, 65)])
def test_beams_and_picks(beams, picks):
    _raises(lambda: cl.Beams(beams, picks=picks), "beams and picks must be in 1..64")


def test_the_ends_of_the_range():
    for beams, picks in ((1, 1), (64, 64), (1, 64)):
        assert len(cl.Beams(beams, picks=picks).packed()) == 24
