"""What the binding hands on of changed scores, on the CPU."""
import pytest

from paper_2307_02628_amd import skd


@pytest.mark.parametrize("window", [1 << 31, (1 << 32) + 5, 5 - (1 << 32), -(1 << 31) - 1])
def test_windows_beyond_32_bits_are_refused(window):
    """(and not cut to another window)"""
    with pytest.raises(ValueError):
        skd.KvScores(window=window)


@pytest.mark.parametrize("window", [0, 1, (1 << 31) - 1, -1, -(1 << 31)])
def test_others_reach_the_call_as_they_are(window):
    assert skd.KvScores(window=window).c.window == window
