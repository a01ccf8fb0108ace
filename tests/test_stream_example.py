"""The example of streams: how it compares its steps, and how far they may be from attention over rows."""
import math
import sys
from pathlib import Path

import pytest
import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))


def test_a_difference_that_is_no_number_is_kept():
    import stream_encoder
    worst, one = torch.zeros(()), torch.ones(3)
    worst = stream_encoder.further(worst, one, one + 0.25)
    assert float(worst) == 0.25
    assert float(stream_encoder.further(worst, one, one)) == 0.25 and float(stream_encoder.further(worst, one[:0], one[:0])) == 0.25
    worst = stream_encoder.further(worst, one, torch.tensor([1.0, math.nan, 1.0]))
    assert math.isnan(worst) and math.isnan(stream_encoder.further(worst, one, one))


@pytest.mark.gpu
@pytest.mark.parametrize("held_as", ["int8", "e4m3"])
def test_steps_against_rows(held_as):
    """A captured step with moments, cap, slopes, causality and streams that end, against attention over the same past as 16-bit rows.  Both sides round to bf16: a
    step of the last product is 2^-6 (results up to 4), of the out-projection's 2^-7 (up to 2).  The attentions differ by 2^-8 of values of size 1 (rows of bf16 next
    to 8-bit values: 2^-9 of a key and of a value, and the results' own 2^-9); with the out-projection's step and that of the norm behind it (2^-7), that
    is 2^-6 through an MLP of gain 2: 2^-5.  Together less than 2^-4, where a pair too many or too few moves results by a few tenths."""
    import stream_encoder
    worst, held, pages, rows = stream_encoder.run(4, 60, held_as)
    assert 0 <= worst <= 2.0 ** -4 and held > 0 and 0 < pages
