"""The work memory that beam selection asks for says how a row is cut: more than
eight candidates a segment go with long segments, of which the join reads few."""
import os

import pytest

from paper_2606_29223_amd import dexlib


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n_out", [9, 12, 16, 32, 64])
@pytest.mark.parametrize("requests,beams,vocab", [(1, 1, 8000), (1, 4, 32000), (1, 16, 32000), (1, 64, 4000)])
def test_many_candidates_come_from_long_segments(requests, beams, vocab, n_out, dtype):
    if not os.path.exists(dexlib.LIB_PATH):
        pytest.skip("libdex.so not built")
    work = dexlib.load().dex_beam_select_work
    rows, segments = requests * beams, -(-vocab // 2048)
    a_segment = 8 * n_out + 16                             # its candidates, its sum and maximum
    assert work(dtype, requests, beams, vocab, n_out) == rows * segments * a_segment
    assert work(dtype, requests, beams, vocab, 8) > 0
