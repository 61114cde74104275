"""The chunked oracle of the selective scan against the recurrence, and which calls of its tests go in segments of several
chunks.  No GPU needed."""
import pytest
import torch

import paper_2606_27748_amd as F
from tests import scan_chunks
from tests.layer_util import scan_oracle
from tests.seq_util import F32


@pytest.mark.parametrize("start", [False, True])
@pytest.mark.parametrize("G,H", [(1, 3), (2, 4)])
def test_chunks_are_the_recurrence(G, H, start):
    """Both are in float64: what is left is a few thousand roundings of 2^-53."""
    x = scan_chunks.inputs([1, 64, 0, 200], G, H, 8, 4, F32, G, "cpu")
    want = scan_oracle(x, start, grads=True)
    got, _ = scan_chunks.results(x, start)
    for n, v in got.items():
        assert (v - want[n]).norm() <= 1e-12 * want[n].norm(), n


@pytest.mark.parametrize("N,P,G,H,lengths", scan_chunks.MANY_CHUNKS)
def test_segments_of_the_tests_have_several_chunks(N, P, G, H, lengths):
    tokens = scan_chunks.tokens_of_a_segment(F, len(lengths), sum(lengths), G, H, N, P)
    assert 128 <= tokens and max(lengths) > 2 * tokens, tokens


def test_one_chunk_of_a_few_tokens():
    """As in the tests of small calls."""
    assert scan_chunks.tokens_of_a_segment(F, 5, 763, 1, 6, 128, 64) == 64
