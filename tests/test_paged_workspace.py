"""The paged calls' workspace queries: one workspace, sized for a program's largest call, serves its smaller ones."""
import pytest

import paper_2511_03092_amd as snap
from pagedhelp import params

HEADS = [(32, 8, 128, "bf16", False), (8, 8, 64, "fp8", False), (16, 1, 576, "fp8", True), (4, 2, 64, "f32", False)]
ROWS = [1, 31, 32, 33, 4095, 4096, 4097, 8191, 8192, 8193, 9000, 12288, 12289, 16384, 16385, 40000, 131071, 131072, 131073,
        131077, 262144, 262145, 1 << 20, (1 << 20) + 1]
COUNTS = [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513, 2000]


def _monotone(query):
    """query(n, rows) never falls as either grows."""
    got = [[query(n, r) for r in ROWS] for n in COUNTS]
    assert all(x > 0 for row in got for x in row)
    for i, n in enumerate(COUNTS):
        for j, r in enumerate(ROWS):
            if i:
                assert got[i][j] >= got[i - 1][j], (COUNTS[i - 1], n, r, got[i - 1][j], got[i][j])
            if j:
                assert got[i][j] >= got[i][j - 1], (n, ROWS[j - 1], r, got[i][j - 1], got[i][j])


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("topk", [0, 4000, 14000])
def test_eviction_needs_no_more_for_fewer_sequences_or_rows(heads, topk):
    p = params(*heads, topk=topk)
    _monotone(lambda n, r: snap.snap_paged_evict_workspace(p, n, r))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("weigh", [False, True])
def test_attention_needs_no_more_for_fewer_sequences_or_rows(heads, weigh):
    p = params(*heads)
    _monotone(lambda n, r: snap.snap_paged_decode_workspace(p, n, r, weigh))


@pytest.mark.parametrize("heads", HEADS)
def test_attention_needs_no_more_without_weights(heads):
    p = params(*heads)
    for n in COUNTS:
        for r in ROWS:
            a, b = (snap.snap_paged_decode_workspace(p, n, r, w) for w in (False, True))
            assert a <= b, (n, r, a, b)
