"""snap_rope refuses outputs that share elements with each other, before anything would be launched (no GPU)."""
import ctypes

import pytest

import paper_2511_03092_amd as snap

FAKE = 0x100000  # aligned, never dereferenced
N, HEADS, TOKENS, D = 2, 4, 8, 64


def _status(ys, heads=HEADS, n=N, tokens=TOKENS, x=FAKE, y=FAKE + (1 << 20)):
    """The status of a call whose heads are apart from their output, with the second operand refused in any case, so that
    nothing is launched; the message names the operand."""
    i3 = ctypes.c_int64 * 3
    xs = (HEADS * TOKENS * D, TOKENS * D, D)
    q = snap.SnapRopeHeads(x, y, i3(*(ys if x == y else xs)), i3(*ys), heads)
    k = snap.SnapRopeHeads(0, 0, i3(*xs), i3(*xs), 1)
    L = snap.lib()
    st = L.snap_rope(ctypes.byref(snap.RopeParams(0, D).c()), snap.SNAP_BF16, n, tokens, D, None, 0, None, None,
                     ctypes.byref(q), ctypes.byref(k), None)
    assert st == snap.SNAP_ERR_INVALID_ARG
    return L.snap_last_error().decode()


@pytest.mark.parametrize("ys", [
    (HEADS * TOKENS * D, TOKENS * D, D),          # head by head
    (HEADS * TOKENS * D, D, HEADS * D),           # token by token
    (D, N * TOKENS * D, N * D),                   # sequences innermost
    (-HEADS * TOKENS * D, TOKENS * D, -D),        # backwards
    (9999, 2000, 72),                             # slices of wider rows
    (1 << 30, 1 << 20, D),
])
def test_outputs_that_are_apart_are_taken(ys):
    assert _status(ys).startswith("k:")


@pytest.mark.parametrize("kw", [
    dict(ys=(HEADS * TOKENS * D, TOKENS * D, D - 1)),      # tokens
    dict(ys=(HEADS * TOKENS * D, TOKENS * D, 1)),
    dict(ys=(HEADS * TOKENS * D, TOKENS * D, 1 - D)),
    dict(ys=(HEADS * TOKENS * D, (TOKENS - 1) * D, D)),    # the last token of a head, the first of the next
    dict(ys=(HEADS * TOKENS * D, D, D)),
    dict(ys=(HEADS * TOKENS * D, D, (HEADS - 1) * D)),
    dict(ys=(TOKENS * D, TOKENS * D, D)),                  # the first sequence's head 1, the second's head 0
    dict(ys=(HEADS * TOKENS * D, TOKENS * D, 1), y=FAKE),  # in place
    dict(ys=(HEADS * TOKENS * D, 0, D), y=FAKE),
])
def test_outputs_that_share_elements_are_refused(kw):
    msg = _status(**kw)
    assert msg.startswith("q:") and "stride" in msg


def test_strides_along_sizes_of_one_are_not_looked_at():
    assert _status((0, 1, D), heads=1, n=1).startswith("k:")
    assert _status((0, TOKENS * D, 3), n=1, tokens=1).startswith("k:")
