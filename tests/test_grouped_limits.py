"""Sizes of the grouped products inside every width's limit whose tiles are too many to number (no GPU: only calls that
are refused, or that have nothing to do)."""
import ctypes

from test_grouped_checks import BF16, FAKE, L, OK, TOO_LARGE  # noqa: F401

ROWS, WIDE = 2 ** 31 - 1, 2 ** 22


def backward(L, n, k, m, dX=None, dW=None, db=None):
    return L.cogdl_grouped_linear_backward(n, 2, k, m, FAKE, FAKE, FAKE, FAKE, None, None, BF16, None, 0, dX, dW, BF16,
                                           db, None, 0, None)


def test_the_widest_sizes_are_allowed(L):  # noqa: F811
    """Nothing to do, so nothing is launched: what is refused below is not refused for its rows or widths."""
    size = ctypes.c_size_t()
    assert L.cogdl_grouped_linear_backward_workspace(ROWS, 2, WIDE, WIDE, ctypes.byref(size)) == OK
    assert L.cogdl_grouped_linear(0, 2, WIDE, WIDE, FAKE, None, None, BF16, None, 0, None, BF16, None, None, None) == OK
    assert L.cogdl_grouped_linear(ROWS, 2, 4, 0, FAKE, FAKE, None, BF16, None, 0, None, BF16, None, None, None) == OK
    assert backward(L, ROWS, WIDE, WIDE) == OK


def test_more_tiles_than_32_bits_number(L):  # noqa: F811
    assert L.cogdl_grouped_linear(ROWS, 2, 4, WIDE, FAKE, FAKE, FAKE, BF16, None, 0, FAKE, BF16, None, None,
                                  None) == TOO_LARGE
    # the checkpoint of X is not written either
    assert L.cogdl_grouped_linear(ROWS, 2, 4, WIDE, FAKE, FAKE, FAKE, BF16, None, 0, FAKE, BF16, FAKE, FAKE,
                                  None) == TOO_LARGE
    assert backward(L, ROWS, WIDE, 4, dX=FAKE) == TOO_LARGE
    assert backward(L, 16, WIDE, WIDE, dW=FAKE) == TOO_LARGE
    assert backward(L, 16, WIDE, WIDE, dW=FAKE, db=FAKE) == TOO_LARGE
