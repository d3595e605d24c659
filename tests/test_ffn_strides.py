"""Row strides, and the workspace's size, as the binding takes them from tensors (no GPU)."""
import pytest
import torch

from paper_1705_01626_amd import ffn, zvc

FAR = ffn.MAX_COLUMNS * 2


def stride_of(t, rows, cols):
    return ffn._matrix(t, rows, cols, t, "call", "t")


@pytest.mark.parametrize("rows", [0, 1])
def test_a_single_row_has_no_stride(rows):
    """One token of a tensor whose rows lie far apart, or at an odd stride: the stride is never used, so it is neither too large nor
    unaligned."""
    for stride in (FAR, FAR + 1, 9, 8, 3, 0):
        t = torch.zeros(FAR + 64).as_strided((rows, 8), (stride, 1))
        assert stride_of(t, rows, 8) == 8
        assert not ffn._loose(t)


def test_columns_of_one_element():
    base = torch.zeros(64, 8)
    assert stride_of(base[:, 3:4], 64, 1) == 8
    assert stride_of(torch.zeros(1, 64).t(), 64, 1) == 1
    assert stride_of(torch.zeros(5).as_strided((1, 1), (0, 0)), 1, 1) == 1


def test_more_rows_keep_theirs():
    for stride in (8, 9, 16, FAR):
        assert stride_of(torch.zeros(FAR + 64).as_strided((2, 8), (stride, 1)), 2, 8) == stride
    assert ffn._loose(torch.zeros(64).as_strided((2, 8), (9, 1)))
    for stride in (0, 7):
        with pytest.raises(zvc.ZvcError, match="strides"):
            stride_of(torch.zeros(64).as_strided((2, 8), (stride, 1)), 2, 8)


def test_the_pair_of_a_single_row():
    a, b = torch.zeros(2, FAR)[:1, :8], torch.zeros(1, 8)
    assert ffn._pair(a, b, 1, 8, a, "call", ("a", "b"))[2] == 8


@pytest.mark.parametrize("ws", [torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20, dtype=torch.uint8)[::2],
                                torch.zeros(64, 64, dtype=torch.uint8)[:, :32]])
def test_a_workspace_with_gaps_or_without_memory_is_refused(ws):
    """Its number of elements says nothing of the memory behind its address."""
    x, w, h = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, 6)
    for call in (lambda: ffn.zvc_glu_forward(x, w, w, h, ws),
                 lambda: ffn.zvc_glu_backward(h, x, w, w, x.clone(), w.clone(), w.clone(), ws)):
        with pytest.raises(zvc.ZvcError, match="contiguous"):
            call()
