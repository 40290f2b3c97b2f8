"""What the weight gradient asks for as workspace: the sums of its ranges of rows, and next to nothing where there is one range."""
import pytest

import paper_2312_08656_amd as maxk


@pytest.mark.parametrize("din,dout", [(1, 1), (100, 47), (384, 384), (4096, 512), (65536, 65536)])
def test_a_single_range_keeps_no_sums(din, dout):
    for N in (0, 1, 31, 32):  # one step of 32 rows is one range whatever tile it is given
        assert 0 < maxk.mx_weight_grad_workspace(N, din, dout) <= 256


@pytest.mark.parametrize("din,dout", [(64, 64), (256, 256), (384, 384)])
def test_ranges_keep_their_sums(din, dout):
    assert maxk.mx_weight_grad_workspace(232965, din, dout) >= 2 * 4 * dout * (din + 1)


def test_too_small_a_workspace_is_named():
    text = maxk.load_library().maxk_status_string(-5)
    assert b"workspace" in text and b"scratch" in text
