"""The workspaces that the operators of a training step ask for, without a GPU."""
import ctypes as C

import pytest

from paper_2605_04478_amd import ccld
from tests.test_step_refusals import _expert_args, _vocab_args


def _bytes(query, args):
    need = C.c_uint64(0)
    assert query(C.addressof(args), 1, C.addressof(need)) == 0
    return need.value


@pytest.mark.parametrize("rows", [1, 64, 127, 128, 129, 255, 256, 8192, 65536, 1 << 18, 1 << 20])
@pytest.mark.parametrize("vocab", [1000, 32000, 1 << 20, 1 << 21, 5_000_003])
def test_dz_is_bounded(rows, vocab):
    """dz is half a gigabyte and a line to a row at most, or 4,096 columns where there are more than 65,536 rows.  Beside it, where neither gradient is
    wanted, there are up to 40 bytes to a row and h of 8 columns, twice."""
    need = _bytes(ccld.lib().ccld_vocab_workspace, _vocab_args(rows=rows, vocab=vocab, dh=None, dw=None))
    rows_of_dz = max(rows, 2 * min(rows, 128))
    dz = 2 * rows_of_dz * 4096 if rows > 65536 else (1 << 29) + 512 * rows_of_dz
    assert need <= dz + (40 + 2 * 16) * rows + (1 << 13)


def test_workspaces_do_not_depend_on_addresses():
    at = 1 << 20
    for off in (2, 4, 8):
        for change in (dict(rows=8000, k=2048, n=2048, ldx=2048, ldw=2048, lddy=2048, ldy=2048, lddx=2048, expert_stride=1 << 22),
                       dict(rows=60, k=8192, n=64, ldx=8192, ldw=8192, lddy=64, ldy=64, lddx=8192, expert_stride=1 << 19)):
            aligned = _expert_args(**change)
            shifted = _expert_args(**change, x=at + off, w=at + off, dy=at + off, dw=at + off)
            assert _bytes(ccld.lib().ccld_expert_workspace, aligned) == _bytes(ccld.lib().ccld_expert_workspace, shifted)
        for change in (dict(rows=4096, d=4096, vocab=8192, ldh=4096, ldw=4096, lddh=4096, lddw=4096), dict(rows=60, d=1976, vocab=3047, ldh=1976, ldw=1976, lddh=1976, lddw=1976)):
            aligned, shifted = _vocab_args(**change), _vocab_args(**change, h=at + off, w=at + off)
            assert _bytes(ccld.lib().ccld_vocab_workspace, aligned) == _bytes(ccld.lib().ccld_vocab_workspace, shifted)
