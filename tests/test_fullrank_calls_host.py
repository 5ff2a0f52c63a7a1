"""Refusals of the full-rank operators that need no GPU, beside those of test_fullrank_host.py."""
import ctypes as C

import pytest

from paper_2602_04396_amd import lordo


def _bytes(**hp):
    size, one = C.c_size_t(0), (lordo.Tensor * 1)(lordo.Tensor(4, 4, 1, 0))
    return lordo.load().lordo_adamw_workspace_bytes(one, 1, C.byref(lordo.adamw_hparams(**hp)), C.byref(size))


@pytest.mark.parametrize("decay, code", [(0.0, lordo.OK), (2.0 ** 64, lordo.OK), (2.0 ** 64 * (1 + 2.0 ** -52), lordo.EINVAL), (float("inf"), lordo.EINVAL)])
def test_weight_decay_has_a_limit(decay, code):
    """It meets the weights in fp32, divided by what the bias corrections make of the learning rate."""
    assert _bytes(weight_decay=decay) == code


def test_steps_taken_needs_a_context():
    assert lordo.load().lordo_adamw_steps_taken(None, C.byref(C.c_int64(0)), None) == lordo.EINVAL
