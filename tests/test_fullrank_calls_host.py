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


def test_the_low_rank_context_refuses_lists_made_for_others():
    """The library reads a pointer for each of its matrices, so a shorter list would be read beyond its end."""
    import torch
    low = lordo.Lordo.__new__(lordo.Lordo)
    low.shapes, low.n, low.ctx = [(4, 8, 2), (8, 4, 2)], 2, C.c_void_p()
    two = [torch.zeros(4, 8), torch.zeros(8, 4)]
    low._check_tensors(lordo.PtrList(two, lordo._ptr_array(two)), torch.float32, "pq")
    for bad in (lordo.PtrList(two[:1], lordo._ptr_array(two[:1])),
                lordo.PtrList(two, lordo._ptr_array(two), (torch.device("cuda", 0), lordo.F32, ((4, 8), (8, 4))))):
        with pytest.raises(ValueError):
            low._check_tensors(bad, torch.float32, "pq")
