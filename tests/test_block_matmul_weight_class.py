"""vvs_block_matmul takes a weight of its class alone: an object that has as many bytes is not one."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2511_13587_b200 import binding as vb

ROWS, COLS, OUTS = 5, 144, 200


def call(w):
    vb.vvs_block_matmul(None, torch.zeros((ROWS, COLS), dtype=torch.uint8), torch.zeros((ROWS, 2)), w, torch.zeros((ROWS, OUTS)), stream=0)


class Other(ctypes.Structure):
    _fields_ = vb.vvs_qweight._fields_


class More(vb.vvs_qweight):
    _fields_ = [("more", ctypes.c_int64)]


@pytest.mark.parametrize("size", [ctypes.sizeof(vb.vvs_qweight), ctypes.sizeof(vb._WeightOnDevice)])
def test_objects_of_as_many_bytes(size):
    for wrong in (b"\0" * size, bytearray(size), np.zeros(size // 4, np.float32), np.zeros(size // 8, np.int64), memoryview(bytes(size)),
                  (ctypes.c_char * size)()):
        with pytest.raises(TypeError, match="vvs_qweight"):
            call(wrong)


def test_other_classes_and_none():
    for wrong in (Other(16, COLS, 16, OUTS, COLS), More(16, COLS, 16, OUTS, COLS, 0), vb.vvs_qweight, torch.zeros(8)):
        with pytest.raises(TypeError, match="vvs_qweight"):
            call(wrong)


def test_the_class_and_what_derives_from_it():
    class Same(vb.vvs_qweight):
        pass
    for right in (vb.vvs_qweight(16, COLS, 16, OUTS, COLS), Same(16, COLS, 16, OUTS, COLS)):
        with pytest.raises(ValueError, match="CUDA"):         # the tensors are looked at next
            call(right)
