"""Empty arrays reach the library whatever strides they carry (an empty array
of numpy's becomes a tensor of strides 0)."""
import os

import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(fp8t.LIB_PATH):
        pytest.skip("libfp8train.so is not built")
    fp8t.lib()


def empty(*shape, dtype=np.uint8):
    return torch.from_numpy(np.zeros(shape, dtype))


def test_no_tokens():
    x, y = empty(0, 2, 8), empty(0, 2, 8)
    assert x.stride() == (0, 0, 0)
    none = torch.zeros(4, dtype=torch.float64)
    assert fp8t.rotary_embed(x, empty(0, dtype=np.int64), none, y, stream=0) is y
    cu = torch.zeros(1, dtype=torch.int64)
    fp8t.attn_fwd_fp8(x, x, x, cu, cu, 0, 0, True, 1.0, None, y, stream=0)
    fp8t.attn_bwd_fp8(x, x, x, cu, cu, 0, 0, True, 1.0, empty(0, 2, 8, dtype=np.int16).view(torch.uint16),
                      x, torch.zeros(2, 0), y, y, y, stream=0)


def test_no_rows_of_logits():
    z = empty(0, 9, dtype=np.float32)
    fp8t.distill_loss(z, empty(0, 3, dtype=np.int64), empty(0, 3, dtype=np.float32), None, 1.0, 1.0,
                      torch.zeros(0), z, stream=0)


def test_others_are_still_refused():
    x = torch.zeros((4, 8, 2), dtype=torch.uint8).transpose(1, 2)
    with pytest.raises(ValueError):
        fp8t.rotary_embed(x, torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.float64), x,
                          stream=0)
