"""distill_loss on logits whose largest is itself a mask value, or far from
zero: only differences between a row's logits decide its softmax."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import say
from tests.lm_util import check, value
from tests.test_gpu_distill import inputs, run

pytestmark = pytest.mark.gpu
LOW32 = np.finfo(np.float32).min
LOW16 = np.uint16(0xFDFF)                              # -(2^32 - 2^22), the lowest FP16 value


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def compare(z, idx, t, w, tau, scale, g_type):
    loss, g = run(z, idx, t, w, tau, scale, g_type)
    want = lm.distill(value(z), idx, value(t), w.astype(np.float64), np.float64(np.float32(tau)), scale)
    check("loss", loss, want[0], want[2])
    check("g", g, want[1], want[3])


@pytest.mark.parametrize("V", [500, 9001, 70001])
@pytest.mark.parametrize("tau", [0.5, 1.0, 4.0])
def test_rows_of_mask_values(tau, V):
    """Every logit at a mask value (a uniform row), or all but some."""
    say(f"distill, masked rows, tau={tau}, V={V}")
    z, idx, t, w = inputs(50, 6, V, 7)
    z[0] = LOW32
    z[1] = -1e30
    z[2] = -1e9
    z[3] = 3e38
    z[4, V // 2:] = LOW32
    idx[4] = np.arange(7)
    z[5] = LOW32
    z[5, idx[5]] = -1.5e38                             # the teacher's, above the others
    compare(z, idx, t, w, tau, 64.0, np.float32)
    z, idx, t, w = inputs(51, 3, V, 7, np.uint16)
    z[0] = LOW16
    z[1] = LOW16 & 0x7FFF
    z[2, 5:] = LOW16
    idx[2, :5] = np.arange(5)
    idx[2, 5:] = -1
    compare(z, idx, t, w, tau, 64.0, np.uint16)


@pytest.mark.parametrize("z_type", [np.float32, np.uint16])
def test_teachers_mask_values(z_type):
    """Teacher's entries all at the lowest value: a uniform target."""
    say("distill, masked teacher")
    z, idx, t, w = inputs(52, 4, 1000, 6, z_type)
    t[0] = LOW32
    t[1, 2:] = LOW32
    t[2] = -1e30
    t[3] = 2e38
    compare(z, idx, t, w, 1.0, 8.0, np.float32)
    z, idx, t, w = inputs(53, 2, 1000, 6, z_type, np.uint16)
    t[0] = LOW16
    compare(z, idx, t, w, 1.0, 8.0, np.float32)


def test_a_target_on_a_masked_logit():
    """Finite logits have a finite loss: q times the distance of the masked one."""
    say("distill, target on a masked logit")
    z, idx, t, w = inputs(54, 2, 300, 3)
    z[0, idx[0, 0]] = -1e38
    z[1, idx[1, 1]] = -1e9
    compare(z, idx, t, w * np.float32(0.25), 1.0, 1.0, np.float32)


@pytest.mark.parametrize("tau", [2.0 ** -30, 2.0 ** -20, 2.0 ** 30])
def test_extreme_temperatures(tau):
    say(f"distill, tau={tau}")
    for z_type in (np.float32, np.uint16):
        z, idx, t, w = inputs(55, 4, 700, 5, z_type, std=30.0)
        z[1] = z[1, 0]                                 # a uniform row
        compare(z, idx, t, w, tau, 1.0, np.float32)
