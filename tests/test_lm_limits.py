"""Attention calls whose tiles pass what one launch may hold are refused before
anything reaches the GPU."""
import os

import pytest

import paper_1812_08011_amd as fp8t

FAKE = 0x10000        # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fp8t.LIB_PATH):
        pytest.skip("libfp8train.so is not built")
    return fp8t.lib()


def sizes(S, Tq, Tk, H, D=16):
    return S, Tq, Tk, 1, 1, H, H, D, 1, 0.5


def fwd(lib, S, Tq, Tk, H):
    rows = (FAKE, H * 16, 16)
    return lib.attn_fwd_fp8(*rows, *rows, *rows, FAKE, FAKE, *sizes(S, Tq, Tk, H), *rows, None, 0, 0, 1.0,
                            None, FAKE, 1, None)


def bwd(lib, S, Tq, Tk, H):
    rows = (FAKE, H * 16, 16)
    return lib.attn_bwd_fp8(*rows, *rows, *rows, FAKE, FAKE, *sizes(S, Tq, Tk, H), *rows, *rows, FAKE,
                            *rows, *rows, *rows, fp8t.FMT_FP16, 1.0, FAKE, 1, None)


@pytest.mark.parametrize("S,Tq,Tk,H", [(2 ** 24, 1, 1, 1), (2 ** 21, 1, 1, 8), (2 ** 31 - 4097, 1, 1, 1),
                                       (2 ** 29, 1, 1, 64)])
def test_too_many_sequences(lib, S, Tq, Tk, H):
    assert fwd(lib, S, Tq, Tk, H) == fp8t.EINVAL
    assert bwd(lib, S, Tq, Tk, H) == fp8t.EINVAL


def test_too_many_tiles(lib):
    assert fwd(lib, 1, 2 ** 30, 1, 16) == fp8t.EINVAL
    assert bwd(lib, 1, 2 ** 24, 1, 64) == fp8t.EINVAL
    assert bwd(lib, 1, 1, 2 ** 26, 64) == fp8t.EINVAL


def test_the_limit_is_not_lower(lib):
    """Up to it the next check answers: the workspace is too small."""
    assert bwd(lib, 2 ** 24 - 3, 1, 1, 1) == fp8t.EWORKSPACE
    assert bwd(lib, 1, 2 ** 22, 1, 64) == fp8t.EWORKSPACE
