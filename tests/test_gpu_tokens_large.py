"""What large inputs select: shares of many sorted tokens in embed_bwd, and results
past the caches (beyond 32 MB) of the gradients.  Sums of small whole numbers are
exact and rows repeat, so that results are compared bit for bit."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, dev, host, say
from tests.token_util import F8, F16, F32, TORCH, Wide, draw, gpu, rounded, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def sums(tok, e, V):
    """The errors (whole numbers) of each row, added."""
    used = np.flatnonzero((tok >= 0) & (tok < V))
    order = used[np.argsort(tok[used], kind="stable")]
    at = np.flatnonzero(np.diff(tok[order], prepend=-1))
    g = np.zeros((V, e.shape[1]), np.int32)
    if len(order):
        g[tok[order][at]] = np.add.reduceat(e[order], at, axis=0)
    return g


def runs(rng, T):
    """T tokens in runs whose lengths lie at the borders of shares, pieces and what
    is not cut, each second token named, in a random order."""
    lengths, n = [], 0
    while n < T:
        lengths.append(min(int(rng.choice([1, 2, 3, 5, 15, 16, 17, 31, 32, 33, 34, 47, 48, 49, 63, 64, 65, 100, 129, 700])), T - n))
        n += lengths[-1]
    return rng.permutation(np.repeat(np.arange(len(lengths)) * 2, lengths)), 2 * len(lengths)


def embed_bwd(tok, e, V, e_ty, g_ty, scale=1.0, pad=0, shift=0):
    say(f"embed_bwd T={len(tok)} V={V} W={e.shape[1]} {e_ty.__name__} -> {g_ty.__name__}")
    ed, g = Wide(*e.shape, e_ty, pad, shift, rounded(e.astype(F32), e_ty)), Wide(V, e.shape[1], g_ty, pad, shift)
    td = dev(tok)
    n = fp8t.embed_bwd_workspace_size(td, ed.view, g.view)
    fp8t.embed_bwd(td, ed.view, g.view, scale, workspace(n), n)
    return g.result()


@pytest.mark.parametrize("share", range(4, 18))
def test_gradient_shares(share):
    """Rows of 512: a group of lanes is a wave, its share T / 2048 of the sorted
    tokens, 16 at most."""
    rng = np.random.default_rng(150)
    tok, V = runs(rng, 2048 * share + 5)
    e = rng.integers(-3, 4, (len(tok), 512), dtype=np.int32)
    assert np.array_equal(embed_bwd(tok, e, V, F8, F32), sums(tok, e, V).astype(F32))


@pytest.mark.parametrize("T,W", [(16400, 1030), (33000, 260), (70000, 130), (262200, 40)])
def test_gradient_of_large_batches(T, W):
    """Shares of 16 in groups of 64, 32 and 8 lanes, several slabs of columns."""
    rng = np.random.default_rng(151)
    tok, V = runs(rng, T)
    e = rng.integers(-3, 4, (T, W), dtype=np.int32)
    for e_ty, g_ty in ((F16, F32), (F8, F16)):
        want = rounded(sums(tok, e, V).astype(F32), g_ty, 2.0)
        assert np.array_equal(embed_bwd(tok, e, V, e_ty, g_ty, 2.0, 3, 1), want)


@pytest.mark.parametrize("ty,V", [(F32, 9001), (F16, 18003), (F8, 34001)])
def test_embedding_gradient_past_the_caches(ty, V):
    rng = np.random.default_rng(152)
    tok = rng.integers(0, V, 6000)
    tok[:900], tok[2000:2050] = 17, V - 1
    e = rng.integers(-3, 4, (6000, 1003), dtype=np.int32)
    for pad, shift in ((0, 0), (3, 1)):
        assert np.array_equal(embed_bwd(tok, e, V, F16, ty, 1.0, pad, shift), rounded(sums(tok, e, V).astype(F32), ty))


def same_blocks(big, small):
    """Every block of rows of the large result against the small one."""
    raw = torch.int16 if big.dtype == torch.uint16 else torch.int32 if big.dtype == torch.float32 else big.dtype
    n = len(big) // len(small)
    return bool((big.view(raw).view(n, *small.shape) == small.view(raw)).all())


def repeated(a, n):
    d = dev(a)
    raw = d.view(torch.int16) if d.dtype == torch.uint16 else d
    big = raw.repeat(n, *[1] * (raw.dim() - 1))
    return d, big.view(torch.uint16) if d.dtype == torch.uint16 else big


@pytest.mark.parametrize("rows,times,W", [(400, 84, 1003), (40, 190, 4500), (20, 190, 9001), (20, 100, 17001)])
@pytest.mark.parametrize("ty", [F32, F16])
def test_norm_gradients_past_the_caches(ty, rows, times, W):
    rng = np.random.default_rng(153)
    say(f"rms_norm_bwd past the caches {rows * times}x{W} {ty.__name__}")
    h, H = repeated(draw(rng, (rows, W), F16), times)
    dy, DY = repeated(draw(rng, (rows, W), F8), times)
    dr, DR = repeated(draw(rng, (rows, W), ty), times)
    rstd, RSTD = repeated(np.exp(rng.standard_normal(rows)).astype(F32), times)
    w = dev(draw(rng, W, F16))
    out = lambda t, dtype: torch.empty(t.shape, dtype=dtype, device=DEV)
    dx, DX, dx8, DX8 = out(dr, dr.dtype), out(DR, dr.dtype), out(dr, torch.uint8), out(DR, torch.uint8)
    fp8t.rms_norm_bwd(h, w, rstd, dy, dr, dx, dx8, 3.0)
    fp8t.rms_norm_bwd(H, w, RSTD, DY, DR, DX, DX8, 3.0)
    assert same_blocks(DX, dx) and same_blocks(DX8, dx8)
    fp8t.rms_norm_bwd(H, w, RSTD, DY, DR, DR)               # in place
    assert same_blocks(DR, dx)


@pytest.mark.parametrize("z_ty,g_ty,times", [(F32, F32, 9), (F16, F16, 18), (F16, F8, 36), (F32, F8, 36), (F32, F16, 18)])
@pytest.mark.parametrize("V", [50001, 50008])
def test_logit_gradients_past_the_caches(z_ty, g_ty, times, V):
    rng = np.random.default_rng(154)
    say(f"token_logprobs_bwd past the caches {20 * times}x{V} {z_ty.__name__} -> {g_ty.__name__}")
    z, Z = repeated(draw(rng, (20, V), z_ty, 2.0), times)
    idx, IDX = repeated(rng.integers(-1, V, (20, 3)), times)
    dl, DL = repeated(draw(rng, (20, 3), F32), times)
    dh, DH = repeated(draw(rng, 20, F32), times)
    stats, H = torch.empty((20, 2), device=DEV), torch.empty(20, device=DEV)
    fp8t.token_logprobs(z, None, 1.0, entropy=H, stats=stats)
    g, G = (torch.empty(t.shape, dtype=TORCH[g_ty], device=DEV) for t in (z, Z))
    fp8t.token_logprobs_bwd(z, idx, 1.0, stats, H, dl, dh, 1e4, g)
    STATS, HH = stats.repeat(times, 1), H.repeat(times)
    fp8t.token_logprobs_bwd(Z, IDX, 1.0, STATS, HH, DL, DH, 1e4, G)
    assert same_blocks(G, g)
    if z_ty == g_ty:
        fp8t.token_logprobs_bwd(Z, IDX, 1.0, STATS, HH, DL, DH, 1e4, Z)
        assert same_blocks(Z, g)
