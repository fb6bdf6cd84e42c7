"""Sums of dcd_logits_fp8 for bf16 logits: held in fp32 at every number of rows, and rounded once.

The wider bound that test_gpu_logits_fp8 gives bf16 logits of more than 64 rows is not used here.
"""
import numpy as np
import pytest
import torch

import proposal_oracle as oracle
from tests.test_gpu_logits_fp8 import _dev, _inputs, _run

pytestmark = pytest.mark.gpu
CODE = {-448: 0xFE, -2: 0xC0, -1: 0xB8, 0: 0, 1: 0x38, 2: 0x40, 448: 0x7E}
ENC = np.vectorize(CODE.get, otypes=[np.uint8])


def _integers(M, N, K, pairs, seed):
    """Codes of small whole numbers, with `pairs` neighbouring columns of +-448 that cancel."""
    rng = np.random.RandomState(seed)
    h, w = rng.randint(-2, 3, (M, K)), rng.randint(-2, 3, (N, K))
    at = 8 * rng.permutation(K // 8)[:pairs] + 2 * rng.randint(0, 4, pairs)
    h[:, at] = h[:, at + 1] = 448
    w[:, at], w[:, at + 1] = 448, -448
    codes = (ENC(h), np.ones((M, -(-K // 128)), np.float32), ENC(w), np.ones((-(-N // 128), -(-K // 128)), np.float32),
             np.zeros(N, np.float32))
    return codes, h @ w.T


@pytest.mark.parametrize("pairs", [0, 16])
@pytest.mark.parametrize("M, N, K", [(5, 300, 512), (64, 700, 256), (65, 1000, 256), (100, 777, 400), (190, 3000, 1040),
                                     (285, 1100, 2000), (520, 600, 384)])
def test_whole_numbers(M, N, K, pairs):
    """Products of whole numbers whose magnitudes add up to less than 2^24 (16 pairs: 2 * 16 * 448^2 + 4 K):
    sums in fp32 are exact in any order, and the bf16 logit is that sum rounded once."""
    a, z = _integers(M, N, K, pairs, M)
    assert 2 * pairs * 448 ** 2 + 4 * K < 2 ** 24
    exact = torch.from_numpy(z.astype(np.float32))
    assert torch.equal(_run(a, M, N, K, "f32").cpu(), exact)
    assert torch.equal(_run(a, M, N, K, "bf16").cpu(), exact.bfloat16())


@pytest.mark.parametrize("M, N, K", [(1, 4099, 272), (17, 900, 1040), (64, 3001, 1024), (65, 1000, 512), (100, 2050, 976),
                                     (160, 33000, 256), (190, 3000, 8176), (285, 2000, 2000), (520, 2000, 256),
                                     (1000, 515, 384)])
def test_bf16_logits_are_the_fp32_ones_rounded(M, N, K):
    t = _dev(*_inputs(M, N, K, M))
    assert torch.equal(_run(t, M, N, K, "bf16"), _run(t, M, N, K, "f32").bfloat16())


@pytest.mark.parametrize("M, N, K", [(66, 1500, 2000), (128, 4096, 512), (200, 999, 1536), (300, 300, 8192)])
def test_more_than_64_rows_within_fp32_sums(M, N, K):
    """The bound of fp32 sums of exact products ((130 + groups) * 2^-23 of the magnitudes) and half a step."""
    a = _inputs(M, N, K, M + 1)
    out = _run(a, M, N, K, "bf16").double().cpu().numpy()
    z, mag = oracle.logits(*a[:4], a[4].astype(np.float64))
    tol = (130 + -(-K // 128)) * 2.0 ** -23 * (mag + np.abs(a[4]))
    assert (np.abs(out - z) <= tol + 2.0 ** -8 * (np.abs(z) + tol)).all()


@pytest.mark.parametrize("M", [66, 140, 300])
def test_nan_stays_in_its_row_and_token(M):
    N, K = 700, 400
    a = _inputs(M, N, K, 3)
    clean = _run(a, M, N, K, "bf16").float().cpu().numpy()
    a[1][1, 2] = np.nan
    a[2][300, 17] = 0x7F
    out = _run(a, M, N, K, "bf16").float().cpu().numpy()
    hit = np.zeros((M, N), bool)
    hit[1, :] = hit[:, 300] = True
    assert np.isnan(out[hit]).all()
    assert np.array_equal(out[~hit], clean[~hit])


@pytest.mark.parametrize("M", [40, 100, 180])
def test_repeats_and_replays(M):
    """Bit-identical repeats, and replays of a captured call on new inputs with eager calls in between."""
    N, K = 5003, 1040
    t = _dev(*_inputs(M, N, K, 4))
    first = _run(t, M, N, K, "bf16")
    assert torch.equal(first, _run(t, M, N, K, "bf16"))
    out = torch.empty_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _run(t, M, N, K, "bf16", out=out, stream=torch.cuda.current_stream())
    for seed in (5, 6, 7):
        for dst, src in zip(t, _dev(*_inputs(M, N, K, seed))):
            dst.copy_(src)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, _run(t, M, N, K, "bf16"))


@pytest.mark.parametrize("M, more", [(5, 16), (20, 60), (70, 128), (300, 520)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_do_not_depend_on_the_rows_beside_them(M, more, dtype):
    """A batch's first rows alone: the same bits, where both batches add the blocks of K in one order (up to
    64 rows; one tile of 128 rows, which every number of rows up to that takes; several tiles)."""
    N, K = 13000, 1024
    h, hs, w, ws, bias = _dev(*_inputs(more, N, K, M))
    some = [h[:M].contiguous(), hs[:M].contiguous(), w, ws, bias]
    assert torch.equal(_run(some, M, N, K, dtype), _run([h, hs, w, ws, bias], more, N, K, dtype)[:M])
