"""dcd_quantize_fp8 against the definition in 64 bits: codes and scales bit for bit."""
import numpy as np
import pytest
import torch

import proposal_oracle as oracle
from paper_2608_12913_amd import dcd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _run(x, block, dtype, stream=None):
    rows, cols = x.shape
    q = torch.full((rows, cols), 99, dtype=torch.uint8, device=DEV)
    s = torch.full((-(-rows // block), -(-cols // 128)), 7.0, device=DEV)
    dcd.quantize_fp8(x, q, s, rows=rows, cols=cols, dtype=dtype, block_rows=block,
                     stream=stream or torch.cuda.current_stream())
    return q, s


def _check(x, block, dtype):
    q, s = _run(x, block, dtype)
    qo, so = oracle.quantize(x.double().cpu().numpy(), block)
    assert np.array_equal(s.cpu().numpy(), so, equal_nan=True)
    assert np.array_equal(q.cpu().numpy(), qo)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows, cols", [(1, 16), (1, 128), (3, 144), (127, 256), (128, 1008), (129, 112), (515, 2000),
                                        (5000, 4096)])
def test_codes_and_scales(dtype, block, rows, cols):
    gen = torch.Generator(device=DEV).manual_seed(rows * 7 + cols)
    x = torch.randn(rows, cols, generator=gen, device=DEV) * 4
    _check(x.bfloat16() if dtype == "bf16" else x, block, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [1, 128])
def test_ends_of_the_range(dtype, block):
    """Groups of zeros, of tiny and subnormal values, of the largest ones; with infinities and NaN."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(1152, 256, generator=gen, device=DEV)
    for i, f in enumerate([0.0, 1e-38, 1e-42, 1e-30, 1e36, 3e37, 1e-18, 2.0 ** -126]):
        x[128 * i:128 * (i + 1)] *= f
    x = x.bfloat16() if dtype == "bf16" else x
    x[1024] = torch.finfo(x.dtype).max
    x[1030, 3], x[1031, 200], x[1032, 130] = float("inf"), float("nan"), -float("inf")
    x[1040, :128] = -0.0
    _check(x, block, dtype)


def test_every_border():
    """Quotients on and one unit beside every border between two codes, and on the codes."""
    v = oracle.e4m3_values()
    mid = np.concatenate([v, (v[1:] + v[:-1]) / 2]).astype(np.float32)
    near = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(500))])
    near = np.concatenate([near, -near])
    near = near[np.abs(near) <= 448]
    near = np.resize(near, (-(-len(near) // 127), 127))
    for f in (1.0, 3.0, 0.7, 1 / 3, 2.0 ** -100, 2.0 ** -120):
        x = np.concatenate([np.full((len(near), 1), 448.0, np.float32), near], axis=1) * np.float32(f)
        _check(torch.from_numpy(x).to(DEV), 1, "f32")


def test_many_groups_and_repeats():
    """The variant of several groups per lane (above 65,536 groups), a group count that is no
    multiple of its step, on another stream and twice."""
    gen = torch.Generator(device=DEV).manual_seed(9)
    x = (torch.randn(33000, 400, generator=gen, device=DEV) * 3).bfloat16()
    _check(x, 1, "bf16")
    q0, s0 = _run(x, 1, "bf16")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        q1, s1 = _run(x, 1, "bf16", st)
    st.synchronize()
    assert torch.equal(q0, q1) and torch.equal(s0, s1)
