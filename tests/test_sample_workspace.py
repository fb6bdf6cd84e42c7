"""dcd_sample_workspace_bytes never falls as the rows grow: what a largest batch needs, every smaller one
runs in."""
import pytest

from paper_2608_12913_amd import dcd


def _need(rows, vocab, dtype="f32"):
    return dcd.sample_workspace_bytes(dcd.make_sample_problem(rows, vocab, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 3, 4, 100, 2048, 2049, 5000, 8192, 8193, 32003, 50257, 128256, 151936, 262144,
                                   (1 << 20) - 1, 1 << 20, (1 << 20) + 1])
def test_never_falls(vocab, dtype):
    rows = list(range(1, 1100)) + [2047, 2048, 4096, 20000]
    need = [_need(r, vocab, dtype) for r in rows if (vocab // 2048 + 1) * r < 1 << 24]
    assert all(n > 0 for n in need)
    assert all(a <= b for a, b in zip(need, need[1:]))
