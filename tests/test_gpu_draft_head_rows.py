"""A DraftHead takes every number of rows up to its largest one."""
import numpy as np
import pytest
import torch

import proposal_oracle
from paper_2608_12913_amd.runner import DraftHead

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V, max_rows, rows", [(128256, 64, (1, 17, 18, 32, 33, 64)), (32003, 200, (66, 67, 128, 129, 200)),
                                               (5000, 600, (1, 512, 513, 600))])
def test_rows_up_to_the_largest(V, max_rows, rows):
    d, gen = 128, torch.Generator(device="cuda:0").manual_seed(V)
    head = DraftHead(torch.randn(V, d, generator=gen, device="cuda:0") * 3 / d ** 0.5, max_rows=max_rows)
    for n in rows:
        h = torch.randn(n, d, generator=gen, device="cuda:0")
        u = np.random.default_rng(n).random(n).astype(np.float32)
        g = head.propose(h, u, top_k=np.full(n, 50, np.int32), top_p=np.full(n, 0.9, np.float32))
        z = head.logits[:n].double().cpu().numpy()
        for r in range(0, n, max(1, n // 8)):
            t, kept, p, _ = proposal_oracle.sample_row(z[r], float(u[r]), k=50, p=float(np.float32(0.9)))
            assert (g["tokens"][r], g["kept"][r]) == (t, kept), (n, r)
            assert (np.abs(g["probs"][r] - p) <= 2.0 ** -23 * p + 2.0 ** -149).all()
