"""Verification of fewer drafts than a call has room for: what stands behind a candidate's last draft."""
import math

import pytest
import torch

from tests.test_gpu_verify import gen, rows, sevo  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dist", [False, True])
@pytest.mark.parametrize("temp", [0.0, 0.8])
@pytest.mark.parametrize("T,v", [(3, 5000), (16, 2500)])
def test_rows_behind_the_last_draft_do_not_matter(sevo, T, v, temp, dist):  # noqa: F811
    """Logits, draft ids and uniform numbers behind the count: any bits give the same result."""
    g = gen(T)
    n = 7
    z, y = rows(n, T + 1, v, g), rows(n, T, v, g)
    x = z[:, :T].argmax(2).to(torch.int32)
    u = torch.rand(n, T + 1, generator=g)
    count = torch.tensor([0, 1, T, T - 1, 2, 0, 1], dtype=torch.int32)

    def call():
        ws = torch.full((sevo.sevo_verify_workspace_bytes(n, T, v),), 255, dtype=torch.uint8, device=DEV)
        return sevo.sevo_verify_drafts(z.to(DEV), x.to(DEV), u.to(DEV), temp, draft_logits=y.to(DEV) if dist else None,
                                       n_drafts=count.to(DEV), workspace=ws)
    want = [t.cpu() for t in call()]
    for bad, num in ((math.nan, v - 1), (math.inf, 0), (3.4e38, 2 ** 31 - 1)):
        for i, m in enumerate(count.tolist()):
            z[i, m + 1:], y[i, m:], x[i, m:], u[i, m:T] = bad, bad, num, bad
        assert all(torch.equal(a, b.cpu()) for a, b in zip(want, call()))
