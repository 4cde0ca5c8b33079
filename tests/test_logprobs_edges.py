"""kv_logprobs (include/kvr_logprob.h) on logits whose differences no fp32 number holds:
scale times a difference may still be an ordinary one."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_logprobs import DT, Call  # noqa: E402


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -124, 0.5])
@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("V", [700, 20000])
def test_logits_far_apart(V, dt, scale):
    """Rows over -3.3e38 .. 3.3e38: within a chunk, chunks as a whole, one logit above all."""
    i = torch.arange(V)
    g = torch.Generator().manual_seed(V)
    rows = [torch.where(i < V // 2, 2e38, -2e38), torch.where(i < V // 2, -2e38, 2e38), torch.where(i % 2 == 0, 2e38, -2e38),
            (torch.rand(V, generator=g, dtype=torch.float64) * 2 - 1) * 3.3e38, torch.where(i == V - 9, 3.3e38, -3.3e38),
            torch.where(i < V // 2, -1e38, -3.3e38), torch.where(i == 3, -np.inf, torch.where(i < 9, 3.3e38, -3.3e38))]
    z = torch.stack([r.double() for r in rows]).to(DT[dt])
    c = Call(z, scale, [V - 1, 0, 1, V // 3, 5, V - 1, 3], 12)
    c.run()
    c.check()
