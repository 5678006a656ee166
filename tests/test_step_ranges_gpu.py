"""The operators around the decoder layers at the ends of what their arguments may hold.  Oracles and bounds are those of test_ce_gpu
and test_norm_gpu."""
import numpy as np
import pytest

from tests import test_ce_gpu as tc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [60, 4500])
def test_tokens_of_weight_zero_have_no_gradient_from_the_caller_either(T):
    import torch
    off = [0, 25, 25, T]
    H, W, y = tc._inputs(51, T, 64, 300, 304, ignored=0.1)
    rng = np.random.default_rng(2)
    w = rng.uniform(0.5, 2.0, T).astype(np.float32)
    idle = np.array([3, 24, 30, T - 1])
    w[idle] = [0.0, -0.0, 0.0, 0.0]
    y[idle] = [1, 0, 299, 7]
    dl = rng.normal(size=T).astype(np.float32)
    counted = np.where(w == 0, 0.0, dl.astype(np.float64))
    r = tc._oracle(H, W, y, 300, off, w, dloss=counted)
    H[3], H[T - 1, 7] = np.nan, np.inf
    head = tc._head(H, W, y, 300, off, w)
    loss, lse, job, dH = tc._outs(head)
    print(f"fwd_bwd {T}", flush=True)
    head.fwd_bwd(loss, lse, job, dH, dloss=torch.from_numpy(dl).cuda())
    torch.cuda.synchronize()
    assert not dH[torch.from_numpy(idle).cuda()].any()
    for t in (3, T - 1):                                # (for the comparison of the rest)
        loss[t], lse[t] = float(r["loss"][t]), float(r["lse"][t])
    tc._check((loss, lse, job, dH), r, np.nan_to_num(H, nan=0.0, posinf=0.0), W, y, 300)
