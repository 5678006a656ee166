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


@pytest.mark.parametrize("shift,size", [(50.0, 1e-13), (50.0, 1e-20), (50.0, 1e-30), (-27.0, 1e31), (0.0, 1e-30), (0.0, 1e30)])
def test_upstream_gradients_far_from_one(shift, size):
    """Rows whose logarithm of the sum is 57 or -20, with gradients of which the product with exp(57) or exp(-20) is no ordinary number,
    beside rows of gradients near one and of zero.  (A row that is brought to another reference has its exponentials rounded twice.)"""
    import torch
    T, d, V = 70, 64, 1111
    off = [0, 30, 70]
    H, W, y = tc._inputs(52, T, d, V, 1112, std=1.0, shift=shift, ignored=0.1)
    dl = (np.random.default_rng(3).normal(size=T) * size).astype(np.float32)
    dl[::5] = np.random.default_rng(4).normal(size=14).astype(np.float32)
    dl[::7] = 0.0
    r = tc._oracle(H, W, y, V, off, dloss=dl.astype(np.float64))
    head = tc._head(H, W, y, V, off)
    out = tc._outs(head)
    print(f"fwd_bwd {shift} {size}", flush=True)
    head.fwd_bwd(*out, dloss=torch.from_numpy(dl).cuda())
    torch.cuda.synchronize()
    tc._check(out, r, H, W, y, V, roundings=2)
    # That bound has a floor for what rounds to zero, so the smallest gradients are held to their own size as well, without the feature
    # that holds the shift (its gradient is a difference of equal numbers): two roundings of an exponential and the logits' error leave
    # (2^-7 + 4 exp_err) sum_v |P_v| |W_v| of a row, the last rounding 2^-8 of it.
    rows = np.flatnonzero(dl[r["live"]])
    at, W64 = r["live"][rows], W[:-1, :V].astype(np.float64)
    exp_err = tc._bounds(r, H, W[:, :V])[2][at]
    size_of = lambda a: np.linalg.norm(a, axis=1)
    want = r["dH"][at, :-1]
    bound = (2.0 ** -7 + 4 * exp_err) * (np.abs(r["P"][rows]) @ size_of(W64.T)) + 2.0 ** -8 * size_of(want)
    err = size_of(out[3].double().cpu().numpy()[at, :-1] - want)
    assert np.all(err <= 1.01 * bound), (err / bound).max()
    assert np.all(bound <= 0.2 * size_of(want))
