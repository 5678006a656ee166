"""The operators around the decoder layers at the ends of what their arguments may hold.  Oracles and bounds are those of test_ce_gpu
and test_norm_gpu."""
import numpy as np
import pytest

from oracle import norm_oracle as no
from tests import test_ce_gpu as tc
from tests import test_norm_gpu as tn

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


# Mean squares of 2^80 and 2^-80, with gradients from above whose products with powers of 1 / rms leave fp32 where two or three of them
# come together, although each result is an ordinary number.  Widths of every variant of the backward.
WIDTHS = [("bf16", 256), ("f32", 1544), ("bf16", 8200), ("f32", 4104), ("bf16", 17408)]


@pytest.mark.parametrize("alone,size,upstream", [(True, 40, -60), (True, -40, 60), (False, 40, -50), (False, -40, 20)])
@pytest.mark.parametrize("dtype,d", WIDTHS, ids=[f"{t}_{d}" for t, d in WIDTHS])
def test_norm_of_rows_far_from_unit_size(dtype, d, alone, size, upstream):
    import torch
    from paper_2602_07263_amd import tlora
    T, off, half = 9, [0, 5, 9], 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    v = tn._draw(61 + d, dtype, T, d, 2, post=not alone, gates=not alone, X=not alone)
    for k in ("X", "Y"):
        v[k] = None if v[k] is None else np.ldexp(v[k], size)
    for k in ("dH", "dXn"):
        v[k] = np.ldexp(v[k], upstream)
    if alone:
        v["dH"] = None
    kw = dict(gamma_post=v["gamma_post"], gamma_pre=v["gamma_pre"], gates=v["gates"])
    r = no.backward(v["X"], v["Y"], off, 0.0, v["dH"], v["dXn"], 0.5, **kw)
    up = lambda a: tn._up(a, dtype)
    n = tlora.ResidualNorm(dtype, off, up(v["X"]), up(v["Y"]), up(v["gamma_pre"]), 0.0, gamma_post=up(v["gamma_post"]),
                           gates=None if alone else [up(g) for g in v["gates"]], res_scale=0.5)
    Y = n._keep[1]
    dX, dY = tn._nan_like(Y), tn._nan_like(Y)
    sums = [tn._nan_like(Y, d, True) for _ in range(4)]
    print(f"bwd {dtype} {d} {alone} {size}", flush=True)
    n.bwd(up(v["dH"]), up(v["dXn"]), dX, dY, dgamma_pre=sums[0], dgamma_post=None if alone else sums[1],
          dgates=None if alone else sums[2:])
    torch.cuda.synchronize()
    tn._near(dX, r["dX"], r["abs_dX"], half, "dX")
    tn._near(dY, r["dY"], r["abs_dY"], half, "dY")
    chain = 1 + (T / 512 + 64) / 64
    tn._near(sums[0], r["dgamma_pre"], chain * r["abs_dgamma_pre"], 2.0 ** -24, "dgamma_pre")
    if not alone:
        tn._near(sums[1], r["dgamma_post"], chain * r["abs_dgamma_post"], 2.0 ** -24, "dgamma_post")
        for j in range(2):
            tn._near(sums[2 + j], r["dgates"][j], chain * r["abs_dgates"][j], 2.0 ** -24, f"dgate {j}")
