"""Pins of the oracles of the operators around the decoder layers: torch autograd on the CPU in float64, central
differences, closed forms."""
import numpy as np
import torch

from oracle import ce_oracle as ce
from oracle import ckpt_oracle as ck
from oracle import norm_oracle as no


def _ce_problem(seed=0):
    rng = np.random.default_rng(seed)
    H, W = rng.normal(size=(11, 6)), rng.normal(size=(6, 9))
    y = np.array([3, -100, 8, 0, 9, 5, -1, 2, 2, 7, 1])           # 9 and the negative ones: no loss
    return H, W, y, [0, 4, 4, 7, 11], rng.uniform(0.5, 2.0, 11)


def test_cross_entropy_against_autograd():
    H, W, y, off, w = _ce_problem()
    r = ce.cross_entropy(H, W, y, off, w)
    t = torch.tensor(H, requires_grad=True)
    total = 0.0
    for j, (a, b) in enumerate(zip(off[:-1], off[1:])):
        rows = [i for i in range(a, b) if 0 <= y[i] < 9]
        if not rows:
            assert r["job_loss"][j] == 0.0
            continue
        l = torch.nn.functional.cross_entropy(t[rows] @ torch.tensor(W), torch.tensor(y[rows]), reduction="none")
        np.testing.assert_allclose(r["loss"][rows], l.detach().numpy(), rtol=1e-12)
        mean = (l * torch.tensor(w[rows])).sum() / w[rows].sum()
        np.testing.assert_allclose(r["job_loss"][j], mean.item(), rtol=1e-12)
        total = total + mean
    total.backward()
    np.testing.assert_allclose(r["dH"], t.grad.numpy(), rtol=1e-11, atol=1e-14)


def test_cross_entropy_against_differences_and_closed_forms():
    H, W, y, off, w = _ce_problem(1)
    dl = np.random.default_rng(2).normal(size=11)
    r = ce.cross_entropy(H, W, y, off, w, dloss=dl)
    h = 1e-6
    for t, i in ((0, 2), (5, 0), (10, 5), (1, 1)):
        up, dn = H.copy(), H.copy()
        up[t, i] += h
        dn[t, i] -= h
        f = lambda A: (ce.cross_entropy(A, W, y, off, w)["loss"] * dl).sum()
        assert abs((f(up) - f(dn)) / (2 * h) - r["dH"][t, i]) < 1e-7
    assert not r["dH"][[1, 4, 6]].any() and not r["loss"][[1, 4, 6]].any()
    z = ce.cross_entropy(np.zeros((2, 6)), W, [0, 5], [0, 2])      # equal logits: log of the vocabulary's size
    np.testing.assert_allclose(z["loss"], np.log(9.0), rtol=1e-14)
    np.testing.assert_allclose(z["dH"][1], 0.5 * (W.mean(axis=1) - W[:, 5]), rtol=1e-12)


def test_norm_against_autograd_and_differences():
    rng = np.random.default_rng(3)
    T, d, off = 7, 5, [0, 3, 3, 7]
    for post in (True, False):
        for pre in (True, False):
            v = {k: rng.normal(size=(T, d)) for k in ("X", "Y", "dH", "dXn")}
            gp = rng.normal(size=d) if post else None
            gn = rng.normal(size=d) if pre else None
            gates = [rng.normal(size=d), None, rng.normal(size=d)]
            H, Xn = no.forward(v["X"], v["Y"], off, 1e-3, 0.7, gp, gn, gates)
            r = no.backward(v["X"], v["Y"], off, 1e-3, v["dH"], v["dXn"] if pre else None, 0.7, gp, gn, gates)
            t = {k: torch.tensor(a, requires_grad=True) for k, a in
                 dict(X=v["X"], Y=v["Y"], gp=gp if post else np.ones(d), gn=gn if pre else np.ones(d), g0=gates[0], g2=gates[2]).items()}
            norm = lambda V: V * torch.rsqrt((V * V).mean(dim=1, keepdim=True) + 1e-3)
            N = norm(t["Y"]) * t["gp"] if post else t["Y"]
            tH = t["X"] + 0.7 * torch.cat([t["g0"].expand(3, d), t["g2"].expand(4, d)]) * N
            np.testing.assert_allclose(H, tH.detach().numpy(), rtol=1e-12, atol=1e-13)
            L = (tH * torch.tensor(v["dH"])).sum()
            if pre:
                tXn = norm(tH) * t["gn"]
                np.testing.assert_allclose(Xn, tXn.detach().numpy(), rtol=1e-12, atol=1e-13)
                L = L + (tXn * torch.tensor(v["dXn"])).sum()
            L.backward()
            same = lambda a, b: np.testing.assert_allclose(a, b.grad.numpy(), rtol=1e-10, atol=1e-12)
            same(r["dX"], t["X"])
            same(r["dY"], t["Y"])
            same(r["dgates"][0], t["g0"])
            same(r["dgates"][2], t["g2"])
            assert not r["dgates"][1].any()
            if post:
                same(r["dgamma_post"], t["gp"])
            if pre:
                same(r["dgamma_pre"], t["gn"])
    # one derivative by differences: of sum(dH H) + sum(dXn Xn) for Y[4, 1]
    f = lambda Y: sum((a * b).sum() for a, b in zip((v["dH"], v["dXn"]), no.forward(v["X"], Y, off, 1e-3, 0.7, gp, np.ones(d), gates)))
    r = no.backward(v["X"], v["Y"], off, 1e-3, v["dH"], v["dXn"], 0.7, gp, np.ones(d), gates)
    up, dn = v["Y"].copy(), v["Y"].copy()
    up[4, 1] += 1e-6
    dn[4, 1] -= 1e-6
    assert abs((f(up) - f(dn)) / 2e-6 - r["dY"][4, 1]) < 1e-7


def test_checkpoint_codes():
    rng = np.random.default_rng(4)
    x = rng.normal(size=(40, 300)).astype(np.float32)
    x[3, 128:256] = 0
    x[5, 7] = 1e30
    codes, s = ck.pack(x)
    v = ck.unpack(codes, s)
    step = np.repeat(s.astype(np.float64), 128, axis=1)[:, :300]
    assert np.abs(codes.astype(int)).max() == 127
    assert np.all(np.abs(v - x) <= step / 2 * (1 + 1e-6))
    assert s[3, 1] == np.float32(2.0 ** -100) and not codes[3, 128:256].any()
    # the scale is a bf16 number, holds the largest value, and the bf16 number below it does not
    bits = s.view(np.uint32)
    assert not (bits & 0xFFFF).any()
    below = (bits - np.uint32(0x10000)).view(np.float32).astype(np.float64)
    top = np.stack([np.abs(x[:, a:a + 128]).max(axis=1) for a in (0, 128, 256)], axis=1).astype(np.float64)
    live = top > 0
    assert np.all(127 * s.astype(np.float64) >= top) and np.all(127 * below[live] < top[live])
    for bad in (np.inf, -np.inf, np.nan, 2.0 ** 127):
        y = x[:2].copy()
        y[1, 130] = bad
        c, s2 = ck.pack(y)
        assert np.isnan(s2[1, 1]) and not c[1, 128:256].any() and np.isfinite(np.delete(s2.ravel(), 4)).all()
    # ties: 2.5 and 3.5 steps
    t = np.zeros((1, 128), dtype=np.float32)
    t[0, :4] = [127, 2.5, 3.5, -2.5]
    c, s3 = ck.pack(t)
    assert s3[0, 0] == 1.0 and list(c[0, :4]) == [127, 2, 4, -2]
