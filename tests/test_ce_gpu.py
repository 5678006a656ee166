"""Cross entropy of the vocabulary projection against the fp64 oracle on the same bf16 inputs.

Bounds.  A logit is an fp32 sum of d products: |dz| <= (d / 16 + 16) 2^-24 max_v sum_k |h_k w_kv| =: e (products of one matrix
instruction are added at once, so the chain has d / 32 links; the factor doubles that).  loss and lse: 2 e, the rounding of z log2(e)
and of the logarithm, 2^-22 (1 + |value| + max |z|).  dH: an exponential is rounded once, 2^-8 of itself (twice where its tile is
scaled), and is off by e^(2 e) - 1 and 2^-22 (1 + max |z|) from the logits' error: sum_v |P_v| |W_v| times that; then the row is
rounded once, 2^-8."""
import numpy as np
import pytest

from oracle import ce_oracle as ce
from paper_2602_07263_amd import workloads as wk

pytestmark = pytest.mark.gpu


def _inputs(seed, T, d, V, ld, std=2.0, ignored=0.3, shift=0.0):
    rng = np.random.default_rng(seed)
    r = wk.round_to_bf16
    H = r(rng.normal(size=(T, d)).astype(np.float32))
    W = r((rng.normal(size=(d, ld)) * std / np.sqrt(d)).astype(np.float32))
    if shift:                                   # a common shift of all logits: the last feature is 1 and its weights are the shift
        H[:, -1] = 1.0
        W[-1, :] = r(np.full(ld, shift, dtype=np.float32))
    y = rng.integers(0, V, T)
    y[rng.uniform(size=T) < ignored] = -100
    return H, W, y.astype(np.int32)


def _head(H, W, y, V, off, weights=None, with_grad=True):
    import torch
    from paper_2602_07263_amd import tlora
    up = lambda a: torch.from_numpy(a).to("cuda", torch.bfloat16)
    w = None if weights is None else torch.from_numpy(weights.astype(np.float32)).cuda()
    return tlora.LossHead(off, up(H), up(W), V, torch.from_numpy(y).cuda(), w, with_grad=with_grad)


def _outs(head):
    import torch
    T, J = head.offsets[-1], len(head.offsets) - 1
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    return nan(T), nan(T), nan(J), torch.full_like(head._keep[0], float("nan"))


def _bounds(r, H, W):
    live = r["live"]
    d = H.shape[1]
    e = np.zeros(H.shape[0])
    e[live] = (d / 16 + 16) * 2.0 ** -24 * (np.abs(H[live]).astype(np.float64) @ np.abs(W).astype(np.float64)).max(axis=1)
    zmax = np.zeros(H.shape[0])
    zmax[live] = np.abs(r["z"]).max(axis=1)
    exp_err = np.expm1(2 * e) + 2.0 ** -22 * (1 + zmax)
    reach = np.zeros(H.shape)
    reach[live] = np.abs(r["P"]) @ np.abs(W).astype(np.float64).T
    # the softmax itself enters the target's difference: p - 1 is made from p
    own = np.zeros(H.shape)
    own[live] = r["share_g"][live, None] * (np.abs(W).astype(np.float64).T[r["y"][live]])
    return e, zmax, exp_err, reach, own


def _check(out, r, H, W, y, V, roundings=1):
    import torch
    loss, lse, job, dH = [t.double().cpu().numpy() for t in out]
    W = W[:, :V]
    r["y"] = y
    r["share_g"] = np.abs(r["g"])
    e, zmax, exp_err, reach, own = _bounds(r, H, W)
    for got, ref in ((loss, r["loss"]), (lse, r["lse"])):
        assert np.all(np.abs(got - ref) <= 2 * e + 2.0 ** -22 * (1 + np.abs(ref) + zmax)), np.abs(got - ref).max()
    tol = np.array([(2 * e + 2.0 ** -22 * (1 + r["lse"] + zmax))[a:b].max(initial=0) for a, b in zip(r["off"][:-1], r["off"][1:])])
    assert np.all(np.abs(job - r["job_loss"]) <= 2 * tol + 2.0 ** -23 * np.abs(r["job_loss"]))
    bound = (roundings * 2.0 ** -8 + 2 * exp_err[:, None]) * reach + 2 * exp_err[:, None] * own
    bound += 2.0 ** -8 * (np.abs(r["dH"]) + bound) + 1e-37
    over = np.abs(dH - r["dH"]) / bound
    assert np.all(over <= 1.0), (over.max(), np.unravel_index(over.argmax(), over.shape))
    dead = np.setdiff1d(np.arange(len(y)), r["live"])
    assert not loss[dead].any() and not lse[dead].any() and not dH[dead].any()


def _oracle(H, W, y, V, off, weights=None, dloss=None):
    r = ce.cross_entropy(H, W[:, :V], y, off, weights, dloss)
    g = r["share"] if dloss is None else np.zeros(len(y))
    if dloss is not None:
        g[r["live"]] = dloss[r["live"]]
    r["g"], r["off"] = g, off
    return r


# tokens, d, vocab, ld: one token; vocabularies of 1, of less than a step, of odd sizes and row strides; d that is no multiple of 32;
# several row and column tiles; more rows than a tile with a ragged end
CASES = [([1], 64, 1, 8), ([1], 8, 5, 8), ([3, 0, 5], 40, 31, 40), ([7], 96, 33, 40), ([1, 4, 7, 1], 256, 1000, 1000),
         ([130, 0, 141, 300], 128, 777, 784), ([257], 1000, 300, 512), ([90, 420], 512, 2049, 2056), ([64], 2048, 8193, 8200)]


@pytest.mark.parametrize("tokens,d,V,ld", CASES, ids=[f"{sum(c[0])}x{c[1]}x{c[2]}" for c in CASES])
@pytest.mark.parametrize("weighted", [False, True])
def test_loss_and_gradient_match_the_oracle(tokens, d, V, ld, weighted):
    import torch
    T, off = sum(tokens), np.concatenate([[0], np.cumsum(tokens)])
    H, W, y = _inputs(T + d + V, T, d, V, ld)
    W[:, V:] = np.nan                           # columns that do not count hold anything
    y[-1] = V - 1
    if T > 3:
        y[1] = V                                # not a column: no loss
    H[y < 0] = np.nan                           # rows without a loss hold anything
    w = np.random.default_rng(5).uniform(0.25, 4.0, T).astype(np.float32) if weighted else None
    r = _oracle(np.nan_to_num(H), np.nan_to_num(W), y, V, off, w)
    head = _head(H, W, y, V, off, w)
    out = _outs(head)
    print(f"fwd_bwd {tokens} {d} {V} {ld}", flush=True)
    head.fwd_bwd(*out)
    torch.cuda.synchronize()
    _check(out, r, np.nan_to_num(H), np.nan_to_num(W), y, V)
    ev = _head(H, W, y, V, off, w, with_grad=False)
    fwd = _outs(ev)
    print("fwd", flush=True)
    ev.fwd(*fwd[:3])
    torch.cuda.synchronize()
    for a, b in zip(fwd[:3], out[:3]):
        assert torch.equal(a, b)                # the same statistics, the same bits


@pytest.mark.parametrize("std,shift", [(40.0, 0.0), (2.0, 200.0), (2.0, -200.0), (30.0, -60.0), (0.0, 0.0), (3.0, 56.0), (3.0, -36.0)],
                         ids=["wide", "high", "low", "mixed", "equal", "at_the_top", "at_the_bottom"])
def test_logits_far_from_zero(std, shift):
    """Rows whose exponentials need references of their own: logits of hundreds, of either sign, and all equal."""
    import torch
    T, d, V = 70, 64, 1111
    off = [0, 30, 70]
    H, W, y = _inputs(17, T, d, V, 1112, std=std, shift=shift, ignored=0.1)
    r = _oracle(H, W, y, V, off)
    head = _head(H, W, y, V, off)
    out = _outs(head)
    head.fwd_bwd(*out)
    torch.cuda.synchronize()
    _check(out, r, H, W, y, V, roundings=2)


def test_upstream_gradient_and_optional_outputs():
    import torch
    off = [0, 100, 300]
    H, W, y = _inputs(3, 300, 128, 500, 504)
    dl = np.random.default_rng(1).normal(size=300).astype(np.float32)
    dl[7] = 0.0
    head = _head(H, W, y, 500, off)
    loss, lse, job, dH = _outs(head)
    head.fwd_bwd(loss, lse, job, dH, dloss=torch.from_numpy(dl).cuda())
    r = _oracle(H, W, y, 500, off, dloss=dl.astype(np.float64))
    _check((loss, lse, job, dH), r, H, W, y, 500)
    only = torch.empty_like(dH)
    head.fwd_bwd(None, None, None, only, dloss=torch.from_numpy(dl).cuda())
    torch.cuda.synchronize()
    assert torch.equal(only, dH)


@pytest.mark.parametrize("which", ["none", "all_ignored", "zero_weights"])
def test_batches_without_a_loss(which):
    import torch
    T = 0 if which == "none" else 40
    off = [0, 0, 0] if T == 0 else [0, 15, 40]
    H, W, y = _inputs(9, T, 64, 100, 104, ignored=0.0)
    if which == "all_ignored":
        y[:] = -1
    w = np.zeros(T, dtype=np.float32) if which == "zero_weights" else None
    head = _head(H, W, y, 100, off, w)
    loss, lse, job, dH = _outs(head)
    head.fwd_bwd(loss, lse, job, dH)
    torch.cuda.synchronize()
    assert not job.any() and not dH.any()
    if which == "all_ignored":
        assert not loss.any() and not lse.any()


def test_infinite_and_nan_rows_stay_their_own():
    import torch
    off = [0, 60]
    H, W, y = _inputs(21, 60, 64, 300, 304, ignored=0.0)
    clean = _head(H, W, y, 300, off)
    a = _outs(clean)
    dl = torch.ones(60, device="cuda")
    clean.fwd_bwd(*a, dloss=dl)
    H[5, 3], H[9, 0] = np.nan, np.inf
    b = _outs(clean)
    bad = _head(H, W, y, 300, off)
    bad.fwd_bwd(*b, dloss=dl)
    torch.cuda.synchronize()
    keep = np.setdiff1d(np.arange(60), [5, 9])
    for s, t in ((a[0], b[0]), (a[1], b[1]), (a[3], b[3])):
        assert torch.equal(s[keep], t[keep])
    assert torch.isnan(b[0][5]) and torch.isnan(b[3][5]).all() and torch.isnan(b[2][0])


def test_tokens_of_weight_zero_enter_nothing():
    import torch
    off = [0, 25, 60]
    H, W, y = _inputs(22, 60, 64, 300, 304, ignored=0.0)
    w = np.random.default_rng(1).uniform(0.5, 2.0, 60).astype(np.float32)
    w[[3, 30, 59]] = 0.0
    r = _oracle(H, W, y, 300, off, w)
    H[3], H[59, 7] = np.nan, np.inf
    head = _head(H, W, y, 300, off, w)
    loss, lse, job, dH = _outs(head)
    head.fwd_bwd(loss, lse, job, dH)
    torch.cuda.synchronize()
    assert not torch.isfinite(loss[[3, 59]]).any() and not dH[[3, 30, 59]].any()
    loss[[3, 59]] = torch.from_numpy(r["loss"][[3, 59]]).float().cuda()      # (for the comparison of the rest)
    lse[[3, 59]] = torch.from_numpy(r["lse"][[3, 59]]).float().cuda()
    _check((loss, lse, job, dH), r, np.nan_to_num(H, nan=0.0, posinf=0.0), W, y, 300)


def test_pieces_of_a_long_batch():
    """More tokens with a loss than a piece holds (4096): a piece boundary inside a job, and a last piece of few rows."""
    import torch
    T, d, V = 9000, 64, 640
    off = [0, 4000, 9000]
    H, W, y = _inputs(33, T, d, V, V, ignored=0.05)
    r = _oracle(H, W, y, V, off)
    assert 4096 < len(r["live"]) < 8192 + 600
    head = _head(H, W, y, V, off)
    out = _outs(head)
    head.fwd_bwd(*out)
    torch.cuda.synchronize()
    _check(out, r, H, W, y, V)


def test_more_jobs_than_an_argument_takes_and_one_workspace_for_both_calls():
    import torch
    rng = np.random.default_rng(2)
    tokens = rng.integers(0, 4, 300)
    off, T = np.concatenate([[0], np.cumsum(tokens)]), int(tokens.sum())
    H, W, y = _inputs(40, T, 512, 200, 200)
    r = _oracle(H, W, y, 200, off)
    head = _head(H, W, y, 200, off)
    out, ev = _outs(head), _outs(head)
    head.fwd_bwd(*out)
    head.fwd(*ev[:3])
    torch.cuda.synchronize()
    _check(out, r, H, W, y, 200)
    for a, b in zip(ev[:3], out[:3]):
        assert torch.equal(a, b)


def test_repeated_calls_give_the_same_bits_on_a_larger_workspace_and_another_stream():
    import torch
    off = [0, 200, 517]
    H, W, y = _inputs(4, 517, 256, 3000, 3000)
    head = _head(H, W, y, 3000, off)
    a, b = _outs(head), _outs(head)
    head.fwd_bwd(*a)
    torch.cuda.synchronize()
    head.ws.fill_(0xFF)                                 # whatever lay in the workspace
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        head.fwd_bwd(*b)
    torch.cuda.synchronize()
    for x, z in zip(a, b):
        assert torch.equal(x, z)


def test_replays_from_a_captured_stream():
    import torch
    off = [0, 90, 300]
    H, W, y = _inputs(8, 300, 128, 1000, 1000)
    head = _head(H, W, y, 1000, off)
    ref, out = _outs(head), _outs(head)
    head.fwd_bwd(*ref)
    H2, W2, y2 = _inputs(80, 300, 128, 1000, 1000, ignored=0.8)
    other = _head(H2, W2, y2, 1000, off)
    other.ws = head.ws                                  # two calls that share a workspace, ordered on one stream
    ref2, out2 = _outs(other), _outs(other)
    other.fwd_bwd(*ref2)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    print("capture", flush=True)
    with torch.cuda.graph(graph, stream=side):
        head.fwd_bwd(*out)
    for rep in range(3):
        for t in out + out2:
            t.fill_(float("nan"))
        other.fwd_bwd(*out2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        print(f"replay {rep}", flush=True)
        for a, b in zip(out + out2, ref + ref2):
            assert torch.equal(a, b)


def test_the_targets_rounding_is_not_the_gradients_error():
    # The error along W_y, in units of W_y: of the target's element at most N / (T + N) half steps are left, with N below the sum of
    # the tiles' squares; a half step of each other element and one more of all of them enter through <W_v, W_y>; and the output's
    # roundings add up as independent ones do, of which 8 standard deviations are allowed (each uniform in half a step).
    T, d, V = 64, 1024, 4096
    H, W, y = _inputs(31, T, d, V, V, std=1.0, ignored=0.0)
    head = _head(H, W, y, V, [0, T])
    import torch
    loss, lse, job, dH = _outs(head)
    print("fwd_bwd", flush=True)
    head.fwd_bwd(loss, lse, job, dH, dloss=torch.ones(T, device="cuda"))
    torch.cuda.synchronize()
    r = _oracle(H, W, y, V, [0, T], dloss=np.ones(T))
    W64, rows = W.astype(np.float64), np.arange(T)
    z = H.astype(np.float64) @ W64
    p = np.exp(z - np.log(np.exp(z).sum(axis=1, keepdims=True)))
    py = p[rows, y]
    tiles = p.reshape(T, V // 256, 256).sum(axis=2)
    tiles[rows, y // 256] -= py
    N, left = (tiles ** 2).sum(axis=1), (1 - py) ** 2
    Wy = W64.T[y]
    size = (Wy * Wy).sum(axis=1)
    others = np.abs(Wy @ W64) * p
    others[rows, y] = 0.0
    half = 2.0 ** -8
    bound = half * (1 - py) * N / (left + N) + 2 * half * others.sum(axis=1) / size
    bound += 8 * half * np.sqrt((r["dH"] ** 2 * Wy ** 2).sum(axis=1) / 3) / size + 1e-5
    err = np.abs(((dH.double().cpu().numpy() - r["dH"]) * Wy).sum(axis=1) / size)
    assert np.all(err <= bound), (err / bound).max()
    # without it most rows would be off by more: a half step is spread evenly, and the bound is less than half of one
    assert bound.max() < half / 2

