"""The operators around the decoder layers on tensors beyond 4 GiB: rows at the far end have the bits that a call on those rows
alone gives them (a row's result depends on its own values; the loss lists the same tokens in the same order)."""
import pytest

pytestmark = pytest.mark.gpu

T, LAST = 1_100_000, 300


def _fill(t, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for a in range(0, t.shape[0], 100_000):                     # drawn in pieces: no fp32 copy of a whole tensor
        t[a:a + 100_000] = torch.randn(min(100_000, t.shape[0] - a), t.shape[1], device="cuda", generator=g).to(t.dtype)
    return t


def test_norms():
    import torch
    from paper_2602_07263_amd import tlora
    d, bf = 2048, torch.bfloat16
    X, Y = _fill(torch.empty(T, d, dtype=bf, device="cuda"), 1), _fill(torch.empty(T, d, dtype=bf, device="cuda"), 2)
    gamma = torch.ones(d, dtype=bf, device="cuda") * 1.25
    gates = [gamma * 0.5, gamma]
    off = [0, T - 100, T]
    H, Xn = torch.empty_like(X), torch.empty_like(X)
    big = tlora.ResidualNorm("bf16", off, X, Y, gamma, 1e-5, gamma_post=gamma, gates=gates)
    print("norm forward", flush=True)
    big.fwd(H, Xn)
    tail = lambda t: t[T - LAST:].contiguous()
    small = tlora.ResidualNorm("bf16", [0, LAST - 100, LAST], tail(X), tail(Y), gamma, 1e-5, gamma_post=gamma, gates=gates)
    h, xn = torch.empty(LAST, d, dtype=bf, device="cuda"), torch.empty(LAST, d, dtype=bf, device="cuda")
    small.fwd(h, xn)
    torch.cuda.synchronize()
    assert torch.equal(tail(H), h) and torch.equal(tail(Xn), xn)
    # H and Xn serve as upstream gradients
    dX, dY = torch.empty_like(X), torch.empty_like(X)
    dg = [torch.empty(d, device="cuda") for _ in range(2)]
    print("norm backward", flush=True)
    big.bwd(H, Xn, dX, dY, dgates=dg)
    a, b = torch.empty_like(h), torch.empty_like(h)
    sg = [torch.empty(d, device="cuda") for _ in range(2)]
    small.bwd(h, xn, a, b, dgates=sg)
    torch.cuda.synchronize()
    assert torch.equal(tail(dX), a) and torch.equal(tail(dY), b)
    # the last job has the same 100 tokens in both: the same sums but for their order (100 terms, 2^-24 each, of terms below ~50)
    torch.testing.assert_close(dg[1], sg[1], rtol=1e-4, atol=100 * 50 * 2 ** -24)


def test_eight_bits():
    import torch
    from paper_2602_07263_amd import tlora
    d, bf = 4096, torch.bfloat16
    X = _fill(torch.empty(T, d, dtype=bf, device="cuda"), 3)
    c = tlora.Checkpoint("bf16", T, d, "cuda")
    print("pack, unpack", flush=True)
    c.pack(X)
    out = torch.empty_like(X)
    c.unpack(out)
    s = tlora.Checkpoint("bf16", LAST, d, "cuda")
    x, y = X[T - LAST:].contiguous(), torch.empty(LAST, d, dtype=bf, device="cuda")
    s.pack(x)
    s.unpack(y)
    torch.cuda.synchronize()
    assert torch.equal(out[T - LAST:], y)


def test_loss():
    import torch
    from paper_2602_07263_amd import tlora
    d, V, bf = 2048, 500, torch.bfloat16
    H = _fill(torch.empty(T, d, dtype=bf, device="cuda"), 4)
    W = _fill(torch.empty(d, 504, dtype=bf, device="cuda"), 5) * 0.05
    y = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    y[T - LAST:] = torch.arange(LAST, device="cuda", dtype=torch.int32)
    f32 = lambda n: torch.empty(n, device="cuda")
    head = tlora.LossHead([0, 10, T - 50, T], H, W, V, y)
    loss, lse, job, dH = f32(T), f32(T), f32(3), torch.full_like(H, float("nan"))
    print("loss", flush=True)
    head.fwd_bwd(loss, lse, job, dH)
    alone = tlora.LossHead([0, LAST - 50, LAST], H[T - LAST:].contiguous(), W, V, y[T - LAST:].contiguous())
    l, e, j, g = f32(LAST), f32(LAST), f32(2), torch.empty(LAST, d, dtype=bf, device="cuda")
    alone.fwd_bwd(l, e, j, g)
    torch.cuda.synchronize()
    assert torch.equal(loss[T - LAST:], l) and torch.equal(lse[T - LAST:], e) and torch.equal(dH[T - LAST:], g)
    assert not loss[:T - LAST].any() and job[0] == 0
    assert torch.equal(job[1:], j)
    for a in range(0, T - LAST, 200_000):
        assert not dH[a:min(a + 200_000, T - LAST)].any()


def test_norm_of_more_rows_than_a_launch_takes():
    # 2^22 rows of 1024 threads are 2^32 threads.  Rows of a few kinds, other ones in the second half; one row's result does not
    # depend on where it lies.
    import torch
    from paper_2602_07263_amd import tlora
    rows, d, bf = 1 << 22, 8192, torch.bfloat16
    torch.cuda.empty_cache()
    kinds = _fill(torch.empty(16, d, dtype=bf, device="cuda"), 5)
    gamma = torch.ones(d, dtype=bf, device="cuda") * 1.25
    few = torch.empty_like(kinds)
    tlora.ResidualNorm("bf16", [0, 16], None, kinds, gamma, 1e-5).fwd(None, few)
    Y, Xn = torch.empty(rows, d, dtype=bf, device="cuda"), torch.empty(rows, d, dtype=bf, device="cuda")
    for h in range(2):
        Y[h * rows // 2:(h + 1) * rows // 2].view(-1, 8, d).copy_(kinds[8 * h:8 * h + 8])
    Xn.fill_(float("nan"))
    print("norm forward, 2^22 rows", flush=True)
    tlora.ResidualNorm("bf16", [0, rows], None, Y, gamma, 1e-5).fwd(None, Xn)
    torch.cuda.synchronize()
    for h in range(2):
        got = Xn[h * rows // 2:(h + 1) * rows // 2].view(-1, 8, d)
        for a in range(0, got.shape[0], 1 << 14):
            assert torch.equal(got[a:a + (1 << 14)], few[8 * h:8 * h + 8].expand(1 << 14, 8, d)), (h, a)
