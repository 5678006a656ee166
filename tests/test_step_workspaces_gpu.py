"""Workspaces of just the stated size: the bits that larger ones give, and nothing behind them written."""
import pytest

from paper_2602_07263_amd import workloads as wk

pytestmark = pytest.mark.gpu


# S_j kept; and, of the last, made again from the codes
@pytest.mark.parametrize("d_in,ranks,tokens,reuse_S", [(4096, [16, 32], [512, 1001], True), (144, [200], [130], True),
                                                       (320, [40, 130, 8], [7000, 5000, 301], True),
                                                       (320, [40, 130, 8], [7000, 5000, 301], False)])
def test_the_plain_workspace_is_enough(d_in, ranks, tokens, reuse_S):
    import torch
    from paper_2602_07263_amd import tlora
    p = wk.generate(wk.custom("ckpt", "bf16", d_in, 256, ranks, tokens, [1.0] * len(ranks)), seed=3)
    lp = tlora.LayerProblem.from_numpy(p)
    c = tlora.Checkpoint("bf16", lp.T, d_in, "cuda")
    c.pack(lp.X)
    dY = torch.from_numpy(p.dY).to("cuda", torch.bfloat16)
    plain, results = lp.ws_bytes, []
    for guarded in (False, True):
        if guarded:
            lp.ws_bytes = plain
            lp.ws = torch.full((plain + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
        else:
            lp.bwd_ckpt_workspace()
            assert lp.ws_bytes > plain
        Y, dX, dA, dB = lp.new_outputs()
        print(f"{d_in} {tokens} {reuse_S} {guarded}", flush=True)
        lp.fwd(Y)
        lp.bwd_ckpt(c.packed, dY, dX, dA, dB, reuse_S=reuse_S)
        torch.cuda.synchronize()
        results.append([dX] + dA + dB)
    assert (lp.ws[plain:] == 0xAB).all()
    for a, b in zip(*results):
        assert torch.equal(a, b)
    lp.bwd_ckpt_workspace(reuse_S=True)                 # asks for nothing more
    assert lp.ws_bytes == plain


def test_a_workspace_that_grows_behind_the_forward_keeps_its_S():
    import torch
    from paper_2602_07263_amd import tlora
    p = wk.generate(wk.custom("ckpt", "f32", 136, 72, [4, 7], [50, 81], [2.0, 1.0]), seed=5)
    dY, results = torch.from_numpy(p.dY).cuda(), []
    for late in (False, True):
        lp = tlora.LayerProblem.from_numpy(p)
        c = tlora.Checkpoint("f32", lp.T, 136, "cuda")
        c.pack(lp.X)
        Y, _, dA, dB = lp.new_outputs()
        if not late:
            lp.bwd_ckpt_workspace()
        lp.fwd(Y)
        if late:
            with pytest.raises(tlora.TloraError):       # (a workspace that is too small: refused, nothing is launched)
                lp.bwd_ckpt(c.packed, dY, None, dA, dB, reuse_S=True)
            lp.bwd_ckpt_workspace()
        print(f"late {late}", flush=True)
        lp.bwd_ckpt(c.packed, dY, None, dA, dB, reuse_S=True)
        torch.cuda.synchronize()
        results.append(dA + dB)
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,d,V", [(5, 64, 200), (61, 4096, 32000), (300, 512, 50000), (700, 8192, 259), (257, 72, 5000), (5000, 256, 3001)])
def test_the_losses_workspace_is_enough(T, d, V):
    import torch
    from paper_2602_07263_amd import tlora
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    rn = lambda *n: torch.randn(*n, device="cuda", generator=g).to(torch.bfloat16)
    H, W = rn(T, d), rn(d, (V + 7) // 8 * 8) * (2 * d ** -0.5)
    y = torch.randint(-1, V, (T,), device="cuda", generator=g, dtype=torch.int32)
    head, results = tlora.LossHead([0, T // 3, T], H, W, V, y), []
    for guard in (1 << 27, 4096):
        head.ws = torch.full((head.ws_bytes + guard,), 0xAB, dtype=torch.uint8, device="cuda")
        out = [torch.full(n, float("nan"), device="cuda") for n in ((T,), (T,), (2,))] + [torch.full_like(H, float("nan"))]
        print(f"{T} {d} {V} {guard}", flush=True)
        head.fwd_bwd(*out)
        torch.cuda.synchronize()
        assert (head.ws[head.ws_bytes:] == 0xAB).all()
        results.append(out)
    for a, b in zip(*results):
        assert torch.isfinite(a).all() and torch.equal(a, b)
