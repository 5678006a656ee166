"""The backward from 8 bits on the plain workspace, where that is enough: the bits that a larger one gives, and nothing behind it written."""
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
