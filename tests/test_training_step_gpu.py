"""A whole training step of two jobs on a small decoder, assembled from the library's calls: the layers' inputs are kept in 8 bits alone;
after the loss each layer is run again from them and then backward; the adapters take an optimizer step.

The step's gradients are compared with those of the same step whose layer inputs are kept as they are: what the 8 bits change is
the layers' input by at most half a step, s / 2 <= max |x| / 254 + its bf16 rounding in every group.  And the step with unrounded
inputs is compared with differences of the loss along the gradient of one adapter matrix."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

D, FF, HEADS, KV, V, SEQ = 512, 1024, 4, 2, 3001, [0, 150, 290, 420]
OFF, RANKS, LAYERS = [0, 290, 420], [8, 16], 2


class _Model:
    def __init__(self, seed):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        bf = torch.bfloat16
        rn = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(bf)
        shapes = dict(q=(D, HEADS * 128), k=(D, KV * 128), v=(D, KV * 128), o=(HEADS * 128, D), gate=(D, FF), up=(D, FF), down=(FF, D))
        self.layers = [{n: (rn(i, o, std=i ** -0.5), [rn(i, r, std=i ** -0.5) for r in RANKS], [rn(r, o, std=0.05) for r in RANKS])
                        for n, (i, o) in shapes.items()} for _ in range(LAYERS)]
        self.gamma = [1 + rn(D, std=0.1) for _ in range(2 * LAYERS + 1)]
        self.head = rn(D, (V + 7) // 8 * 8, std=D ** -0.5)
        self.X = rn(OFF[-1], D)
        self.y = torch.randint(0, V, (OFF[-1],), device="cuda", generator=g, dtype=torch.int32)
        self.y[::3] = -100


def _layer(m, i, X):
    from paper_2602_07263_amd import tlora
    return tlora.DecoderLayer(D, FF, HEADS, KV, 10000.0, RANKS, OFF, [1.0, 2.0], SEQ, X, m.gamma[2 * i], m.gamma[2 * i + 1], 1e-5, m.layers[i])


def _step(m, eight_bits):
    """(job losses, gradients of every layer)"""
    import torch
    from paper_2602_07263_amd import tlora
    T = OFF[-1]
    x, kept = m.X, []
    for i in range(LAYERS):
        if eight_bits:
            c = tlora.Checkpoint("bf16", T, D, "cuda")
            c.pack(x)
            kept.append(c)
        else:
            kept.append(x.clone())
        out = torch.empty_like(x)
        _layer(m, i, x).fwd(out)
        x = out
    norm = tlora.ResidualNorm("bf16", OFF, None, x, m.gamma[-1], 1e-5)
    xn = torch.empty_like(x)
    norm.fwd(None, xn)
    head = tlora.LossHead(OFF, xn, m.head, V, m.y)
    loss, dxn = torch.empty(len(OFF) - 1, device="cuda"), torch.empty_like(x)
    head.fwd_bwd(None, None, loss, dxn)
    dx = torch.empty_like(x)
    norm.bwd(None, dxn, None, dx)
    grads = []
    for i in reversed(range(LAYERS)):
        if eight_bits:
            x = torch.empty_like(m.X)
            kept[i].unpack(x)
        else:
            x = kept[i]
        layer, again, g = _layer(m, i, x), torch.empty_like(m.X), None
        layer.fwd(again)
        g = layer.new_grads()
        back = torch.empty_like(dx)
        layer.bwd(dx, back, g)
        dx = back
        grads.insert(0, g)
    return loss, grads


def test_step_from_eight_bits_is_close_to_the_step_from_whole_inputs():
    import torch
    m = _Model(1)
    l8, g8 = _step(m, True)
    l16, g16 = _step(m, False)
    torch.cuda.synchronize()
    assert torch.equal(l8, l16)                         # the forward does not see what is kept
    for a, b in zip(g8, g16):
        for n in a:
            for ab in (0, 1):
                for x, y in zip(a[n][ab], b[n][ab]):
                    # a group of 128 normal values has max |x| about 2.7 deviations: half a step is 1.1 % of a deviation at most, 0.6 % in
                    # the mean square; through the norm into a product's operands, with the Jacobians of order one behind it, a few per cent
                    assert float((x - y).norm()) <= 0.05 * float(y.norm()), n


def test_gradients_against_differences_of_the_loss():
    """bf16 weights move in steps of 2^-8 of themselves, so the difference is taken over what they really became.  A step of 0.3 of the
    matrix is far above those steps; along it d(h) = f(h) - f(-h) = 2 h f' + h^3 f3 / 3 (f3: the third derivative) + ..., and of two steps, h and h / 2, the
    combination (8 d(h / 2) - d(h)) / 3 is free of the cubic term."""
    import torch
    m = _Model(2)
    _, grads = _step(m, False)
    for i, n, ab, j in ((0, "q", 0, 1), (1, "down", 1, 0)):
        g = grads[i][n][ab][j]
        w = m.layers[i][n][1 + ab][j]
        old = w.clone()
        got, expect = [], []
        for part in (0.3, 0.15):
            h = part * float(old.float().norm()) / float(g.norm())
            ends = []
            for sign in (1, -1):
                w.copy_((old.float() + sign * h * g).to(torch.bfloat16))
                ends.append((_step(m, False)[0].sum().double().item(), w.float().clone()))
            expect.append(float(((ends[0][1] - ends[1][1]) * g).sum()))
            got.append(ends[0][0] - ends[1][0])
        w.copy_(old)
        without_cubic = lambda d: (8 * d[1] - d[0]) / 3
        assert abs(without_cubic(got) - without_cubic(expect)) <= 0.1 * abs(without_cubic(expect)), (n, got, expect)


def test_adapters_take_the_optimizer_step():
    import torch
    from paper_2602_07263_amd import tlora
    m = _Model(3)
    _, grads = _step(m, True)
    tens, keep = [], []
    for i in range(LAYERS):
        for n, ab in grads[i].items():
            for k in (0, 1):
                for p, g in zip(m.layers[i][n][1 + k], ab[k]):
                    master, a, b = p.float(), torch.zeros_like(g), torch.zeros_like(g)
                    keep.append((p, p.clone(), g, master, a, b))
                    tens.append(dict(param=p.data_ptr(), master=master.data_ptr(), grad=g.data_ptr(), m=a.data_ptr(), v=b.data_ptr(),
                                     n=p.numel(), lr=1e-2, step=1))
    ws = torch.empty(tlora.tlora_adamw_workspace_bytes(len(tens)), dtype=torch.uint8, device="cuda")
    tlora.tlora_adamw_step(tens, tlora.TLORA_BF16, ws.data_ptr(), ws.numel(), int(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    for p, old, g, master, _, _ in keep:
        # the first step of AdamW without decay moves a weight by lr g / (|g| + eps)
        expect = old.float() - 1e-2 * g / (g.abs() + 1e-8)
        torch.testing.assert_close(master, expect, rtol=1e-4, atol=1e-5)
        assert torch.isfinite(p.float()).all() and torch.isfinite(g).all()
