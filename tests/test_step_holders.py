"""The holders of the operators around the decoder layers refuse tensors of a call that are not what the kernels would take them for.
(The tensors here are on the CPU, which a call that is otherwise right is refused for last: nothing is ever launched.)"""
import pytest
import torch

from paper_2602_07263_amd import tlora

BF, F32 = torch.bfloat16, torch.float32


def _b(*n):
    return torch.zeros(*n, dtype=BF)


def _f(*n):
    return torch.zeros(*n)


def _refused(call, good, bad, fields):
    """`good` is refused for its device alone, and with any of `bad` (argument -> tensor) in its place for that argument."""
    with pytest.raises(tlora.TloraError, match="must be on a GPU"):
        call(**good)
    for name, tensors in bad.items():
        for t in tensors:
            with pytest.raises(tlora.TloraError, match=fields.get(name, name)):
                call(**{**good, name: t})


ROWS = [_b(3, 16), _b(4, 24), _f(4, 16), _b(16, 4).t(), _b(8, 16)[::2], _b(4, 32)[:, :16]]      # of [4, 16] bf16
VECTOR = [_b(16), _f(15), _f(32)[::2], torch.zeros(16, dtype=torch.float64)]                    # of [16] fp32


def test_residual_norm():
    n = tlora.ResidualNorm("bf16", [0, 1, 4], _b(4, 16), _b(4, 16), _b(16), 1e-5, gamma_post=_b(16), gates=[_b(16), None])
    _refused(n.fwd, dict(H=_b(4, 16), Xn=_b(2, 3, 16)), dict(H=ROWS, Xn=ROWS), {})
    good = dict(dH=_b(4, 16), dXn=_b(5, 16), dX=_b(4, 16), dY=None, dgamma_post=_f(16), dgamma_pre=_f(1, 16), dgates=[_f(16), None])
    bad = {k: ROWS for k in ("dH", "dXn", "dX", "dY")}
    bad.update(dgamma_post=VECTOR, dgamma_pre=VECTOR, dgates=[[_f(16)], [_f(16)] * 3, [_f(16), _f(8)], [_b(16), None]])
    _refused(n.bwd, good, bad, {})
    single = tlora.ResidualNorm("f32", [0, 4], None, _f(4, 16), _f(16), 1e-5)
    _refused(single.fwd, dict(H=None, Xn=_f(4, 16)), dict(Xn=[_b(4, 16), _f(3, 16)]), {})


def test_loss_head():
    y = torch.zeros(4, dtype=torch.int32)
    h = tlora.LossHead([0, 1, 4], _b(4, 16), _b(16, 24), 20, y)
    tokens, jobs = [_f(3), _b(4), _f(8)[::2]], [_f(1), _b(2)]
    good = dict(loss=_f(4), lse=_f(5), job_loss=_f(2))
    bad = dict(loss=tokens, lse=tokens, job_loss=jobs)
    _refused(h.fwd, good, bad, {"loss": "LossHead.fwd: loss"})
    _refused(h.fwd_bwd, dict(good, dH=_b(4, 16), dloss=None), dict(bad, dH=ROWS, dloss=tokens), {"loss": "LossHead.fwd_bwd: loss"})
    _refused(h.fwd_bwd, dict(loss=None, lse=None, job_loss=None, dH=_b(4, 16), dloss=_f(4)), {}, {})


def test_checkpoint():
    c = tlora.Checkpoint("bf16", 4, 16, "cpu")
    for call in (c.pack, c.unpack):
        _refused(call, dict(X=_b(4, 16)), dict(X=[_b(3, 16), _f(4, 16), _b(16, 4).t()]), {"X": "Checkpoint"})


def test_backward_from_eight_bits():
    layer = tlora.LayerProblem("bf16", 16, 24, [4, 0], [0, 3, 4], [1.0, 1.0], _b(4, 16), _b(16, 24), [_b(16, 4), None], [_b(4, 24), None])
    packed = torch.zeros(int(tlora.lib().tlora_ckpt_bytes(4, 16)), dtype=torch.uint8)
    good = dict(packed=packed, dY=_b(4, 24), dX=_b(4, 16), dA=[_f(16, 4), _f(16, 0)], dB=[_f(4, 24), _f(0, 24)])
    bad = dict(packed=[packed[:-1], torch.zeros(2 * len(packed), dtype=torch.uint8)[::2]], dX=ROWS,
               dY=[_b(3, 24), _f(4, 24), _b(24, 4).t(), _b(4, 16)],
               dA=[[_f(16, 4)], [_f(15, 4), None], [_b(16, 4), None], [_f(4, 16).t(), None]], dB=[[_f(4, 24)], [_f(4, 23), None]])
    _refused(layer.bwd_ckpt, good, bad, {})
    _refused(layer.bwd_ckpt, dict(good, dX=None, dA=None, dB=None), dict(dA=[good["dA"]], dB=[good["dB"]]), {})


def test_inputs_on_several_devices():
    y = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(tlora.TloraError, match="another device"):
        tlora._one_device("holder", (("X", None), ("Y", y)), 0)
    with pytest.raises(tlora.TloraError, match="must be on a GPU"):
        tlora._call_stream(torch, -1, "holder")


def test_two_jobs_with_one_gradient_of_a_gate_are_refused():
    import ctypes
    P, L = ctypes.c_void_p, tlora.lib()
    off = (ctypes.c_int64 * 4)(0, 1, 2, 4)
    gates = (P * 3)(0x5000, 0x5000, None)                # (a gate that two jobs share is read alone)
    q = tlora.tlora_norm_t(tlora.TLORA_BF16, 3, 64, off, 1e-5, 1.0, None, P(0x2000), None, None, gates)
    n = L.tlora_norm_workspace_bytes(ctypes.byref(q))
    # (the size of the workspace is looked at last: a call whose gradients are apart is refused for it)
    call = lambda dg, ws: L.tlora_norm_bwd(ctypes.byref(q), P(0x8000), None, P(0xA000), None, None, None, (P * 3)(*dg), 0, P(0x100000), ws, None)
    for dg in ((0xE000, 0xE000, None), (0xE000, 0xF000, 0xE000), (None, 0xF000, 0xF000)):
        assert call(dg, n) == -1
    for dg in ((0xE000, 0xF000, 0xE100), (None, 0xF000, None), (None, None, None)):
        assert call(dg, n - 1) == -4
