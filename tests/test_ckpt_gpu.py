"""Activations kept in 8 bits: codes and scales equal the oracle's bit for bit, the values their rounding; the layer's backward from
them equals the plain backward whose X are those values."""
import numpy as np
import pytest

from oracle import ckpt_oracle as ck
from oracle import tlora_oracle as orc
from paper_2602_07263_amd import workloads as wk
from tests import parity_util as pu

pytestmark = pytest.mark.gpu


def _values(seed, T, d, dtype):
    rng = np.random.default_rng(seed)
    x = (rng.normal(size=(T, d)) * np.exp2(rng.integers(-8, 9, size=(T, 1)))).astype(np.float32)
    x[:, ::41] *= 30
    if dtype == "bf16":
        # multiples of half a step: ties
        x[::3] = np.round(x[::3] * 4) / 4
        x = wk.round_to_bf16(x)
    return x


def _pack(x, dtype):
    import torch
    from paper_2602_07263_amd import tlora
    T, d = x.shape
    t = torch.from_numpy(x).to("cuda", torch.bfloat16 if dtype == "bf16" else torch.float32)
    c = tlora.Checkpoint(dtype, T, d, "cuda")
    c.packed.fill_(0xAB)
    c.pack(t)
    out = torch.full_like(t, float("nan"))
    c.unpack(out)
    torch.cuda.synchronize()
    raw = c.packed.cpu().numpy()
    at, G = (T * d + 255) // 256 * 256, (d + 127) // 128
    codes = raw[:T * d].view(np.int8).reshape(T, d)
    scales = (raw[at:at + 2 * T * G].view(np.uint16).astype(np.uint32) << 16).view(np.float32).reshape(T, G)
    return c, codes, scales, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 8), (1, 128), (3, 136), (77, 1000), (130, 4096), (5, 17408), (999, 24)])
def test_codes_scales_and_values(T, d, dtype):
    import torch
    x = _values(T + d, T, d, dtype)
    _, codes, scales, out = _pack(x, dtype)
    rc, rs = ck.pack(x)
    assert np.array_equal(scales, rs)
    assert np.array_equal(codes, rc), int((codes != rc).sum())
    v = ck.unpack(rc, rs)
    ref = wk.round_to_bf16(v.astype(np.float32)) if dtype == "bf16" else v.astype(np.float32)    # (products of 7 and 8 bits: exact)
    assert np.array_equal(out.float().cpu().numpy(), ref)


def test_extreme_and_not_finite_groups():
    x = np.zeros((8, 256), dtype=np.float32)
    x[0, :3] = [2.0 ** -130, -2.0 ** -110, 2.0 ** -101]
    x[1, 5], x[1, 130] = np.inf, 7.0
    x[2, 200], x[2, 1] = np.nan, -3.0
    x[3, 0], x[3, 128] = 2.0 ** 127, 1.5 * 2.0 ** 126
    x[4, :] = -0.0
    x[5, 255] = -np.inf
    x[6, :128] = 127.0
    _, codes, scales, out = _pack(wk.round_to_bf16(x), "bf16")
    rc, rs = ck.pack(x)
    assert np.array_equal(codes, rc) and np.array_equal(scales, rs, equal_nan=True)
    o = out.float().cpu().numpy()
    for r, g in ((1, 0), (2, 1), (3, 0), (5, 1)):
        assert np.isnan(o[r, g * 128:(g + 1) * 128]).all()
    assert np.isfinite(o[[0, 4, 6, 7]]).all() and o[1, 130] != 0 and np.isfinite(o[1, 128:]).all()


def _layer(dtype, d_in, d_out, ranks, tokens, scales, seed):
    from paper_2602_07263_amd import tlora
    p = wk.generate(wk.custom("ckpt", dtype, d_in, d_out, ranks, tokens, scales), seed=seed)
    p.X[:, ::37] *= 8
    return p, tlora.LayerProblem.from_numpy(p)


LAYERS = [("bf16", 256, 384, [3, 16, 40, 0, 130], [70, 300, 129, 40, 260], [2.0, 0.5, 1.0, 2.0, 1.5]),
          ("bf16", 1000, 264, [8], [1], [2.0]), ("bf16", 4096, 1024, [16, 32], [512, 1001], [2.0, 1.0]),
          ("bf16", 512, 512, [8, 5], [70, 33], [2.0, 3.0]), ("f32", 136, 72, [4, 7], [50, 81], [2.0, 1.0]),
          ("bf16", 136, 1024, [1, 128, 32], [0, 700, 65], [1.0, 1.0, 2.0]),
          # a last tile of 16 columns, units of more tokens than one takes, ranks of several blocks
          ("bf16", 272, 64, [40, 4], [9000, 31], [1.0, 2.0]), ("bf16", 144, 128, [200], [130], [1.0]),
          # batches whose S_j is made again from the codes: units of 64 and of 128 rows, low and high ranks, a half group at the end
          ("bf16", 320, 64, [40, 130, 8], [7000, 5000, 301], [1.0, 2.0, 0.5]),
          ("bf16", 448, 64, [16, 64, 160], [20000, 4001, 2300], [1.0, 2.0, 0.5])]


@pytest.mark.parametrize("case", LAYERS, ids=[f"{c[0]}_{c[1]}_{c[2]}_{sum(c[4])}" for c in LAYERS])
@pytest.mark.parametrize("reuse_S", [False, True])
@pytest.mark.parametrize("want_dX", [False, True])
def test_backward_from_eight_bits(case, reuse_S, want_dX):
    import torch
    from paper_2602_07263_amd import tlora
    p, lp = _layer(*case, seed=11)
    c = tlora.Checkpoint(p.dtype, lp.T, lp.d_in, "cuda")
    c.pack(lp.X)
    lp.bwd_ckpt_workspace()
    Y, dX, dA, dB = lp.new_outputs()
    for t in [dX] + dA + dB:
        t.fill_(float("nan"))
    dY = torch.from_numpy(p.dY).to("cuda", lp.X.dtype)
    X = lp.X.clone()
    if reuse_S:
        lp.fwd(Y)
    lp.X.fill_(float("nan"))                            # X is not read
    print(f"bwd_ckpt {case} reuse {reuse_S} dX {want_dX}", flush=True)
    lp.bwd_ckpt(c.packed, dY, dX if want_dX else None, dA, dB, reuse_S=reuse_S)
    torch.cuda.synchronize()
    X8 = torch.empty_like(X)
    c.unpack(X8)
    torch.cuda.synchronize()
    v = X8.float().cpu().numpy()
    ref = orc.backward(v, p.W, p.A, p.B, p.scales, p.offsets, p.dY)
    rX, rA, rB = ref[0], ref[1], ref[2]
    if reuse_S:
        rB = orc.backward(X.float().cpu().numpy(), p.W, p.A, p.B, p.scales, p.offsets, p.dY)[2]
    tol = pu.BF16_TOL if p.dtype == "bf16" else pu.F32_TOL
    if want_dX:
        assert pu.worst_ratio(dX.float().cpu().numpy(), rX, tol) <= 1.0
    else:
        assert torch.isnan(dX.float()).all()
    for j, r in enumerate(p.ranks):
        if r:
            assert pu.worst_ratio(dA[j].cpu().numpy(), rA[j], pu.F32_TOL if p.dtype == "f32" else tol) <= 1.0
            assert pu.worst_ratio(dB[j].cpu().numpy(), rB[j], pu.F32_TOL if p.dtype == "f32" else tol) <= 1.0
    # sums of two backwards
    acc = [t.clone() for t in dA + dB]
    lp.bwd_ckpt(c.packed, dY, None, dA, dB, reuse_S=reuse_S, flags=tlora.TLORA_BWD_ACCUMULATE)
    torch.cuda.synchronize()
    for a, b in zip(acc, dA + dB):
        torch.testing.assert_close(b, 2 * a, rtol=2 ** -20, atol=2 ** -20 * float(a.abs().max()) if a.numel() else 0)


def test_dX_alone_does_not_read_the_packed_values():
    import torch
    p, lp = _layer(*LAYERS[2], seed=12)
    lp.bwd_ckpt_workspace()
    _, dX, _, _ = lp.new_outputs()
    ref = torch.empty_like(dX)
    dY = torch.from_numpy(p.dY).to("cuda", torch.bfloat16)
    bad = torch.full((1 << 23,), 0x7F, dtype=torch.uint8, device="cuda")
    lp.bwd_ckpt(bad, dY, dX, None, None)
    lp.bwd(dY, ref, None, None)
    torch.cuda.synchronize()
    assert torch.equal(dX, ref)


def test_pack_and_unpack_replay_from_a_captured_stream():
    import torch
    from paper_2602_07263_amd import tlora
    x = torch.randn(200, 1160, device="cuda").to(torch.bfloat16)
    c = tlora.Checkpoint("bf16", 200, 1160, "cuda")
    ref, out = torch.empty_like(x), torch.empty_like(x)
    c.pack(x)
    c.unpack(ref)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        c.pack(x)
        c.unpack(out)
    for rep in range(3):
        out.fill_(float("nan"))
        c.packed.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
