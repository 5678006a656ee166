"""Workspaces of the operators around the decoder layers: what they hold beside the plain ones, on the host."""
import ctypes

import numpy as np
import pytest

from paper_2602_07263_amd import tlora
from paper_2602_07263_amd import workloads as wk

P = ctypes.c_void_p
WS = 0x100000
EWORKSPACE, ENOUGH = -4, -7


def _problem(tokens, ranks, d_in, d_out=4096, dtype=tlora.TLORA_BF16):
    off = np.concatenate([[0], np.cumsum(tokens)]).astype(np.int64)
    n = len(ranks)
    return tlora.make_problem(dtype, d_in, d_out, ranks, off, [1.0] * n, 0, 0x2000, [0x3000] * n, [0x4000] * n)


def _sizes(q):
    L = tlora.lib()
    return L.tlora_workspace_bytes(ctypes.byref(q[0])), L.tlora_ckpt_workspace_bytes(ctypes.byref(q[0]))


def _rc(q, n, flags=0, grads=True):
    """EWORKSPACE, or what a call whose workspace is large enough is refused for next: packed values that are not aligned."""
    g = (P * q[0].num_jobs)(*[0x6000] * q[0].num_jobs) if grads else None
    return tlora.lib().tlora_bwd_ckpt(ctypes.byref(q[0]), P(WS + 16), P(0x5000), P(0x8000), g, g, flags, P(WS), n, None)


BATCH_8B = [[int(v) for v in x] for x in (wk.config(2).tokens, wk.config(2).ranks)]      # the benchmark's eight jobs, 31744 tokens


def test_a_kept_S_needs_no_room_for_the_values():
    for d_in in (4096, 12288, 17408, 144):
        q = _problem(*BATCH_8B, d_in)
        plain, with_values = _sizes(q)
        assert _rc(q, plain - 1, tlora.TLORA_BWD_REUSE_S) == EWORKSPACE
        assert _rc(q, plain, tlora.TLORA_BWD_REUSE_S) == ENOUGH
        assert _rc(q, plain, grads=False) == ENOUGH
        assert with_values > plain


def test_large_batches_have_room_for_what_small_ones_unpack():
    T = sum(BATCH_8B[0])
    for d_in in (4096, 12288):
        plain, with_values = _sizes(_problem(*BATCH_8B, d_in))
        assert with_values - plain <= 2 * 12288 * d_in + 512 < 2 * T * d_in
        q = _problem(*BATCH_8B, d_in)
        assert _rc(q, plain) == ENOUGH              # (S_j is made again from the codes)


@pytest.mark.parametrize("kw", [dict(d_in=4096), dict(d_in=4096, d_out=4104), dict(d_in=1000), dict(d_in=144), dict(d_in=24576),
                                dict(d_in=512, dtype=tlora.TLORA_F32)], ids=lambda k: "_".join(str(v) for v in k.values()))
@pytest.mark.parametrize("ranks", [[8, 16, 0], [130, 4, 700]])
def test_a_workspace_serves_every_smaller_batch(kw, ranks):
    sizes, tokens = [], ([1, 0, 3], [60, 1, 60], [61, 200, 200], [3000, 200, 200], [6000, 3000, 200], [6000, 6000, 6000], [12000, 12000, 6000],
                         [30000, 12000, 6000], [30000, 40000, 6001])
    for t in tokens:
        q = _problem(t, ranks, **kw)
        plain, most = _sizes(q)
        # what any call on this batch needs: found by its refusals
        for flags in (0, tlora.TLORA_BWD_REUSE_S):
            assert _rc(q, most, flags) == ENOUGH
        sizes.append(most)
        values = (4 if kw.get("dtype") == tlora.TLORA_F32 else 2) * sum(t) * kw["d_in"]
        behind = (plain + 255) // 256 * 256
        small = _rc(q, plain) == EWORKSPACE
        if small:                                       # the call unpacks: no byte less than the values take
            assert _rc(q, behind + values - 1) == EWORKSPACE
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_a_holder_keeps_what_its_workspace_held():
    import torch
    bf = torch.bfloat16
    z = lambda *n: torch.zeros(*n, dtype=bf)
    layer = tlora.LayerProblem("bf16", 16, 16, [4], [0, 4], [1.0], z(4, 16), z(16, 16), [z(16, 4)], [z(4, 16)])
    layer.ws.copy_(torch.arange(layer.ws_bytes) % 251)
    before = layer.ws.clone()
    layer.bwd_ckpt_workspace(reuse_S=True)
    assert layer.ws_bytes == before.numel()
    layer.bwd_ckpt_workspace()
    assert layer.ws_bytes == layer.ws.numel() > before.numel()
    assert torch.equal(layer.ws[:before.numel()], before)


@pytest.mark.parametrize("behind,groups,tokens", [(-65, 439, 2445881), (-64, 64, 16777215), (-62, 131, 8196502), (-1, 77, 13944699)])
def test_eight_bits_of_a_full_launch(behind, groups, tokens):
    # 64 groups to a workgroup: 2^24 - 1 workgroups of 256 threads are the most below 2^32 threads
    L = tlora.lib()
    assert groups * tokens == (1 << 30) + behind
    fits = -(-groups * tokens // 64) * 256 < 1 << 32
    assert (L.tlora_ckpt_bytes(tokens, 128 * groups) > 0) == fits == (behind <= -64)
    if not fits:
        assert L.tlora_ckpt_pack(1, P(0x1000), tokens, 128 * groups, P(WS), None) == -1
        assert L.tlora_ckpt_unpack(1, P(WS), tokens, 128 * groups, P(0x1000), None) == -1


def _shares(rows, tiles_n, steps):
    """Tiles of fp32 sums that a product of `rows` rows leaves: whole rounds of 256 tiles as they are, the rest in shares."""
    rest = -(-rows // 256) * tiles_n % 256
    if not rest:
        return 0
    extra, most = 32 * min(rows, 256) // 256, min(64, max(steps // 8, 1))
    s1, s2 = min(256 // rest, most), min(512 // rest, most)
    cost1 = -(-steps // s1) + extra if s1 > 1 else steps
    cost2 = 2 * (-(-steps // s2) + extra)
    n = s2 if cost2 < cost1 and rest * s2 > 256 else s1 if s1 > 1 and cost1 < steps else 1
    return rest * n if n > 1 else 0


def _ce_sizes(T, d, V):
    ld = (V + 7) // 8 * 8
    off = (ctypes.c_int64 * 2)(0, T)
    q = tlora.tlora_ce_t(tlora.TLORA_BF16, 1, d, V, ld, off, P(0x1000), P(0x2000), P(0x3000), None)
    return [tlora.lib().tlora_ce_workspace_bytes(ctypes.byref(q), g) for g in (0, 1)], ld


@pytest.mark.parametrize("d,V", [(64, 9), (64, 1000), (72, 5000), (1024, 600), (512, 50000), (4096, 32000), (8192, 259)])
def test_the_losses_workspace_holds_the_shares_of_any_number_of_rows(d, V):
    tile = 256 * 256 * 4
    last = [0, 0]
    for T in (1, 61, 256, 257, 1500, 4096, 5000, 20000):
        sizes, ld = _ce_sizes(T, d, V)
        for g in (0, 1):
            piece = min(4096 if g else 16384, -(-T // 256) * 256)
            logits = max(_shares(r, -(-V // 256), d // 32) for r in range(1, min(piece, T) + 1, 1 if T < 300 else 17)) if d % 32 == 0 else 0
            grads = max(_shares(r, -(-d // 256), -(-V // 32)) for r in range(1, min(piece, T) + 1, 1 if T < 300 else 17)) if g else 0
            # beside them a piece's rows, exponentials and statistics
            others = 2 * piece * d + 8 * piece * -(-V // 256) + (2 * piece * ld if g else 0)
            assert sizes[g] >= others + tile * max(logits, grads)
            assert sizes[g] >= last[g]
        last = sizes
    assert sizes[1] <= 2 * 16384 * d + 8 * 16384 * -(-V // 256) + 2 * 4096 * ld + 512 * tile + (1 << 20)


def test_a_small_loss_has_a_small_workspace():
    for T, d, V in ((61, 64, 200), (500, 128, 250), (61, 72, 255)):
        sizes, _ = _ce_sizes(T, d, V)
        assert max(sizes) < 1 << 20
