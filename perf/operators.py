"""The operators around the decoder layers of a training step, as cases: what is timed, in plain torch and as the library runs it.

kind      one pass
"loss"    softmax cross entropy of the vocabulary projection of the last hidden states, per job: token losses, each job's mean
          loss and, with "grad", the gradient of the sum of those means for the hidden states (tlora_ce_fwd, tlora_ce_fwd_bwd)
"norm"    residual stream and norms between two blocks: H = X + res_scale * gate_j * norm(Y; gamma_post), Xn = norm(H; gamma_pre)
          (tlora_norm_fwd), or with "grad" its gradient for the stream, the block's output, both gammas and the gates (tlora_norm_bwd)
"act8"    an activation into 8 bits and back (tlora_ckpt_pack, tlora_ckpt_unpack)
"bwd8"    the fused layer's backward whose X was kept in 8 bits (tlora_bwd_ckpt)

Lists of per-job numbers are texts ("8,16,32").  Hidden states and upstream gradients are N(0, 1), the vocabulary projection
N(0, 1 / d_model) times 2 (logits of standard deviation 2), gammas and gates N(1, 0.1), adapters as in the benchmark's workloads.
"""
import math

import torch

own = False      # False: the plain forms; True: the library's calls

GROUP = 128      # values of a row that share a scale in the 8-bit form
IGNORE = -100    # target of a token that has no loss


def _ints(text):
    return [int(v) for v in text.split(",")]


def _text(values):
    return ",".join(str(v) for v in values)


def _offsets(tokens):
    out = [0]
    for t in tokens:
        out.append(out[-1] + t)
    return out


# The tokens of the benchmark's 8B-class workload of eight jobs (its configuration 2) and their ranks
TOKENS_8B, RANKS_8B = "5120,512,2048,3584,3072,6144,5120,6144", "4,8,8,16,32,32,64,128"


def listed():
    return [
        # loss and gradient of a few short answers of eight jobs: the smallest training call, bound by reading the projection twice
        {"name": "loss_grad_61", "kind": "loss", "grad": True, "d": 4096, "vocab": 32000, "tokens": "1,4,7,1,16,12,11,9",
         "ignored": 0.0, "weighted": False},
        # three jobs' instruction samples: prompts are ignored (about half of the tokens), a vocabulary of odd size, token weights
        {"name": "loss_grad_ragged_1500", "kind": "loss", "grad": True, "d": 4096, "vocab": 49999, "tokens": "517,802,181",
         "ignored": 0.5, "weighted": True},
        # four jobs' micro-batch on a large vocabulary, every token counts; the largest call
        {"name": "loss_grad_7680", "kind": "loss", "grad": True, "d": 4096, "vocab": 128000, "tokens": "2048,1024,4096,512",
         "ignored": 0.0, "weighted": False},
        # validation: losses alone, feature size of the 14B-class layer
        {"name": "loss_eval_4095", "kind": "loss", "grad": False, "d": 5120, "vocab": 64000, "tokens": "1365,2730",
         "ignored": 0.1, "weighted": False},
        # one step of a few tokens through the norms of an 8B-class layer: latency
        {"name": "norm_fwd_13", "kind": "norm", "grad": False, "dtype": "bf16", "d": 4096, "tokens": "5,1,7", "post": True,
         "gates": True},
        # the benchmark's 8B-class batch, forward
        {"name": "norm_fwd_31744", "kind": "norm", "grad": False, "dtype": "bf16", "d": 4096, "tokens": TOKENS_8B, "post": True,
         "gates": True},
        # the same batch backward, gammas and the jobs' gates trained
        {"name": "norm_grad_31744", "kind": "norm", "grad": True, "dtype": "bf16", "d": 4096, "tokens": TOKENS_8B, "post": True,
         "gates": True},
        # fp32 stream, ragged jobs (one without tokens), odd feature size, no norm behind the block and no gates
        {"name": "norm_grad_f32_1001", "kind": "norm", "grad": True, "dtype": "f32", "d": 1544, "tokens": "333,0,668",
         "post": False, "gates": False},
        # the input of one job's layer as a checkpoint
        {"name": "act8_512", "kind": "act8", "dtype": "bf16", "d": 4096, "tokens": "512"},
        # the widest activation of the 8B-class batch (input of the down projection)
        {"name": "act8_31744", "kind": "act8", "dtype": "bf16", "d": 12288, "tokens": TOKENS_8B},
        # backward of an attention projection (benchmark's configuration 1) from 8 bits, S_j kept from the forward
        {"name": "bwd8_7680", "kind": "bwd8", "dtype": "bf16", "dims": "4096x4096", "ranks": "8,16,32,64",
         "tokens": "2048,1024,4096,512", "reuse_S": True, "want_dX": True},
        # the 8B-class batch at the first layer's gate projection (no gradient for X wanted), S_j made again from the 8 bits
        {"name": "bwd8_first_layer_31744", "kind": "bwd8", "dtype": "bf16", "dims": "4096x12288", "ranks": RANKS_8B,
         "tokens": TOKENS_8B, "reuse_S": False, "want_dX": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, total, jobs):
    """`total` tokens cut at random into at most `jobs` segments of at least one token."""
    jobs = min(jobs, total)
    cuts = sorted(rng.sample(range(1, total), jobs - 1)) if jobs > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def draw(rng):
    kind = rng.choice(["loss", "loss", "norm", "norm", "act8", "bwd8"])
    if kind == "loss":
        d, vocab = rng.choice([1024, 2048, 4096, 5120, 8 * _log_uniform(rng, 64, 640)]), _log_uniform(rng, 4000, 128000)
        # no more products than the largest listed case has
        top = min(8192, 7680 * 4096 * 128000 // (d * vocab))
        tok = _split(rng, _log_uniform(rng, 1, top), rng.randint(1, 12))
        return {"kind": kind, "grad": rng.random() < 0.7, "d": d, "vocab": vocab, "tokens": _text(tok),
                "ignored": rng.choice([0.0, 0.0, 0.1, 0.5, 0.9]), "weighted": rng.random() < 0.3}
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([1024, 4096, 5120, 8 * _log_uniform(rng, 16, 1600)])
        top = min(32768, 31744 * 4096 // d // (1 if dtype == "bf16" else 2))
        tok = _split(rng, _log_uniform(rng, 1, top), rng.randint(1, 16))
        return {"kind": kind, "grad": rng.random() < 0.6, "dtype": dtype, "d": d, "tokens": _text(tok),
                "post": rng.random() < 0.7, "gates": rng.random() < 0.6}
    if kind == "act8":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([4096, 12288, 17408, 8 * _log_uniform(rng, 16, 2048)])
        top = min(32768, 31744 * 12288 // d // (1 if dtype == "bf16" else 2))
        return {"kind": kind, "dtype": dtype, "d": d, "tokens": str(_log_uniform(rng, 1, top))}
    width = lambda: rng.choice([1024, 4096, 4096, 5120, 8 * _log_uniform(rng, 32, 1536)])
    d_in, d_out = width(), width()
    tok = _split(rng, _log_uniform(rng, 16, min(16384, 31744 * 4096 * 12288 // (4 * d_in * d_out))), rng.randint(1, 12))
    ranks = [rng.choice([1, 2, 3, 4, 8, 8, 16, 16, 32, 48, 64, 96, 128]) for _ in tok]
    return {"kind": kind, "dtype": "bf16", "dims": f"{d_in}x{d_out}", "ranks": _text(ranks), "tokens": _text(tok),
            "reuse_S": rng.random() < 0.5, "want_dX": rng.random() < 0.7}


class _Inputs:
    """Seeded device tensors."""

    def __init__(self, seed, dtype="bf16"):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(self, *shape, std=1.0, mean=0.0):
        t = torch.randn(*shape, device="cuda", generator=self.g, dtype=self.dtype)
        return t if std == 1.0 and mean == 0.0 else t.mul_(std).add_(mean)

    def uniform(self, *shape):
        return torch.rand(*shape, device="cuda", generator=self.g)


def _prepare_loss(case, seed):
    x = _Inputs(seed)
    tokens, d, vocab = _ints(case["tokens"]), case["d"], case["vocab"]
    T, ld = sum(tokens), (vocab + 7) // 8 * 8
    st = {"H": x.normal(T, d), "W": x.normal(d, ld, std=2.0 / d ** 0.5), "offsets": _offsets(tokens)}
    y = torch.randint(0, vocab, (T,), device="cuda", generator=x.g, dtype=torch.int32)
    st["targets"] = torch.where(x.uniform(T) < case["ignored"], torch.full_like(y, IGNORE), y)
    st["weights"] = 0.5 + x.uniform(T) if case["weighted"] else None
    return st


def _prepare_norm(case, seed):
    x = _Inputs(seed, case["dtype"])
    tokens, d = _ints(case["tokens"]), case["d"]
    T = sum(tokens)
    st = {"X": x.normal(T, d), "Y": x.normal(T, d, std=0.5), "offsets": _offsets(tokens), "eps": 1e-5, "res_scale": 0.5}
    st["gamma_post"] = x.normal(d, std=0.1, mean=1.0) if case["post"] else None
    st["gates"] = [x.normal(d, std=0.1, mean=1.0) for _ in tokens] if case["gates"] else None
    st["gamma_pre"] = x.normal(d, std=0.1, mean=1.0)
    if case["grad"]:
        st["dH"], st["dXn"] = x.normal(T, d), x.normal(T, d)
    return st


def _activations(x, T, d):
    """Rows as a layer sees them: unit scale with a few feature columns that are larger by far."""
    X = x.normal(T, d)
    X[:, :: 97] *= 8
    return X


def _prepare_bwd8(case, seed):
    x = _Inputs(seed, case["dtype"])
    ranks, tokens = _ints(case["ranks"]), _ints(case["tokens"])
    d_in, d_out = _ints(case["dims"].replace("x", ","))
    T = sum(tokens)
    st = {"X": _activations(x, T, d_in), "dY": x.normal(T, d_out), "W": x.normal(d_in, d_out, std=0.02), "offsets": _offsets(tokens),
          "ranks": ranks, "scales": [2.0] * len(ranks)}
    st["A"] = [((x.uniform(d_in, r) * 2 - 1) / d_in ** 0.5).to(x.dtype) for r in ranks]
    st["B"] = [x.normal(r, d_out, std=0.01) for r in ranks]
    codes, scales = _quantise(st["X"])
    # the packed form as tlora_ckpt_pack lays it out: all codes, then the scales from the next multiple of 256 bytes on
    at = (codes.numel() + 255) // 256 * 256
    st["packed"] = torch.zeros((at + 2 * scales.numel() + 255) // 256 * 256, dtype=torch.uint8, device="cuda")
    st["packed"][:codes.numel()] = codes.reshape(-1).view(torch.uint8)
    st["packed"][at:at + 2 * scales.numel()] = scales.to(torch.bfloat16).reshape(-1).view(torch.uint8)
    return st


def prepare(case, seed):
    kind = case["kind"]
    if kind == "loss":
        st = _prepare_loss(case, seed)
    elif kind == "norm":
        st = _prepare_norm(case, seed)
    elif kind == "act8":
        st = {"X": _activations(_Inputs(seed, case["dtype"]), sum(_ints(case["tokens"])), case["d"])}
    else:
        st = _prepare_bwd8(case, seed)
    st["case"] = case
    if own:
        _prepare_own(case, st)
    return st


def _prepare_own(case, st):
    """The holders and output buffers that a training program keeps from step to step."""
    from paper_2602_07263_amd import tlora
    kind, f32 = case["kind"], dict(dtype=torch.float32, device="cuda")
    if kind == "loss":
        T, J = st["offsets"][-1], len(st["offsets"]) - 1
        st["head"] = tlora.LossHead(st["offsets"], st["H"], st["W"], case["vocab"], st["targets"], st["weights"],
                                    with_grad=case["grad"])
        st["out"] = {"loss": torch.empty(T, **f32), "lse": torch.empty(T, **f32), "job_loss": torch.empty(J, **f32)}
        if case["grad"]:
            st["out"]["dH"] = torch.empty_like(st["H"])
    elif kind == "norm":
        st["norm"] = tlora.ResidualNorm(case["dtype"], st["offsets"], st["X"], st["Y"], st["gamma_pre"], st["eps"],
                                        gamma_post=st["gamma_post"], gates=st["gates"], res_scale=st["res_scale"])
        if case["grad"]:
            d = case["d"]
            st["out"] = {"dX": torch.empty_like(st["X"]), "dY": torch.empty_like(st["Y"]), "dgamma_pre": torch.empty(d, **f32),
                         "dgamma_post": torch.empty(d, **f32) if case["post"] else None,
                         "dgates": [torch.empty(d, **f32) for _ in st["gates"]] if case["gates"] else None}
        else:
            st["out"] = {"H": torch.empty_like(st["X"]), "Xn": torch.empty_like(st["X"])}
    elif kind == "act8":
        T, d = st["X"].shape
        st["act8"] = tlora.Checkpoint(case["dtype"], T, d, "cuda")
        st["out"] = torch.empty_like(st["X"])
    else:
        d_in, d_out = _ints(case["dims"].replace("x", ","))
        st["layer"] = tlora.LayerProblem(case["dtype"], d_in, d_out, st["ranks"], st["offsets"], st["scales"], st["X"], st["W"],
                                         st["A"], st["B"])
        Y, dX, dA, dB = st["layer"].new_outputs()
        st["layer"].bwd_ckpt_workspace()
        if case["reuse_S"]:
            st["layer"].fwd(Y)
        st["out"] = {"dX": dX if case["want_dX"] else None, "dA": dA, "dB": dB}


def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    return {"loss": _plain_loss, "norm": _plain_norm, "act8": _plain_act8, "bwd8": _plain_bwd8}[case["kind"]](case, st)


def _run_own(case, st):
    kind = case["kind"]
    if kind == "loss":
        out = st["out"]
        if case["grad"]:
            st["head"].fwd_bwd(out["loss"], out["lse"], out["job_loss"], out["dH"])
        else:
            st["head"].fwd(out["loss"], out["lse"], out["job_loss"])
        return out
    if kind == "norm":
        out = st["out"]
        if case["grad"]:
            st["norm"].bwd(st["dH"], st["dXn"], out["dX"], out["dY"], dgamma_post=out["dgamma_post"], dgamma_pre=out["dgamma_pre"],
                           dgates=out["dgates"])
        else:
            st["norm"].fwd(out["H"], out["Xn"])
        return {k: v for k, v in out.items() if v is not None}
    if kind == "act8":
        st["act8"].pack(st["X"])
        st["act8"].unpack(st["out"])
        return st["out"]
    out = st["out"]
    st["layer"].bwd_ckpt(st["packed"], st["dY"], out["dX"], out["dA"], out["dB"], reuse_S=case["reuse_S"])
    return {k: v for k, v in out.items() if v is not None}


# ---- plain forms: elementary torch operations in 32 bits, rounded once at the end ----------------------------------------

_PIECE = 1024        # rows of logits held at a time


def _plain_loss(case, st):
    H, y, vocab = st["H"], st["targets"].long(), case["vocab"]
    W = st["W"][:, :vocab].float()
    counted = y >= 0
    y0 = torch.where(counted, y, torch.zeros_like(y))
    w = torch.where(counted, st["weights"] if st["weights"] is not None else torch.ones_like(y, dtype=torch.float32), 0.0)
    loss, lse = torch.zeros_like(w), torch.zeros_like(w)
    share = torch.zeros_like(w)                    # what a token's loss counts for in its job's mean
    bounds = list(zip(st["offsets"][:-1], st["offsets"][1:]))
    for a, b in bounds:
        total = w[a:b].sum()
        share[a:b] = torch.where(total != 0, w[a:b] / total, torch.zeros_like(w[a:b]))
    dH = torch.empty_like(H) if case["grad"] else None
    for a in range(0, H.shape[0], _PIECE):
        s = slice(a, min(a + _PIECE, H.shape[0]))
        z = H[s].float() @ W
        top = z.max(dim=1, keepdim=True).values
        l = top[:, 0] + torch.exp(z - top).sum(dim=1).log()
        zy = z.gather(1, y0[s, None])[:, 0]
        zero = torch.zeros_like(l)
        lse[s] = torch.where(counted[s], l, zero)
        loss[s] = torch.where(counted[s], l - zy, zero)
        if case["grad"]:
            p = z.sub_(l[:, None]).exp_()
            p.scatter_add_(1, y0[s, None], -torch.ones_like(l)[:, None])
            p *= share[s, None]
            dH[s] = (p @ W.t()).to(H.dtype)
    job_loss = torch.stack([(loss[a:b] * share[a:b]).sum() for a, b in bounds])
    out = {"loss": loss, "lse": lse, "job_loss": job_loss}
    if case["grad"]:
        out["dH"] = dH
    return out


def _spread(st, T, d, like):
    """The gate of every token: its job's."""
    if st["gates"] is None:
        return torch.ones(1, d, dtype=like, device="cuda")
    n = torch.tensor([b - a for a, b in zip(st["offsets"][:-1], st["offsets"][1:])], device="cuda")
    return torch.stack(st["gates"]).to(like).repeat_interleave(n, dim=0, output_size=T)


def _plain_norm(case, st):
    X, Y, alpha, eps = st["X"].float(), st["Y"].float(), st["res_scale"], st["eps"]
    T, d = X.shape
    gate, g_pre = _spread(st, T, d, torch.float32), st["gamma_pre"].float()
    post = st["gamma_post"]
    if post is not None:
        r1 = 1.0 / torch.sqrt((Y * Y).mean(dim=1, keepdim=True) + eps)
        Yh = Y * r1
        N = Yh * post.float()
    else:
        N = Y
    H = X + alpha * (gate * N)
    r2 = 1.0 / torch.sqrt((H * H).mean(dim=1, keepdim=True) + eps)
    Hh = H * r2
    if not case["grad"]:
        return {"H": H.to(st["X"].dtype), "Xn": (Hh * g_pre).to(st["X"].dtype)}
    dXn = st["dXn"].float()
    gd = dXn * g_pre
    D = st["dH"].float() + r2 * (gd - Hh * (gd * Hh).mean(dim=1, keepdim=True))
    dN = alpha * (gate * D)
    out = {"dX": D.to(st["X"].dtype), "dgamma_pre": (dXn * Hh).sum(dim=0)}
    if post is not None:
        pd = dN * post.float()
        out["dY"] = (r1 * (pd - Yh * (pd * Yh).mean(dim=1, keepdim=True))).to(st["X"].dtype)
        out["dgamma_post"] = (dN * Yh).sum(dim=0)
    else:
        out["dY"] = dN.to(st["X"].dtype)
    if st["gates"] is not None:
        dg = alpha * D * N
        out["dgates"] = [dg[a:b].sum(dim=0) for a, b in zip(st["offsets"][:-1], st["offsets"][1:])]
    return out


def _quantise(X):
    """(codes int8 [T, d], scales fp32 [T, groups]): for each group of 128 values of a row the smallest bfloat16 s >= 2^-100 with
    127 s >= max |x|, and the whole numbers next to x / s, ties to even."""
    T, d = X.shape
    G = (d + GROUP - 1) // GROUP
    x = torch.zeros(T, G * GROUP, dtype=torch.float32, device=X.device)
    x[:, :d] = X
    x = x.view(T, G, GROUP)
    top = x.abs().amax(dim=2)
    up = lambda v: ((v.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)     # bfloat16, away from zero
    s = up((top / 127.0).contiguous())
    s = torch.where(127.0 * s < top, up((s * (1 + 2.0 ** -12)).contiguous()), s).clamp_min(2.0 ** -100)
    q = torch.round(x / s[:, :, None]).to(torch.int8).view(T, G * GROUP)[:, :d].contiguous()
    return q, s


def _restore(codes, scales, dtype):
    T, d = codes.shape
    s = scales.repeat_interleave(GROUP, dim=1)[:, :d]
    return (codes.float() * s).to(dtype)


def _plain_act8(case, st):
    return _restore(*_quantise(st["X"]), st["X"].dtype)


def _unpack(st, dtype):
    T, d = st["X"].shape
    n, G = T * d, (d + GROUP - 1) // GROUP
    at = (n + 255) // 256 * 256
    scales = st["packed"][at:at + 2 * T * G].view(torch.bfloat16).float().view(T, G)
    return _restore(st["packed"][:n].view(torch.int8).view(T, d), scales, dtype)


def _plain_bwd8(case, st):
    X8 = _unpack(st, st["X"].dtype).float()
    dY = st["dY"].float()
    S_from = st["X"].float() if case["reuse_S"] else X8
    dX = dY @ st["W"].float().t() if case["want_dX"] else None
    dA, dB = [], []
    for j, (a, b) in enumerate(zip(st["offsets"][:-1], st["offsets"][1:])):
        A, B, s = st["A"][j].float(), st["B"][j].float(), st["scales"][j]
        dS = dY[a:b] @ B.t()
        dA.append(s * (X8[a:b].t() @ dS))
        dB.append(s * ((S_from[a:b] @ A).t() @ dY[a:b]))
        if dX is not None:
            dX[a:b] += s * (dS @ A.t())
    out = {"dA": dA, "dB": dB}
    if dX is not None:
        out["dX"] = dX.to(st["X"].dtype)
    return out


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------

def exact(case, seed):
    kind = case["kind"]
    if kind == "loss":
        return _exact_loss(case, _prepare_loss(case, seed))
    if kind == "norm":
        return _exact_norm(case, _prepare_norm(case, seed))
    if kind == "act8":
        X = _activations(_Inputs(seed, case["dtype"]), sum(_ints(case["tokens"])), case["d"])
        return _exact_act8(X)
    return _exact_bwd8(case, _prepare_bwd8(case, seed))


def _exact_loss(case, st):
    V, grad = case["vocab"], case["grad"]
    T, d = st["H"].shape
    W = st["W"].double()[:, :V].contiguous()
    Wt = W.t().contiguous() if grad else None
    loss = torch.zeros(T, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    weight = torch.ones_like(loss) if st["weights"] is None else st["weights"].double()
    live = (st["targets"] >= 0).nonzero()[:, 0]
    share = torch.zeros_like(loss)
    job_loss = torch.zeros(len(st["offsets"]) - 1, dtype=torch.float64, device="cuda")
    for a, b in zip(st["offsets"][:-1], st["offsets"][1:]):
        mine = live[(live >= a) & (live < b)]
        if len(mine):
            share[mine] = weight[mine] / weight[mine].sum()
    dH = torch.zeros(T, d, dtype=torch.float64, device="cuda") if grad else None
    for rows in live.split(512):
        z = st["H"][rows].double().matmul(W)
        y = st["targets"][rows].long()
        L = torch.logsumexp(z, dim=1)
        k = torch.arange(len(rows), device="cuda")
        lse[rows], loss[rows] = L, L - z[k, y]
        if grad:
            P = (z - L[:, None]).exp()
            P[k, y] -= 1.0
            dH[rows] = share[rows, None] * P.matmul(Wt)
    for j, (a, b) in enumerate(zip(st["offsets"][:-1], st["offsets"][1:])):
        job_loss[j] = (share[a:b] * loss[a:b]).sum()
    out = {"loss": loss, "lse": lse, "job_loss": job_loss}
    if grad:
        out["dH"] = dH
    return out


def _exact_norm(case, st):
    """The gradient by the chain rule job by job, from the derivative of v / sqrt(mean(v^2) + eps)."""
    f = lambda t: None if t is None else t.double()
    outs = {"H": [], "Xn": [], "dX": [], "dY": []}
    post, pre = f(st["gamma_post"]), f(st["gamma_pre"])
    one = torch.ones_like(pre)
    dpost, dpre, dgates = torch.zeros_like(pre), torch.zeros_like(pre), []
    a_, e = st["res_scale"], st["eps"]

    def unit(v):
        n = (v.square().mean(dim=1) + e).rsqrt()[:, None]
        return v * n, n

    def back(u, n, g):                       # gradient through unit()
        return n * g - u * n * (g * u).mean(dim=1, keepdim=True)

    for j, (a, b) in enumerate(zip(st["offsets"][:-1], st["offsets"][1:])):
        X, Y = f(st["X"][a:b]), f(st["Y"][a:b])
        gate = one if st["gates"] is None else f(st["gates"][j])
        u, n = unit(Y) if post is not None else (Y, None)
        N = u * post if post is not None else Y
        H = X + a_ * gate * N
        v, m = unit(H)
        outs["H"].append(H)
        outs["Xn"].append(v * pre)
        if case["grad"]:
            gn = f(st["dXn"][a:b])
            D = f(st["dH"][a:b]) + back(v, m, gn * pre)
            dpre += (gn * v).sum(dim=0)
            dgates.append((a_ * D * N).sum(dim=0))
            dN = a_ * gate * D
            outs["dX"].append(D)
            if post is None:
                outs["dY"].append(dN)
            else:
                dpost += (dN * u).sum(dim=0)
                outs["dY"].append(back(u, n, dN * post))
    if not case["grad"]:
        return {k: torch.cat(outs[k]) for k in ("H", "Xn")}
    out = {"dX": torch.cat(outs["dX"]), "dY": torch.cat(outs["dY"]), "dgamma_pre": dpre}
    if post is not None:
        out["dgamma_post"] = dpost
    if st["gates"] is not None:
        out["dgates"] = dgates
    return out


def _exact_act8(X):
    T, d = X.shape
    G = (d + GROUP - 1) // GROUP
    out = torch.empty(T, d, dtype=torch.float64, device="cuda")
    for a in range(0, T, 2048):
        x = torch.nn.functional.pad(X[a:a + 2048].double(), (0, G * GROUP - d)).view(-1, G, GROUP)
        m, k = torch.frexp(x.abs().amax(dim=2) / 127.0)
        # ceil to 8 significant bits (a quotient on the grid is exact: it has no more bits than the largest value)
        s = torch.ldexp(torch.ceil(m * 256.0) / 256.0, k).clamp_min(2.0 ** -100)[:, :, None]
        out[a:a + 2048] = (torch.round(x / s) * s).reshape(-1, G * GROUP)[:, :d]
    return out


def _exact_bwd8(case, st):
    # the activation that the packed form stands for: code times scale, rounded to the tensor's type
    T, d = st["X"].shape
    at, G = -(-T * d // 256) * 256, -(-d // GROUP)
    step = st["packed"][at:at + 2 * T * G].view(torch.bfloat16).view(T, G, 1).double().expand(T, G, GROUP).reshape(T, -1)[:, :d]
    X8 = (st["packed"][:T * d].view(torch.int8).view(T, d).double() * step).to(st["X"].dtype).double()
    X = st["X"].double() if case["reuse_S"] else X8
    dY = st["dY"].double()
    res = {"dA": [], "dB": []}
    parts = []
    Wt = st["W"].double().t().contiguous() if case["want_dX"] else None
    for j, (a, b) in enumerate(zip(st["offsets"][:-1], st["offsets"][1:])):
        A, B, s = st["A"][j].double(), st["B"][j].double(), st["scales"][j]
        g = dY[a:b]
        dS = s * g.matmul(B.t().contiguous())
        res["dA"].append(X8[a:b].t().contiguous().matmul(dS))
        res["dB"].append(s * X[a:b].matmul(A).t().contiguous().matmul(g))
        if Wt is not None:
            parts.append(g.matmul(Wt) + dS.matmul(A.t().contiguous()))
    if Wt is not None:
        res["dX"] = torch.cat(parts)
    return res


def work(case):
    """Inputs read once, outputs written once; the products that the definition asks for."""
    kind, tokens = case["kind"], _ints(case["tokens"])
    T = sum(tokens)
    if kind == "loss":
        d, V = case["d"], case["vocab"]
        live = T * (1.0 - case["ignored"])
        nbytes = 2 * d * V + 2 * live * d + 4 * T + 8 * T + (2 * T * d if case["grad"] else 0) + (4 * T if case["weighted"] else 0)
        # logits; with the gradient the product with the transposed projection too
        return {"bytes": nbytes, "flops": (4 if case["grad"] else 2) * live * d * V}
    elt = 2 if case["dtype"] == "bf16" else 4
    if kind == "norm":
        d = case["d"]
        vectors = 1 + (1 if case["post"] else 0) + (len(tokens) if case["gates"] else 0)
        if case["grad"]:
            return {"bytes": 6 * elt * T * d + (elt + 4) * vectors * d, "flops": 40 * T * d}
        return {"bytes": 4 * elt * T * d + elt * vectors * d, "flops": 14 * T * d}
    if kind == "act8":
        d = case["d"]
        packed = T * d + 2 * T * ((d + GROUP - 1) // GROUP)
        return {"bytes": 2 * (elt * T * d + packed), "flops": 6 * T * d}
    d_in, d_out = _ints(case["dims"].replace("x", ","))
    ranks = _ints(case["ranks"])
    tr, R = sum(t * r for t, r in zip(tokens, ranks)), sum(ranks)
    # dY and the packed X in, dA and dB out; dX out and W in if wanted; S_j kept or made again
    nbytes = 2 * T * d_out + T * d_in + 2 * T * ((d_in + 127) // 128) + (2 + 4) * R * (d_in + d_out)
    flops = 2 * tr * (d_out + d_in + d_out)
    if case["want_dX"]:
        nbytes += 2 * T * d_in + 2 * d_in * d_out
        flops += 2 * T * d_in * d_out + 2 * tr * d_in
    if not case["reuse_S"]:
        flops += 2 * tr * d_in
    return {"bytes": nbytes, "flops": flops}
