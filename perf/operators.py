"""What a training step needs beside a VeLoRA linear layer, as cases to be timed and compared.

A case is one of four kinds of pass.

  keep   an input X that the rank-1 projection is not used on is kept for the backward pass in 8 bits and read back:
         velora_checkpoint_store, velora_checkpoint_load.
  grad   the same, but the backward pass takes the layer's weight gradient from the 8 bits: velora_checkpoint_store in the
         forward pass, velora_checkpoint_weight_grad in the backward pass.
  loss   softmax cross entropy of a linear head, without keeping its logits: velora_head_loss.
  step   the same and its gradients: velora_head_loss, velora_head_loss_backward.

The operators' formulas.

  Checkpoint.  A row of X is cut into blocks of 32 columns (the last one may be shorter).  With a = max |x| over a block, its step is
  the smallest power of two s = 2^e, -126 <= e <= 121, with a <= 127 s (e = 121 where there is none), and
      q = min(127, max(-127, round(x / s)))  (ties to even),      Xhat = q s.
  A block that holds an infinity or a NaN reads back as NaN.    dW[o, d] = sum_n dY[n, o] Xhat[n, d]

  Head.  l[n, v] = sum_d X[n, d] W[v, d],  lse[n] = log sum_v exp l[n, v],  loss[n] = lse[n] - l[n, t[n]];  a token with a target below
  zero has no part in it: its loss, its lse, its row of dX and its share of dW are zero.  With the gradient g[n] of loss[n]:
      G[n, v] = g[n] (exp(l[n, v] - lse[n]) - [v = t[n]]),      dX = G W,      dW = G^T X

Sizes are those of ``velora_inputs`` where a layer's are meant (activations N(0, 1) with a scale per channel, W ~ N(0, 1 / D)); vocabularies are
of the usual sizes, 32000 and odd ones beside it.
"""
import math

import torch

own = False                              # True: the framework's kernels; False: the plain form

DEV = "cuda"
BLOCK = 32
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _keep(name, N, D, dtype="bf16"):
    return dict({"name": name} if name else {}, kind="keep", N=N, D=D, dtype=dtype)


def _grad(name, N, D, O, dtype="bf16"):
    return dict({"name": name} if name else {}, kind="grad", N=N, D=D, O=O, dtype=dtype)


def _head(name, kind, N, D, V, masked=0.0, dtype="bf16"):
    return dict({"name": name} if name else {}, kind=kind, N=N, D=D, V=V, masked=masked, dtype=dtype)


def listed():
    return [
        # A small batch in front of a narrow layer: a few microseconds of work, so calls and launches count.
        _keep("keep_256x512", 256, 512),
        # The input of a LLaMA-7B-shaped block's down projection, the widest activation that a block keeps.
        _keep("keep_8192x11008", 8192, 11008),
        # A ViT-B/16-shaped block's activations (64 images of 197 tokens) in fp32.
        _keep("keep_12608x768_fp32", 64 * 197, 768, "f32"),
        # A width that is no multiple of anything, rows as torch.empty lays them: LLaMA-1B-shaped MLP.
        _keep("keep_4096x5461", 4096, 5461),
        # Key or output projection of a LLaMA-7B-shaped block, whose input the method does not compress.
        _grad("grad_8192x4096_to_4096", 8192, 4096, 4096),
        # Down projection with 5461 inputs, unpadded rows.
        _grad("grad_4096x5461_to_2048", 4096, 5461, 2048),
        # Gate projection of a LLaMA-60M-shaped block: a few output tiles, a long sum over tokens.
        _grad("grad_8192x512_to_1376", 8192, 512, 1376),
        # Scoring the next token of one sequence: the head's weights are read once, nothing else counts.
        _head("loss_1x4096_of_32000", "loss", 1, 4096, 32000),
        # Pre-training step of a LLaMA-60M-shaped model: a narrow head over a large vocabulary.
        _head("step_8192x512_of_32000", "step", 8192, 512, 32000),
        # The head of a LLaMA-7B-shaped model, the largest case.
        _head("step_8192x4096_of_32000", "step", 8192, 4096, 32000),
        # Instruction tuning: prompt tokens have no target, an odd number of tokens, a vocabulary with a token added.
        _head("step_3001x2048_of_32001", "step", 3001, 2048, 32001, masked=0.6),
        # Classifier of a ViT-B/16-shaped model in fp32: 64 images, 1000 classes.
        _head("step_64x768_of_1000_fp32", "step", 64, 768, 1000, dtype="f32"),
    ]


def _log_size(rng, low, high, multiple=1):
    return max(multiple, int(round(math.exp(rng.uniform(math.log(low), math.log(high))) / multiple)) * multiple)


def draw(rng):
    kind = rng.choice(["keep", "grad", "loss", "step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    multiple = rng.choice([8, 8, 8, 64, 1])                   # of the widths: odd ones among them
    while True:
        N = _log_size(rng, 1, 16384)
        if kind in ("keep", "grad"):
            D = _log_size(rng, 64, 11008, multiple)
            if kind == "keep":
                return _keep(None, N, D, dtype)
            O = _log_size(rng, 64, 11008, multiple)
            if N * D * O <= 8192 * 4096 * 4096:
                return _grad(None, N, D, O, dtype)
        else:
            D, V = _log_size(rng, 64, 4096, multiple), _log_size(rng, 100, 65536)
            if N * D * V <= (1 if dtype == "bf16" else 0.125) * 8192 * 4096 * 32000:
                return _head(None, kind, N, D, V, rng.choice([0.0, 0.1, 0.6]), dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    N, D, dt = case["N"], case["D"], _TORCH[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    X = normal(N, D) * torch.exp(0.5 * normal(D))            # log-normal channel scales
    state = {"case": case, "kept": {}}                        # kept: workspaces, as a training program keeps them
    if case["kind"] in ("keep", "grad"):
        state["X"] = X.to(dt)
        if case["kind"] == "grad":
            state["dY"] = normal(N, case["O"]).to(dt)
        return state
    V = case["V"]
    W = normal(V, D) / math.sqrt(D)
    target = torch.randint(V, (N,), generator=g, device=DEV)
    X = normal(N, D) + 6.0 * W[target] * torch.rand((N, 1), generator=g, device=DEV)     # a trained head is often right
    if case["masked"]:
        masked = torch.rand(N, generator=g, device=DEV) < case["masked"]
        masked[-1] = False                                    # a batch has a token to learn from
        target = torch.where(masked, -100, target)
    count = (target >= 0).sum().clamp(min=1)
    state.update(X=X.to(dt), W=W.to(dt), target=target, dloss=(torch.ones(N, device=DEV) / count).contiguous())   # of the mean
    return state


# ---- plain form ----
def _kept(X):
    """Xhat in fp32."""
    N, D = X.shape
    x = torch.nn.functional.pad(X.float(), (0, -D % BLOCK)).view(N, -1, BLOCK)
    a = x.abs().amax(dim=2, keepdim=True)
    m, k = torch.frexp(a)                                     # a = m 2^k, 1/2 <= m < 1; a <= 127 * 2^(k - 7) where m <= 127 / 128
    e = (k - 7 + (m > 127 / 128)).clamp(-126, 121)
    step = ((e + 127) << 23).view(torch.float32)              # exact powers of two
    inverse = ((127 - e) << 23).view(torch.float32)
    y = torch.round(x * inverse).clamp(-127, 127) * step
    y = torch.where(torch.isfinite(a), y, torch.nan)
    return y.view(N, -1)[:, :D]


def _head_plain(state, gradients):
    X, W, target = state["X"].float(), state["W"].float(), state["target"]
    live = target >= 0
    rows, t = torch.arange(X.shape[0], device=X.device), target.clamp(min=0)
    l = X @ W.t()
    m = l.amax(dim=1, keepdim=True)
    lse = m + torch.log(torch.exp(l - m).sum(dim=1, keepdim=True))
    loss = torch.where(live, lse[:, 0] - l[rows, t], 0.0)
    if not gradients:
        return {"loss": loss, "lse": torch.where(live, lse[:, 0], 0.0)}
    g = torch.where(live, state["dloss"], 0.0)
    G = torch.exp(l - lse) * g[:, None]
    G[rows, t] -= g
    return {"loss": loss, "dX": (G @ W).to(state["X"].dtype), "dW": (G.t() @ X).to(state["W"].dtype)}


def _run_plain(state):
    kind, dt = state["case"]["kind"], state["X"].dtype
    if kind == "keep":
        return _kept(state["X"]).to(dt)
    if kind == "grad":
        return (state["dY"].float().t() @ _kept(state["X"])).to(dt)
    return _head_plain(state, kind == "step")


# ---- the framework's operators ----
def _run_own(state):
    import paper_2405_17991_b200 as vl
    case, kept, X = state["case"], state["kept"], state["X"]
    kind, N, D, f32 = case["kind"], case["N"], case["D"], case["dtype"] == "f32"

    def workspace(op, width):
        if op not in kept:
            kept[op] = vl.velora_workspace_alloc(vl.velora_workspace_bytes(op | (vl.OP_F32 if f32 else 0), N, D, width, 1, D % 8 != 0 or width % 8 != 0), DEV)
        return kept[op]

    if kind in ("keep", "grad"):
        Q, E = vl.velora_checkpoint_store(X)
        if kind == "keep":
            return vl.velora_checkpoint_load(Q, E, x_dtype=X.dtype)
        return vl.velora_checkpoint_weight_grad(state["dY"], Q, E, ws=workspace(vl.OP_CHECKPOINT_WEIGHT_GRAD, case["O"]))
    W, target = state["W"], state["target"]
    loss, lse = vl.velora_head_loss(X, W, target, ws=workspace(vl.OP_HEAD_LOSS, case["V"]))
    if kind == "loss":
        return {"loss": loss, "lse": lse}
    dX, dW = vl.velora_head_loss_backward(X, W, target, lse, state["dloss"], ws=workspace(vl.OP_HEAD_LOSS_BACKWARD, case["V"]))
    return {"loss": loss, "dX": dX, "dW": dW}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    N, D, b = case["N"], case["D"], _BYTES[case["dtype"]]
    code = 1 + 1 / BLOCK                                      # a byte and a block's share of its step's exponent
    if case["kind"] == "keep":
        return {"bytes": N * D * 2 * (b + code), "flops": 0}
    if case["kind"] == "grad":
        O = case["O"]
        return {"bytes": N * D * (b + 2 * code) + N * O * b + O * D * b, "flops": 2 * N * D * O}
    V = case["V"]
    live = N * (1 - case["masked"])
    if case["kind"] == "loss":
        return {"bytes": (live * D + V * D) * b + 12 * N, "flops": 2 * live * D * V}
    # The logits are not kept, so they are formed twice: four products.
    return {"bytes": 2 * (N * D + V * D) * b + 16 * N, "flops": 8 * live * D * V}


# ---- the definition in 64 bits ----
def _exact_kept(X):
    N, D = X.shape
    blocks = -(-D // BLOCK)
    x = torch.zeros((N, blocks * BLOCK), dtype=torch.float64, device=X.device)
    x[:, :D] = X.double()
    x = x.reshape(N * blocks, BLOCK)
    a = x.abs().max(dim=1).values
    e = torch.ceil(torch.log2(a / 127.0)).clamp(-126, 121)
    e = torch.where((e < 121) & (127.0 * torch.exp2(e) < a), e + 1, e)                 # where the logarithm's rounding crossed a border
    e = torch.where((e > -126) & (127.0 * torch.exp2(e - 1) >= a), e - 1, e)
    s = torch.exp2(e)[:, None]
    y = torch.round(x / s).clamp(-127, 127) * s
    y[~torch.isfinite(a)] = float("nan")
    return y.reshape(N, blocks * BLOCK)[:, :D].contiguous()


def exact(case, seed):
    state = prepare(case, seed)
    kind, X = case["kind"], state["X"].double()
    if kind == "keep":
        return _exact_kept(state["X"])
    if kind == "grad":
        return torch.einsum("no,nd->od", state["dY"].double(), _exact_kept(state["X"]))
    W, target = state["W"].double(), state["target"]
    with_target = (target >= 0).nonzero()[:, 0]
    x, t = X[with_target], target[with_target]
    logits = torch.einsum("nd,vd->nv", x, W)
    top = logits.max(dim=1).values
    logits -= top[:, None]
    at_target = logits.gather(1, t[:, None])[:, 0]
    total = logits.exp_().sum(dim=1)                          # logits now holds exp(l - top)
    loss = torch.zeros(X.shape[0], dtype=torch.float64, device=X.device)
    loss[with_target] = torch.log(total) - at_target
    if kind == "loss":
        lse = torch.zeros_like(loss)
        lse[with_target] = torch.log(total) + top
        return {"loss": loss, "lse": lse}
    g = state["dloss"].double()[with_target]
    logits *= (g / total)[:, None]
    logits.scatter_add_(1, t[:, None], -g[:, None])
    dX = torch.zeros_like(X)
    dX[with_target] = torch.einsum("nv,vd->nd", logits, W)
    return {"loss": loss, "dX": dX, "dW": torch.einsum("nv,nd->vd", logits, x)}
