"""Layer norm, and distillation into a linear head from a teacher's top logits, as cases to be timed and compared.

A case is one of four kinds of pass.

  norm          layer norm of the rows of X, or of a residual stream X + R that is handed on as well: velora_layer_norm.
  norm_step     the same and its gradients: velora_layer_norm, velora_layer_norm_backward.
  distill       a student's loss against what a teacher holds likely, without keeping the student's logits: velora_head_distill.
  distill_step  the same and its gradients: velora_head_distill, velora_head_distill_backward.

The operators' formulas.

  Layer norm.  H = X + R, rounded to the type of X (H = X without R);  over a row of H
      m = mean h,  r = 1 / sqrt(mean (h - m)^2 + eps),  xhat = (h - m) r,  Y = xhat w + b
  and, with the gradients dY of Y and dH of H (from the layers that H is handed on to; none without R)
      c = dY w,  dX = dH + r (c - mean c - xhat mean(c xhat)),  dw[d] = sum_n dY xhat,  db[d] = sum_n dY

  Distillation.  l[n, v] = sum_d X[n, d] W[v, d] / T,  lse[n] = log sum_v exp l[n, v].  The teacher gives K columns i[n, k] (below zero: no
  entry) and its logits there, t[n, k]; with s[n] = log sum_k exp(t[n, k] / T), or, where it is given, the log sum over the teacher's whole vocabulary,
      p[n, k] = exp(t[n, k] / T - s[n]),   loss[n] = sum_k p[n, k] (log p[n, k] - l[n, i[n, k]] + lse[n])
      G[n, v] = dloss[n] / T (exp(l[n, v] - lse[n]) sum_k p[n, k] - sum_{k: i[n, k] = v} p[n, k]),   dX = G W,   dW = G^T X
  A token without any entry (a prompt, padding) has no part in it: its loss, its row of dX and its share of dW are zero.

Sizes are those of ``velora_inputs`` where a layer's are meant; vocabularies and numbers of entries are of the usual sizes, odd ones beside them.
"""
import math

import torch

own = False                              # True: the framework's kernels; False: the plain form

DEV = "cuda"
EPS = 1e-5
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _norm(name, kind, N, D, residual=False, dtype="bf16", params="f32"):
    return dict({"name": name} if name else {}, kind=kind, N=N, D=D, residual=residual, dtype=dtype, params=params)


def _distill(name, kind, N, D, V, K, T=1.0, masked=0.0, whole=False, dtype="bf16"):
    """whole: the teacher's log sum over its whole vocabulary is given."""
    return dict({"name": name} if name else {}, kind=kind, N=N, D=D, V=V, K=K, T=T, masked=masked, whole=whole, dtype=dtype)


def listed():
    return [
        # One token of a LLaMA-7B-shaped model while it answers: a call's latency.
        _norm("norm_1x4096", "norm", 1, 4096, params="bf16"),
        # Evaluation of a LLaMA-60M-shaped model on a short batch, the residual stream added on the way.
        _norm("norm_256x512_residual", "norm", 256, 512, residual=True),
        # Training step of a ViT-B/16-shaped block in fp32: 64 images of 197 tokens.
        _norm("norm_step_12608x768_fp32", "norm_step", 64 * 197, 768, dtype="f32"),
        # Pre-norm of a LLaMA-7B-shaped block in training: residual in, residual's gradient back.
        _norm("norm_step_8192x4096_residual", "norm_step", 8192, 4096, residual=True),
        # A norm inside the MLP of a LLaMA-1B-shaped block: rows without padding that start on any boundary.
        _norm("norm_step_4096x5461", "norm_step", 4096, 5461),
        # The same for a LLaMA-7B-shaped block, the widest rows.
        _norm("norm_step_8192x11008", "norm_step", 8192, 11008, params="bf16"),
        # Scoring one token against a teacher: the head's weights are read once, nothing else counts.
        _distill("distill_1x4096_of_32000", "distill", 1, 4096, 32000, 64),
        # A LLaMA-60M-shaped student in training: a narrow head over a large vocabulary, the teacher softened.
        _distill("distill_step_8192x512_of_32000", "distill_step", 8192, 512, 32000, 64, T=2.0),
        # A LLaMA-7B-shaped student, the largest case.
        _distill("distill_step_8192x4096_of_32000", "distill_step", 8192, 4096, 32000, 32),
        # Instruction tuning: prompt tokens have no entries, an odd number of tokens, the teacher's mass outside its top logits counted.
        _distill("distill_step_3001x2048_of_32001", "distill_step", 3001, 2048, 32001, 100, T=1.5, masked=0.6, whole=True),
        # A classifier of 1000 classes in fp32, 64 images, taught the ten likeliest.
        _distill("distill_step_64x768_of_1000_fp32", "distill_step", 64, 768, 1000, 10, T=4.0, dtype="f32"),
    ]


def _log_size(rng, low, high, multiple=1):
    return max(multiple, int(round(math.exp(rng.uniform(math.log(low), math.log(high))) / multiple)) * multiple)


def draw(rng):
    kind = rng.choice(["norm", "norm_step", "distill", "distill_step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    multiple = rng.choice([8, 8, 8, 64, 1])                   # of the widths: odd ones among them
    while True:
        N = _log_size(rng, 1, 16384)
        if kind in ("norm", "norm_step"):
            D = _log_size(rng, 64, 12288, multiple)
            if N * D * _BYTES[dtype] <= 8192 * 11008 * 2:
                return _norm(None, kind, N, D, rng.choice([False, True]), dtype, rng.choice(["f32", dtype]))
        else:
            D, V = _log_size(rng, 64, 4096, multiple), _log_size(rng, 100, 65536)
            K = min(_log_size(rng, 1, 256), V // 4)
            if N * D * V <= (1 if dtype == "bf16" else 0.125) * 8192 * 4096 * 32000:
                return _distill(None, kind, N, D, V, K, rng.choice([1.0, 1.0, 2.0, 1.5]), rng.choice([0.0, 0.1, 0.6]), rng.choice([False, True]), dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 6271 + 29)
    N, D, dt = case["N"], case["D"], _TORCH[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    state = {"case": case, "kept": {}}                        # kept: workspaces, as a training program keeps them
    if case["kind"] in ("norm", "norm_step"):
        pt = _TORCH[case["params"]]
        spread = torch.exp(0.5 * normal(D))                   # log-normal channel scales, as a residual stream has them
        state["X"] = (normal(N, D) * spread + 0.3 * normal(N, 1)).to(dt)
        state["R"] = (0.5 * normal(N, D) * spread).to(dt) if case["residual"] else None
        state["w"], state["b"] = (1.0 + 0.2 * normal(D)).to(pt), (0.1 * normal(D)).to(pt)
        if case["kind"] == "norm_step":
            state["dY"] = normal(N, D).to(dt)
            state["dH"] = normal(N, D).to(dt) if case["residual"] else None
        return state
    V, K, T = case["V"], case["K"], case["T"]
    W = normal(V, D) / math.sqrt(D)
    # K columns a token, all different: random steps from a random start, in an order of no meaning.
    steps = torch.randint(1, V // K + 1, (N, K), generator=g, device=DEV)
    steps[:, 0] = torch.randint(V, (N,), generator=g, device=DEV)
    index = (steps.cumsum(1) % V)[:, torch.randperm(K, generator=g, device=DEV)]
    # Logits from the likeliest down, and a student that has learned some of it.
    t = 14.0 + 2.0 * normal(N, 1) - torch.cumsum(-torch.log(uniform(N, K).clamp(min=1e-6)) * 1.5 / torch.arange(1, K + 1, device=DEV), 1)
    X = normal(N, D)
    for k in range(min(3, K)):
        X += 5.0 / (k + 1) * uniform(N, 1) * W[index[:, k]]
    last = (uniform(N, 1) * K).long() if K > 1 else torch.zeros((N, 1), dtype=torch.int64, device=DEV)
    short = (uniform(N, 1) < 0.2) & (torch.arange(K, device=DEV) > last)               # lists cut short where little is left
    index = torch.where(short, -1, index)
    if case["masked"]:
        masked = uniform(N) < case["masked"]
        masked[-1] = False                                    # a batch has a token to learn from
        index = torch.where(masked[:, None], -1, index)
    count = (index >= 0).any(1).sum().clamp(min=1)
    state.update(X=X.to(dt), W=W.to(dt), index=index.contiguous(), teacher=t.to(dt).contiguous(), teacher_lse=None,
                 dloss=(T * T * torch.ones(N, device=DEV) / count).contiguous())        # of the mean, with the usual T^2
    if case["whole"]:
        mass = torch.where(index >= 0, state["teacher"].float() / T, -math.inf)
        state["teacher_lse"] = torch.where((index >= 0).any(1), torch.logsumexp(mass, 1) + 0.3 * uniform(N), 0.0).contiguous()
    return state


# ---- plain form ----
def _norm_plain(state):
    X, R = state["X"], state["R"]
    dt, (N, D) = X.dtype, X.shape
    H = (X.float() + R.float()).to(dt) if R is not None else X
    h, w, b = H.float(), state["w"].float(), state["b"].float()
    m = h.sum(dim=1, keepdim=True) / D
    r = 1.0 / torch.sqrt(((h - m) * (h - m)).sum(dim=1, keepdim=True) / D + EPS)
    xhat = (h - m) * r
    out = {"Y": (xhat * w + b).to(dt)}
    if R is not None:
        out["H"] = H
    if state["case"]["kind"] == "norm":
        return out
    dy = state["dY"].float()
    c = dy * w
    dx = r * (c - c.sum(dim=1, keepdim=True) / D - xhat * ((c * xhat).sum(dim=1, keepdim=True) / D))
    if R is not None:
        dx = dx + state["dH"].float()
    out.update(dX=dx.to(dt), dweight=(dy * xhat).sum(dim=0).to(state["w"].dtype), dbias=dy.sum(dim=0).to(state["b"].dtype))
    return out


def _distill_plain(state):
    X, W, index, T = state["X"].float(), state["W"].float(), state["index"], state["case"]["T"]
    some = index >= 0
    live = some.any(dim=1)
    columns = index.clamp(min=0)
    l = (X @ W.t()) / T
    m = l.amax(dim=1, keepdim=True)
    lse = m + torch.log(torch.exp(l - m).sum(dim=1, keepdim=True))
    u = torch.where(some, state["teacher"].float() / T, -math.inf)
    if state["teacher_lse"] is None:
        top = torch.where(live[:, None], u.amax(dim=1, keepdim=True), 0.0)
        logp = u - top - torch.log(torch.exp(u - top).sum(dim=1, keepdim=True))
    else:
        logp = u - state["teacher_lse"][:, None]
    logp = torch.where(some, logp, 0.0)
    p = torch.where(some, torch.exp(logp), 0.0)
    loss = (p * (logp - (l.gather(1, columns) - lse))).sum(dim=1)
    if state["case"]["kind"] == "distill":
        return {"loss": loss, "lse": torch.where(live, lse[:, 0], 0.0)}
    g = (torch.where(live, state["dloss"], 0.0) / T)[:, None]
    G = torch.exp(l - lse) * (g * p.sum(dim=1, keepdim=True))
    G.scatter_add_(1, columns, -g * p)
    return {"loss": loss, "dX": (G @ W).to(state["X"].dtype), "dW": (G.t() @ X).to(state["W"].dtype)}


# ---- the framework's operators ----
def _run_own(state):
    import paper_2405_17991_b200 as vl
    case, kept, X = state["case"], state["kept"], state["X"]
    N, D = case["N"], case["D"]

    def workspace(op, columns=1, entries=1, any_rows=False):
        if op not in kept:
            op_and_type = op | (vl.OP_F32 if case["dtype"] == "f32" else 0)
            kept[op] = vl.velora_workspace_alloc(vl.velora_workspace_bytes(op_and_type, N, D, columns, entries, any_rows), DEV)
        return kept[op]

    if case["kind"] in ("norm", "norm_step"):
        Y, H, mean, rstd = vl.velora_layer_norm(X, state["w"], state["b"], eps=EPS, residual=state["R"])
        out = {"Y": Y} if state["R"] is None else {"Y": Y, "H": H}
        if case["kind"] == "norm_step":
            dX, dw, db = vl.velora_layer_norm_backward(state["dY"], H, mean, rstd, state["w"], dH=state["dH"], ws=workspace(vl.OP_LAYER_NORM_BACKWARD))
            out.update(dX=dX, dweight=dw, dbias=db)
        return out
    W, teacher, V, K = state["W"], (state["index"], state["teacher"]), case["V"], case["K"]
    more = {"temperature": case["T"], "teacher_lse": state["teacher_lse"]}
    loss, lse = vl.velora_head_distill(X, W, *teacher, ws=workspace(vl.OP_HEAD_DISTILL, V, K, D % 8 != 0), **more)
    if case["kind"] == "distill":
        return {"loss": loss, "lse": lse}
    dX, dW = vl.velora_head_distill_backward(X, W, *teacher, lse, state["dloss"], ws=workspace(vl.OP_HEAD_DISTILL_BACKWARD, V, K, D % 8 != 0), **more)
    return {"loss": loss, "dX": dX, "dW": dW}


def run(state):
    if own:
        return _run_own(state)
    return _norm_plain(state) if state["case"]["kind"] in ("norm", "norm_step") else _distill_plain(state)


def work(case):
    N, D, b = case["N"], case["D"], _BYTES[case["dtype"]]
    if case["kind"] in ("norm", "norm_step"):
        streams = 4 if case["residual"] else 2                # X, R, H, Y
        if case["kind"] == "norm_step":
            streams += 4 if case["residual"] else 3           # dY, H, dH, dX
        vectors = 2 if case["kind"] == "norm" else 5          # w, b; w, dw, db
        return {"bytes": N * D * b * streams + D * _BYTES[case["params"]] * vectors, "flops": 0}
    V, K = case["V"], case["K"]
    live = N * (1 - case["masked"])
    lists = live * K * (8 + b)
    if case["kind"] == "distill":
        return {"bytes": (live * D + V * D) * b + lists + 8 * N, "flops": 2 * live * D * V}
    # The logits are not kept, so they are formed twice: four products.
    return {"bytes": 2 * (N * D + V * D) * b + 2 * lists + 12 * N, "flops": 8 * live * D * V}


# ---- the definition in 64 bits ----
def _exact_norm(state):
    X, R, D = state["X"], state["R"], state["case"]["D"]
    h = X.double()
    if R is not None:
        h = (h + R.double()).to(X.dtype).double()
    centred = h - h.mean(dim=1, keepdim=True)
    xhat = centred / torch.sqrt(torch.einsum("nd,nd->n", centred, centred)[:, None] / D + EPS)
    r = 1.0 / torch.sqrt(torch.einsum("nd,nd->n", centred, centred)[:, None] / D + EPS)
    w = state["w"].double()
    out = {"Y": xhat * w + state["b"].double()}
    if R is not None:
        out["H"] = h
    if state["case"]["kind"] == "norm":
        return out
    dy = state["dY"].double()
    # The norm's derivative as a projection: what lies along the row of ones and along xhat goes, the scale is left.
    c = dy * w
    c = c - c.mean(dim=1, keepdim=True)
    dx = r * (c - xhat * (torch.einsum("nd,nd->n", c, xhat) / D)[:, None])
    if R is not None:
        dx = dx + state["dH"].double()
    out.update(dX=dx, dweight=torch.einsum("nd,nd->d", dy, xhat), dbias=torch.einsum("nd->d", dy))
    return out


def _exact_distill(state):
    T, index = state["case"]["T"], state["index"]
    rows = (index >= 0).any(dim=1).nonzero()[:, 0]
    x, W, i = state["X"].double()[rows], state["W"].double(), index[rows]
    none = i < 0
    u = (state["teacher"].double()[rows] / T).masked_fill(none, float("-inf"))
    s = torch.logsumexp(u, dim=1) if state["teacher_lse"] is None else state["teacher_lse"].double()[rows]
    p = torch.exp(u - s[:, None])
    q = torch.einsum("nd,vd->nv", x, W) / T
    top = q.max(dim=1).values
    q -= top[:, None]
    at = q.gather(1, i.masked_fill(none, 0))
    total = q.exp_().sum(dim=1)                               # q now holds exp(l - top)
    terms = p * ((u - s[:, None]).masked_fill(none, 0.0) - at + torch.log(total)[:, None])
    loss = torch.zeros(index.shape[0], dtype=torch.float64, device=index.device)
    loss[rows] = terms.sum(dim=1)
    if state["case"]["kind"] == "distill":
        lse = torch.zeros_like(loss)
        lse[rows] = torch.log(total) + top
        return {"loss": loss, "lse": lse}
    g = state["dloss"].double()[rows] / T
    q *= (g * p.sum(dim=1) / total)[:, None]
    q.scatter_add_(1, i.masked_fill(none, 0), -g[:, None] * p)
    dX = torch.zeros((index.shape[0], W.shape[1]), dtype=torch.float64, device=index.device)
    dX[rows] = torch.einsum("nv,vd->nd", q, W)
    return {"loss": loss, "dX": dX, "dW": torch.einsum("nv,nd->vd", q, x)}


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_norm(state) if case["kind"] in ("norm", "norm_step") else _exact_distill(state)
