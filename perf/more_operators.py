"""More operators around the expert layer, as calls that can be timed and compared: the whole layer for a few tokens, the dense
product that a shared expert beside the routed ones is made of, and the gradients' norm and clipping at the end of a step.

  few         logits = x Wg + gate_bias; the router's choices and weights; y = sum over a token's choices of
              w * gelu(x W1[e]) W2[e]: nothing has a capacity and nothing is dropped (moe_few_forward)
  linear      z = x W + bias; y = act(z) + residual (moe_linear_fwd)
  act_bwd     dz = dy * act'(z) and the bias's gradient (moe_act_bwd)
  linear_bwd  dx = dz W^T; dW = x^T dz (moe_linear_bwd)
  grad_norm   the root of the sum of squares of all elements of many tensors (moe_grad_norm)
  grad_clip   the same, and every element times min(1, most / norm) (moe_grad_clip)

Sizes are those of the workloads in paper_2506_22175_amd/synth.py (512/2048, 1024/4096, 2048/8192; 8, 16 and 64 experts; up
to 32768 tokens), wider gates of 256 experts, and generic odd sizes between them.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}

FEW = dict(kind="few", T=1, M=2048, H=8192, E=16, k=2, scores="softmax", gate_bias=False, bias=False, groups=1, group_k=1,
           renorm=True, scale=1.0, dtype="bf16")
LINEAR = dict(kind="linear", T=1, K=2048, N=8192, act="gelu", bias=True, residual=False, keep=False, dtype="bf16")
GRADS = dict(kind="grad_clip", layer=0, tensors=100, most=100000, mixed=True, clip=0.3)


def listed():
    return [
        # one new token through the large layer: two experts' weights have to come
        dict(FEW, name="few_token"),
        # a decoding batch over many experts with a balancing bias and groups: nearly all weights have to come
        dict(FEW, name="few_batch", T=48, M=1024, H=4096, E=64, k=4, scores="sigmoid", bias=True, groups=8, group_k=4, scale=2.5),
        # odd sizes in float32, a gate that adds its own bias
        dict(FEW, name="few_odd", T=7, M=520, H=1000, E=33, k=3, gate_bias=True, renorm=False, dtype="f32"),
        # one new token through the shared expert's second product, onto the routed experts' sum
        dict(LINEAR, name="linear_token", K=8192, N=2048, act="none", residual=True),
        # a training batch through its first product, what backward needs kept
        dict(LINEAR, name="linear_train", T=8192, keep=True),
        # the training batch's gradient through the activation
        dict(LINEAR, name="act_grad", kind="act_bwd", T=16384),
        # odd rows in float32
        dict(LINEAR, name="act_grad_odd", kind="act_bwd", T=777, N=1000, act="silu", dtype="f32"),
        # the training batch's gradients of rows and weights
        dict(LINEAR, name="linear_grad", kind="linear_bwd", T=8192),
        # many rows of a small layer in odd numbers: the weights' gradient is a long sum over few columns
        dict(LINEAR, name="linear_grad_long", kind="linear_bwd", T=30011, K=520, N=1000),
        # a small layer's gradients on their way to a log line: latency is all there is
        dict(GRADS, name="norm_small", kind="grad_norm", tensors=12, most=20000),
        # a model's worth of small tensors of both types in odd numbers
        dict(GRADS, name="clip_many", tensors=300, most=300000),
        # a block's own gradients: gain, gate and both weights of 16 experts of 1024/4096
        dict(GRADS, name="clip_block", layer=16, tensors=0, mixed=False),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["few", "few", "few", "linear", "linear", "act_bwd", "linear_bwd", "grad_norm", "grad_clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "few":
        E = rng.choice([1, 4, 8, 16, 16, 33, 64, 64, 100, 256])
        groups = rng.choice([g for g in (1, 1, 4, 8) if E % g == 0])
        group_k = rng.choice([1, 2, groups // 2, groups]) if groups > 1 else 1
        k = rng.choice([q for q in (1, 2, 2, 3, 4, 6, 8) if q <= min(E, E // groups * group_k)])
        while True:
            M, H = 8 * _logu(rng, 8, 512), 8 * _logu(rng, 8, 1024)
            if E * M * H <= (64 if dtype == "bf16" else 32) * 1024 * 4096:
                break
        return dict(FEW, T=_logu(rng, 1, 128), M=M, H=H, E=E, k=k, scores=rng.choice(["softmax", "sigmoid"]),
                    gate_bias=rng.random() < 0.3, bias=rng.random() < 0.4, groups=groups, group_k=group_k,
                    renorm=rng.random() < 0.5, scale=rng.choice([1.0, 1.0, 2.5]), dtype=dtype)
    if kind in ("linear", "act_bwd", "linear_bwd"):
        while True:
            T, K, N = _logu(rng, 1, 32768), 8 * _logu(rng, 8, 1024), 8 * _logu(rng, 8, 1024)
            if rng.random() < 0.3:
                T = min(T, 64)
            if T * K * N <= (8192 if dtype == "bf16" else 1024) * 2048 * 8192 and T * max(K, N) <= 16384 * 8192:
                break
        return dict(LINEAR, kind=kind, T=T, K=K, N=N, act=rng.choice(["none", "gelu", "gelu", "silu"]), bias=rng.random() < 0.7,
                    residual=rng.random() < 0.5, keep=rng.random() < 0.5, dtype=dtype)
    tensors = _logu(rng, 1, 400)
    return dict(GRADS, kind=kind, tensors=tensors, most=_logu(rng, 100, min(60000000, 400000000 // tensors)),
                mixed=rng.random() < 0.6, clip=rng.choice([0.01, 0.3, 2.0]))


# ---- inputs -----------------------------------------------------------------------------------

def _config(c):
    """The configuration that a program keeps beside its weights."""
    if not own or c["kind"].startswith("grad"):
        return None
    from paper_2506_22175_amd import binding as B
    code = {"f32": B.MOE_F32, "bf16": B.MOE_BF16}[c["dtype"]]
    if c["kind"] == "few":
        return B.make_few_config(c["T"], c["M"], c["H"], c["E"], c["k"], code,
                                 B.MOE_SIGMOID if c["scores"] == "sigmoid" else B.MOE_SOFTMAX, c["groups"], c["group_k"], 2,
                                 int(c["renorm"]), c["scale"])
    act = {"none": B.MOE_ACT_NONE, "gelu": B.MOE_ACT_GELU, "silu": B.MOE_ACT_SILU}[c["act"]]
    return B.make_linear_config(c["T"], c["K"], c["N"], code, act, grad_overwrite=1)


def _tensor_sizes(c):
    """Elements and types of a list of gradients: those of one block's layer, or many of sizes spread over their logarithm."""
    if c["layer"]:
        E, M, H = c["layer"], 1024, 4096
        return [(M, "f32"), (M * E, "f32"), (E * M * H, "f32"), (E * H * M, "f32")]
    sizes = []
    for j in range(c["tensors"]):
        u = (j * 0.6180339887498949 + 0.37) % 1.0
        n = int(math.exp(u * math.log(c["most"]))) | 1
        sizes.append((0 if j % 37 == 20 else n, "bf16" if c["mixed"] and j % 3 == 1 else "f32"))
    return sizes


def _places(c):
    """Where each tensor lies in its type's buffer, and the buffers' sizes: at multiples of 64 elements, every fifth one
    behind one element more."""
    at, end = [], {"f32": 0, "bf16": 0}
    for j, (n, d) in enumerate(_tensor_sizes(c)):
        at.append(end[d] + (1 if j % 5 == 4 else 0))
        end[d] = -(-(at[-1] + n) // 64) * 64
    return at, {d: n for d, n in end.items() if n}


def _views(c, buffers):
    return [buffers[d][at:at + n] for at, (n, d) in zip(_places(c)[0], _tensor_sizes(c))]


def _inputs(c, seed):
    """Everything random, from the seed alone, on the GPU."""
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    randn = lambda *dims: torch.randn(dims, generator=g, device=DEVICE, dtype=torch.float32)  # noqa: E731
    i = {}
    if c["kind"].startswith("grad"):
        i["grads"] = {d: torch.zeros(n, device=DEVICE, dtype=DT[d]) for d, n in _places(c)[1].items()}
        for v in _views(c, i["grads"]):                      # each tensor's gradients have a size of their own
            v.copy_(randn(v.numel()) * torch.exp(randn(1)) * 0.01)
        i["most"] = c["clip"] * math.sqrt(sum(float(v.double().square().sum()) for v in i["grads"].values()))
        return i
    dt = DT[c["dtype"]]
    if c["kind"] == "few":
        T, M, H, E = c["T"], c["M"], c["H"], c["E"]
        i["x"] = randn(T, M).to(dt)
        i["Wg"] = (randn(M, E) * (1.5 / math.sqrt(M))).to(dt)
        i["gate_bias"] = 0.5 * randn(E) if c["gate_bias"] else None
        i["bias"] = 0.1 * randn(E) if c["bias"] else None
        i["W1"], i["W2"] = torch.empty((E, M, H), device=DEVICE, dtype=dt), torch.empty((E, H, M), device=DEVICE, dtype=dt)
        for e in range(E):
            i["W1"][e] = randn(M, H) * (1.0 / math.sqrt(M))
            i["W2"][e] = randn(H, M) * (1.0 / math.sqrt(H))
        return i
    T, K, N = c["T"], c["K"], c["N"]
    if c["kind"] == "act_bwd":
        i["dy"], i["z"] = randn(T, N).to(dt), (1.5 * randn(T, N)).to(dt)
        return i
    i["x"], i["W"] = randn(T, K).to(dt), (randn(K, N) * (1.0 / math.sqrt(K))).to(dt)
    if c["kind"] == "linear":
        i["bias"] = 0.5 * randn(N) if c["bias"] else None
        i["residual"] = randn(T, N).to(dt) if c["residual"] else None
    else:
        i["dz"] = randn(T, N).to(dt)
    return i


def prepare(case, seed):
    c = case
    i = _inputs(c, seed)
    empty = lambda *dims, dtype: torch.empty(dims, device=DEVICE, dtype=dtype)  # noqa: E731
    cfg = _config(c)
    s = {"case": c, "cfg": cfg, "in": i, "scratch": None}
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    if c["kind"].startswith("grad"):
        o = {"norm": empty(1, dtype=f32)}
        if c["kind"] == "grad_clip":
            o["grads"] = {d: torch.zeros_like(v) for d, v in i["grads"].items()}
        if own:
            from paper_2506_22175_amd import binding as B
            s["cfg"] = B.make_grad_list(_views(c, i["grads"]), _views(c, o["grads"]) if "grads" in o else None)
            s["scratch"] = empty(max(1, B.moe_grad_scratch_bytes(s["cfg"])), dtype=u8)
        s["out"] = o
        return s
    dt = DT[c["dtype"]]
    if c["kind"] == "few":
        T, M, E, k = c["T"], c["M"], c["E"], c["k"]
        o = {"y": empty(T, M, dtype=dt), "logits": empty(T, E, dtype=f32), "topk_idx": empty(T, k, dtype=i32),
             "topk_w": empty(T, k, dtype=f32)}
    elif c["kind"] == "linear":
        o = {"y": empty(c["T"], c["N"], dtype=dt)}
        if c["keep"]:
            o["z"] = empty(c["T"], c["N"], dtype=dt)
    elif c["kind"] == "act_bwd":
        o = {"dz": empty(c["T"], c["N"], dtype=dt), "dbias": empty(c["N"], dtype=f32)}
    else:
        o = {"dx": empty(c["T"], c["K"], dtype=dt), "dW": empty(c["K"], c["N"], dtype=f32)}
    if own:
        from paper_2506_22175_amd import binding as B
        need = B.moe_few_scratch_bytes(cfg) if c["kind"] == "few" else B.moe_linear_scratch_bytes(cfg)
        s["scratch"] = empty(max(1, need), dtype=u8)
    s["out"] = o
    return s


# ---- the calls --------------------------------------------------------------------------------

def run(state):
    c, i, o = state["case"], state["in"], state["out"]
    if own:
        return _own(state["cfg"], c, i, o, state["scratch"])
    return {"few": _plain_few, "linear": _plain_linear, "act_bwd": _plain_act_bwd, "linear_bwd": _plain_linear_bwd,
            "grad_norm": _plain_grads, "grad_clip": _plain_grads}[c["kind"]](c, i)


def _own(cfg, c, i, o, scratch):
    from paper_2506_22175_amd import binding as B
    if c["kind"] == "few":
        B.moe_few_forward(cfg, i["x"], i["Wg"], i["gate_bias"], i["bias"], i["W1"], i["W2"], o["y"], o["logits"], o["topk_idx"],
                          o["topk_w"], scratch)
    elif c["kind"] == "linear":
        B.moe_linear_fwd(cfg, i["x"], i["W"], i["bias"], i["residual"], o.get("z"), o["y"], scratch)
    elif c["kind"] == "act_bwd":
        B.moe_act_bwd(cfg, i["dy"], i["z"], o["dz"], o["dbias"], scratch)
    elif c["kind"] == "linear_bwd":
        B.moe_linear_bwd(cfg, i["dz"], i["x"], i["W"], o["dx"], o["dW"], scratch)
    elif c["kind"] == "grad_norm":
        B.moe_grad_norm(cfg, o["norm"], scratch)
    else:
        B.moe_grad_clip(cfg, i["most"], o["norm"], scratch)
    return o


def _route(c, logits, bias):
    """Choices and weights of float logits; scores in 64 bits: which of two experts comes first is decided by their last bits."""
    T, E = logits.shape
    l = logits.double()
    if c["scores"] == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-l))
    else:
        s = torch.exp(l - l.amax(1, keepdim=True))
        s = s / s.sum(1, keepdim=True)
    v = s if bias is None else s + bias.double()
    rank = v if bias is not None else l
    if c["groups"] > 1:
        score = torch.sort(v.reshape(T, c["groups"], -1), dim=2, descending=True)[0][..., :2].sum(2)
        best = torch.sort(score, dim=1, descending=True, stable=True)[1][:, :c["group_k"]]
        stays = torch.zeros_like(score, dtype=torch.bool).scatter(1, best, True)
        rank = torch.where(stays[..., None].expand(T, c["groups"], E // c["groups"]).reshape(T, E), rank, -math.inf)
    idx = torch.sort(rank, dim=1, descending=True, stable=True)[1][:, :c["k"]]
    w = s.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return idx, w * c["scale"]


def _logits(i):
    """In 64 bits, rounded to float: what is chosen hangs on their last bits."""
    l = i["x"].double() @ i["Wg"].double()
    return (l if i["gate_bias"] is None else l + i["gate_bias"].double()).float()


def _gelu(z):
    return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))


def _plain_few(c, i):
    T, M, E, k = c["T"], c["M"], c["E"], c["k"]
    logits = _logits(i)
    idx, w = _route(c, logits, i["bias"])
    w = w.float()
    x = i["x"].float()
    if T * k <= E:                                        # the chosen experts' weights alone
        at = idx.reshape(-1)
        a = _gelu(torch.bmm(x.repeat_interleave(k, 0)[:, None], i["W1"][at].float()))
        y = torch.bmm(a, i["W2"][at].float()).reshape(T, k, M)
        y = (w[..., None] * y).sum(1)
    else:                                                 # every token through every expert
        share = torch.zeros((T, E), device=x.device).scatter(1, idx, w)
        y = torch.zeros((T, M), device=x.device)
        for e in range(E):
            y += share[:, e, None] * (_gelu(x @ i["W1"][e].float()) @ i["W2"][e].float())
    return {"y": y.to(DT[c["dtype"]]), "logits": logits, "topk_idx": idx.to(torch.int32), "topk_w": w}


def _act(c, z):
    return z if c["act"] == "none" else _gelu(z) if c["act"] == "gelu" else z / (1.0 + torch.exp(-z))


def _plain_linear(c, i):
    z = i["x"].float() @ i["W"].float()
    if i["bias"] is not None:
        z = z + i["bias"]
    y = _act(c, z)
    if i["residual"] is not None:
        y = y + i["residual"].float()
    out = {"y": y.to(DT[c["dtype"]])}
    if c["keep"]:
        out["z"] = z.to(DT[c["dtype"]])
    return out


def _plain_act_bwd(c, i):
    dz, z = i["dy"].float(), i["z"].float()
    if c["act"] == "gelu":
        dz = dz * (0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
    elif c["act"] == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        dz = dz * (s * (1.0 + z * (1.0 - s)))
    return {"dz": dz.to(DT[c["dtype"]]), "dbias": dz.sum(0)}


def _plain_linear_bwd(c, i):
    dz = i["dz"].float()
    return {"dx": (dz @ i["W"].float().t()).to(DT[c["dtype"]]), "dW": i["x"].float().t() @ dz}


def _plain_grads(c, i):
    norm = sum(g.double().square().sum() for g in i["grads"].values()).sqrt().float()       # a long sum
    out = {"norm": norm.reshape(1)}
    if c["kind"] == "grad_clip":
        most = float(torch.tensor(i["most"], dtype=torch.float32))
        factor = (most / norm.double()).clamp(max=1.0)
        out["grads"] = {d: (g.double() * factor).to(g.dtype) if d == "f32" else (g.float() * factor.float()).to(g.dtype)
                        for d, g in i["grads"].items()}
    return out


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    """Every input read once and every output written once; of the experts' weights those that are expected to be chosen (each
    token has k different ones out of E).  Clipping reads its input twice: the factor is not known before the first reading ends."""
    c = case
    if c["kind"].startswith("grad"):
        sizes = _tensor_sizes(c)
        n = sum(s * (4 if d == "f32" else 2) for s, d in sizes)
        return {"bytes": (n if c["kind"] == "grad_norm" else 3 * n) + 4, "flops": 2.0 * sum(s for s, _ in sizes)}
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "few":
        T, M, H, E, k = c["T"], c["M"], c["H"], c["E"], c["k"]
        experts = E * (1.0 - (1.0 - k / E) ** T)
        return {"bytes": (experts * 2 * M * H + M * E + 2 * T * M) * es + T * E * 4 + T * k * 8,
                "flops": 4.0 * T * k * M * H + 2.0 * T * M * E}
    T, K, N = c["T"], c["K"], c["N"]
    if c["kind"] == "linear":
        outs = 1 + int(c["keep"]) + int(c["residual"])
        return {"bytes": (T * K + K * N + outs * T * N) * es + (4 * N if c["bias"] else 0), "flops": 2.0 * T * K * N}
    if c["kind"] == "act_bwd":
        return {"bytes": 3 * T * N * es + 4 * N, "flops": 12.0 * T * N}
    return {"bytes": (2 * T * K + T * N + K * N) * es + 4 * K * N, "flops": 4.0 * T * K * N}


# ---- the same in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    c = case
    i = _inputs(c, seed)
    f64 = torch.float64
    if c["kind"].startswith("grad"):
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.to(f64)) for g in i["grads"].values()]))
        out = {"norm": norm.reshape(1)}
        if c["kind"] == "grad_clip":
            ratio = torch.tensor(i["most"], dtype=torch.float32).to(f64).to(DEVICE) / norm
            out["grads"] = {d: torch.where(ratio < 1.0, g.to(f64) * ratio, g.to(f64)) for d, g in i["grads"].items()}
        return out
    if c["kind"] == "few":
        T, M, E = c["T"], c["M"], c["E"]
        x = i["x"].to(f64)
        logits = (x[:, :, None] * i["Wg"].to(f64)[None]).sum(1) if T * M * E <= 1 << 26 else x @ i["Wg"].to(f64)
        if c["gate_bias"]:
            logits = logits + i["gate_bias"].to(f64)
        idx = _route(c, _logits(i), i["bias"])[0]          # the choices themselves are whole numbers
        chosen = logits.gather(1, idx)
        if c["scores"] == "sigmoid":
            log_s = torch.nn.functional.logsigmoid(chosen)
        else:
            log_s = chosen - torch.logsumexp(logits, 1, keepdim=True)
        if c["renorm"]:
            log_s = log_s - torch.logsumexp(log_s, 1, keepdim=True)
        w = torch.exp(log_s) * c["scale"]
        y = torch.zeros((T, M), dtype=f64, device=DEVICE)
        for e in range(E):
            t, j = torch.nonzero(idx == e, as_tuple=True)
            if t.numel():
                z = x[t] @ i["W1"][e].to(f64)
                y.index_add_(0, t, (z * torch.special.ndtr(z)) @ i["W2"][e].to(f64) * w[t, j, None])
        return {"y": y, "logits": logits, "topk_idx": None, "topk_w": w}
    act = {"none": lambda z: z, "gelu": lambda z: z * torch.special.ndtr(z), "silu": lambda z: z * torch.sigmoid(z)}[c["act"]]
    if c["kind"] == "linear":
        z = i["x"].to(f64) @ i["W"].to(f64)
        z = z + i["bias"].to(f64) if c["bias"] else z
        y = act(z)
        y = y + i["residual"].to(f64) if c["residual"] else y
        return {"y": y, "z": z} if c["keep"] else {"y": y}
    if c["kind"] == "act_bwd":
        # by differentiation of the sum of dy * act(z), some rows at a time
        dz = torch.empty((c["T"], c["N"]), dtype=f64, device=DEVICE)
        with torch.enable_grad():
            for at in range(0, c["T"], 2048):
                z = i["z"][at:at + 2048].to(f64).requires_grad_()
                (dz[at:at + 2048],) = torch.autograd.grad((act(z) * i["dy"][at:at + 2048].to(f64)).sum(), z)
        return {"dz": dz, "dbias": torch.ones(c["T"], dtype=f64, device=DEVICE) @ dz}
    dz = i["dz"].to(f64)
    return {"dx": torch.mm(i["W"].to(f64), dz.t()).t().contiguous(), "dW": torch.mm(dz.t().contiguous(), i["x"].to(f64)).t().contiguous()}
