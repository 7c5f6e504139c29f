"""The operators around the expert layer, as calls that can be timed and compared: the norm in front of the gate, the router
behind it, and the experts' products on 4-bit weights that serve a trained layer.

  norm      h = x + residual; y = h / sqrt(mean(h^2) + eps) * gain, stored as it came or in 8 bits (e4m3) with a float scale
            for each 128 columns or for the row (moe_norm_fwd)
  norm_bwd  the gradients of both inputs and of the gain (moe_norm_bwd)
  route     softmax or sigmoid scores of the logits, a bias that moves the choice and not the weight, groups of experts of
            which the best stay, k choices, their weights, renormalised or not, scaled (moe_router_fwd)
  route_bwd the logits' gradient from that of the weights (moe_router_bwd)
  w4        products of routed rows with their experts' 4-bit weights (e2m1, a power of two for each 32), with GeLU behind
            the first and the weighted sum over a token's choices behind the second (moe_w4_product)

Sizes are those of the workloads in paper_2506_22175_amd/synth.py (512/2048, 1024/4096, 2048/8192; 8, 16 and 64 experts; up
to 32768 tokens), wider gates of 256 experts, and generic odd sizes between them.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
EPS = 1e-6
E4M3_MOST = 448.0
TINY = 2.0 ** -126

NORM = dict(kind="norm", T=4096, M=1024, dtype="bf16", out="bf16", group=0, residual=True, gain=True)
ROUTE = dict(kind="route", T=4096, E=64, k=2, scores="softmax", bias=False, groups=1, group_k=1, renorm=False, scale=1.0,
             dtype="f32", masked=False, load=True)
W4 = dict(kind="w4", T=1, k=2, E=16, K=1024, N=4096, dtype="bf16", out="bf16", group=0, per_choice=False, combine=False,
          gelu=False, masked=False)


def listed():
    return [
        # one new token in front of the large layer's experts, 8-bit rows for their products: latency is all there is
        dict(NORM, name="norm_token", T=1, M=2048, out="e4m3", group=128),
        # the large layer's training batch
        dict(NORM, name="norm_train", T=32768, M=2048),
        # a prompt on its way to 8-bit products, the last scale's columns not full
        dict(NORM, name="norm_prompt_e4m3", T=7001, M=4040, out="e4m3", group=128),
        # the training batch's gradients
        dict(NORM, name="norm_grad", kind="norm_bwd", T=32768, M=2048),
        # odd rows in float32, no residual branch
        dict(NORM, name="norm_grad_odd", kind="norm_bwd", T=3003, M=777, dtype="f32", out="f32", residual=False),
        # one new token's choice
        dict(ROUTE, name="route_token", T=1, E=64, k=8, scores="sigmoid", bias=True, groups=8, group_k=4, renorm=True,
             scale=2.5, load=False),
        # the training batch's choices as the layer's own gate makes them, with the experts' loads
        dict(ROUTE, name="route_train", T=32768, E=64, k=2),
        # a wide gate with a balancing bias and groups; padding tokens and unavailable experts
        dict(ROUTE, name="route_groups", T=16384, E=256, k=8, scores="sigmoid", bias=True, groups=8, group_k=4, renorm=True,
             scale=2.5, masked=True),
        # the training batch's gradient
        dict(ROUTE, name="route_grad", kind="route_bwd", T=32768, E=64, k=2),
        # one new token through its experts' first product
        dict(W4, name="w4_token_first", T=1, k=2, E=16, K=2048, N=8192, gelu=True),
        # a batch of sequences through the second product, joined over the choices
        dict(W4, name="w4_batch_second", T=64, k=2, E=16, K=8192, N=2048, per_choice=True, combine=True),
        # 8-bit rows, odd numbers of tokens and columns, some tokens without all of their choices
        dict(W4, name="w4_rows_e4m3", T=37, k=4, E=64, K=1024, N=4093, dtype="e4m3", group=128, out="f32", masked=True),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "route", "route_bwd", "w4", "w4", "w4"])
    if kind.startswith("norm"):
        while True:
            T, M = _logu(rng, 1, 32768), _logu(rng, 64, 8192)
            M = rng.choice([M, M // 8 * 8, M // 64 * 64])
            if T * M <= 32768 * 2048:
                break
        dtype = rng.choice(["bf16", "bf16", "f32"])
        out = rng.choice([dtype, "e4m3"]) if kind == "norm" else dtype
        if dtype == "f32" and T * M > 16384 * 2048:
            T = max(1, T // 2)
        return dict(NORM, kind=kind, T=T, M=M, dtype=dtype, out=out, group=rng.choice([0, 128]) if out == "e4m3" else 0,
                    residual=rng.random() < 0.7, gain=rng.random() < 0.9)
    if kind.startswith("route"):
        E = rng.choice([8, 16, 33, 64, 64, 100, 128, 256])
        groups = rng.choice([g for g in (1, 1, 4, 8) if E % g == 0])
        group_k = rng.choice([1, 2, groups // 2, groups]) if groups > 1 else 1
        k = rng.choice([q for q in (1, 2, 2, 3, 4, 6, 8) if q <= min(E, E // groups * group_k)])
        T = min(_logu(rng, 1, 32768), 32768 * 128 // E)
        return dict(ROUTE, kind=kind, T=T, E=E, k=k, scores=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                    groups=groups, group_k=group_k, renorm=rng.random() < 0.5, scale=rng.choice([1.0, 1.0, 2.5]),
                    dtype=rng.choice(["f32", "f32", "bf16"]), masked=rng.random() < 0.3, load=rng.random() < 0.7)
    E = rng.choice([1, 4, 8, 8, 16, 16, 32, 64])
    k = rng.choice([q for q in (1, 2, 2, 4, 8) if q <= E])
    T = _logu(rng, 1, 256)
    dtype = rng.choice(["bf16", "bf16", "f32", "e4m3"])
    while True:
        K, N = 32 * _logu(rng, 4, 256), _logu(rng, 64, 8192)
        N = rng.choice([N, N // 16 * 16, N // 64 * 64])
        if E * K * N <= 16 * 2048 * 8192 and T * k * E * N <= 1 << 29:
            break
        if T > 1:
            T = (T + 1) // 2
    combine = rng.random() < 0.5
    return dict(W4, T=T, k=k, E=E, K=K, N=N, dtype=dtype, out="bf16" if dtype == "bf16" else rng.choice(["f32", "bf16"]),
                group=rng.choice([0, 128]) if dtype == "e4m3" else 0, per_choice=rng.random() < 0.5, combine=combine,
                gelu=not combine and rng.random() < 0.6, masked=rng.random() < 0.3)


# ---- inputs -----------------------------------------------------------------------------------

def _config(c):
    """The configuration that a program keeps beside its weights."""
    if not own:
        return None
    from paper_2506_22175_amd import binding as B
    code = {"f32": B.MOE_F32, "bf16": B.MOE_BF16, "e4m3": B.MOE_E4M3}
    if c["kind"].startswith("norm"):
        return B.make_norm_config(c["T"], c["M"], EPS, code[c["dtype"]], code[c["out"]], c["group"], grad_overwrite=1)
    if c["kind"].startswith("route"):
        return B.make_router_config(c["T"], c["E"], c["k"], B.MOE_SIGMOID if c["scores"] == "sigmoid" else B.MOE_SOFTMAX,
                                    c["groups"], c["group_k"], 2, int(c["renorm"]), c["scale"], code[c["dtype"]])
    return B.make_w4_config(c["T"], c["k"], c["E"], c["K"], c["N"], code[c["dtype"]], code[c["out"]], c["group"],
                            int(c["per_choice"]), int(c["combine"]), int(c["gelu"]))


def _inputs(c, seed):
    """Everything random, from the seed alone, on the GPU."""
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    randn = lambda *dims: torch.randn(dims, generator=g, device=DEVICE, dtype=torch.float32)  # noqa: E731
    rand = lambda *dims: torch.rand(dims, generator=g, device=DEVICE, dtype=torch.float32)  # noqa: E731
    i = {}
    if c["kind"].startswith("norm"):
        T, M, dt = c["T"], c["M"], DT[c["dtype"]]
        wide = 1.0 + 15.0 * (rand(M) < 0.004)             # a few columns carry most of a row, as in trained models
        i["x"] = (randn(T, M) * wide).to(dt)
        i["gain"] = 1.0 + 0.2 * randn(M) if c["gain"] else None
        if c["kind"] == "norm":
            i["residual"] = randn(T, M).mul_(2.0).to(dt) if c["residual"] else None
            return i
        # backward: x is the h that forward left, with its row statistics
        i["rstd"] = (i["x"].double().square().mean(1) + EPS).rsqrt().float()
        i["dy"] = randn(T, M).to(dt)
        i["dh"] = randn(T, M).to(dt) if c["residual"] else None
        return i
    if c["kind"].startswith("route"):
        T, E, k, dt = c["T"], c["E"], c["k"], DT[c["dtype"]]
        l = randn(T, E) * 1.5 + 0.5 * randn(E)            # some experts are more popular
        if c["masked"]:
            l[rand(T, E) < 0.1] = -math.inf               # experts that a token may not have
            l[rand(T) < 0.05] = -math.inf                 # padding tokens
        i["logits"] = l.to(dt)
        i["bias"] = 0.1 * randn(E) if c["bias"] else None
        if c["kind"] == "route_bwd":
            i["topk_idx"] = _plain_route(c, i["logits"], i["bias"])[0]
            i["dw"] = randn(T, k)
        return i
    T, k, E, K, N = c["T"], c["k"], c["E"], c["K"], c["N"]
    x = randn(T * k, K) if c["per_choice"] else randn(T, K)
    if c["dtype"] == "e4m3":
        cols = c["group"] or K
        pad = torch.nn.functional.pad(x, (0, -K % cols)).reshape(x.shape[0], -1, cols)
        i["x_scales"] = (pad.abs().amax(2) / E4M3_MOST).contiguous()
        i["x"] = (pad / i["x_scales"][..., None]).reshape(x.shape[0], -1)[:, :K].to(DT["e4m3"]).contiguous()
    else:
        i["x"], i["x_scales"] = x.to(DT[c["dtype"]]), None
    choice = torch.topk(randn(T, E) + 0.5 * randn(E), k, dim=1)
    i["topk_idx"], i["topk_w"] = choice.indices.to(torch.int32), torch.softmax(choice.values, 1)
    if c["masked"]:
        i["topk_idx"][rand(T, k) < 0.1] = -1
    # weights as a quantiser leaves them: two columns of K in a byte, the first in the low half, and for each 32 of them the
    # power of two under which the largest magnitude is at most 6
    i["Wq"] = torch.empty((E, N, K // 2), dtype=torch.uint8, device=DEVICE)
    i["Ws"] = torch.empty((E, N, K // 32), dtype=torch.uint8, device=DEVICE)
    for e in range(E):
        w = randn(N, K // 32, 32) * 0.02
        p = torch.ceil(torch.log2(w.abs().amax(2) / 6.0)).clamp(-126, 127)
        v = w.abs() * torch.exp2(-p)[..., None]
        q = torch.bucketize(v, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEVICE)).to(torch.uint8)
        q = (q | ((w < 0).to(torch.uint8) << 3)).reshape(N, K // 2, 2)
        i["Wq"][e] = q[..., 0] | (q[..., 1] << 4)
        i["Ws"][e] = (p + 127).to(torch.uint8)
    return i


def prepare(case, seed):
    c = case
    i = _inputs(c, seed)
    empty = lambda *dims, dtype: torch.empty(dims, device=DEVICE, dtype=dtype)  # noqa: E731
    cfg = _config(c)
    s = {"case": c, "cfg": cfg, "in": i, "scratch": None}
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    if c["kind"] == "norm":
        T, M = c["T"], c["M"]
        o = {"y": empty(T, M, dtype=DT[c["out"]]), "rstd": empty(T, dtype=f32)}
        if c["residual"]:
            o["h"] = empty(T, M, dtype=DT[c["dtype"]])
        if c["out"] == "e4m3":
            o["scales"] = empty(T, -(-M // c["group"]) if c["group"] else 1, dtype=f32)
    elif c["kind"] == "norm_bwd":
        T, M = c["T"], c["M"]
        o = {"dx": empty(T, M, dtype=DT[c["dtype"]]), "dgain": empty(M, dtype=f32)}
    elif c["kind"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        o = {"topk_idx": empty(T, k, dtype=i32), "topk_w": empty(T, k, dtype=f32)}
        if c["load"]:
            o["load"] = empty(E, dtype=i32)
    elif c["kind"] == "route_bwd":
        o = {"dlogits": empty(c["T"], c["E"], dtype=DT[c["dtype"]])}
    else:
        T, k, N = c["T"], c["k"], c["N"]
        o = {"y": empty(*((T, N) if c["combine"] else (T, k, N)), dtype=DT[c["out"]])}
    if own and c["kind"] in ("norm_bwd", "w4"):
        from paper_2506_22175_amd import binding as B
        need = B.moe_norm_scratch_bytes(cfg) if c["kind"] == "norm_bwd" else B.moe_w4_scratch_bytes(cfg)
        s["scratch"] = empty(max(1, need), dtype=u8)
    s["out"] = o
    return s


# ---- the calls --------------------------------------------------------------------------------

def run(state):
    c, i, o = state["case"], state["in"], state["out"]
    if own:
        return _own(state["cfg"], c, i, o, state["scratch"])
    if c["kind"] == "norm":
        return _plain_norm(c, i)
    if c["kind"] == "norm_bwd":
        return _plain_norm_bwd(c, i)
    if c["kind"] == "route":
        idx, w = _plain_route(c, i["logits"], i["bias"])
        out = {"topk_idx": idx, "topk_w": w}
        if c["load"]:
            out["load"] = (idx[..., None] == torch.arange(c["E"], device=idx.device, dtype=idx.dtype)).sum((0, 1)).to(torch.int32)
        return out
    if c["kind"] == "route_bwd":
        return _plain_route_bwd(c, i)
    return _plain_w4(c, i)


def _own(cfg, c, i, o, scratch):
    from paper_2506_22175_amd import binding as B
    if c["kind"] == "norm":
        B.moe_norm_fwd(cfg, i["x"], i["residual"], i["gain"], o.get("h"), o["y"], o.get("scales"), o["rstd"])
    elif c["kind"] == "norm_bwd":
        B.moe_norm_bwd(cfg, i["dy"], i["x"], i["gain"], i["rstd"], i["dh"], o["dx"], o["dgain"], scratch)
    elif c["kind"] == "route":
        if c["load"]:
            o["load"].zero_()                             # the call adds to it
        B.moe_router_fwd(cfg, i["logits"], i["bias"], o["topk_idx"], o["topk_w"], o.get("load"))
    elif c["kind"] == "route_bwd":
        B.moe_router_bwd(cfg, i["logits"], i["topk_idx"], i["dw"], o["dlogits"])
    else:
        B.moe_w4_product(cfg, i["x"], i["x_scales"], i["topk_idx"], i["topk_w"] if c["combine"] else None, i["Wq"], i["Ws"],
                         o["y"], scratch)
    return o


def _plain_norm(c, i):
    h = i["x"].float()
    if i["residual"] is not None:
        h = h + i["residual"].float()
    rstd = torch.rsqrt((h * h).mean(1) + EPS)
    y = h * rstd[:, None]
    if i["gain"] is not None:
        y = y * i["gain"]
    out = {"rstd": rstd}
    if c["residual"]:
        out["h"] = h.to(DT[c["dtype"]])
    if c["out"] == "e4m3":
        T, M = h.shape
        cols = c["group"] or M
        y = torch.nn.functional.pad(y, (0, -M % cols)).reshape(T, -1, cols)
        scales = (y.abs().amax(2) / E4M3_MOST).clamp(min=TINY)
        y = (y / scales[..., None]).reshape(T, -1)[:, :M]
        out["scales"] = scales
    out["y"] = y.to(DT[c["out"]])
    return out


def _plain_norm_bwd(c, i):
    h, dy, r = i["x"].float(), i["dy"].float(), i["rstd"][:, None]
    n = h * r
    dn = dy if i["gain"] is None else dy * i["gain"]
    dx = r * (dn - n * (dn * n).mean(1, keepdim=True))
    if i["dh"] is not None:
        dx = dx + i["dh"].float()
    return {"dx": dx.to(DT[c["dtype"]]), "dgain": (dy * n).sum(0)}


def _plain_route(c, logits, bias):
    """Scores in 64 bits: which of two experts comes first is decided by the last bits of their scores."""
    T, E = logits.shape
    l = logits.double()
    l = torch.where(torch.isnan(l), -math.inf, l)
    s = _scores(c, l)
    open_ = l > -math.inf
    v = s if bias is None else s + bias.double()
    open_ = open_ & (v > -math.inf)
    v = torch.where(open_, v, -math.inf)
    rank = v if bias is not None else l
    if c["groups"] > 1:
        by = torch.sort(v.reshape(T, c["groups"], -1), dim=2, descending=True)[0][..., :2]
        score = torch.where(by == -math.inf, 0.0, by).sum(2)
        score = torch.where(by[..., 0] == -math.inf, -math.inf, score)
        best = torch.sort(score, dim=1, descending=True, stable=True)[1][:, :c["group_k"]]
        stays = torch.zeros_like(score, dtype=torch.bool).scatter(1, best, True)
        rank = torch.where(stays[..., None].expand(T, c["groups"], E // c["groups"]).reshape(T, E), rank, -math.inf)
    rank, idx = torch.sort(rank, dim=1, descending=True, stable=True)
    rank, idx = rank[:, :c["k"]], idx[:, :c["k"]]
    chosen = rank > -math.inf
    w = torch.where(chosen, s.gather(1, idx), 0.0)
    if c["renorm"]:
        w = w / torch.clamp(w.sum(1, keepdim=True), min=1e-300)
    return torch.where(chosen, idx, -1).to(torch.int32), (w * c["scale"]).float()


def _scores(c, l):
    """Of logits without NaN, in their own type; none has -inf."""
    if c["scores"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    m = l.amax(1, keepdim=True)
    p = torch.where(l == -math.inf, 0.0, torch.where(l == m, 1.0, torch.exp(l - m)))
    return p / torch.clamp(p.sum(1, keepdim=True), min=1.0)


def _plain_route_bwd(c, i):
    l = i["logits"].float()
    l = torch.where(torch.isnan(l), -math.inf, l)
    s = _scores(c, l)
    chosen = i["topk_idx"] >= 0
    idx = i["topk_idx"].clamp(min=0).long()
    dw = torch.where(chosen, i["dw"] * c["scale"], 0.0)
    w = torch.where(chosen, s.gather(1, idx), 0.0)
    if c["renorm"]:
        total = torch.clamp(w.sum(1, keepdim=True), min=1e-30)
        dw = (dw - (dw * w).sum(1, keepdim=True) / total) / total
        dw = torch.where(chosen, dw, 0.0)
    ds = torch.zeros_like(s).scatter_add_(1, idx, dw)
    if c["scores"] == "sigmoid":
        dl = ds * s * torch.sigmoid(-l)
    else:
        dl = s * (ds - (ds * s).sum(1, keepdim=True))
    return {"dlogits": dl.to(DT[c["dtype"]])}


def _plain_weights(q, s):
    """[..., N, K] float of packed weights."""
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=q.device)
    w = torch.stack([values[(q & 15).int()], values[(q >> 4).int()]], dim=-1).reshape(*s.shape, 32)
    return (w * torch.exp2(s.float() - 127.0)[..., None]).reshape(*q.shape[:-1], -1)


def _plain_rows(c, i):
    if c["dtype"] != "e4m3":
        return i["x"].float()
    cols = c["group"] or c["K"]
    return i["x"].float() * i["x_scales"].repeat_interleave(cols, 1)[:, :c["K"]]


def _plain_w4(c, i):
    T, k, E, K, N = c["T"], c["k"], c["E"], c["K"], c["N"]
    x = _plain_rows(c, i)
    chosen = i["topk_idx"] >= 0
    idx = i["topk_idx"].clamp(min=0).long()
    if T * k <= E:                                        # the chosen experts' weights alone
        W = _plain_weights(i["Wq"][idx.reshape(-1)], i["Ws"][idx.reshape(-1)])
        x = x if c["per_choice"] else x.repeat_interleave(k, 0)
        y = torch.matmul(W, x[..., None]).reshape(T, k, N)
    else:                                                 # every row with every expert, in one product
        W = _plain_weights(i["Wq"].reshape(E * N, -1), i["Ws"].reshape(E * N, -1))
        y = torch.matmul(x, W.t()).reshape(-1, k if c["per_choice"] else 1, E, N)
        y = y.expand(T, k, E, N).gather(2, idx[..., None, None].expand(T, k, 1, N)).reshape(T, k, N)
    y = torch.where(chosen[..., None], y, 0.0)
    if c["gelu"]:
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if c["combine"]:
        y = (i["topk_w"][..., None] * y).sum(1)
    return {"y": y.to(DT[c["out"]])}


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    """Every input read once and every output written once; of the packed weights those of the experts that are expected to
    be chosen (each token has k different ones out of E)."""
    c = case
    size = {"f32": 4, "bf16": 2, "e4m3": 1}
    if c["kind"].startswith("norm"):
        n, es = c["T"] * c["M"], size[c["dtype"]]
        if c["kind"] == "norm_bwd":
            return {"bytes": n * es * (4 if c["residual"] else 3) + 8 * c["M"] + 4 * c["T"], "flops": 8.0 * n}
        scales = c["T"] * (-(-c["M"] // c["group"]) if c["group"] else 1) * 4 if c["out"] == "e4m3" else 0
        return {"bytes": n * es * (3 if c["residual"] else 1) + n * size[c["out"]] + scales + 4 * c["M"] + 4 * c["T"], "flops": 5.0 * n}
    if c["kind"] == "route":
        return {"bytes": c["T"] * (c["E"] * size[c["dtype"]] + 8 * c["k"]) + 8 * c["E"], "flops": 5.0 * c["T"] * c["E"]}
    if c["kind"] == "route_bwd":
        return {"bytes": c["T"] * (2 * c["E"] * size[c["dtype"]] + 8 * c["k"]), "flops": 6.0 * c["T"] * c["E"]}
    T, k, E, K, N = c["T"], c["k"], c["E"], c["K"], c["N"]
    experts = E * (1.0 - (1.0 - k / E) ** T)
    rows = T * k if c["per_choice"] else T
    return {"bytes": experts * N * K * (0.5 + 1 / 32) + rows * K * size[c["dtype"]] + (T if c["combine"] else T * k) * N * size[c["out"]],
            "flops": 2.0 * T * k * N * K}


# ---- the same in 64 bits ----------------------------------------------------------------------------

def _to_e4m3(v):
    """64-bit values rounded to the 8-bit type's, ties to even."""
    _, p = torch.frexp(v)
    step = torch.exp2((p.double() - 1.0).clamp(min=-6.0) - 3.0)
    return torch.round(v / step) * step


def exact(case, seed):
    c = case
    i = _inputs(c, seed)
    f64 = torch.float64
    if c["kind"] == "norm":
        h = i["x"].to(f64)
        h = h + i["residual"].to(f64) if c["residual"] else h
        norm = torch.linalg.vector_norm(h, dim=1)
        root = torch.sqrt(norm ** 2 / c["M"] + EPS)
        y = h / root[:, None]
        y = y * i["gain"].to(f64) if c["gain"] else y
        out = {"rstd": 1.0 / root, "y": y}
        if c["residual"]:
            out["h"] = h
        if c["out"] == "e4m3":
            cols = c["group"] or c["M"]
            parts = torch.split(y, cols, dim=1)
            scales = [torch.clamp(p.abs().max(dim=1, keepdim=True)[0] / E4M3_MOST, min=TINY) for p in parts]
            out["y"] = torch.cat([_to_e4m3(p / s) for p, s in zip(parts, scales)], 1)
            out["scales"] = torch.cat(scales, 1)
        return out
    if c["kind"] == "norm_bwd":
        h, dy, r = i["x"].to(f64), i["dy"].to(f64), i["rstd"].to(f64)
        up = dy * i["gain"].to(f64) if c["gain"] else dy
        # d/dh of up . h r, where dr/dh = -r^3 h / M
        dx = up * r[:, None] - h * ((up * h).sum(1) * r ** 3 / c["M"])[:, None]
        return {"dx": dx + i["dh"].to(f64) if c["residual"] else dx, "dgain": torch.mv((dy * h).t(), r)}
    if c["kind"] == "route":
        # the weights of the choices that the definition gives; the choices themselves are whole numbers
        l = i["logits"].to(f64).nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
        idx = _plain_route(c, i["logits"], i["bias"])[0].long()
        there = idx >= 0
        mine = torch.where(there, l.gather(1, idx.clamp(min=0)), -math.inf)
        if c["scores"] == "sigmoid":
            log_s = torch.nn.functional.logsigmoid(mine)
        else:
            log_s = mine - torch.logsumexp(l, 1, keepdim=True)
        log_s = torch.where(there, log_s, -math.inf)
        if c["renorm"]:
            log_s = log_s - torch.logsumexp(log_s, 1, keepdim=True)
        w = torch.where(there, torch.exp(log_s), 0.0) * c["scale"]
        return {"topk_idx": None, "topk_w": w, "load": None} if c["load"] else {"topk_idx": None, "topk_w": w}
    if c["kind"] == "route_bwd":
        # by differentiation of the loss sum(dw * weights)
        l = i["logits"].to(f64).nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
        shut = l == -math.inf
        with torch.enable_grad():
            z = torch.where(shut, 0.0, l).requires_grad_()
            if c["scores"] == "sigmoid":
                s = torch.sigmoid(z).masked_fill(shut, 0.0)
            else:
                s = torch.softmax(z.masked_fill(shut, -1e4), 1).masked_fill(shut, 0.0)
            there = i["topk_idx"] >= 0
            w = s.gather(1, i["topk_idx"].clamp(min=0).long()).masked_fill(~there, 0.0)
            if c["renorm"]:
                total = w.sum(1, keepdim=True)
                w = w / torch.where(total > 0, total, 1.0)
            (dl,) = torch.autograd.grad((w * i["dw"].to(f64) * c["scale"]).sum(), z)
        return {"dlogits": dl}
    T, k, E, K, N = c["T"], c["k"], c["E"], c["K"], c["N"]
    x = i["x"].to(f64)
    if c["dtype"] == "e4m3":
        cols = c["group"] or K
        x = torch.cat([p * s for p, s in zip(torch.split(x, cols, dim=1), i["x_scales"].to(f64).split(1, dim=1))], 1)
    rows = torch.zeros((T * k, N), dtype=f64, device=DEVICE)
    idx = i["topk_idx"].reshape(-1)
    for e in range(E):
        r = torch.nonzero(idx == e)[:, 0]
        if r.numel() == 0:
            continue
        W = torch.empty((N, K), dtype=f64, device=DEVICE)
        for half in (0, 1):
            q = (i["Wq"][e] >> (4 * half)) & 15
            up, odd = ((q >> 1) & 3).to(f64), (q & 1).to(f64)
            size = torch.where(up > 0, (1.0 + 0.5 * odd) * torch.exp2(up - 1.0), 0.5 * odd)
            W[:, half::2] = torch.where(q >= 8, -size, size)
        W.mul_(torch.exp2(i["Ws"][e].to(f64) - 127.0).repeat_interleave(32, 1))
        rows[r] = x[r if c["per_choice"] else r // k] @ W.t()
    if c["gelu"]:
        rows = rows * torch.special.ndtr(rows)
    y = rows.reshape(T, k, N)
    return {"y": torch.einsum("tj,tjn->tn", i["topk_w"].to(f64), y) if c["combine"] else y}
