"""The dense half of a pruned network and the loss that trains it, as measurable cases: one pass each through an operator,
in elementary torch operations or, where `own` is true, through the entry points of paper_2001_07710_amd.

Kinds of work
  linear       y = act(x w^T + bias) with a residual behind or in front of the activation; z, the activation's argument, is
               kept where the layer is being trained
  linear_grad  the same layer backwards: dx = (dz w) * act'(z of the layer before) + a gradient that comes round the layer,
               dw and db in 32 bits
  norm         layer norm over the last axis, forward
  norm_step    layer norm forward and backward with the gradients of its weight and bias
  distill      distillation from a teacher's top logits: the loss of every row and the gradient of the logits
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one image's pooled features into class scores: a launch and its latency
        {"name": "head_1x512_1000_f32", "kind": "linear", "dtype": "f32", "M": 1, "N": 1000, "K": 512, "pad": 0, "act": "none",
         "residual": "none", "keep_z": False},
        # the first fully connected layer behind VGG-16's last pooling (512 x 7 x 7 features) on one image: weights once through
        {"name": "fc_1x25088_4096_f16", "kind": "linear", "dtype": "f16", "M": 1, "N": 4096, "K": 25088, "pad": 0, "act": "relu",
         "residual": "none", "keep_z": False},
        # the last 1x1 layer of a bottleneck on channel-minor maps of 14 x 14, batch 32: residual, then ReLU
        {"name": "conv1x1_6272x256_1024_f16", "kind": "linear", "dtype": "f16", "M": 6272, "N": 1024, "K": 256, "pad": 0,
         "act": "relu", "residual": "first", "keep_z": False},
        # sizes that no tile divides, rows that are not aligned: a slice of a wider tensor
        {"name": "ragged_777x1001_333_f16", "kind": "linear", "dtype": "f16", "M": 777, "N": 333, "K": 1001, "pad": 5, "act": "silu",
         "residual": "behind", "keep_z": False},
        # the widening layer of a large feed-forward block in training: the product is all that counts
        {"name": "mlp_8192x4096_16384_bf16", "kind": "linear", "dtype": "bf16", "M": 8192, "N": 16384, "K": 4096, "pad": 0,
         "act": "gelu_tanh", "residual": "none", "keep_z": True},
        # fine-tuning in 32 bits on a small batch
        {"name": "grad_1000x520_300_f32", "kind": "linear_grad", "dtype": "f32", "M": 1000, "N": 300, "K": 520, "pad": 0, "act": "relu",
         "add": True},
        # fine-tuning of a large layer whose input went through an activation
        {"name": "grad_8192x4096_4096_bf16", "kind": "linear_grad", "dtype": "bf16", "M": 8192, "N": 4096, "K": 4096, "pad": 0,
         "act": "gelu_tanh", "add": False},
        # the norm in front of a head, for one image or token at a time
        {"name": "norm_1x4096_bf16", "kind": "norm", "dtype": "bf16", "M": 1, "D": 4096, "pad": 0},
        # the norm over the channels of channel-minor maps of 56 x 56, batch 64, in training
        {"name": "norm_step_200704x64_f16", "kind": "norm_step", "dtype": "f16", "M": 200704, "D": 64, "pad": 0},
        # the norm in front of a large feed-forward block, in training
        {"name": "norm_step_16384x4096_bf16", "kind": "norm_step", "dtype": "bf16", "M": 16384, "D": 4096, "pad": 0},
        # a batch of class scores against the twenty best of the unpruned network
        {"name": "distill_256x1000_f16", "kind": "distill", "dtype": "f16", "R": 256, "V": 1000, "k": 20, "T": 4.0, "pad": 0,
         "short": False},
        # logits over a vocabulary of odd length, padded rows and short lists among them
        {"name": "distill_8192x32001_bf16", "kind": "distill", "dtype": "bf16", "R": 8192, "V": 32001, "k": 64, "T": 1.0, "pad": 0,
         "short": True},
    ]


# -------------------------------------------------------------------------------------------- more of the same ranges

_MOST_FLOPS = 1.0e12       # (the largest listed product has 1.1e12)
_MOST_VALUES = 6.0e7       # of one tensor of the kinds that memory bounds


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A length spread over its logarithm; half of the time a multiple of 8, as networks have them."""
    n = _log(rng, lo, hi)
    return n if n < 8 or rng.random() < 0.5 else max(8, n // 8 * 8)


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_grad", "norm", "norm_step", "distill"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    pad = rng.choice([0, 0, 0, 8, rng.randint(1, 15)])
    if kind in ("linear", "linear_grad"):
        while True:
            M, N, K = _size(rng, 1, 16384), _size(rng, 16, 16384), _size(rng, 16, 25088)
            if 2.0 * M * N * K * (1 if kind == "linear" else 2) <= _MOST_FLOPS:
                break
        act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
        if kind == "linear":
            return {"kind": kind, "dtype": dtype, "M": M, "N": N, "K": K, "pad": pad, "act": act,
                    "residual": rng.choice(["none", "first", "behind"]), "keep_z": rng.random() < 0.4}
        return {"kind": kind, "dtype": dtype, "M": M, "N": N, "K": K, "pad": pad, "act": act, "add": rng.random() < 0.4}
    if kind in ("norm", "norm_step"):
        while True:
            M, D = _size(rng, 1, 250000), _size(rng, 16, 20000)
            if M * D <= _MOST_VALUES:
                return {"kind": kind, "dtype": dtype, "M": M, "D": D, "pad": pad}
    while True:
        R, V = _size(rng, 1, 16384), _size(rng, 200, 200000)
        if R * V <= _MOST_VALUES:
            break
    return {"kind": kind, "dtype": dtype, "R": R, "V": V, "k": _log(rng, 1, 128), "T": rng.choice([1.0, 2.0, 4.0]), "pad": pad,
            "short": rng.random() < 0.5}


# -------------------------------------------------------------------------------------------- inputs

def _rows(g, rows, cols, pad, dtype, scale=1.0, offset=0.0):
    """[rows][cols] normal values; a row begins `pad` values behind the end of the row before."""
    t = torch.empty((rows, cols + pad), dtype=_TYPES[dtype], device="cuda")
    step = max(1, (1 << 26) // (cols + pad))
    for at in range(0, rows, step):
        part = t[at:at + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(scale).add_(offset))
    return t[:, :cols]


def _like(rows, cols, pad, dtype):
    return torch.zeros((rows, cols + pad), dtype=_TYPES[dtype], device="cuda")[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s, kind, pad = {"case": case}, case["kind"], case["pad"]
    vec = lambda n, scale, offset=0.0: torch.randn(n, generator=g, device="cuda").mul_(scale).add_(offset)  # noqa: E731
    if kind in ("linear", "linear_grad"):
        M, N, K, dt = case["M"], case["N"], case["K"], case["dtype"]
        s["w"] = _rows(g, N, K, pad, dt, math.sqrt(2.0 / K))
    if kind == "linear":
        s["x"] = _rows(g, M, K, pad, dt)
        s["bias"] = vec(N, 0.1)
        s["residual"] = _rows(g, M, N, pad, dt) if case["residual"] != "none" else None
        s["y"] = _like(M, N, pad, dt)
        s["z"] = _like(M, N, pad, dt) if case["keep_z"] else None
    elif kind == "linear_grad":
        s["dz"] = _rows(g, M, N, pad, dt)
        s["x"] = _rows(g, M, K, pad, dt)
        s["z"] = _rows(g, M, K, pad, dt) if case["act"] != "none" else None
        s["add"] = _rows(g, M, K, pad, dt) if case["add"] else None
        s["dx"] = _like(M, K, pad, dt)
        s["dw"] = torch.zeros((N, K), device="cuda")
        s["db"] = torch.zeros(N, device="cuda")
    elif kind in ("norm", "norm_step"):
        M, D, dt = case["M"], case["D"], case["dtype"]
        s["x"] = _rows(g, M, D, pad, dt, 1.5, 0.5)
        s["gamma"], s["beta"] = vec(D, 0.1, 1.0), vec(D, 0.1)
        s["y"] = _like(M, D, pad, dt)
        if kind == "norm_step":
            s["dy"] = _rows(g, M, D, pad, dt)
            s["dx"] = _like(M, D, pad, dt)
            s["mean"], s["rstd"] = torch.zeros(M, device="cuda"), torch.zeros(M, device="cuda")
            s["dgamma"], s["dbeta"] = torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda")
    else:
        R, V, k, dt = case["R"], case["V"], case["k"], case["dtype"]
        s["logits"] = _rows(g, R, V, pad, dt, 3.0)
        s["values"] = torch.empty((R, k), device="cuda")
        s["indices"] = torch.empty((R, k), dtype=torch.int32, device="cuda")
        step = max(1, (1 << 26) // V)
        for at in range(0, R, step):                          # the teacher has learnt much the same, and keeps its best
            part = s["logits"][at:at + step].float()
            part += torch.randn(part.shape, generator=g, device="cuda")
            v, i = torch.topk(part, k, dim=1)
            s["values"][at:at + step], s["indices"][at:at + step] = v, i.int()
        s["weight"] = torch.full((R,), 1.0 / R, device="cuda")
        if case["short"]:
            length = torch.randint(0, 2 * k, (R, 1), generator=g, device="cuda")      # half of the lists are shorter than k
            length[0] = k                                                             # (the first row is never empty)
            s["indices"].masked_fill_(torch.arange(k, device="cuda")[None, :] >= length, -1)
            s["weight"][1:].masked_fill_(torch.rand(R - 1, generator=g, device="cuda") < 0.1, 0.0)      # padding
        s["loss"] = torch.zeros(R, device="cuda")
        s["grad"] = _like(R, V, pad, dt)
    return s


# -------------------------------------------------------------------------------------------- the plain forms

def _act(z, act):
    if act == "relu":
        return z * (z > 0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _plain_linear(s, case):
    z = s["x"].float() @ s["w"].float().t() + s["bias"]
    if case["residual"] == "first":
        z = z + s["residual"].float()
    y = _act(z, case["act"])
    if case["residual"] == "behind":
        y = y + s["residual"].float()
    dt = _TYPES[case["dtype"]]
    return {"y": y.to(dt), "z": z.to(dt) if case["keep_z"] else None}


def _plain_linear_grad(s, case):
    dz = s["dz"].float()
    dx = dz @ s["w"].float()
    if case["act"] != "none":
        dx = dx * _act_grad(s["z"].float(), case["act"])
    if case["add"]:
        dx = dx + s["add"].float()
    return {"dx": dx.to(_TYPES[case["dtype"]]), "dw": dz.t() @ s["x"].float(), "db": dz.sum(0)}


_EPS = 1e-5


def _plain_norm(s, case):
    x, dt = s["x"].float(), _TYPES[case["dtype"]]
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + _EPS)
    h = x * rstd
    out = {"y": (h * s["gamma"] + s["beta"]).to(dt)}
    if case["kind"] == "norm_step":
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        out.update(dx=dx.to(dt), dgamma=(dy * h).sum(0), dbeta=dy.sum(0))
    return out


def _plain_distill(s, case):
    T, k = case["T"], case["k"]
    there = s["indices"] >= 0
    t = (s["values"] / T).masked_fill(~there, -math.inf)
    some = there.any(1, keepdim=True) & (s["weight"][:, None] != 0)
    top = torch.where(some, t.max(1, keepdim=True).values, torch.zeros_like(t[:, :1]))
    e = torch.where(there & some, torch.exp(t - top), torch.zeros_like(t))
    total = torch.where(some, e.sum(1, keepdim=True), torch.ones_like(top))
    p = e / total
    log_p = torch.where(there, t - top - torch.log(total), torch.zeros_like(t))
    z = s["logits"].float() / T
    z = z - z.max(1, keepdim=True).values
    u = torch.exp(z)
    norm = u.sum(1, keepdim=True)
    at = s["indices"].clamp(min=0).long()
    loss = (p * (log_p - (z.gather(1, at) - torch.log(norm)))).sum(1) * (s["weight"] * T * T)
    scale = s["weight"][:, None] * T
    grad = u.mul_(scale * some / norm)
    grad.scatter_add_(1, at, -scale * p)
    return {"loss": loss, "grad": grad.to(_TYPES[case["dtype"]])}


# -------------------------------------------------------------------------------------------- the framework's calls

def _workspace(s, name, nbytes):
    if s.get(name) is None:
        s[name] = torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")
    return s[name]


def _own_linear(s, case):
    import paper_2001_07710_amd as pc
    dt, M, N, K, pad = _code(pc, case), case["M"], case["N"], case["K"], case["pad"]
    nbytes = pc.linear_workspace(dt, M, N, K)
    pc.linear(s["x"], s["w"], s["y"], dt, M, N, K, bias=s["bias"], residual=s["residual"], z=s["z"], act=_act_code(pc, case),
              flags=pc.FLAG_RESIDUAL_FIRST if case["residual"] == "first" else 0, ldx=K + pad, ldw=K + pad, ldr=N + pad, ldy=N + pad,
              workspace=_workspace(s, "ws", nbytes), workspace_bytes=nbytes, stream=torch.cuda.current_stream().cuda_stream)
    return {"y": s["y"], "z": s["z"]}


def _own_linear_grad(s, case):
    import paper_2001_07710_amd as pc
    dt, M, N, K, pad = _code(pc, case), case["M"], case["N"], case["K"], case["pad"]
    stream = torch.cuda.current_stream().cuda_stream
    n1, n2 = pc.linear_grad_input_workspace(dt, M, N, K), pc.linear_grad_weight_workspace(dt, M, N, K)
    ws = _workspace(s, "ws", max(n1, n2))
    pc.linear_grad_input(s["dz"], s["w"], s["dx"], dt, M, N, K, z=s["z"], act=_act_code(pc, case), add=s["add"], lddz=N + pad,
                         ldw=K + pad, ldz=K + pad, lda=K + pad, lddx=K + pad, workspace=ws, workspace_bytes=n1, stream=stream)
    pc.linear_grad_weight(s["dz"], s["x"], s["dw"], dt, M, N, K, db=s["db"], lddz=N + pad, ldx=K + pad, workspace=ws,
                          workspace_bytes=n2, stream=stream)
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_norm(s, case):
    import paper_2001_07710_amd as pc
    dt, M, D, pad = _code(pc, case), case["M"], case["D"], case["pad"]
    stream, ld = torch.cuda.current_stream().cuda_stream, case["D"] + case["pad"]
    pc.layer_norm(s["x"], s["y"], dt, M, D, gamma=s["gamma"], beta=s["beta"], eps=_EPS, mean=s.get("mean"), rstd=s.get("rstd"), ldx=ld,
                  ldy=ld, stream=stream)
    if case["kind"] == "norm":
        return {"y": s["y"]}
    nbytes = pc.layer_norm_grad_workspace(dt, M, D)
    pc.layer_norm_grad(s["dy"], s["x"], s["dx"], s["mean"], s["rstd"], dt, M, D, gamma=s["gamma"], dgamma=s["dgamma"],
                       dbeta=s["dbeta"], lddy=ld, ldx=ld, lddx=ld, workspace=_workspace(s, "ws", nbytes), workspace_bytes=nbytes,
                       stream=stream)
    return {"y": s["y"], "dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _own_distill(s, case):
    import paper_2001_07710_amd as pc
    ld = case["V"] + case["pad"]
    pc.distill(s["logits"], s["indices"], s["values"], _code(pc, case), case["R"], case["V"], case["k"], case["T"], weight=s["weight"],
               loss=s["loss"], grad=s["grad"], ldl=ld, ldg=ld, stream=torch.cuda.current_stream().cuda_stream)
    return {"loss": s["loss"], "grad": s["grad"]}


def _code(pc, case):
    return {"f32": pc.F32, "f16": pc.F16, "bf16": pc.BF16}[case["dtype"]]


def _act_code(pc, case):
    return {"none": pc.ACT_NONE, "relu": pc.ACT_RELU, "gelu": pc.ACT_GELU, "gelu_tanh": pc.ACT_GELU_TANH, "silu": pc.ACT_SILU}[case["act"]]


def run(state):
    case = state["case"]
    kind = "norm" if case["kind"] == "norm_step" else case["kind"]
    if own:
        return {"linear": _own_linear, "linear_grad": _own_linear_grad, "norm": _own_norm, "distill": _own_distill}[kind](state, case)
    return {"linear": _plain_linear, "linear_grad": _plain_linear_grad, "norm": _plain_norm, "distill": _plain_distill}[kind](state, case)


# -------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        outs = 1 + (case["residual"] != "none") + case["keep_z"]
        return {"bytes": e * (M * K + N * K + outs * M * N) + 4 * N, "flops": 2.0 * M * N * K}
    if kind == "linear_grad":
        M, N, K = case["M"], case["N"], case["K"]
        maps = 2 + (case["act"] != "none") + case["add"]                 # x and dx, z, add
        return {"bytes": e * (M * N + N * K + maps * M * K) + 4 * (N * K + N), "flops": 4.0 * M * N * K}
    if kind in ("norm", "norm_step"):
        M, D = case["M"], case["D"]
        both = kind == "norm_step"
        return {"bytes": e * M * D * (4 if both else 2) + 4 * D * (4 if both else 2), "flops": M * D * (20.0 if both else 8.0)}
    R, V, k = case["R"], case["V"], case["k"]
    return {"bytes": 2 * e * R * V + R * (8 * k + 8), "flops": 6.0 * R * V}


# -------------------------------------------------------------------------------------------- the definition in 64 bits

def _phi(z):
    return torch.special.ndtr(z)


def _curve(z, act):
    """(act(z), act'(z)) in the type of z."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.clamp(z, min=0), torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    if act == "gelu":
        return z * _phi(z), _phi(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    a = 2 * math.sqrt(2 / math.pi)                      # (1 + tanh(v)) / 2 = sigmoid(2 v)
    s, r = torch.sigmoid(a * (z + 0.044715 * z ** 3)), torch.sigmoid(-a * (z + 0.044715 * z ** 3))
    return z * s, s + z * s * r * a * (1 + 3 * 0.044715 * z ** 2)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    d = {n: v.double() for n, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()
         and n in ("x", "w", "bias", "residual", "dz", "add", "gamma", "beta", "dy", "weight", "values") or n == "z" and kind == "linear_grad" and v is not None}
    if kind == "linear":
        z = torch.addmm(d["bias"], d["x"], d["w"].t())
        if case["residual"] == "first":
            z += d["residual"]
        y = _curve(z, case["act"])[0]
        if case["residual"] == "behind":
            y = y + d["residual"]
        return {"y": y, "z": z if case["keep_z"] else None}
    if kind == "linear_grad":
        dx = torch.mm(d["dz"], d["w"])
        if d.get("z") is not None:
            dx *= _curve(d["z"], case["act"])[1]
        if case["add"]:
            dx += d["add"]
        return {"dx": dx, "dw": torch.mm(d["dz"].t().contiguous(), d["x"]), "db": d["dz"].t().contiguous().sum(1)}
    if kind in ("norm", "norm_step"):
        var, mean = torch.var_mean(d["x"], dim=1, unbiased=False, keepdim=True)
        sd = torch.sqrt(var + _EPS)
        h = (d["x"] - mean) / sd
        out = {"y": torch.addcmul(d["beta"], h, d["gamma"])}
        if kind == "norm_step":
            g = d["dy"] * d["gamma"]
            D = case["D"]
            out["dx"] = (D * g - g.sum(1, keepdim=True) - h * torch.linalg.vecdot(g, h)[:, None]) / (D * sd)
            out["dgamma"], out["dbeta"] = torch.linalg.vecdot(d["dy"], h, dim=0), d["dy"].sum(0)
        return out
    # the rows a few at a time: the teacher's distribution spread over the vocabulary, its sum with log(p / q)
    R, V, T = case["R"], case["V"], case["T"]
    loss = torch.zeros(R, dtype=torch.float64, device="cuda")
    grad = torch.zeros((R, V), dtype=torch.float32 if R * V > 1 << 29 else torch.float64, device="cuda")
    step = max(1, (1 << 26) // V)
    for at in range(0, R, step):
        part = slice(at, at + step)
        idx, w = s["indices"][part].long(), d["weight"][part]
        log_t = torch.full((idx.shape[0], V + 1), -math.inf, dtype=torch.float64, device="cuda")
        log_t.scatter_(1, torch.where(idx < 0, V, idx), d["values"][part] / T)
        log_t = log_t[:, :V]
        used = (idx >= 0).any(1) & (w != 0)
        log_p = torch.log_softmax(torch.where(used[:, None], log_t, torch.zeros_like(log_t)), dim=1)
        log_q = torch.log_softmax(s["logits"][part].double() / T, dim=1)
        p = torch.exp(log_p)
        each = torch.where(p > 0, p * (log_p - log_q), torch.zeros_like(p)).sum(1)
        loss[part] = torch.where(used, w * T * T * each, torch.zeros_like(each))
        grad[part] = torch.where(used[:, None], (w * T)[:, None] * (torch.exp(log_q) - p), torch.zeros_like(p)).to(grad.dtype)
    return {"loss": loss, "grad": grad}
