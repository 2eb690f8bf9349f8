"""Group normalization and learning from a teacher's top logits, as cases that can be timed and compared.

A case names one call of the framework (its "op") and its sizes:

  gn_fwd    group normalization of a channels-last tensor with the residual add and the activation behind it, and the
            statistics that the backward pass needs
  gn_bwd    its backward pass: gradients of the input, the residual, gamma and beta
  topk      the largest logits of each row with their class indices, in falling order: what is kept of a teacher
  distill   cross-entropy with the label and with the teacher's kept logits at a temperature: the loss and the gradient of
            the logits

Group normalization takes the statistics of a group of neighbouring channels of one image, so a worker's result does not
depend on how many images it has.  With m = H*W*C/G values to a group:
  mean = sum x / m,  var = sum (x - mean)^2 / m,  xhat = (x - mean) / sqrt(var + eps)
  u = gamma*xhat + beta [+ residual],  y = act(u)
  dz = (dy [+ dy2]) * act'(u),  dresidual = dz,  dbeta = sum dz,  dgamma = sum dz*xhat
  dx = (gamma*dz - mean(gamma*dz) - xhat*mean(gamma*dz*xhat)) / sqrt(var + eps)      (means over the group)

A row of the distillation loss, with q = softmax(z), r = softmax(z/tau), p = softmax(v/tau) over the teacher's kept logits v
(class index i_t each; an index of -1 keeps nothing, a row without any has no soft term, one with label -1 no hard term):
  hard = -log q[label],  soft = tau^2 * sum_t p_t (log p_t - log r[i_t])
  loss = scale * sum over rows of (1 - alpha)*hard + alpha*soft
  dz = scale * ((1 - alpha)*(q - onehot) + alpha*tau*(r - sum over t with i_t = k of p_t))

dtype: "f32" or "bf16" (the activations or the logits; parameters, statistics, the teacher's logits and losses are fp32).
"""
import math

import torch

DEV = "cuda:0"
EPS = 1e-5
own = False


def listed():
    return [
        # evaluation of one image in the last stage: the call itself is what it costs
        {"name": "gn_fwd_n1_c512_h7", "op": "gn_fwd", "n": 1, "c": 512, "h": 7, "w": 7, "g": 32, "act": "relu", "res": True, "dtype": "f32"},
        # the end of a stage-2 block at a large batch, activations kept as bf16
        {"name": "gn_fwd_n128_c256_h56_bf16", "op": "gn_fwd", "n": 128, "c": 256, "h": 56, "w": 56, "g": 32, "act": "relu", "res": True, "dtype": "bf16"},
        # a few large images of odd sizes, groups of ten channels, the smooth activation
        {"name": "gn_fwd_n3_c320_h129_w131", "op": "gn_fwd", "n": 3, "c": 320, "h": 129, "w": 131, "g": 32, "act": "silu", "res": False, "dtype": "f32"},
        # the first layer's output on the paper's 32 images: groups of two channels and the most pixels
        {"name": "gn_bwd_n32_c64_h112", "op": "gn_bwd", "n": 32, "c": 64, "h": 112, "w": 112, "g": 32, "act": "relu", "res": False, "dy2": False, "dtype": "f32"},
        # the end of a stage-4 block: both gradients of the fork arrive, the shortcut's leaves
        {"name": "gn_bwd_n64_c1024_h14_bf16", "op": "gn_bwd", "n": 64, "c": 1024, "h": 14, "w": 14, "g": 32, "act": "relu", "res": True, "dy2": True, "dtype": "bf16"},
        # a few small images of odd sizes
        {"name": "gn_bwd_n2_c320_h33_w35", "op": "gn_bwd", "n": 2, "c": 320, "h": 33, "w": 35, "g": 32, "act": "silu", "res": False, "dy2": False, "dtype": "f32"},
        # a teacher's logits of one worker's 32 images
        {"name": "topk_n32_k1000_t10", "op": "topk", "n": 32, "k": 1000, "pad": 0, "t": 10, "dtype": "f32"},
        # a teacher's logits of many positions over a large vocabulary
        {"name": "topk_n4096_k32768_t64_bf16", "op": "topk", "n": 4096, "k": 32768, "pad": 0, "t": 64, "dtype": "bf16"},
        # one long row of odd length
        {"name": "topk_n1_k131071_t32", "op": "topk", "n": 1, "k": 131071, "pad": 1, "t": 32, "dtype": "f32"},
        # the loss of one worker's 32 images
        {"name": "distill_n32_k1000_t10", "op": "distill", "n": 32, "k": 1000, "pad": 0, "t": 10, "alpha": 0.5, "tau": 4.0, "dtype": "f32"},
        # many positions over a large vocabulary
        {"name": "distill_n4096_k32768_t64_bf16", "op": "distill", "n": 4096, "k": 32768, "pad": 0, "t": 64, "alpha": 0.75, "tau": 2.0, "dtype": "bf16"},
        # a few rows of an odd length, padded in memory, from the teacher alone
        {"name": "distill_n7_k100003_t50", "op": "distill", "n": 7, "k": 100003, "pad": 5, "t": 50, "alpha": 1.0, "tau": 1.0, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op, dtype = rng.choice(("gn_fwd", "gn_bwd", "topk", "distill")), rng.choice(("f32", "bf16"))
    if op in ("gn_fwd", "gn_bwd"):
        g = rng.choice((1, 2, 4, 8, 16, 32, 32, 32))
        per = _log(rng, 1, 64)
        while g * per % 4 or g * per > 2048:
            per = _log(rng, 1, 64)
        c, h = g * per, _log(rng, 1, 132)
        w = h if rng.random() < 0.5 else _log(rng, 1, 132)
        if per * h * w < 16:   # of so few values little is left behind mean and variance: dx is a difference of near-equal numbers
            h = w = 4
        most = (102_000_000 if dtype == "bf16" else 25_000_000) if op == "gn_fwd" else 25_000_000   # values of the largest listed case
        n = _log(rng, 1, max(1, min(128, most // (c * h * w))))
        case = {"op": op, "n": n, "c": c, "h": h, "w": w, "g": g, "act": rng.choice(("none", "relu", "silu")), "res": rng.random() < 0.5, "dtype": dtype}
        if op == "gn_bwd":
            case["dy2"] = rng.random() < 0.5
        return case
    n, k = _log(rng, 1, 4096), _log(rng, 2, 131072)
    while n * k > (134_000_000 if dtype == "bf16" else 67_000_000):
        n, k = _log(rng, 1, 4096), _log(rng, 2, 131072)
    case = {"op": op, "n": n, "k": k, "pad": rng.choice((0, 0, 1, 6, 64)), "t": _log(rng, 1, min(256, k)), "dtype": dtype}
    if op == "distill":
        case.update(alpha=rng.choice((0.25, 0.5, 0.75, 1.0)), tau=rng.choice((1.0, 1.5, 2.0, 4.0)))
    return case


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ---- group normalization --------------------------------------------------------------------------------------------------
def _grouped(v, g):
    """N x H x W x C as N x H*W x G x C/G."""
    n, h, w, c = v.shape
    return v.reshape(n, h * w, g, c // g)


def _gn_stats(x, g):
    v = _grouped(x.float(), g)
    mean = v.mean((1, 3))
    var = (v - mean[:, None, :, None]).square().mean((1, 3))
    return mean, (var + EPS).rsqrt()


def _gn_pre(x, g, gamma, beta, mean, invstd, residual):
    """(xhat, u), both N x H x W x C in 32 bits."""
    xhat = ((_grouped(x.float(), g) - mean[:, None, :, None]) * invstd[:, None, :, None]).reshape(x.shape)
    u = xhat * gamma + beta
    return xhat, u if residual is None else u + residual.float()


def _gn_fwd(x, g, gamma, beta, residual, act):
    mean, invstd = _gn_stats(x, g)
    u = _gn_pre(x, g, gamma, beta, mean, invstd, residual)[1]
    y = u if act == "none" else u.clamp(min=0) if act == "relu" else u * torch.sigmoid(u)
    return y.to(x.dtype), mean, invstd


def _gn_bwd(x, dy, dy2, g, gamma, beta, mean, invstd, residual, act):
    xhat, u = _gn_pre(x, g, gamma, beta, mean, invstd, residual)
    dz = dy.float() if dy2 is None else dy.float() + dy2.float()
    if act == "relu":
        dz = dz * (u > 0)
    elif act == "silu":
        s = torch.sigmoid(u)
        dz = dz * (s * (1 + u * (1 - s)))
    dgamma, dbeta = (dz * xhat).sum((0, 1, 2)), dz.sum((0, 1, 2))
    a, xg = _grouped(dz * gamma, g), _grouped(xhat, g)
    dx = (a - a.mean((1, 3), keepdim=True) - xg * (a * xg).mean((1, 3), keepdim=True)) * invstd[:, None, :, None]
    return dx.reshape(x.shape).to(x.dtype), dz.to(x.dtype) if residual is not None else None, dgamma, dbeta


def _off_corner(s, g):
    x = s["x"].float()
    u = _gn_pre(x, g, s["gamma"], s["beta"], *_gn_stats(x, g), s["res"])[1]
    away = torch.where(u < 0, -0.02, 0.02) * (1 + x.abs())   # beyond the spacing of bf16 numbers there
    s["x"] = torch.where(u.abs() < 2e-3, x + away, x).to(s["x"].dtype)


def _gn_inputs(case, gen):
    n, c, h, w, g = (case[k] for k in "nchwg")
    shape, dt = (n, h, w, c), _type(case)

    def normal(*size):
        return torch.randn(size, generator=gen, device=DEV)

    # channels of different scales and means, as a convolution leaves them
    x = (normal(*shape) * (0.5 + torch.rand(c, generator=gen, device=DEV)) + normal(c)).to(dt)
    s = {"case": case, "x": x, "gamma": 1 + 0.1 * normal(c), "beta": 0.1 * normal(c), "res": normal(*shape).to(dt) if case["res"] else None}
    if case["op"] == "gn_bwd":
        if case["act"] == "relu":
            # a value within rounding of the ReLU's corner has either gradient: such values (some in a thousand) are moved off it;
            # that moves the statistics a little, and with them a few others
            _off_corner(s, g)
            _off_corner(s, g)
        s["mean"], s["invstd"] = _gn_stats(s["x"], g)
        s["dy"] = normal(*shape).to(dt)
        s["dy2"] = normal(*shape).to(dt) if case["dy2"] else None
    return s


def _gn_exact(case, seed):
    n, c, h, w, g = (case[k] for k in "nchwg")
    s = prepare(case, seed)
    per = c // g

    def images(t):
        return t.double().view(n, h * w, c).transpose(1, 2).reshape(n * g, per * h * w)   # a row for each group

    def back(t):
        return t.view(n, c, h * w).transpose(1, 2).reshape(n, h, w, c)

    def channels(t):
        return t.double().view(1, g, per, 1).expand(n, g, per, h * w).reshape(n * g, per * h * w)

    x = images(s["x"])
    if case["op"] == "gn_fwd":
        mean = x.sum(1, keepdim=True) / x.shape[1]
        sigma = ((x * x).sum(1, keepdim=True) / x.shape[1] - mean * mean + EPS).sqrt()
    else:
        mean, sigma = s["mean"].double().view(-1, 1), 1 / s["invstd"].double().view(-1, 1)
    xhat = (x - mean) / sigma
    del x
    u = channels(s["gamma"]) * xhat + channels(s["beta"])
    if s["res"] is not None:
        u = u + images(s["res"])
    if case["op"] == "gn_fwd":
        y = u if case["act"] == "none" else torch.maximum(u, torch.zeros_like(u)) if case["act"] == "relu" else u / (1 + torch.exp(-u))
        return {"y": back(y), "mean": mean.view(n, g), "invstd": 1 / sigma.view(n, g)}
    dz = images(s["dy"])
    if s["dy2"] is not None:
        dz = dz + images(s["dy2"])
    if case["act"] == "relu":
        dz = torch.where(u > 0, dz, torch.zeros_like(dz))
    elif case["act"] == "silu":
        e = torch.exp(-u)
        dz = dz * ((1 + e + u * e) / (1 + e) ** 2)
    del u
    dgamma = (dz * xhat).view(n, c, h * w).sum(2).sum(0)
    dbeta = dz.view(n, c, h * w).sum(2).sum(0)
    a = channels(s["gamma"]) * dz
    m = a.shape[1]
    dx = (a - (a.sum(1, keepdim=True) + xhat * (a * xhat).sum(1, keepdim=True)) / m) / sigma
    return {"dx": back(dx), "dgamma": dgamma, "dbeta": dbeta, **({"dres": back(dz)} if s["res"] is not None else {})}


# ---- the teacher's top logits ---------------------------------------------------------------------------------------------
def _topk(z, t):
    """Values (32 bits) and indices of the t largest of each row, falling; equal ones by rising index."""
    k = z.shape[1]
    bits = z.float().contiguous().view(torch.int32)
    bits = torch.where(bits == -2 ** 31, torch.zeros_like(bits), bits)   # -0 and 0 are equal
    order = (bits ^ ((bits >> 31) & 0x7fffffff)).to(torch.int64)
    order = torch.where(torch.isnan(z), torch.full_like(order, 0x7fffffff), order)
    keys = (order << 32) | (0xffffffff - torch.arange(k, device=z.device))
    best = 0xffffffff - (torch.topk(keys, t, dim=1).values & 0xffffffff)
    return z.float().gather(1, best), best.to(torch.int32)


def _logits(case, gen):
    """n x (k + pad) in memory: normal logits, some classes far above the rest, the padding filled with a value that nobody may read."""
    n, k, pad = case["n"], case["k"], case["pad"]
    z = torch.randn((n, k + pad), generator=gen, device=DEV) * 2
    peaks = torch.randint(0, k, (n, 1 + k // 200), generator=gen, device=DEV)
    hit = torch.zeros_like(z).scatter_(1, peaks, 10.0)   # one value for all, so that it does not matter which of two comes last
    z.addcmul_(hit, torch.rand(z.shape, generator=gen, device=DEV))
    del hit
    z[:, k:] = 1e4
    return z.to(_type(case))


# ---- distillation ---------------------------------------------------------------------------------------------------------
def _distill(z, labels, idx, val, alpha, tau, scale):
    n, k = z.shape
    zf = z.float()
    shifted = zf - zf.amax(1, keepdim=True)
    hot = shifted / tau
    e = torch.exp(hot)
    total = e.sum(1, keepdim=True)
    kept = idx >= 0
    at = idx.clamp(min=0).long()
    v = torch.where(kept, val, torch.full_like(val, -math.inf)) / tau
    some = kept.any(1, keepdim=True)
    v = torch.where(some, v - v.amax(1, keepdim=True), torch.zeros_like(v))
    ev = torch.where(kept, torch.exp(v), torch.zeros_like(v))
    p = torch.where(some, ev / ev.sum(1, keepdim=True), torch.zeros_like(ev))
    log_p = v - torch.log(ev.sum(1, keepdim=True))
    log_r = hot.gather(1, at) - torch.log(total)
    soft = tau * tau * torch.where(p > 0, p * (log_p - log_r), torch.zeros_like(p)).sum(1)
    grad = torch.where(some, alpha * tau * (e / total), torch.zeros_like(e))
    grad.scatter_add_(1, at, -alpha * tau * p)
    if labels is None:
        hard = torch.zeros_like(soft)
    else:
        has = (labels >= 0)[:, None]
        y = labels.clamp(min=0).long()[:, None]
        e1 = torch.exp(shifted)
        sum1 = e1.sum(1, keepdim=True)
        hard = torch.where(has, torch.log(sum1) - shifted.gather(1, y), torch.zeros_like(sum1))[:, 0]
        grad = grad + torch.where(has, (1 - alpha) * (e1 / sum1), torch.zeros_like(e1))
        grad.scatter_add_(1, y, torch.where(has, torch.full_like(sum1, alpha - 1), torch.zeros_like(sum1)))
    hard, soft = hard.double().sum() * scale, soft.double().sum() * scale
    return torch.stack(((1 - alpha) * hard + alpha * soft, hard, soft)).float(), (grad * scale).to(z.dtype)


def _distill_exact(case, seed):
    n, k, t, alpha, tau = (case[key] for key in ("n", "k", "t", "alpha", "tau"))
    s = prepare(case, seed)
    z, labels, idx, val = s["z"][:, :k].double(), s["labels"], s["idx"], s["val"].double()
    grad = torch.zeros_like(z)
    soft = hard = torch.zeros((), dtype=torch.float64, device=DEV)
    rows = (idx >= 0).any(1).nonzero()[:, 0]
    log_r = torch.log_softmax(z / tau, 1)
    grad[rows] = alpha * tau * log_r[rows].exp()
    log_p = torch.log_softmax(torch.where(idx >= 0, val / tau, torch.full_like(val, -math.inf))[rows], 1)
    i = idx[rows].clamp(min=0).long()
    there = idx[rows] >= 0
    soft = (tau * tau * torch.where(there, log_p.exp() * (log_p - log_r[rows].gather(1, i)), torch.zeros_like(log_p))).sum()
    grad.index_put_((rows[:, None].expand_as(i), i), torch.where(there, -alpha * tau * log_p.exp(), torch.zeros_like(log_p)), accumulate=True)
    del log_r
    if labels is not None:
        rows = (labels >= 0).nonzero()[:, 0]
        y = labels[rows].long()
        log_q = torch.log_softmax(z[rows], 1)
        hard = -log_q.gather(1, y[:, None]).sum()
        log_q = log_q.exp_()
        log_q[torch.arange(len(rows), device=DEV), y] -= 1
        grad.index_add_(0, rows, log_q, alpha=1 - alpha)
    hard, soft = hard * s["scale"], soft * s["scale"]
    return {"loss": torch.stack(((1 - alpha) * hard + alpha * soft, hard, soft)), "dlogits": grad * s["scale"]}


# ---- what the tools call --------------------------------------------------------------------------------------------------
def _room(n, *shape_type):
    return torch.empty(n, *shape_type[:-1], dtype=shape_type[-1], device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    op, n, dt = case["op"], case["n"], _type(case)
    if op in ("gn_fwd", "gn_bwd"):
        s = _gn_inputs(case, gen)
        c, g = case["c"], case["g"]
        # the caller's own buffers, which the framework's calls write
        s["out"] = torch.empty_like(s["x"])
        s["dres"] = torch.empty_like(s["x"]) if op == "gn_bwd" and s["res"] is not None else None
        s["stats"] = (_room(n, g, torch.float32), _room(n, g, torch.float32))
        s["params"] = (_room(c, torch.float32), _room(c, torch.float32))
        if own:
            from paper_1711_04325_amd import binding as rn
            s["ws"] = _room(max(16, rn.rn50_gn_workspace_bytes(n, c, case["h"], case["w"], g)), torch.uint8)
        return s
    k, t = case["k"], case["t"]
    s = {"case": case, "z": _logits(case, gen)}
    if op == "topk":
        s["val"], s["idx"] = _room(n, t, torch.float32), _room(n, t, torch.int32)
    else:
        # a teacher that agrees with the student in part; one row in sixteen keeps fewer logits, one in sixteen none
        teacher = s["z"][:, :k].float() * 0.7 + torch.randn((n, k), generator=gen, device=DEV)
        s["val"], idx = torch.topk(teacher, t, dim=1)
        del teacher
        few = torch.rand(n, generator=gen, device=DEV)
        keep = torch.where(few < 1 / 16, 0, torch.where(few < 1 / 8, (t + 1) // 2, t)) if n > 1 else torch.full((1,), t, device=DEV)
        s["idx"] = torch.where(torch.arange(t, device=DEV) < keep[:, None], idx, -1).to(torch.int32)
        s["labels"] = None
        if case["alpha"] < 1:
            labels = torch.randint(0, k, (n,), generator=gen, device=DEV, dtype=torch.int32)
            # one position in eight is padding without a label
            s["labels"] = torch.where(torch.rand(n, generator=gen, device=DEV) < 1 / 8, -1, labels).to(torch.int32) if n > 1 else labels
        s["scale"] = float(torch.tensor(1 / n, dtype=torch.float32))
        s["loss"], s["dz"] = _room(3, torch.float32), _room(n, k + case["pad"], dt)
    if own:
        from paper_1711_04325_amd import binding as rn
        need = rn.rn50_topk_workspace_bytes(n, k, t) if op == "topk" else rn.rn50_distill_workspace_bytes(n, k, t)
        s["ws"] = _room(max(16, need), torch.uint8)
    return s


def run(s):
    case = s["case"]
    op, n = case["op"], case["n"]
    if own:
        return _run_own(s, case, op, n)
    if op == "gn_fwd":
        y, mean, invstd = _gn_fwd(s["x"], case["g"], s["gamma"], s["beta"], s["res"], case["act"])
        return {"y": y, "mean": mean, "invstd": invstd}
    if op == "gn_bwd":
        dx, dres, dgamma, dbeta = _gn_bwd(s["x"], s["dy"], s["dy2"], case["g"], s["gamma"], s["beta"], s["mean"], s["invstd"], s["res"], case["act"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta, **({"dres": dres} if dres is not None else {})}
    z = s["z"][:, :case["k"]]
    if op == "topk":
        val, idx = _topk(z, case["t"])
        return {"val": val, "idx": idx}
    loss, dz = _distill(z, s["labels"], s["idx"], s["val"], case["alpha"], case["tau"], s["scale"])
    return {"loss": loss, "dlogits": dz}


def _run_own(s, case, op, n):
    from paper_1711_04325_amd import binding as rn
    bf16 = case["dtype"] == "bf16"
    if op in ("gn_fwd", "gn_bwd"):
        c, h, w, g = (case[k] for k in "chwg")
        act = {"none": rn.ACT_NONE, "relu": rn.ACT_RELU, "silu": rn.ACT_SILU}[case["act"]]
        if op == "gn_fwd":
            fwd = rn.gn_fwd_bf16 if bf16 else rn.gn_fwd
            fwd(n, c, h, w, g, s["x"], s["gamma"], s["beta"], EPS, s["res"], act, s["out"], *s["stats"], s["ws"])
            return {"y": s["out"], "mean": s["stats"][0], "invstd": s["stats"][1]}
        bwd = rn.gn_bwd_bf16 if bf16 else rn.gn_bwd
        bwd(n, c, h, w, g, s["x"], s["dy"], s["dy2"], s["res"], s["gamma"], s["beta"], s["mean"], s["invstd"], act, s["out"], s["dres"],
            *s["params"], s["ws"])
        return {"dx": s["out"], "dgamma": s["params"][0], "dbeta": s["params"][1], **({"dres": s["dres"]} if s["dres"] is not None else {})}
    k, t = case["k"], case["t"]
    ld = k + case["pad"]
    if op == "topk":
        top = rn.logits_topk_bf16 if bf16 else rn.logits_topk
        top(n, k, t, s["z"], ld, s["val"], s["idx"], s["ws"])
        return {"val": s["val"], "idx": s["idx"]}
    distill = rn.distill_ce_bf16 if bf16 else rn.distill_ce
    distill(n, k, t, s["z"], ld, s["labels"], s["idx"], s["val"], case["alpha"], case["tau"], s["scale"], s["loss"], s["dz"], ld, s["ws"])
    return {"loss": s["loss"], "dlogits": s["dz"][:, :k]}


def exact(case, seed):
    """The same outputs by their definitions in 64 bits."""
    if case["op"] in ("gn_fwd", "gn_bwd"):
        return _gn_exact(case, seed)
    if case["op"] == "distill":
        return _distill_exact(case, seed)
    z = prepare(case, seed)["z"][:, :case["k"]]
    return {"val": z.double().sort(1, descending=True).values[:, :case["t"]], "idx": None}


def work(case):
    op, n, size = case["op"], case["n"], 4 if case["dtype"] == "f32" else 2
    if op in ("gn_fwd", "gn_bwd"):
        values, c, stats = n * case["c"] * case["h"] * case["w"], case["c"], 2 * n * case["g"]
        if op == "gn_fwd":
            tensors = 2 + case["res"]                              # x, y, the residual
            return {"bytes": values * size * tensors + 4 * (2 * c + stats), "flops": values * (8 + (5 if case["act"] == "silu" else 0))}
        tensors = 3 + case["dy2"] + 2 * case["res"]                # x, dy, dx, the second gradient, the residual and its gradient
        return {"bytes": values * size * tensors + 4 * (4 * c + stats), "flops": values * (16 + (10 if case["act"] == "silu" else 0))}
    k, t = case["k"], case["t"]
    if op == "topk":
        return {"bytes": n * k * size + n * t * 8, "flops": n * k}
    kinds = (2 if case["alpha"] < 1 and case["tau"] != 1 else 1)   # softmaxes of a row
    return {"bytes": 2 * n * k * size + n * (8 * t + 4) + 12, "flops": n * k * 6 * kinds}
