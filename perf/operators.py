"""The operators of a router's training step, as cases that can be timed.

  balance  eqb_balance_loss: per-expert counts, the balance loss with its
           z-loss, and their gradient with respect to the router logits
  rgrad    eqb_router_grad: the gradient of the router projection with respect
           to its input (dx) and its weight (dW)
  adamw    EqbAdamW.step: one AdamW step over many tensors, with states in 32
           or in 8 bits

`run` computes them in plain torch operations in 32 bits, or with the
package's calls where `own` is true; `exact` from the formulas in 64 bits.
Sizes are the repository's configurations (tiny, mid, global, router, wide),
its serving and ragged shapes, and generic ones between them.
"""
import math

import torch

own = False

ALPHA = 0.1    # weight of the balance loss
ZETA = 1e-3    # weight of the z-loss
LR, BETA1, BETA2, EPS, WD, STEP = 2e-4, 0.9, 0.95, 1e-8, 0.1, 1000
BLOCK = 256    # elements that share a scale in 8-bit states
TOP = 448.0    # largest e4m3 value
LEAST = 2.0 ** -9  # least positive e4m3 value


def listed():
    return [
        # The smallest training step's loss and gradient, added to the score gradients in place: latency.
        {"name": "balance_tiny", "kind": "balance", "T": 4096, "E": 8, "K": 2, "M": 4, "score": "softmax", "zeta": 0.0, "z": "bf16", "grad": "add", "mask": False},
        # Monitoring a run: counts, mean probabilities and loss, no gradient.
        {"name": "balance_value", "kind": "balance", "T": 524288, "E": 128, "K": 8, "M": 32, "score": "sigmoid", "zeta": 0.0, "z": "bf16", "grad": "none", "mask": False},
        # The headline training shape: loss, z-loss and a bf16 gradient for the projection's backward pass.
        {"name": "balance_global", "kind": "balance", "T": 2097152, "E": 256, "K": 8, "M": 64, "score": "softmax", "zeta": ZETA, "z": "bf16", "grad": "bf16", "mask": False},
        # A loss per sequence: 700 uneven sequences (some empty), padding tokens that hold garbage, fp32 logits.
        {"name": "balance_seqs", "kind": "balance", "T": 200003, "E": 96, "K": 6, "M": 700, "score": "sigmoid", "zeta": 0.0, "z": "fp32", "grad": "add", "mask": True},
        # A short microbatch of a small router.
        {"name": "rgrad_short", "kind": "rgrad", "T": 300, "d": 1024, "E": 64, "add": False},
        # A prefill-sized batch, no multiple of a tile, many experts.
        {"name": "rgrad_ragged", "kind": "rgrad", "T": 16411, "d": 2048, "E": 256, "add": False},
        # One of the 16 microbatches of the router configuration, added to the gradients that are there.
        {"name": "rgrad_router", "kind": "rgrad", "T": 65536, "d": 4096, "E": 128, "add": True},
        # One layer's router and its norm weight: latency.
        {"name": "adamw_layer", "kind": "adamw", "sizes": "layer", "count": 2, "n": 525000, "p": "fp32", "g": "fp32", "bits": 32, "copy": True, "shift": 0},
        # The routers of 48 MoE layers: fp32 masters, bf16 copies for the projection.
        {"name": "adamw_routers", "kind": "adamw", "sizes": "even", "count": 48, "n": 48 * 128 * 4096, "p": "fp32", "g": "fp32", "bits": 32, "copy": True, "shift": 0},
        # One layer's experts: 64 x 3 matrices, bf16 gradients, some experts without a token.
        {"name": "adamw_experts", "kind": "adamw", "sizes": "even", "count": 192, "n": 192 * 2048 * 1024, "p": "fp32", "g": "bf16", "bits": 32, "copy": True, "shift": 0},
        # The same experts where memory is short: bf16 weights, states in 8 bits.
        {"name": "adamw_experts8", "kind": "adamw", "sizes": "even", "count": 192, "n": 192 * 2048 * 1024, "p": "bf16", "g": "bf16", "bits": 8, "copy": False, "shift": 0},
        # Adapters, norms and biases of odd sizes (some empty), views that start one element late in their buffer.
        {"name": "adamw_odd8", "kind": "adamw", "sizes": "odd", "count": 300, "n": 6000000, "p": "bf16", "g": "fp32", "bits": 8, "copy": False, "shift": 1},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["balance", "balance", "rgrad", "rgrad", "adamw", "adamw"])
    if kind == "balance":
        E = rng.choice([8, 16, 40, 64, 96, 128, 160, 256, 256, 264, 384, 512, 1000, 1024])
        T = _log_int(rng, 1, min(2097152, (1 << 29) // E))
        score = rng.choice(["softmax", "softmax", "sigmoid"])
        return {"kind": kind, "T": T, "E": E, "K": rng.choice([k for k in (1, 2, 6, 8, 12) if k < E]),
                "M": _log_int(rng, 1, max(1, min(2000, T // 8))), "score": score,
                "zeta": ZETA if score == "softmax" and rng.random() < 0.5 else 0.0, "z": rng.choice(["bf16", "bf16", "fp32"]),
                "grad": rng.choice(["none", "add", "fp32", "bf16"]), "mask": rng.random() < 0.4}
    if kind == "rgrad":
        d = 64 * _log_int(rng, 1, 64)
        return {"kind": kind, "T": _log_int(rng, 1, 65536), "d": 4096 if d == 3072 else d,
                "E": rng.choice([16, 48, 64, 96, 128, 128, 256]), "add": rng.random() < 0.5}
    count = _log_int(rng, 1, 400)
    bits = rng.choice([8, 32])
    p = rng.choice(["fp32", "bf16"])
    return {"kind": kind, "sizes": rng.choice(["even", "odd"]) if count > 1 else "even", "count": count,
            "n": _log_int(rng, max(1000, 4 * count), 300000000), "p": p, "g": rng.choice(["fp32", "bf16"]), "bits": bits,
            "copy": p == "fp32" and rng.random() < 0.5, "shift": 1 if rng.random() < 0.2 else 0}


# ---- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(std)


def _offsets(case, g):
    T, M = case["T"], case["M"]
    if not case["mask"]:
        return torch.div(torch.arange(M + 1, device="cuda") * T, M, rounding_mode="floor")
    cuts = torch.randint(0, T + 1, (M - 1,), generator=g, device="cuda").sort().values
    ends = torch.tensor([0, T], device="cuda")
    return torch.cat([ends[:1], cuts, ends[1:]])


def _prepare_balance(case, seed):
    g = _gen(seed)
    T, E, K, M = case["T"], case["E"], case["K"], case["M"]
    z = _normal((T, E), g) + _normal((E,), g, 0.5)  # some experts are liked more than others
    # a list of K distinct experts: the largest of the logits with some noise, in descending order
    idx = torch.empty((T, K), dtype=torch.int32, device="cuda")
    for a in range(0, T, 1 << 18):
        idx[a:a + (1 << 18)] = torch.topk(z[a:a + (1 << 18)] + _normal((min(T - a, 1 << 18), E), g, 0.1), K).indices.int()
    off = _offsets(case, g)
    s = {"case": case, "idx": idx, "off": off, "mask": None}
    if case["mask"]:
        s["mask"] = torch.rand(T, generator=g, device="cuda") < 0.8
        z[~s["mask"]] = math.nan         # nobody has computed these rows
        idx[~s["mask"]] = -1
        z[::7, E // 2] = -math.inf       # an expert that is closed to some tokens
        z[3::1009] = torch.where(s["mask"][3::1009, None], -math.inf, z[3::1009])  # and all of them
        idx[5::11, K - 1] = -1           # lists that a capacity limit has cut short
    s["z"] = z.bfloat16() if case["z"] == "bf16" else z
    s["grad_in"] = _normal((T, E), g, 1e-5) if case["grad"] in ("add", "bf16") else None
    # the loss is summed over the tokens of a microbatch, not averaged
    s["scale"] = torch.full((1,), float(max(1, T // M)), device="cuda")
    s["grad_out"] = {"none": None, "add": s["grad_in"], "fp32": torch.empty((T, E), device="cuda") if case["grad"] == "fp32" else None,
                     "bf16": torch.empty((T, E), dtype=torch.bfloat16, device="cuda") if case["grad"] == "bf16" else None}[case["grad"]]
    s["counts"] = torch.empty((M, E), dtype=torch.int32, device="cuda")
    s["prob"] = torch.empty((M, E), device="cuda")
    s["loss"] = torch.empty((M, 2), device="cuda")
    if own:
        import paper_2609_28053_gb300 as eqb
        s["workspace"] = torch.empty(eqb.eqb_balance_loss_workspace_bytes(T, E, M), dtype=torch.uint8, device="cuda")
    return s


def _prepare_rgrad(case, seed):
    g = _gen(seed)
    T, d, E = case["T"], case["d"], case["E"]
    s = {"case": case, "dz": _normal((T, E), g, 1e-2).bfloat16(), "x": _normal((T, d), g).bfloat16(),
         "W": _normal((E, d), g, d ** -0.5).bfloat16()}
    s["dx"] = _normal((T, d), g, 1e-2).bfloat16() if case["add"] else torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    s["dW"] = _normal((E, d), g) if case["add"] else torch.empty((E, d), device="cuda")
    if own:
        import paper_2609_28053_gb300 as eqb
        s["workspace"] = torch.empty(eqb.eqb_router_grad_workspace_bytes(T, d, E), dtype=torch.uint8, device="cuda")
    return s


def _sizes(case):
    """The tensors' lengths, from the case alone."""
    n, c = case["n"], case["count"]
    if case["sizes"] == "even":
        return [n // c] * c
    if case["sizes"] == "layer":
        return [n - 1000, 1000]
    # odd lengths over four decades, every 29th tensor empty
    w = [0.0 if i % 29 == 28 else math.exp(9.2 * ((i * 0.618034) % 1.0)) for i in range(c)]
    return [int(n * x / sum(w)) | 1 if x else 0 for x in w]


def _blocks(case):
    return sum((n + BLOCK - 1) // BLOCK for n in _sizes(case))


def _views(flat, sizes):
    """Each tensor's part of a flat buffer in which every tensor starts at a multiple of BLOCK elements."""
    got, at = [], 0
    for n in sizes:
        got.append(flat[at:at + n])
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    return got


def _prepare_adamw(case, seed):
    g = _gen(seed)
    sizes = _sizes(case)
    nb = _blocks(case)
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}
    # zero in the gaps between tensors
    lens = torch.tensor(sizes, device="cuda")
    blk = torch.div(lens + BLOCK - 1, BLOCK, rounding_mode="floor")
    first = torch.cumsum(blk, 0) - blk
    which = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), blk)
    left = lens[which] - (torch.arange(nb, device="cuda") - first[which]) * BLOCK
    live = torch.arange(BLOCK, device="cuda")[None] < left[:, None]

    def flat(v, dtype):
        buf = torch.zeros(nb * BLOCK + case["shift"], dtype=dtype, device="cuda")
        out = buf[case["shift"]:]
        out.copy_((v * live).view(-1))
        return out

    size = torch.exp(_normal((nb, 1), g))                    # gradients differ from block to block
    size = size * (which % 13 != 12)[:, None]                # an expert without a token
    s = {"case": case}
    s["p"] = flat(_normal((nb, BLOCK), g, 0.02), dt[case["p"]])
    s["g"] = flat(_normal((nb, BLOCK), g, 1e-3) * size, dt[case["g"]])
    m = _normal((nb, BLOCK), g, 3e-4) * size * live
    v = (_normal((nb, BLOCK), g, 1e-3) * size).square_().add_(1e-8 * size * size).mul_(live)
    if case["bits"] == 32:
        s["m"], s["v"] = m.view(-1), v.view(-1)
    else:
        s["m"], s["ms"] = _to8(m, False)
        s["v"], s["vs"] = _to8(v.sqrt(), True)
    s["scale"] = torch.full((1,), 0.5, device="cuda")        # the clipping factor of this step
    s["copy"] = s["p"].bfloat16() if case["copy"] else None
    if own:
        import paper_2609_28053_gb300 as eqb
        s["grads"] = _views(s["g"], sizes)
        more = {"copies": _views(s["copy"], sizes)} if case["copy"] else {}
        if case["bits"] == 8:
            each = [(n + BLOCK - 1) // BLOCK for n in sizes]
            more |= {"avg_scale": list(s["ms"].split(each)), "sq_scale": list(s["vs"].split(each))}
        s["opt"] = eqb.EqbAdamW(_views(s["p"], sizes), state_bits=case["bits"], exp_avg=_views(s["m"], sizes),
                                exp_avg_sq=_views(s["v"], sizes), **more)
    return s


def prepare(case, seed):
    return {"balance": _prepare_balance, "rgrad": _prepare_rgrad, "adamw": _prepare_adamw}[case["kind"]](case, seed)


# ---- the plain forms

def _balance_plain(s):
    c = s["case"]
    T, E, K, M = c["T"], c["E"], c["K"], c["M"]
    z, idx, off = s["z"].float(), s["idx"], s["off"]
    seg = torch.searchsorted(off, torch.arange(T, device=z.device), right=True) - 1
    valid = torch.ones(T, dtype=torch.bool, device=z.device) if s["mask"] is None else s["mask"]
    n = torch.zeros(M, device=z.device).index_add_(0, seg, valid.float())
    n1 = n.clamp(min=1.0)
    use = valid[:, None] & (idx >= 0) & (idx < E)
    place = torch.where(use, seg[:, None] * E + idx, M * E).view(-1)
    counts = torch.zeros(M * E + 1, dtype=torch.int32, device=z.device).index_add_(0, place, torch.ones_like(place, dtype=torch.int32))
    counts = counts[:-1].view(M, E)
    F = counts.float() / (K * n1)[:, None]
    z = torch.where(valid[:, None], z, 0.0)
    if c["score"] == "softmax":
        top = z.amax(1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        e = torch.exp(z - top)
    else:
        e = 1.0 / (1.0 + torch.exp(-z))
    tot = e.sum(1, keepdim=True)
    alive = valid[:, None] & (tot > 0)
    p = torch.where(alive, e / tot, 0.0)
    P = torch.zeros(M, E, device=z.device).index_add_(0, seg, p) / n1[:, None]
    loss = torch.zeros(M, 2, device=z.device)
    loss[:, 0] = ALPHA * (F * P).sum(1)
    if c["zeta"]:
        lse = torch.where(alive, torch.log(tot) + top, 0.0)
        loss[:, 1] = c["zeta"] * torch.zeros(M, device=z.device).index_add_(0, seg, lse[:, 0].square()) / n1
    out = {"counts": counts, "loss": loss, "prob": P}
    if c["grad"] == "none":
        return out
    Ft = F[seg]
    grad = p * (Ft - (p * Ft).sum(1, keepdim=True)) * (ALPHA / n1)[seg][:, None]
    if c["score"] == "sigmoid":
        grad = grad * (1.0 - e)
    if c["zeta"]:
        grad = grad + p * lse * (2.0 * c["zeta"] / n1)[seg][:, None]
    grad = grad * s["scale"]
    if s["grad_in"] is not None:
        grad = grad + s["grad_in"]
    out["grad"] = s["grad_out"].copy_(grad)
    return out


def _rgrad_plain(s):
    dz, x, W = s["dz"].float(), s["x"].float(), s["W"].float()
    dx, dW = dz @ W, dz.t() @ x
    if s["case"]["add"]:
        dx, dW = dx + s["dx"].float(), dW + s["dW"]
    return {"dx": s["dx"].copy_(dx), "dW": s["dW"].copy_(dW)}


def _to8(v, root):
    """Rows of BLOCK values as e4m3 with a scale a row; a root that is not zero does not become zero."""
    scale = v.abs().amax(1) * (1.0 / TOP)
    scale = torch.where(scale < 2.0 ** -126, 0.0, scale)
    inv = torch.where(scale > 0, 1.0 / scale, 0.0)
    u = (v * inv[:, None]).clamp(-TOP, TOP)
    if root:
        u = torch.where((v > 0) & (scale > 0)[:, None], u.clamp(min=LEAST), u)
    return u.to(torch.float8_e4m3fn).view(-1), scale


def _adamw_plain(s):
    c = s["case"]
    p, g = s["p"].float(), s["g"].float() * s["scale"]
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * s["ms"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["vs"][:, None]).view(-1).square()
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * (1.0 - BETA2)) * g
    root = v.sqrt()
    step = LR / (1.0 - BETA1 ** STEP)
    p = p * (1.0 - LR * WD) - (m / (root * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + EPS)) * step
    out = {"p": s["p"].copy_(p)}
    if c["copy"]:
        out["copy"] = s["copy"].copy_(p)
    if c["bits"] == 32:
        return out | {"m": s["m"].copy_(m), "v": s["v"].copy_(v)}
    m8, ms = _to8(m.view(-1, BLOCK), False)
    v8, vs = _to8(root.view(-1, BLOCK), True)
    return out | {"m": s["m"].copy_(m8), "v": s["v"].copy_(v8), "ms": s["ms"].copy_(ms), "vs": s["vs"].copy_(vs)}


# ---- the framework's calls

def _run_own(s):
    import paper_2609_28053_gb300 as eqb
    c = s["case"]
    if c["kind"] == "balance":
        eqb.eqb_balance_loss(s["z"], s["idx"], s["off"], ALPHA, zeta=c["zeta"], score=c["score"], mask=s["mask"],
                             grad_in=s["grad_in"], grad_out=s["grad_out"], grad_scale=s["scale"], counts=s["counts"],
                             prob=s["prob"], loss=s["loss"], workspace=s["workspace"])
        out = {"counts": s["counts"], "loss": s["loss"], "prob": s["prob"]}
        return out if s["grad_out"] is None else out | {"grad": s["grad_out"]}
    if c["kind"] == "rgrad":
        eqb.eqb_router_grad(s["dz"], s["x"], s["W"], dx=s["dx"], dW=s["dW"], accumulate_dx=c["add"], accumulate_dW=c["add"],
                            workspace=s["workspace"])
        return {"dx": s["dx"], "dW": s["dW"]}
    s["opt"].step(s["grads"], lr=LR, step=STEP, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=WD, grad_scale=s["scale"])
    out = {k: s[k] for k in ("p", "m", "v")}
    if c["copy"]:
        out["copy"] = s["copy"]
    if c["bits"] == 8:
        out |= {"ms": s["ms"], "vs": s["vs"]}
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"balance": _balance_plain, "rgrad": _rgrad_plain, "adamw": _adamw_plain}[state["case"]["kind"]](state)


# ---- the definitions in 64 bits

def _balance_exact(case, seed):
    s = _prepare_balance(case, seed)
    T, E, K, M = case["T"], case["E"], case["K"], case["M"]
    off = s["off"].tolist()
    counts = torch.zeros(M, E, dtype=torch.int32, device="cuda")
    prob = torch.zeros(M, E, dtype=torch.float64, device="cuda")
    loss = torch.zeros(M, 2, dtype=torch.float64, device="cuda")
    grad = None
    if case["grad"] != "none":
        grad = torch.zeros(T, E, dtype=torch.float64, device="cuda")
        if s["grad_in"] is not None:
            grad += s["grad_in"].double()
    for l in range(M):
        rows = torch.arange(off[l], off[l + 1], device="cuda")
        if s["mask"] is not None:
            rows = rows[s["mask"][rows]]
        n = rows.numel()
        if n == 0:
            continue
        ids = s["idx"][rows].long().view(-1)
        counts[l] = torch.bincount(ids[ids >= 0], minlength=E).int()
        F = counts[l].double() / (K * n)
        z = s["z"][rows].double()
        rows, z = rows[(z > -math.inf).any(1)], z[(z > -math.inf).any(1)]
        sig = torch.sigmoid(z)
        p = torch.softmax(z, 1) if case["score"] == "softmax" else sig / sig.sum(1, keepdim=True)
        prob[l] = p.sum(0) / n
        loss[l, 0] = ALPHA * (F * prob[l]).sum()
        lse = torch.logsumexp(z, 1, keepdim=True)
        loss[l, 1] = case["zeta"] * lse.square().sum() / n
        if grad is not None:
            d = ALPHA / n * p * (F - (p @ F)[:, None])
            if case["score"] == "sigmoid":
                d = d * torch.sigmoid(-z)
            grad[rows] += (d + 2 * case["zeta"] / n * lse * p) * s["scale"].double()
    out = {"counts": counts, "loss": loss, "prob": prob}
    return out if grad is None else out | {"grad": grad}


def _rgrad_exact(case, seed):
    s = _prepare_rgrad(case, seed)
    dz, x, W = s["dz"].double(), s["x"].double(), s["W"].double()
    dx, dW = dz @ W, dz.t() @ x
    return {"dx": dx + s["dx"].double(), "dW": dW + s["dW"].double()} if case["add"] else {"dx": dx, "dW": dW}


def _adamw_exact(case, seed):
    s = _prepare_adamw(case, seed)
    g = s["g"].double() * s["scale"].double()
    m, v = s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        m = m * s["ms"].double().repeat_interleave(BLOCK)
        v = (v * s["vs"].double().repeat_interleave(BLOCK)) ** 2
    m.mul_(BETA1).add_(g, alpha=1 - BETA1)
    v.mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
    del g
    p = s["p"].double() * (1 - LR * WD) - LR * (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    out = {"p": p, "copy": p} if case["copy"] else {"p": p}
    if case["bits"] == 32:
        return out | {"m": m, "v": v}
    # the values before their rounding to 8 bits
    for name, x in (("m", m), ("v", v.sqrt())):
        x = x.view(-1, BLOCK)
        scale = x.abs().amax(1) / TOP
        out[name] = (x / torch.where(scale > 0, scale, 1.0)[:, None]).view(-1)
        out[name + "s"] = scale
    return out


def exact(case, seed):
    return {"balance": _balance_exact, "rgrad": _rgrad_exact, "adamw": _adamw_exact}[case["kind"]](case, seed)


# ---- what a pass has to read, write and compute

def work(case):
    if case["kind"] == "balance":
        T, E, K, M = case["T"], case["E"], case["K"], case["M"]
        per = {"bf16": 2, "fp32": 4}[case["z"]] + {"none": 0, "add": 8, "fp32": 4, "bf16": 6}[case["grad"]]
        return {"bytes": T * (E * per + 4 * K + case["mask"]) + M * (8 * E + 16), "flops": T * E * (6 if case["grad"] == "none" else 11)}
    if case["kind"] == "rgrad":
        T, d, E = case["T"], case["d"], case["E"]
        twice = 2 if case["add"] else 1
        return {"bytes": 2 * T * E + 2 * T * d * (1 + twice) + E * d * (2 + 4 * twice), "flops": 4 * T * d * E}
    n = sum(_sizes(case))
    per = {"fp32": 8, "bf16": 4}[case["p"]] + {"fp32": 4, "bf16": 2}[case["g"]] + (2 if case["copy"] else 0)
    per += 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * per, "flops": 14 * n}
