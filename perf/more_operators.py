"""The operators of the experts behind a router, as cases that can be timed.

  gate     eqb_gate_topk: experts and gate weights of every token (groups,
           bias for balance, renormalised weights), and eqb_gate_grad: the
           gradient of the weights with respect to the router logits
  rows     eqb_expert_rows: the experts' rows from the tokens' lists, as slots,
           entries and offsets
  quant    eqb_quant_rows, eqb_quant_cols, eqb_quant_blocks: values in 8 bits
           with a scale for each block of 128, along a row (sent to the
           experts' rows on the way), along an expert's rows, in both directions
  matmul   eqb_expert_matmul: every expert's rows times its weights in 8 bits,
           and eqb_expert_wgrad: the gradient of the weights
  combine  eqb_expert_combine: the weighted sum of a token's rows, and
           eqb_expert_combine_grad: its gradients

`run` computes them in plain torch operations in 32 bits, or with the
package's calls where `own` is true; `exact` from the formulas in 64 bits.
Sizes are the repository's configurations (mid, global, router), its serving
and ragged shapes, and generic ones between them.
"""
import math
import random

import torch

own = False

TOP = 448.0    # largest e4m3 value
BLOCK = 128    # values that share a scale
GROUPS = 8


def listed():
    return [
        # A decoding step's gate: 64 tokens, latency.
        {"name": "gate_decode", "kind": "gate", "way": "forward", "T": 64, "E": 256, "K": 8, "groups": 8, "top_groups": 4, "two": True, "score": "sigmoid", "renorm": True, "z": "bf16", "mask": False},
        # The headline training shape: experts in groups, weights renormalised.
        {"name": "gate_global", "kind": "gate", "way": "forward", "T": 2097152, "E": 256, "K": 8, "groups": 8, "top_groups": 4, "two": True, "score": "sigmoid", "renorm": True, "z": "bf16", "mask": False},
        # Backward of the mid configuration's gate: softmax over all experts, a gradient for every logit.
        {"name": "gate_grad_mid", "kind": "gate", "way": "backward", "T": 524288, "E": 128, "K": 8, "score": "softmax", "renorm": False, "z": "bf16", "grad": "fp32", "mask": True},
        # The lists of a decoding step: latency.
        {"name": "rows_decode", "kind": "rows", "T": 64, "E": 256, "K": 8, "drop": 0.0},
        # One microbatch of the router configuration, lists cut short by a capacity limit.
        {"name": "rows_router", "kind": "rows", "T": 65536, "E": 128, "K": 8, "drop": 0.05},
        # A prefill-sized batch on its way to the experts, no multiple of a tile.
        {"name": "quant_prefill", "kind": "quant", "axis": "rows", "T": 16411, "d": 2048, "E": 256, "K": 8, "drop": 0.0},
        # The input of the weights' gradient: a microbatch gathered by expert, turned.
        {"name": "quant_cols", "kind": "quant", "axis": "cols", "T": 16384, "d": 4096, "E": 128, "K": 8, "drop": 0.02},
        # A decoding step's product: 32 tokens with 8 experts each, the weights are what is read.
        {"name": "matmul_decode", "kind": "matmul", "way": "forward", "R": 256, "n": 2048, "d": 4096, "E": 128, "skew": 0.3, "out": "bf16"},
        # A training step's product: 16,384 tokens with 8 experts each.
        {"name": "matmul_train", "kind": "matmul", "way": "forward", "R": 131072, "n": 2048, "d": 4096, "E": 128, "skew": 0.3, "out": "bf16"},
        # The gradient of 64 experts' weights, written in fp32.
        {"name": "matmul_wgrad", "kind": "matmul", "way": "weights", "R": 65536, "n": 1024, "d": 2048, "E": 64, "skew": 0.5, "add": False},
        # The prefill batch's way back.
        {"name": "combine_prefill", "kind": "combine", "way": "forward", "T": 16411, "n": 2048, "E": 256, "K": 8, "drop": 0.0},
        # Its backward pass in training: gradients of the rows and of the gate weights.
        {"name": "combine_grad", "kind": "combine", "way": "backward", "T": 16384, "n": 4096, "E": 128, "K": 8, "drop": 0.02},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A multiple of 16, odd multiples among them."""
    n = 16 * _log_int(rng, lo // 16, hi // 16)
    return n + 16 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["gate", "gate", "rows", "quant", "quant", "matmul", "matmul", "combine"])
    E = rng.choice([8, 16, 40, 64, 96, 128, 160, 256, 256, 384, 512, 1024])
    K = rng.choice([k for k in (1, 2, 4, 6, 8) if k < E])
    if kind == "gate":
        case = {"kind": kind, "way": rng.choice(["forward", "backward"]), "T": _log_int(rng, 1, min(2097152, (1 << 28) // E)), "E": E, "K": K,
                "score": rng.choice(["sigmoid", "softmax"]), "renorm": rng.random() < 0.5, "z": rng.choice(["bf16", "bf16", "fp32"]),
                "mask": rng.random() < 0.4}
        if case["way"] == "backward":
            return case | {"grad": rng.choice(["add", "fp32", "bf16"])}
        if E % GROUPS == 0 and E >= 2 * GROUPS and rng.random() < 0.6:
            open_ = rng.choice([g for g in (1, 2, 4, 8) if g * (E // GROUPS) >= K])
            return case | {"groups": GROUPS, "top_groups": open_, "two": rng.random() < 0.5}
        return case | {"groups": 1, "top_groups": 1, "two": False}
    if kind == "rows":
        return {"kind": kind, "T": _log_int(rng, 1, 1 << 18), "E": E, "K": K, "drop": rng.choice([0.0, 0.0, 0.1])}
    if kind == "quant":
        axis = rng.choice(["rows", "cols", "blocks"])
        if axis == "blocks":
            n, d = _width(rng, 64, 4096), _width(rng, 64, 4096)
            return {"kind": kind, "axis": axis, "E": _log_int(rng, 1, min(256, max(1, (1 << 28) // (n * d)))), "n": n, "d": d,
                    "w": rng.choice(["bf16", "fp32"]), "turned": rng.random() < 0.5}
        d = _width(rng, 64, 8192)
        return {"kind": kind, "axis": axis, "T": _log_int(rng, 1, min(65536, (1 << 28) // (d * K))), "d": d, "E": E, "K": K,
                "drop": rng.choice([0.0, 0.1])}
    if kind == "matmul":
        n, d = _width(rng, 64, 4096), _width(rng, 64, 8192)
        way = rng.choice(["forward", "forward", "weights"])
        E = min(E, (1 << (29 if way == "forward" else 27)) // (n * d))
        R = _log_int(rng, 1, min(131072, (1 << 39) // (n * d)))
        case = {"kind": kind, "way": way, "R": R, "n": n, "d": d, "E": E, "skew": rng.choice([0.0, 0.3, 1.0])}
        return case | ({"out": rng.choice(["bf16", "bf16", "fp32"])} if way == "forward" else {"add": rng.random() < 0.5})
    n = _width(rng, 64, 8192)
    return {"kind": kind, "way": rng.choice(["forward", "backward"]), "T": _log_int(rng, 1, min(65536, (1 << 28) // (n * K))), "n": n, "E": E,
            "K": K, "drop": rng.choice([0.0, 0.1])}


# ---- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(std)


def _lists(T, E, K, drop, g):
    """int32 [T,K]: K distinct experts a token, some liked more than others, some entries dropped."""
    liked = _normal((E,), g, 0.5)
    idx = torch.empty((T, K), dtype=torch.int32, device="cuda")
    for a in range(0, T, 1 << 18):
        idx[a:a + (1 << 18)] = torch.topk(_normal((min(T - a, 1 << 18), E), g) + liked, K).indices.int()
    if drop:
        idx[torch.rand((T, K), generator=g, device="cuda") < drop] = -1
    return idx


def _rows_of(idx, E):
    """offsets, blocks, slot and entry of the lists, by a stable sort."""
    flat = idx.view(-1).long()
    here = (flat >= 0) & (flat < E)
    key = torch.where(here, flat, E)
    lens = torch.zeros(E + 1, dtype=torch.int64, device=idx.device).index_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=idx.device)
    offsets[1:] = torch.cumsum(lens, 0)
    blocks = torch.zeros(E + 1, dtype=torch.int32, device=idx.device)
    blocks[1:] = torch.cumsum(torch.div(lens + BLOCK - 1, BLOCK, rounding_mode="floor"), 0)
    order = torch.sort(key, stable=True).indices
    at = torch.arange(flat.numel(), device=idx.device)
    entry = torch.where(at < offsets[E], order, -1).int()
    slot = torch.empty_like(order)
    slot[order] = at
    return offsets, blocks, torch.where(here, slot, -1).int().view(idx.shape), entry


def _max_blocks(R, E):
    return (R + (BLOCK - 1) * min(R, E)) // BLOCK


def _prepare_gate(case, seed):
    g = _gen(seed)
    T, E, K = case["T"], case["E"], case["K"]
    z = _normal((T, E), g).add_(_normal((E,), g, 0.5))
    s = {"case": case, "mask": None, "scale": 2.5 if case["renorm"] else 1.0}
    if case["mask"]:
        s["mask"] = torch.rand(T, generator=g, device="cuda") < 0.9
    if case["way"] == "forward":
        s["b"] = _normal((E,), g, 0.2)
        if case["mask"]:
            z[~s["mask"]] = math.nan                       # nobody has computed these rows
            z[::7, E // 2:] = -math.inf                    # experts that are closed to some tokens
            z[3::1009] = torch.where(s["mask"][3::1009, None], -math.inf, z[3::1009])  # and all of them
        s["idx"] = torch.empty((T, K), dtype=torch.int32, device="cuda")
        s["weight"] = torch.empty((T, K), device="cuda")
    else:
        s["idx"] = _lists(T, E, K, 0.05 if case["mask"] else 0.0, g)
        if case["mask"]:
            s["idx"][~s["mask"]] = -1
        s["grad_weight"] = _normal((T, K), g, 1e-3)
        s["grad_in"] = None if case["grad"] == "fp32" else _normal((T, E), g, 1e-3)
        s["grad_out"] = s["grad_in"] if case["grad"] == "add" else torch.empty(
            (T, E), dtype=torch.bfloat16 if case["grad"] == "bf16" else torch.float32, device="cuda")
    s["z"] = z.bfloat16() if case["z"] == "bf16" else z
    return s


def _prepare_rows(case, seed):
    T, E, K = case["T"], case["E"], case["K"]
    s = {"case": case, "idx": _lists(T, E, K, case["drop"], _gen(seed))}
    s["offsets"] = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    s["blocks"] = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    s["slot"] = torch.empty((T, K), dtype=torch.int32, device="cuda")
    s["entry"] = torch.empty(T * K, dtype=torch.int32, device="cuda")
    if own:
        import paper_2609_28053_gb300 as eqb
        s["workspace"] = torch.empty(eqb.eqb_expert_rows_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")
    return s


def _values(shape, g):
    """Activations: blocks of different size, a few large values."""
    x = _normal(shape, g)
    x[..., ::67] *= 8.0
    return x


def _prepare_quant(case, seed):
    g = _gen(seed)
    e4m3 = torch.float8_e4m3fn
    if case["axis"] == "blocks":
        E, n, d = case["E"], case["n"], case["d"]
        w = _normal((E, n, d), g, 0.02)
        nb, db = -(-n // BLOCK), -(-d // BLOCK)
        s = {"case": case, "w": w.bfloat16() if case["w"] == "bf16" else w, "q": torch.zeros((E, n, d), dtype=e4m3, device="cuda"),
             "scale": torch.zeros((E, nb, db), device="cuda"), "q_t": None, "scale_t": None}
        if case["turned"]:
            s["q_t"], s["scale_t"] = torch.zeros((E, d, n), dtype=e4m3, device="cuda"), torch.zeros((E, db, nb), device="cuda")
        return s
    T, d, E, K = case["T"], case["d"], case["E"], case["K"]
    s = {"case": case, "x": _values((T, d), g).bfloat16()}
    s["offsets"], s["blocks"], s["slot"], s["entry"] = _rows_of(_lists(T, E, K, case["drop"], g), E)
    if case["axis"] == "rows":
        # one row more, where the plain form puts what has no slot
        s["q"] = torch.zeros((T * K + 1, d), dtype=e4m3, device="cuda")[:-1]
        s["scale"] = torch.zeros((T * K + 1, -(-d // BLOCK)), device="cuda")[:-1]
    else:
        cap = _max_blocks(T * K, E)
        s["q"] = torch.zeros((d, cap * BLOCK), dtype=e4m3, device="cuda")
        s["scale"] = torch.zeros((cap, d), device="cuda")
    return s


def _lens(case, seed):
    """Rows of every expert, uneven."""
    R, E = case["R"], case["E"]
    rng = random.Random(seed)
    share = [math.exp(case["skew"] * rng.gauss(0.0, 1.0)) for _ in range(E)]
    if R < 64 * E:
        lens = [0] * E
        for e in rng.choices(range(E), share, k=R):
            lens[e] += 1
        return lens
    cuts, run = [0], 0.0
    for x in share:
        run += x
        cuts.append(int(R * run / sum(share) + 0.5))
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _codes(shape, g):
    out = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    for part in out.view(-1).split(1 << 28):
        part.copy_(_normal(part.shape, g, 100.0).clamp_(-TOP, TOP))
    return out


def _prepare_matmul(case, seed):
    g = _gen(seed)
    R, n, d, E = case["R"], case["n"], case["d"], case["E"]
    lens = _lens(case, seed)
    first, blk = [0], [0]
    for x in lens:
        first.append(first[-1] + x)
        blk.append(blk[-1] + -(-x // BLOCK))
    s = {"case": case, "lens": lens, "offsets": torch.tensor(first, dtype=torch.int32, device="cuda"),
         "blocks": torch.tensor(blk, dtype=torch.int32, device="cuda")}
    kb = -(-d // BLOCK)
    if case["way"] == "forward":
        s["a"], s["a_scale"] = _codes((R, d), g), torch.exp(_normal((R, kb), g, 0.3)).mul_(1e-2)
        s["w"], s["w_scale"] = _codes((E, n, d), g), torch.exp(_normal((E, -(-n // BLOCK), kb), g, 0.3)).mul_(2e-4)
        s["out"] = torch.zeros((R, n), dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda")
        return s
    cap = _max_blocks(R, E)
    # zero behind the last row of every expert
    at = torch.arange(cap * BLOCK, device="cuda")
    which = torch.searchsorted(s["blocks"].long(), torch.div(at, BLOCK, rounding_mode="floor"), right=True) - 1
    live = which < E
    which = which.clamp(max=E - 1)
    live &= at - s["blocks"].long()[which] * BLOCK < (s["offsets"][1:] - s["offsets"][:-1]).long()[which]
    s["a"], s["b"] = _codes((n, cap * BLOCK), g), _codes((d, cap * BLOCK), g)
    for t in (s["a"], s["b"]):
        t.view(torch.uint8).mul_(live.byte())
    s["a_scale"], s["b_scale"] = torch.exp(_normal((cap, n), g, 0.3)).mul_(1e-5), torch.exp(_normal((cap, d), g, 0.3)).mul_(1e-2)
    s["dW"] = _normal((E, n, d), g) if case["add"] else torch.zeros((E, n, d), device="cuda")
    return s


def _prepare_combine(case, seed):
    g = _gen(seed)
    T, n, E, K = case["T"], case["n"], case["E"], case["K"]
    slot = _rows_of(_lists(T, E, K, case["drop"], g), E)[2]
    s = {"case": case, "slot": slot, "rows": _normal((T * K, n), g).bfloat16(), "weight": torch.rand((T, K), generator=g, device="cuda") / K}
    if case["way"] == "forward":
        s["out"] = torch.empty((T, n), dtype=torch.bfloat16, device="cuda")
    else:
        s["grad"] = _normal((T, n), g, 1e-2).bfloat16()
        s["grad_rows"] = torch.zeros((T * K + 1, n), dtype=torch.bfloat16, device="cuda")[:-1]  # one row more, as above
        s["grad_weight"] = torch.empty((T, K), device="cuda")
    return s


def prepare(case, seed):
    return {"gate": _prepare_gate, "rows": _prepare_rows, "quant": _prepare_quant, "matmul": _prepare_matmul,
            "combine": _prepare_combine}[case["kind"]](case, seed)


# ---- the plain forms

def _sigmoid_shares(z):
    """sigmoid(z), a part of each row's sum of them."""
    m = z.amax(1, keepdim=True).clamp(max=0.0)
    m = torch.where(m == -math.inf, 0.0, m)
    u = torch.where(z > 0, 1.0 / (1.0 + torch.exp(-z)), torch.exp(z - m) / (1.0 + torch.exp(z)))
    tot = u.sum(1, keepdim=True)
    return torch.where(tot > 0, u / tot, 0.0)


def _softmax(z):
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    tot = e.sum(1, keepdim=True)
    return torch.where(tot > 0, e / tot, 0.0)


def _gate_forward(s, z, valid):
    c = s["case"]
    E, K, G = c["E"], c["K"], c["groups"]
    z = torch.where(valid[:, None], z.float(), -math.inf)
    v = z + s["b"]
    if c["top_groups"] < G:
        top = torch.topk(v.view(-1, G, E // G), 2 if c["two"] else 1).values
        score = top[..., 0]
        if c["two"]:
            score = score + torch.where(top[..., 1] == -math.inf, 0.0, top[..., 1])
        best = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        open_ = torch.zeros_like(score, dtype=torch.bool).scatter_(1, best, True)
        v = torch.where(open_[:, :, None], v.view(-1, G, E // G), -math.inf).view(-1, E)
    v, idx = (t[:, :K] for t in torch.sort(v, dim=1, descending=True, stable=True))
    here = v > -math.inf
    zk = torch.where(here, z.gather(1, idx), -math.inf)
    if c["renorm"]:
        w = _sigmoid_shares(zk) if c["score"] == "sigmoid" else _softmax(zk)
    else:
        w = 1.0 / (1.0 + torch.exp(-zk)) if c["score"] == "sigmoid" else torch.where(here, _softmax(z).gather(1, idx), 0.0)
    return torch.where(here, idx, -1).int(), w * s["scale"]


def _gate_backward(s, a, b):
    c = s["case"]
    z, idx, g = s["z"][a:b].float(), s["idx"][a:b].long(), s["grad_weight"][a:b]
    here = idx >= 0
    at = idx.clamp(min=0)
    zk = torch.where(here, z.gather(1, at), -math.inf)
    if c["score"] == "softmax" and not c["renorm"]:
        p = _softmax(z)
        pg = torch.where(here, p.gather(1, at) * g, 0.0)
        d = (p * -pg.sum(1, keepdim=True)).scatter_add_(1, at, pg)
        return d * s["scale"]
    sig = 1.0 / (1.0 + torch.exp(-zk))
    if not c["renorm"]:
        d = g * sig * (1.0 / (1.0 + torch.exp(zk)))
    else:
        w = _sigmoid_shares(zk) if c["score"] == "sigmoid" else _softmax(zk)
        d = w * (g - (w * g).sum(1, keepdim=True))
        if c["score"] == "sigmoid":
            d = d * (1.0 / (1.0 + torch.exp(zk)))
    d = torch.where(here, d * s["scale"], 0.0)
    return torch.zeros_like(z).scatter_add_(1, at, d)


def _gate_plain(s):
    c = s["case"]
    T, step = c["T"], max(1, (1 << 26) // c["E"])
    for a in range(0, T, step):
        b = min(T, a + step)
        if c["way"] == "forward":
            valid = torch.ones(b - a, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][a:b]
            s["idx"][a:b], s["weight"][a:b] = _gate_forward(s, s["z"][a:b], valid)
        else:
            d = _gate_backward(s, a, b)
            s["grad_out"][a:b] = d if s["grad_in"] is None else s["grad_in"][a:b] + d
    return {"idx": s["idx"], "weight": s["weight"]} if c["way"] == "forward" else {"grad": s["grad_out"]}


def _rows_plain(s):
    got = _rows_of(s["idx"], s["case"]["E"])
    return {k: s[k].copy_(t) for k, t in zip(("offsets", "blocks", "slot", "entry"), got)}


def _to8(top):
    """The scale of a block whose largest magnitude is `top`, and its reciprocal."""
    scale = top * (1.0 / TOP)
    scale = torch.where(scale < 2.0 ** -126, 0.0, scale)
    return scale, torch.where(scale > 0, 1.0 / scale, 0.0)


def _padded(x, axis):
    more = -x.shape[axis] % BLOCK
    if not more:
        return x
    shape = list(x.shape)
    shape[axis] = more
    return torch.cat([x, x.new_zeros(shape)], axis)


def _block_rows(s):
    """The row that each place of the blocks has (-1: none), and the blocks there are."""
    E, cap = s["case"]["E"], s["scale"].shape[0]
    at = torch.arange(cap * BLOCK, device="cuda")
    blocks, offsets = s["blocks"].long(), s["offsets"].long()
    which = torch.searchsorted(blocks, torch.div(at, BLOCK, rounding_mode="floor"), right=True) - 1
    which = which.clamp(max=E - 1)
    row = offsets[which] + at - blocks[which] * BLOCK
    return torch.where(row < offsets[which + 1], row, -1), torch.arange(cap, device="cuda") < blocks[E]


def _quant_plain(s):
    c = s["case"]
    if c["axis"] == "blocks":
        E, n, d = c["E"], c["n"], c["d"]
        for e in range(E):
            w = _padded(_padded(s["w"][e].float(), 0), 1)
            w = w.view(w.shape[0] // BLOCK, BLOCK, w.shape[1] // BLOCK, BLOCK)
            scale, inv = _to8(w.abs().amax((1, 3)))
            q = (w * inv[:, None, :, None]).clamp_(-TOP, TOP).reshape(w.shape[0] * BLOCK, w.shape[2] * BLOCK)[:n, :d].to(torch.float8_e4m3fn)
            s["q"][e], s["scale"][e] = q, scale
            if c["turned"]:
                s["q_t"][e], s["scale_t"][e] = q.t(), scale.t()
        out = {"q": s["q"], "scale": s["scale"]}
        return out | {"q_t": s["q_t"], "scale_t": s["scale_t"]} if c["turned"] else out
    d, K = c["d"], c["K"]
    x = s["x"].float()
    if c["axis"] == "rows":
        x = _padded(x, 1).view(c["T"], -1, BLOCK)
        scale, inv = _to8(x.abs().amax(2))
        q = (x * inv[:, :, None]).clamp_(-TOP, TOP).view(c["T"], -1)[:, :d].to(torch.float8_e4m3fn)
        codes, scales = (t.as_strided((t.shape[0] + 1, t.shape[1]), t.stride()) for t in (s["q"].view(torch.uint8), s["scale"]))
        for k in range(K):
            at = s["slot"][:, k].long()
            at = torch.where(at >= 0, at, c["T"] * K)
            codes.index_copy_(0, at, q.view(torch.uint8))
            scales.index_copy_(0, at, scale)
        return {"q": s["q"], "scale": s["scale"]}
    row, there = _block_rows(s)
    entry = s["entry"].long()[row.clamp(min=0)]
    token = torch.div(entry.clamp(min=0), K, rounding_mode="floor")
    for a in range(0, d, 512):
        v = torch.where((row >= 0)[:, None], x[:, a:a + 512][token], 0.0).view(-1, BLOCK, min(512, d - a))
        scale, inv = _to8(v.abs().amax(1))
        q = (v * inv[:, None]).clamp_(-TOP, TOP).to(torch.float8_e4m3fn).view(torch.uint8).permute(2, 0, 1)
        old = s["q"][a:a + 512].view(torch.uint8).view(q.shape)
        old.copy_(torch.where(there[None, :, None], q, old))
        s["scale"][:, a:a + 512] = torch.where(there[:, None], scale, s["scale"][:, a:a + 512])
    return {"q": s["q"], "scale": s["scale"]}


def _matmul_plain(s):
    c = s["case"]
    n, d = c["n"], c["d"]
    at = blk = 0
    for e, rows in enumerate(s["lens"]):
        if c["way"] == "forward":
            if rows:
                a = s["a"][at:at + rows].float() * s["a_scale"][at:at + rows].repeat_interleave(BLOCK, 1)[:, :d]
                w = s["w"][e].float() * s["w_scale"][e].repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :d]
                s["out"][at:at + rows] = a @ w.t()
        else:
            nb = -(-rows // BLOCK)
            a = s["a"][:, blk * BLOCK:(blk + nb) * BLOCK].float() * s["a_scale"][blk:blk + nb].t().repeat_interleave(BLOCK, 1)
            b = s["b"][:, blk * BLOCK:(blk + nb) * BLOCK].float() * s["b_scale"][blk:blk + nb].t().repeat_interleave(BLOCK, 1)
            s["dW"][e] = s["dW"][e] + a @ b.t() if c["add"] else a @ b.t()
            blk += nb
        at += rows
    return {"out": s["out"]} if c["way"] == "forward" else {"dW": s["dW"]}


def _combine_plain(s):
    c = s["case"]
    if c["way"] == "forward":
        out = torch.zeros((c["T"], c["n"]), device="cuda")
        for k in range(c["K"]):
            at = s["slot"][:, k].long()
            w = torch.where(at >= 0, s["weight"][:, k], 0.0)
            out += s["rows"][at.clamp(min=0)].float() * w[:, None]
        return {"out": s["out"].copy_(out)}
    R = s["rows"].shape[0]
    g = s["grad"].float()
    got = s["grad_rows"].as_strided((R + 1, c["n"]), s["grad_rows"].stride())
    for k in range(c["K"]):
        at = s["slot"][:, k].long()
        got.index_copy_(0, torch.where(at >= 0, at, R), (g * s["weight"][:, k, None]).bfloat16())
        s["grad_weight"][:, k] = torch.where(at >= 0, (g * s["rows"][at.clamp(min=0)].float()).sum(1), 0.0)
    return {"grad_rows": s["grad_rows"], "grad_weight": s["grad_weight"]}


# ---- the framework's calls

def _run_own(s):
    import paper_2609_28053_gb300 as eqb
    c = s["case"]
    if c["kind"] == "gate":
        if c["way"] == "forward":
            eqb.eqb_gate_topk(s["z"], s["b"], c["K"], score=c["score"], groups=c["groups"], top_groups=c["top_groups"],
                              group_score="top2" if c["two"] else "max", renorm=c["renorm"], scale=s["scale"], mask=s["mask"],
                              topk_idx=s["idx"], weight=s["weight"])
            return {"idx": s["idx"], "weight": s["weight"]}
        eqb.eqb_gate_grad(s["z"], s["idx"], s["grad_weight"], score=c["score"], renorm=c["renorm"], scale=s["scale"],
                          grad_in=s["grad_in"], grad_out=s["grad_out"])
        return {"grad": s["grad_out"]}
    if c["kind"] == "rows":
        eqb.eqb_expert_rows(s["idx"], c["E"], offsets=s["offsets"], blocks=s["blocks"], slot=s["slot"], entry=s["entry"],
                            workspace=s["workspace"])
        return {k: s[k] for k in ("offsets", "blocks", "slot", "entry")}
    if c["kind"] == "quant":
        if c["axis"] == "blocks":
            eqb.eqb_quant_blocks(s["w"], q=s["q"], scale=s["scale"], q_t=s["q_t"], scale_t=s["scale_t"])
            out = {"q": s["q"], "scale": s["scale"]}
            return out | {"q_t": s["q_t"], "scale_t": s["scale_t"]} if c["turned"] else out
        if c["axis"] == "rows":
            eqb.eqb_quant_rows(s["x"], slot=s["slot"], q=s["q"], scale=s["scale"])
        else:
            eqb.eqb_quant_cols(s["x"], s["offsets"], s["blocks"], entry=s["entry"], K=c["K"], q=s["q"], scale=s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if c["kind"] == "matmul":
        if c["way"] == "forward":
            eqb.eqb_expert_matmul(s["a"], s["a_scale"], s["w"], s["w_scale"], s["offsets"], out=s["out"])
            return {"out": s["out"]}
        eqb.eqb_expert_wgrad(s["a"], s["a_scale"], s["b"], s["b_scale"], s["blocks"], dW=s["dW"], accumulate=c["add"])
        return {"dW": s["dW"]}
    if c["way"] == "forward":
        eqb.eqb_expert_combine(s["rows"], s["slot"], s["weight"], out=s["out"])
        return {"out": s["out"]}
    eqb.eqb_expert_combine_grad(s["grad"], s["rows"], s["slot"], s["weight"], grad_rows=s["grad_rows"], grad_weight=s["grad_weight"])
    return {"grad_rows": s["grad_rows"], "grad_weight": s["grad_weight"]}


def run(state):
    if own:
        return _run_own(state)
    return {"gate": _gate_plain, "rows": _rows_plain, "quant": _quant_plain, "matmul": _matmul_plain,
            "combine": _combine_plain}[state["case"]["kind"]](state)


# ---- the definitions in 64 bits

def _gate_exact(case, seed):
    s = _prepare_gate(case, seed)
    T, E, K = case["T"], case["E"], case["K"]
    step = max(1, (1 << 25) // E)
    sig, out = case["score"] == "sigmoid", {}
    if case["way"] == "forward":
        out = {"idx": torch.full((T, K), -1, dtype=torch.int32, device="cuda"), "weight": torch.zeros((T, K), dtype=torch.float64, device="cuda")}
    else:
        out = {"grad": torch.zeros((T, E), dtype=torch.float64, device="cuda")}
    for a in range(0, T, step):
        z = s["z"][a:a + step].double()
        if case["way"] == "forward":
            if s["mask"] is not None:
                z = z.masked_fill(~s["mask"][a:a + step, None], -math.inf)
            v = (s["z"][a:a + step].float() + s["b"]).masked_fill(torch.isneginf(z), -math.inf)  # the sum that decides is one in fp32
            if case["top_groups"] < case["groups"]:
                by = v.view(len(v), case["groups"], -1).sort(2, descending=True).values
                of = by[..., 0] + by[..., 1].masked_fill(torch.isneginf(by[..., 1]), 0.0) if case["two"] else by[..., 0]
                # a group's place: the groups before it that are as good, and all that are better
                lower = torch.ones((case["groups"],) * 2, dtype=torch.bool, device="cuda").tril(-1)
                ahead = (of[:, None, :] > of[:, :, None]) | ((of[:, None, :] == of[:, :, None]) & lower)
                shut = ahead.sum(2) >= case["top_groups"]
                v = v.masked_fill(shut.repeat_interleave(E // case["groups"], 1), -math.inf)
            idx = torch.argsort(-v, dim=1, stable=True)[:, :K]
            no = torch.isneginf(v.gather(1, idx))
        else:
            idx = s["idx"][a:a + step].long()
            no = idx < 0
            idx = idx.clamp(min=0)
        zk = z.gather(1, idx).masked_fill(no, -math.inf)
        if case["renorm"]:
            w = (torch.nn.functional.logsigmoid(zk) if sig else zk).masked_fill(no, -math.inf).softmax(1)
        else:
            w = zk.sigmoid() if sig else z.softmax(1).gather(1, idx)
        w = w.masked_fill(no, 0.0)
        if case["way"] == "forward":
            out["idx"][a:a + step] = idx.masked_fill(no, -1).int()
            out["weight"][a:a + step] = w * s["scale"]
            continue
        g = s["grad_weight"][a:a + step].double()
        d = w * (g - (w * g).sum(1, keepdim=True) if case["renorm"] else g)
        if sig:
            d = d * torch.sigmoid(-zk)
        full = torch.zeros_like(z).scatter_add_(1, idx, d.masked_fill(no, 0.0))
        if not sig and not case["renorm"]:
            full -= z.softmax(1) * (w * g).sum(1, keepdim=True)
        out["grad"][a:a + step] = full * s["scale"] + (0.0 if s["grad_in"] is None else s["grad_in"][a:a + step].double())
    return out


def _rows_exact(case, seed):
    s = _prepare_rows(case, seed)
    E, K = case["E"], case["K"]
    lists = s["idx"].view(-1).tolist()
    of = [[] for _ in range(E)]
    for i, e in enumerate(lists):
        if e >= 0:
            of[e].append(i)
    offsets, blocks, entry, slot = [0], [0], [], [-1] * len(lists)
    for rows in of:
        for i in rows:
            slot[i] = len(entry)
            entry.append(i)
        offsets.append(len(entry))
        blocks.append(blocks[-1] + (len(rows) + BLOCK - 1) // BLOCK)
    entry += [-1] * (len(lists) - len(entry))
    dev = {"dtype": torch.int32, "device": "cuda"}
    return {"offsets": torch.tensor(offsets, **dev), "blocks": torch.tensor(blocks, **dev), "slot": torch.tensor(slot, **dev).view(-1, K),
            "entry": torch.tensor(entry, **dev)}


def _units(v, axes):
    """Values as parts of their block's scale, before the rounding to 8 bits, and the scales."""
    top = v.abs().amax(axes, keepdim=True) / TOP
    return v / torch.where(top > 0, top, 1.0), top


def _quant_exact(case, seed):
    s = _prepare_quant(case, seed)
    if case["axis"] == "blocks":
        E, n, d = case["E"], case["n"], case["d"]
        out = {"q": torch.zeros((E, n, d), dtype=torch.float64, device="cuda"), "scale": torch.zeros(s["scale"].shape, dtype=torch.float64, device="cuda")}
        for i in range(0, n, BLOCK):
            for j in range(0, d, BLOCK):
                u, top = _units(s["w"][:, i:i + BLOCK, j:j + BLOCK].double(), (1, 2))
                out["q"][:, i:i + BLOCK, j:j + BLOCK], out["scale"][:, i // BLOCK, j // BLOCK] = u, top[:, 0, 0]
        if case["turned"]:
            out |= {"q_t": out["q"].transpose(1, 2).contiguous(), "scale_t": out["scale"].transpose(1, 2).contiguous()}
        return out
    T, d, K = case["T"], case["d"], case["K"]
    x = s["x"].double()
    q = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    scale = torch.zeros(s["scale"].shape, dtype=torch.float64, device="cuda")
    if case["axis"] == "rows":
        has = s["slot"].view(-1) >= 0
        token = torch.arange(T, device="cuda").repeat_interleave(K)[has]
        to = s["slot"].view(-1)[has].long()
        for j in range(0, d, BLOCK):
            u, top = _units(x[:, j:j + BLOCK], 1)
            q[to, j:j + BLOCK], scale[to, j // BLOCK] = u[token], top[token, 0]
        return {"q": q, "scale": scale}
    first, blk = s["offsets"].tolist(), s["blocks"].tolist()
    token = torch.div(s["entry"].long(), K, rounding_mode="floor")
    for e in range(case["E"]):
        for b in range(blk[e], blk[e + 1]):
            r = first[e] + (b - blk[e]) * BLOCK
            rows = token[r:min(r + BLOCK, first[e + 1])]
            u, top = _units(x[rows], 0)
            q[:, b * BLOCK:b * BLOCK + len(rows)], scale[b] = u.t(), top[0]
    return {"q": q, "scale": scale}


def _matmul_exact(case, seed):
    s = _prepare_matmul(case, seed)
    n, d, E = case["n"], case["d"], case["E"]
    if case["way"] == "forward":
        first = s["offsets"].tolist()
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for e in range(E):
            a, w = s["a"][first[e]:first[e + 1]].double(), s["w"][e].double()
            if len(a):
                for k in range(0, d, BLOCK):
                    a[:, k:k + BLOCK] *= s["a_scale"][first[e]:first[e + 1], k // BLOCK, None]
                    for j in range(0, n, BLOCK):
                        w[j:j + BLOCK, k:k + BLOCK] *= s["w_scale"][e, j // BLOCK, k // BLOCK]
                torch.matmul(a, w.t(), out=out[first[e]:first[e + 1]])
        return {"out": out}
    dW, blk = s["dW"].double(), s["blocks"].tolist()
    for e in range(E):
        for b in range(blk[e], blk[e + 1]):
            at = slice(b * BLOCK, (b + 1) * BLOCK)
            dW[e].addmm_(s["a"][:, at].double() * s["a_scale"][b].double()[:, None], (s["b"][:, at].double() * s["b_scale"][b].double()[:, None]).t())
    return {"dW": dW}


def _combine_exact(case, seed):
    s = _prepare_combine(case, seed)
    T, n, K = case["T"], case["n"], case["K"]
    has = s["slot"] >= 0
    token, k = has.nonzero(as_tuple=True)
    at = s["slot"][has].long()
    w = s["weight"][has].double()
    if case["way"] == "forward":
        out = torch.zeros((T, n), dtype=torch.float64, device="cuda")
        for j in range(0, n, 512):
            out[:, j:j + 512].index_add_(0, token, s["rows"][:, j:j + 512][at].double() * w[:, None])
        return {"out": out}
    rows = torch.zeros((T * K, n), dtype=torch.float64, device="cuda")
    dw = torch.zeros((T, K), dtype=torch.float64, device="cuda")
    for i in range(0, len(at), 1 << 15):
        g = s["grad"][token[i:i + (1 << 15)]].double()
        to = at[i:i + (1 << 15)]
        rows[to] = g * w[i:i + (1 << 15), None]
        dw[token[i:i + (1 << 15)], k[i:i + (1 << 15)]] = (g * s["rows"][to].double()).sum(1)
    return {"grad_rows": rows, "grad_weight": dw}


def exact(case, seed):
    return {"gate": _gate_exact, "rows": _rows_exact, "quant": _quant_exact, "matmul": _matmul_exact,
            "combine": _combine_exact}[case["kind"]](case, seed)


# ---- what a pass has to read, write and compute

def work(case):
    kind = case["kind"]
    size = {"bf16": 2, "fp32": 4}
    if kind == "gate":
        T, E, K = case["T"], case["E"], case["K"]
        z = size[case["z"]]
        if case["way"] == "forward":
            return {"bytes": T * (E * z + 8 * K + case["mask"]) + 4 * E, "flops": 4 * T * E}
        dense = case["score"] == "softmax" and not case["renorm"]
        per = {"add": 8 * (E if dense else K), "fp32": 4 * E, "bf16": 6 * E}[case["grad"]]
        return {"bytes": T * ((E if dense else K) * z + 8 * K + per), "flops": T * ((E if dense else K) * 6)}
    if kind == "rows":
        T, E, K = case["T"], case["E"], case["K"]
        return {"bytes": 12 * T * K + 8 * E, "flops": T * K}
    if kind == "quant":
        if case["axis"] == "blocks":
            n = case["E"] * case["n"] * case["d"]
            return {"bytes": n * (size[case["w"]] + 1 + case["turned"]), "flops": 2 * n}
        T, d, K = case["T"], case["d"], case["K"]
        R = T * K * (1.0 - case["drop"])
        out = R * (d + (d / 32 if case["axis"] == "rows" else 0)) + (R * d / 32 if case["axis"] == "cols" else 0)
        return {"bytes": T * d * 2 + out + 4 * T * K, "flops": 2 * T * d}
    if kind == "matmul":
        R, n, d, E = case["R"], case["n"], case["d"], case["E"]
        if case["way"] == "forward":
            used = E * (1.0 - (1.0 - 1.0 / E) ** R)  # experts that have rows
            return {"bytes": R * d * (1 + 1 / 32) + used * n * d + R * n * size[case["out"]], "flops": 2 * R * n * d}
        return {"bytes": R * (n + d) * (1 + 1 / 32) + E * n * d * (8 if case["add"] else 4), "flops": 2 * R * n * d}
    T, n, K = case["T"], case["n"], case["K"]
    R = T * K * (1.0 - case["drop"])
    if case["way"] == "forward":
        return {"bytes": (R + T) * n * 2 + 8 * T * K, "flops": 2 * R * n}
    return {"bytes": (2 * R + T) * n * 2 + 12 * T * K, "flops": 3 * R * n}
