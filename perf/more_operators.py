"""The operators that train a layer of experts, as a program calls them, over the sizes they are used at.

  product  the experts' products in 16 bits, each expert with its own rows: moe_product; with "train" the
           gradients too, moe_product_dx and moe_product_dw.  "gather": the rows are taken from the tokens
           through the grouping's row_token.  "one": a single matrix for every row
  gate     the gated activation of rows that hold gate and up values side by side: moe_gate; with "train"
           moe_gate_backward too
  combine  moe_combine_backward: the gradient of the weighted sum of each token's rows
  clip     moe_squares and moe_clip: the norm of all gradients of a model, and the gradients scaled to at
           most a given norm
"""
from __future__ import annotations

import math

import torch

own = False

WEIGHT_STD = 0.02
EXACT_FLOPS = 5e13        # products of more than this are left without a value in 64 bits


def _product(name, train, tokens, k_in, n_out, experts, k, gather, dw):
    return {"name": name, "kind": "product", "train": train, "tokens": tokens, "k_in": k_in, "n_out": n_out,
            "experts": experts, "k": k, "gather": gather, "dw": dw}


def _gate(name, train, rows, ffn):
    return {"name": name, "kind": "gate", "train": train, "rows": rows, "ffn": ffn}


def _combine(name, tokens, k, hidden):
    return {"name": name, "kind": "combine", "tokens": tokens, "k": k, "hidden": hidden}


def _clip(name, layers, hidden, ffn, experts, dtype, max_norm):
    return {"name": name, "kind": "clip", "layers": layers, "hidden": hidden, "ffn": ffn, "experts": experts,
            "dtype": dtype, "max_norm": max_norm}


def listed():
    return [
        # A few tokens through small experts: the call itself counts.
        _product("product_tiny", False, 3, 320, 576, 8, 2, True, "float32"),
        # Decoding on a rank of 32 experts, gate and up weights together: a read of the weights.
        _product("product_decode", False, 32, 7168, 4096, 32, 8, False, "float32"),
        # The down product of a ragged prefill batch.
        _product("product_prefill", False, 4099, 1408, 2048, 64, 6, False, "float32"),
        # A small training batch, gradients of the weights in 16 bits.
        _product("product_train_small", True, 777, 1024, 1408, 16, 4, True, "bfloat16"),
        # A training step of many small experts, gate and up weights together, fp32 gradients.
        _product("product_train_fine", True, 8192, 2048, 2816, 64, 6, True, "float32"),
        # A training step of few large experts, the down product.
        _product("product_train_large", True, 4096, 14336, 4096, 8, 2, False, "float32"),
        # The activation of a decode batch, and of a training step forward and backward.
        _gate("gate_decode", False, 256, 2048),
        _gate("gate_train", True, 49152, 1408),
        # The combine's gradient for a small batch of a wide model, and for a training batch.
        _combine("combine_small", 64, 8, 7168),
        _combine("combine_train", 8192, 6, 2048),
        # Gradients of a small layer, and of two layers of many experts that hold a matrix each.
        _clip("clip_small", 1, 256, 512, 8, "mixed", 1.0),
        _clip("clip_layers", 2, 2048, 1408, 64, "mixed", 1.0),
    ]


SIZES = [(256, 512, 8, 2), (320, 576, 8, 2), (1024, 1408, 16, 4), (1024, 4096, 16, 2), (2048, 1408, 64, 6), (4096, 7168, 8, 2),
         (7168, 2048, 32, 8)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["product", "product", "product", "gate", "combine", "clip"])
    if kind == "product":
        train = rng.random() < 0.6
        dw = rng.choice(["float32", "bfloat16"])
        if rng.random() < 0.3:
            # One matrix, 16-byte rows: any multiple of 8 features.
            c = _product("", train, _log_int(rng, 1, 8192), 8 * (2 * rng.randint(8, 448) + 1), 8 * _log_int(rng, 8, 900), 1, 1, False, dw)
        else:
            a, b, experts, k = rng.choice(SIZES)
            k_in, n_out = (a, b) if rng.random() < 0.5 else (b, a)
            c = _product("", train, _log_int(rng, 1, 4096), k_in, n_out, experts, k, rng.random() < 0.6, dw)
    elif kind == "gate":
        c = _gate("", rng.random() < 0.6, _log_int(rng, 1, 49152), rng.choice([512, 576, 1408, 2048]) if rng.random() < 0.5 else
                  8 * rng.randint(4, 255))
    elif kind == "combine":
        c = _combine("", _log_int(rng, 1, 4096), rng.randint(1, 8), rng.choice([256, 320, 1024, 2048, 4096, 7168]) if rng.random() < 0.5
                     else 8 * (2 * rng.randint(4, 446) + 1))
    else:
        a, b, experts, _ = rng.choice(SIZES[:5])
        c = _clip("", rng.randint(1, 2), a, b, min(experts, _log_int(rng, 1, 64)), rng.choice(["float32", "bfloat16", "mixed"]),
                  rng.choice([0.1, 1.0, 1e6]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _normal(seed, stream, shape, std, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=_gen(seed, stream))


def _activations(seed, stream, rows, hidden):
    """bf16 rows as a residual stream has them: unit normal, one channel in 128 eight times as large."""
    big = torch.rand(hidden, generator=_gen(seed, stream + 500), device="cuda") < 1 / 128
    return _normal(seed, stream, (rows, hidden), 1.0) * (1.0 + 7.0 * big).to(torch.bfloat16)


def _empty(shape, dtype):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def _choices(case, seed):
    """[tokens, k] different experts of each token; the last tokens of a padded batch have none (-1)."""
    T = case["tokens"]
    ids = torch.rand((T, case["experts"]), generator=_gen(seed, 20), device="cuda").argsort(1)[:, :case["k"]].contiguous()
    if T > 64 and T % 2:
        ids[T - T // 16:] = -1
    return ids


def _order(ids, experts):
    """expert_offsets and the entries of ids by expert."""
    flat = ids.view(-1)
    order = torch.where(flat >= 0, flat, experts).argsort(stable=True)
    off = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    off[1:] = torch.bincount(flat[flat >= 0], minlength=experts)[:experts].cumsum(0)
    return off, order


def _product_inputs(case, seed):
    T, K, N, E, k = (case[n] for n in ("tokens", "k_in", "n_out", "experts", "k"))
    d = {"off": None, "row_token": None, "w": _normal(seed, 2, (E, N, K), WEIGHT_STD)}
    if E == 1:
        d["x"] = _activations(seed, 1, T, K)
    else:
        d["off"], order = _order(_choices(case, seed), E)
        if case["gather"]:
            place = torch.arange(T * k, device="cuda")
            d["row_token"] = torch.where(place < d["off"][E], order // k, -1).int()
        d["x"] = _activations(seed, 1, T if case["gather"] else T * k, K)
    if case["train"]:
        d["dy"] = _normal(seed, 3, (T * k, N), 1e-2)
    return d


def _gate_inputs(case, seed):
    R, F = case["rows"], case["ffn"]
    d = {"gu": _normal(seed, 4, (R, 2 * F), 2.0)}
    if case["train"]:
        d["dact"] = _normal(seed, 5, (R, F), 1e-2)
    return d


def _combine_inputs(case, seed):
    T, k, H = case["tokens"], case["k"], case["hidden"]
    slot = torch.randperm(T * k, generator=_gen(seed, 6), device="cuda").int().view(T, k)
    if T > 64 and T % 2:   # the last tokens of a padded batch have no rows
        slot[T - T // 16:] = -1
    gate = torch.rand((T, k), generator=_gen(seed, 7), device="cuda") + 0.1
    return {"dout": _normal(seed, 8, (T, H), 1e-2), "recv": _normal(seed, 9, (T * k, H), 1.0), "slot": slot.contiguous(),
            "gate": gate / gate.sum(1, keepdim=True)}


def _clip_inputs(case, seed):
    """Gradients of some layers: norm and router weights, then each expert's matrices, tensors of their own."""
    H, F, E = case["hidden"], case["ffn"], case["experts"]
    shapes = []
    for _ in range(case["layers"]):
        shapes += [(H,), (E, H), (E,)] + [(2 * F, H), (H, F)] * E
    mixed = case["dtype"] == "mixed"
    out = []
    for i, s in enumerate(shapes):
        # "mixed": small tensors and every second expert's matrix in 32 bits.
        dt = (torch.float32 if len(s) == 1 or i % 4 < 2 else torch.bfloat16) if mixed else getattr(torch, case["dtype"])
        out.append(_normal(seed, 100 + i, s, 3e-3 * (1 + i % 3), dt))
    return {"grads": out}


def _buckets(grads):
    """A buffer for the results of each type, every tensor's place on 128 bytes or more, and the places."""
    sizes, places = {}, []
    for g in grads:
        at = sizes.get(g.dtype, 0)
        places.append(at)
        sizes[g.dtype] = at + (g.numel() + 63) // 64 * 64
    flat = {dt: _empty(n, dt) for dt, n in sizes.items()}
    return list(flat.values()), [flat[g.dtype][at:at + g.numel()].view(g.shape) for g, at in zip(grads, places)]


def prepare(case, seed):
    kind = case["kind"]
    st = {"case": case}
    if kind == "product":
        K, N, E, rows = case["k_in"], case["n_out"], case["experts"], case["tokens"] * case["k"]
        st.update(_product_inputs(case, seed))
        st["most"] = rows if st["off"] is None else int((st["off"][1:] - st["off"][:-1]).max())   # of the busiest expert
        st["y"] = _empty((rows, N), torch.bfloat16)
        if case["train"]:
            st["dx"], st["dw"] = _empty((rows, K), torch.bfloat16), _empty((E, N, K), getattr(torch, case["dw"]))
    elif kind == "gate":
        R, F = case["rows"], case["ffn"]
        st.update(_gate_inputs(case, seed))
        st["act"], st["dgu"] = _empty((R, F), torch.bfloat16), _empty((R, 2 * F), torch.bfloat16)
    elif kind == "combine":
        st.update(_combine_inputs(case, seed))
        st["drecv"], st["dgate"] = _empty(st["recv"].shape, torch.bfloat16), _empty(st["gate"].shape, torch.float32)
    else:
        st.update(_clip_inputs(case, seed))
        st["flat"], st["out"] = _buckets(st["grads"])
        st["total"], st["norm"] = _empty(1, torch.float64), _empty(1, torch.float32)
    return st


# ------------------------------------------------------------------------------------ plain forms

def _plain_product(st):
    c, bf16 = st["case"], torch.bfloat16
    if st["off"] is None:
        x, w = st["x"].float(), st["w"][0].float()
        out = {"y": (x @ w.t()).to(bf16)}
        if c["train"]:
            dy = st["dy"].float()
            out["dx"], out["dw"] = (dy @ w).to(bf16), (dy.t() @ x).to(st["dw"].dtype)[None]
        return out
    off, E, w = st["off"].long(), c["experts"], st["w"].float()
    rows = c["tokens"] * c["k"]
    # Each expert's rows in a block of as many as the busiest has.
    at = off[:-1, None] + torch.arange(st["most"], device="cuda")
    have = at < off[1:, None]
    at = torch.where(have, at, 0)
    src = st["row_token"].long()[at] if st["row_token"] is not None else at
    x = torch.where(have[:, :, None], st["x"][src].float(), 0.0)
    row = torch.arange(rows, device="cuda")
    e = (row[:, None] >= off[None, 1:]).sum(1).clamp(max=E - 1)
    mine = (row < off[E])[:, None]

    def by_row(blocks):
        return torch.where(mine, blocks[e, (row - off[e]).clamp(max=st["most"] - 1)], 0.0).to(bf16)

    out = {"y": by_row(torch.bmm(x, w.transpose(1, 2)))}
    if c["train"]:
        dy = torch.where(have[:, :, None], st["dy"][at].float(), 0.0)
        out["dx"] = by_row(torch.bmm(dy, w))
        out["dw"] = torch.bmm(dy.transpose(1, 2), x).to(st["dw"].dtype)
    return out


def _plain_gate(st):
    F, bf16 = st["case"]["ffn"], torch.bfloat16
    g, u = st["gu"][:, :F].float(), st["gu"][:, F:].float()
    s = 1.0 / (1.0 + torch.exp(-g))
    out = {"act": (g * s * u).to(bf16)}
    if st["case"]["train"]:
        da = st["dact"].float()
        out["dgu"] = torch.cat([da * u * s * (1.0 + g * (1.0 - s)), da * g * s], 1).to(bf16)
    return out


def _plain_combine(st):
    k = st["case"]["k"]
    slot = st["slot"].view(-1).long()
    have = slot >= 0
    dout = st["dout"].float().repeat_interleave(k, 0)
    rows = st["recv"][slot.clamp(min=0)].float()
    dgate = torch.where(have, (dout * rows).sum(1), 0.0)
    drecv = torch.zeros(st["recv"].shape, dtype=torch.bfloat16, device="cuda")
    drecv[slot[have]] = (dout * st["gate"].view(-1, 1)).to(torch.bfloat16)[have]
    return {"drecv": drecv, "dgate": dgate.view(-1, k)}


def _plain_clip(st):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in st["grads"]:
        total = total + (g.double() * g.double()).sum()
    norm = total.sqrt()
    scale = torch.where(norm > st["case"]["max_norm"], st["case"]["max_norm"] / norm, 1.0).float()
    for g, o in zip(st["grads"], st["out"]):
        o.copy_((g.float() * scale).to(g.dtype))
    return [norm.float().view(1)] + st["flat"]


def _plain(st):
    return {"product": _plain_product, "gate": _plain_gate, "combine": _plain_combine, "clip": _plain_clip}[st["case"]["kind"]](st)


# ------------------------------------------------------------------------------------ the framework's calls

def _own(st):
    from paper_2607_19539_amd import binding as B
    c = st["case"]
    kind = c["kind"]
    if kind == "product":
        B.moe_product(st["x"], st["w"], st["y"], row_index=st["row_token"], expert_offsets=st["off"])
        if not c["train"]:
            return {"y": st["y"]}
        B.moe_product_dx(st["dy"], st["w"], st["dx"], expert_offsets=st["off"])
        B.moe_product_dw(st["dy"], st["x"], st["dw"], row_index=st["row_token"], expert_offsets=st["off"])
        return {n: st[n] for n in ("y", "dx", "dw")}
    if kind == "gate":
        B.moe_gate(st["gu"], st["act"])
        if not c["train"]:
            return {"act": st["act"]}
        B.moe_gate_backward(st["gu"], st["dact"], st["dgu"])
        return {"act": st["act"], "dgu": st["dgu"]}
    if kind == "combine":
        B.moe_combine_backward(st["dout"], st["recv"], st["slot"], st["gate"], st["drecv"], st["dgate"])
        return {"drecv": st["drecv"], "dgate": st["dgate"]}
    B.moe_squares(st["grads"], st["total"])
    B.moe_clip(st["grads"], st["total"], c["max_norm"], out=st["out"], norm=st["norm"])
    return [st["norm"]] + st["flat"]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------ what a pass needs

def work(case):
    kind = case["kind"]
    if kind == "product":
        T, K, N, E, k = (case[n] for n in ("tokens", "k_in", "n_out", "experts", "k"))
        rows = T * k
        busy = E * (1.0 - (1.0 - k / E) ** T)
        n = 2 * (T if case["gather"] else rows) * K + 2 * busy * N * K + 2 * rows * N
        if not case["train"]:
            return {"bytes": n, "flops": 2 * rows * K * N}
        return {"bytes": n + 2 * rows * N + 2 * rows * K + (4 if case["dw"] == "float32" else 2) * E * N * K, "flops": 6 * rows * K * N}
    if kind == "gate":
        n = case["rows"] * case["ffn"]
        return {"bytes": 12 * n, "flops": 20 * n} if case["train"] else {"bytes": 6 * n, "flops": 6 * n}
    if kind == "combine":
        T, k, H = case["tokens"], case["k"], case["hidden"]
        return {"bytes": 2 * T * H + 4 * T * k * H + 12 * T * k, "flops": 3 * T * k * H}
    H, F, E, L = case["hidden"], case["ffn"], case["experts"], case["layers"]
    n = L * (H + E * H + E + 3 * E * F * H)
    size = {"float32": 4, "bfloat16": 2, "mixed": 3}[case["dtype"]]
    return {"bytes": 2 * size * n, "flops": 3 * n}


# ------------------------------------------------------------------------------------ in 64 bits

def _exact_product(case, seed):
    if work(case)["flops"] > EXACT_FLOPS:
        return None
    d = _product_inputs(case, seed)
    E, K, N, rows = case["experts"], case["k_in"], case["n_out"], case["tokens"] * case["k"]
    off = [0, rows] if d["off"] is None else d["off"].tolist()
    f64 = {"dtype": torch.float64, "device": "cuda"}
    out = {"y": torch.zeros((rows, N), **f64)}
    if case["train"]:
        out["dx"], out["dw"] = torch.zeros((rows, K), **f64), torch.zeros((E, N, K), **f64)
    for i in range(E):
        lo, hi = off[i], off[i + 1]
        if lo == hi:
            continue
        x = (d["x"][lo:hi] if d["row_token"] is None else d["x"][d["row_token"][lo:hi].long()]).double()
        w = d["w"][i].double()
        out["y"][lo:hi] = torch.mm(x, w.t())
        if case["train"]:
            dy = d["dy"][lo:hi].double()
            out["dx"][lo:hi] = torch.mm(dy, w)
            out["dw"][i] = torch.mm(dy.t(), x)
    return out


def _exact_gate(case, seed):
    d = _gate_inputs(case, seed)
    g, u = d["gu"].double().split(case["ffn"], 1)
    s = torch.sigmoid(g)
    out = {"act": g * s * u}
    if case["train"]:
        da = d["dact"].double()
        # The derivative of g / (1 + e^-g) as s + g s s'.
        out["dgu"] = torch.cat([da * u * (s + g * s * torch.sigmoid(-g)), da * (g * s)], 1)
    return out


def _exact_combine(case, seed):
    d = _combine_inputs(case, seed)
    T, k = case["tokens"], case["k"]
    drecv = torch.zeros(d["recv"].shape, dtype=torch.float64, device="cuda")
    dgate = torch.zeros((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        t = torch.nonzero(d["slot"][:, j] >= 0)[:, 0]
        at = d["slot"][t, j].long()
        drecv[at] = d["dout"][t].double() * d["gate"][t, j].double()[:, None]
        dgate[t, j] = torch.linalg.vecdot(d["dout"][t].double(), d["recv"][at].double())
    return {"drecv": drecv, "dgate": dgate}


def _exact_clip(case, seed):
    grads = _clip_inputs(case, seed)["grads"]
    norm = math.sqrt(math.fsum(float(torch.linalg.vecdot(g.double().flatten(), g.double().flatten())) for g in grads))
    scale = min(1.0, case["max_norm"] / norm)
    flat, places = {}, []
    for g in grads:
        flat.setdefault(g.dtype, []).append(g)
    for same in flat.values():
        places.append(torch.cat([torch.nn.functional.pad(g.double().flatten() * scale, (0, -g.numel() % 64)) for g in same]))
    return [torch.tensor([norm], dtype=torch.float64, device="cuda")] + places


def exact(case, seed):
    return {"product": _exact_product, "gate": _exact_gate, "combine": _exact_combine, "clip": _exact_clip}[case["kind"]](case, seed)
