"""The operators around the expert stage as a program calls them, over the sizes they are used at.

  norm    moe_norm: the residual's addition and the root-mean-square norm.  "q8": rows in 8 bits with a
          scale each, and back (moe_q8_restore), as they cross between ranks; "train": the 16-bit rows
          and, with moe_norm_backward, the gradients
  route   moe_route: scores, the balance bias, groups, the best k experts and their weights; with
          "train" moe_route_backward too
  group   moe_group: the order of the rows by expert, and the place of each token's choices in it
  linear  moe_q8_rows, then moe_q8_product with one weight matrix for every row
  ffn     an expert's gated FFN in 8 bits: moe_q8_gated, moe_q8_rows, moe_q8_product, each expert with
          its own rows; "gather": the rows are taken from the tokens through the grouping's row_token
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
WEIGHT_STD = 0.02
EXACT_FLOPS = 5e13        # products of more than this are left without a value in 64 bits


def _norm(name, mode, tokens, hidden):
    return {"name": name, "kind": "norm", "mode": mode, "tokens": tokens, "hidden": hidden}


def _route(name, train, tokens, experts, k, score, groups, top_groups, best, dtype):
    return {"name": name, "kind": "route", "train": train, "tokens": tokens, "experts": experts, "k": k, "score": score,
            "groups": groups, "top_groups": top_groups, "best": best, "dtype": dtype}


def _group(name, tokens, experts, k):
    return {"name": name, "kind": "group", "tokens": tokens, "experts": experts, "k": k}


def _linear(name, tokens, hidden, features):
    return {"name": name, "kind": "linear", "tokens": tokens, "hidden": hidden, "features": features}


def _ffn(name, tokens, hidden, ffn, experts, k, gather):
    return {"name": name, "kind": "ffn", "tokens": tokens, "hidden": hidden, "ffn": ffn, "experts": experts, "k": k,
            "gather": gather}


def listed():
    return [
        # A decode step's norm: a few rows, so the call itself counts.
        _norm("norm_q8_decode", "q8", 16, 4096),
        # A prefill batch of the widest model, its rows sent in 8 bits.
        _norm("norm_q8_prefill", "q8", 4096, 7168),
        # A training step's norm, forward and backward.
        _norm("norm_train", "train", 8192, 2048),
        # A decode step's router: sigmoid scores, a bias for balance, four of eight groups.
        _route("route_decode", False, 32, 256, 8, "sigmoid", 8, 4, 2, "float32"),
        # A ragged prefill batch's router: softmax of 16-bit logits, some experts masked out.
        _route("route_prefill", False, 4099, 64, 6, "softmax", 1, 1, 1, "bfloat16"),
        # A training step's router of a large batch, forward and backward.
        _route("route_train", True, 32768, 256, 8, "sigmoid", 8, 4, 2, "float32"),
        # The order of the rows after the two routers above.
        _group("group_decode", 48, 256, 8),
        _group("group_prefill", 32768, 256, 8),
        # One weight matrix for a handful of tokens: a read of the weights.
        _linear("linear_decode", 5, 4096, 14336),
        # Decoding on a rank of 32 experts: about eight dispatched rows for each.
        _ffn("ffn_decode", 32, 7168, 2048, 32, 8, False),
        # A prefill batch of many small experts.
        _ffn("ffn_fine", 8192, 2048, 1408, 64, 6, True),
        # A prefill batch of few large experts.
        _ffn("ffn_mixtral", 4096, 4096, 14336, 8, 2, True),
    ]


HIDDEN = [256, 320, 1024, 2048, 4096, 7168]
FFNS = [(256, 512, 8, 2), (320, 576, 8, 2), (1024, 4096, 16, 2), (2048, 1408, 64, 6), (4096, 14336, 8, 2), (7168, 2048, 32, 8)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "route", "route", "group", "linear", "ffn", "ffn"])
    if kind == "norm":
        hidden = rng.choice(HIDDEN) if rng.random() < 0.5 else 8 * (2 * rng.randint(4, 512) + 1)
        c = _norm("", rng.choice(["q8", "train"]), _log_int(rng, 1, 8192), hidden)
    elif kind == "route":
        experts, groups, top_groups = rng.choice([(8, 1, 1), (60, 1, 1), (64, 1, 1), (128, 4, 2), (160, 8, 3), (256, 8, 4), (384, 1, 1)])
        k = rng.randint(1, 8)
        c = _route("", rng.random() < 0.5, _log_int(rng, 1, 32768), experts, k, rng.choice(["softmax", "sigmoid"]),
                   groups, top_groups, 1 if groups == 1 else rng.randint(1, 2), rng.choice(["float32", "bfloat16"]))
    elif kind == "group":
        c = _group("", _log_int(rng, 1, 32768), rng.choice([8, 16, 60, 64, 128, 256, 384]), rng.randint(1, 8))
    elif kind == "linear":
        # 16-byte rows: any multiple of 16 of features going in, of 8 coming out.
        hidden = rng.choice(HIDDEN) if rng.random() < 0.5 else 16 * (2 * rng.randint(8, 224) + 1)
        features = rng.choice(HIDDEN) if rng.random() < 0.5 else 8 * (2 * rng.randint(16, 448) + 1)
        c = _linear("", _log_int(rng, 1, 8192), hidden, features)
    else:
        hidden, ffn, experts, k = rng.choice(FFNS)
        c = _ffn("", _log_int(rng, 1, 4096), hidden, ffn, experts, k, rng.random() < 0.7)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _activations(seed, stream, rows, hidden):
    """bf16 rows as a residual stream has them: unit normal, one channel in 128 eight times as large."""
    g = _gen(seed, stream)
    big = torch.rand(hidden, generator=g, device="cuda") < 1 / 128
    x = torch.empty((rows, hidden), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)
    return x * (1.0 + 7.0 * big).to(torch.bfloat16)


def _q8_inputs(seed, stream, rows, hidden):
    """int8 rows and a scale each, as a quantiser makes them of unit normal rows."""
    x = torch.empty((rows, hidden), device="cuda").normal_(0.0, 1.0, generator=_gen(seed, stream))
    top = x.abs().amax(1, keepdim=True)
    return (x * (127.0 / top)).round().to(torch.int8), (top / 127.0).view(-1)


def _q8_weights(seed, stream, experts, n, k):
    """int8 weights [experts, n, k] and a scale per output channel."""
    w = torch.empty((experts, n, k), dtype=torch.int8, device="cuda")
    s = torch.empty((experts, n), device="cuda")
    g = _gen(seed, stream)
    for e in range(experts):
        x = torch.empty((n, k), device="cuda").normal_(0.0, WEIGHT_STD, generator=g)
        top = x.abs().amax(1, keepdim=True)
        w[e] = (x * (127.0 / top)).round().to(torch.int8)
        s[e] = (top / 127.0).view(-1)
    return w, s


def _choices(case, seed):
    """[tokens, k] different experts of each token, int32."""
    u = torch.rand((case["tokens"], case["experts"]), generator=_gen(seed, 20), device="cuda")
    return u.argsort(1)[:, :case["k"]].int().contiguous()


def _empty(shape, dtype):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def _norm_inputs(case, seed):
    T, H = case["tokens"], case["hidden"]
    d = {"x": _activations(seed, 1, T, H), "residual": _activations(seed, 2, T, H),
         "weight": (1.0 + 0.1 * torch.randn(H, generator=_gen(seed, 3), device="cuda")).to(torch.bfloat16)}
    if case["mode"] == "train":
        for i, n in enumerate(("dy", "dsum")):
            d[n] = torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1e-2, generator=_gen(seed, 4 + i))
    return d


def _route_inputs(case, seed):
    T, E = case["tokens"], case["experts"]
    g = _gen(seed, 10)
    dt = getattr(torch, case["dtype"])
    logits = (1.5 * torch.randn((T, E), generator=g, device="cuda")).to(dt)
    if case["score"] == "softmax":   # experts that are out of service
        logits[:, torch.rand(E, generator=g, device="cuda") < 0.05] = -math.inf
    bias = 0.05 * torch.randn(E, generator=g, device="cuda") if case["score"] == "sigmoid" else None
    d = {"logits": logits.contiguous(), "bias": bias}
    if case["train"]:
        d["dweights"] = torch.randn((T, case["k"]), generator=g, device="cuda")
    return d


def _ffn_rows(case, seed):
    """expert_offsets, row_token (None without a gather) and the rows of the tokens' tensor."""
    ids = _choices(case, seed).long()
    T, E, k = case["tokens"], case["experts"], case["k"]
    order = ids.view(-1).argsort(stable=True)
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    off[1:] = torch.bincount(ids.view(-1), minlength=E).cumsum(0)
    return (off, (order // k).int(), T) if case["gather"] else (off, None, T * k)


def _ffn_inputs(case, seed):
    H, F, E = case["hidden"], case["ffn"], case["experts"]
    off, row_token, n = _ffn_rows(case, seed)
    xq, xs = _q8_inputs(seed, 30, n, H)
    d = {"off": off, "row_token": row_token, "xq": xq, "xs": xs}
    for i, (name, shape) in enumerate((("w1", (F, H)), ("w3", (F, H)), ("w2", (H, F)))):
        d[name], d["s" + name[1]] = _q8_weights(seed, 31 + i, E, *shape)
    return d


def _route_scale(case):
    return 2.5 if case["score"] == "sigmoid" else 1.0


def prepare(case, seed):
    kind = case["kind"]
    st = {"case": case}
    if kind == "norm":
        T, H = case["tokens"], case["hidden"]
        st.update(_norm_inputs(case, seed))
        st["sum"], st["out"] = _empty((T, H), torch.bfloat16), _empty((T, H), torch.bfloat16)
        st["q"], st["scale"] = _empty((T, H), torch.int8), _empty(T, torch.float32)
        st["rstd"], st["dx"], st["dweight"] = _empty(T, torch.float32), _empty((T, H), torch.bfloat16), _empty(H, torch.float32)
    elif kind == "route":
        T, E, k = case["tokens"], case["experts"], case["k"]
        st.update(_route_inputs(case, seed))
        st["ids"], st["weights"] = _empty((T, k), torch.int32), _empty((T, k), torch.float32)
        st["dlogits"] = _empty((T, E), st["logits"].dtype)
    elif kind == "group":
        T, E, k = case["tokens"], case["experts"], case["k"]
        ids = _choices(case, seed)
        if T > 16:   # the last tokens of a padded batch have no choices
            ids[T - T // 16:] = -1
        st["ids"] = ids
        st["off"], st["row_token"] = _empty(E + 1, torch.int32), _empty(T * k, torch.int32)
        st["slot"] = _empty((T, k), torch.int32)
    elif kind == "linear":
        T, K, N = case["tokens"], case["hidden"], case["features"]
        st["x"] = _activations(seed, 1, T, K)
        st["w"], st["ws"] = _q8_weights(seed, 2, 1, N, K)
        st["q"], st["scale"], st["y"] = _empty((T, K), torch.int8), _empty(T, torch.float32), _empty((T, N), torch.bfloat16)
    else:
        H, F, rows = case["hidden"], case["ffn"], case["tokens"] * case["k"]
        st.update(_ffn_inputs(case, seed))
        st["most"] = int((st["off"][1:] - st["off"][:-1]).max())   # the rows of the busiest expert
        st["act"], st["y"] = _empty((rows, F), torch.bfloat16), _empty((rows, H), torch.bfloat16)
        st["q"], st["scale"] = _empty((rows, F), torch.int8), _empty(rows, torch.float32)
    return st


# ------------------------------------------------------------------------------------ plain forms

def _rows_to_q8(y):
    """Rows of floats as whole numbers up to 127 (held as floats) and a scale each."""
    top = y.abs().amax(1, keepdim=True)
    return torch.where(top > 0, y * (127.0 / top), 0.0).round(), top / 127.0


def _plain_norm(st):
    mode = st["case"]["mode"]
    h = (st["x"].float() + st["residual"].float()).to(torch.bfloat16)
    hf, w = h.float(), st["weight"].float()
    r = torch.rsqrt((hf * hf).mean(1, keepdim=True) + EPS)
    y = hf * r * w
    if mode == "q8":
        q, s = _rows_to_q8(y)
        return {"sum": h, "out": (q * s).to(torch.bfloat16)}
    dy = st["dy"].float()
    g = dy * w
    c = (g * hf).mean(1, keepdim=True)
    dx = r * (g - hf * (r * r * c)) + st["dsum"].float()
    return {"sum": h, "out": y.to(torch.bfloat16), "rstd": r.view(-1), "dx": dx.to(torch.bfloat16), "dweight": (dy * hf * r).sum(0)}


def _plain_scores(st):
    l = st["logits"].float()
    if st["case"]["score"] == "sigmoid":
        return l, 1.0 / (1.0 + torch.exp(-l))
    m = l.amax(1, keepdim=True)
    e = torch.exp(l - torch.where(m == -math.inf, 0.0, m))
    # In 64 bits, so that a score does not depend on the order of the sum and near ties fall alike.
    s = e.double().sum(1, keepdim=True).float()
    return l, torch.where(s > 0, e / s, 0.0)


def _best(v, k):
    """Indices of the k largest of each row, the lowest index first among equals."""
    return torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]


def _plain_route(st):
    c = st["case"]
    T, E, G, k = c["tokens"], c["experts"], c["groups"], c["k"]
    l, p = _plain_scores(st)
    sel = p + st["bias"] if st["bias"] is not None else p
    sel = torch.where(l == -math.inf, -math.inf, sel)
    if G > 1:
        by_group = torch.sort(sel.view(T, G, E // G), dim=2, descending=True).values[:, :, :c["best"]].sum(2)
        keep = torch.zeros((T, G), dtype=torch.bool, device="cuda").scatter_(1, _best(by_group, c["top_groups"]), True)
        sel = torch.where(keep.repeat_interleave(E // G, 1), sel, -math.inf)
    ids = _best(sel, k)
    have = sel.gather(1, ids) > -math.inf
    chosen = torch.where(have, p.gather(1, ids), 0.0)
    total = chosen.sum(1, keepdim=True)
    share = torch.where(total > 0, chosen / total, 0.0)
    out = {"ids": torch.where(have, ids, -1).int(), "weights": share * _route_scale(c)}
    if c["train"]:
        dw = st["dweights"]
        dp = torch.where(have & (total > 0), _route_scale(c) / total * (dw - (dw * share).sum(1, keepdim=True)), 0.0)
        dscore = torch.zeros((T, E), device="cuda").scatter_add_(1, ids, dp)
        if c["score"] == "sigmoid":
            dl = dscore * p * (1.0 - p)
        else:
            dl = p * (dscore - (dscore * p).sum(1, keepdim=True))
        out["dlogits"] = dl.to(st["logits"].dtype)
    return out


def _plain_group(st):
    c = st["case"]
    E, k = c["experts"], c["k"]
    flat = st["ids"].view(-1).long()
    flat = torch.where((flat >= 0) & (flat < E), flat, E)
    order = torch.sort(flat, stable=True).indices
    n = torch.zeros(E + 1, dtype=torch.int64, device="cuda").scatter_add_(0, flat, torch.ones_like(flat))
    off = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
    off[1:] = n[:E].cumsum(0)
    place = torch.arange(flat.numel(), device="cuda")
    slot = torch.empty_like(flat)
    slot[order] = place
    return {"off": off.int(), "row_token": torch.where(place < off[E], order // k, -1).int(),
            "slot": torch.where(flat < E, slot, -1).int().view(-1, k)}


def _plain_linear(st):
    q, s = _rows_to_q8(st["x"].float())
    return {"y": (q @ st["w"][0].float().t() * s * st["ws"]).to(torch.bfloat16)}


def _plain_ffn(st):
    c, off = st["case"], st["off"].long()
    rows, E = c["tokens"] * c["k"], c["experts"]
    # Each expert's rows in a block of as many as the busiest has.
    at = off[:-1, None] + torch.arange(st["most"], device="cuda")
    at = torch.where(at < off[1:, None], at, 0)
    src = st["row_token"].long()[at] if st["row_token"] is not None else at
    x, xs = st["xq"][src].float(), st["xs"][src][:, :, None]
    g = torch.bmm(x, st["w1"].float().transpose(1, 2)) * xs * st["s1"][:, None, :]
    u = torch.bmm(x, st["w3"].float().transpose(1, 2)) * xs * st["s3"][:, None, :]
    a = (g / (1.0 + torch.exp(-g)) * u).to(torch.bfloat16).float()
    q, s = _rows_to_q8(a.view(-1, c["ffn"]))
    y = torch.bmm(q.view(a.shape), st["w2"].float().transpose(1, 2)) * s.view(E, -1, 1) * st["s2"][:, None, :]
    row = torch.arange(rows, device="cuda")
    e = (row[:, None] >= off[None, 1:]).sum(1)
    return {"y": y[e, row - off[e]].to(torch.bfloat16)}


def _plain(st):
    return {"norm": _plain_norm, "route": _plain_route, "group": _plain_group, "linear": _plain_linear,
            "ffn": _plain_ffn}[st["case"]["kind"]](st)


# ------------------------------------------------------------------------------------ the framework's calls

def _own(st):
    from paper_2607_19539_amd import binding as B
    c = st["case"]
    kind = c["kind"]
    if kind == "norm":
        if c["mode"] == "q8":
            B.moe_norm(st["x"], st["weight"], EPS, residual=st["residual"], sum_out=st["sum"], out_q=st["q"], scale=st["scale"])
            B.moe_q8_restore(st["q"], st["scale"], st["out"])
            return {"sum": st["sum"], "out": st["out"]}
        B.moe_norm(st["x"], st["weight"], EPS, residual=st["residual"], sum_out=st["sum"], out=st["out"], rstd=st["rstd"])
        B.moe_norm_backward(st["dy"], st["sum"], st["weight"], st["rstd"], st["dx"], st["dweight"], dsum=st["dsum"])
        return {n: st[n] for n in ("sum", "out", "rstd", "dx", "dweight")}
    if kind == "route":
        cfg = B.make_route_config(c["experts"], c["k"], score=B.MOE_SCORE_SIGMOID if c["score"] == "sigmoid" else B.MOE_SCORE_SOFTMAX,
                                  groups=c["groups"], top_groups=c["top_groups"], group_best=c["best"], renormalise=True,
                                  scale=_route_scale(c))
        B.moe_route(cfg, st["logits"], st["ids"], st["weights"], bias=st["bias"])
        if not c["train"]:
            return {"ids": st["ids"], "weights": st["weights"]}
        B.moe_route_backward(cfg, st["logits"], st["ids"], st["dweights"], st["dlogits"])
        return {"ids": st["ids"], "weights": st["weights"], "dlogits": st["dlogits"]}
    if kind == "group":
        B.moe_group(st["ids"], c["experts"], st["off"], st["row_token"], st["slot"])
        return {"off": st["off"], "row_token": st["row_token"], "slot": st["slot"]}
    if kind == "linear":
        B.moe_q8_rows(st["x"], st["q"], st["scale"])
        B.moe_q8_product(st["q"], st["scale"], st["w"], st["ws"], st["y"])
        return {"y": st["y"]}
    B.moe_q8_gated(st["xq"], st["xs"], st["w1"], st["s1"], st["w3"], st["s3"], st["act"], row_index=st["row_token"],
                   expert_offsets=st["off"])
    B.moe_q8_rows(st["act"], st["q"], st["scale"])
    B.moe_q8_product(st["q"], st["scale"], st["w2"], st["s2"], st["y"], expert_offsets=st["off"])
    return {"y": st["y"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------ what a pass needs

def work(case):
    kind, T = case["kind"], case["tokens"]
    if kind == "norm":
        n = T * case["hidden"]
        if case["mode"] == "q8":
            return {"bytes": 8 * n, "flops": 6 * n}
        return {"bytes": 14 * n + 6 * case["hidden"] + 4 * T, "flops": 17 * n}
    if kind == "route":
        n, size = T * case["experts"], 4 if case["dtype"] == "float32" else 2
        if case["train"]:
            return {"bytes": 2 * size * n + 12 * T * case["k"], "flops": 10 * n}
        return {"bytes": size * n + 8 * T * case["k"], "flops": 6 * n}
    if kind == "group":
        return {"bytes": 12 * T * case["k"] + 4 * case["experts"], "flops": 4 * T * case["k"]}
    if kind == "linear":
        K, N = case["hidden"], case["features"]
        return {"bytes": 2 * T * K + K * N + 4 * N + 2 * T * N, "flops": 2 * T * K * N}
    H, F, E, k = case["hidden"], case["ffn"], case["experts"], case["k"]
    rows = T * k
    busy = E * (1.0 - (1.0 - k / E) ** T)
    return {"bytes": 3 * busy * H * F + (T if case["gather"] else rows) * H + 2 * rows * H, "flops": 6 * rows * H * F}


# ------------------------------------------------------------------------------------ in 64 bits

def _exact_q8(y):
    top = y.abs().max(dim=1, keepdim=True).values
    step = top / 127.0
    return torch.round(y / torch.where(step > 0, step, torch.ones_like(step))), step


def _exact_norm(case, seed):
    d = _norm_inputs(case, seed)
    h64 = d["x"].double() + d["residual"].double()
    h = h64.to(torch.bfloat16).double()      # the rounded sum is what is normed
    w = d["weight"].double()
    n = torch.sqrt(h.pow(2).sum(1, keepdim=True) / case["hidden"] + EPS)
    y = h / n * w
    if case["mode"] == "q8":
        q, step = _exact_q8(y)
        return {"sum": h64, "out": q * step}
    dy = d["dy"].double()
    unit = h / n
    g = dy * w
    dx = (g - unit * (g * unit).sum(1, keepdim=True) / case["hidden"]) / n + d["dsum"].double()
    return {"sum": h64, "out": y, "rstd": (1.0 / n).view(-1), "dx": dx, "dweight": (dy * unit).sum(0)}


def _exact_route(case, seed):
    d = _route_inputs(case, seed)
    T, E, G, k = case["tokens"], case["experts"], case["groups"], case["k"]
    l = d["logits"].double()
    p = torch.sigmoid(l) if case["score"] == "sigmoid" else torch.softmax(l, 1).nan_to_num(0.0)
    # Experts are chosen by their score in 32 bits plus the bias in 32 bits.
    pick = p.float() if d["bias"] is None else p.float() + d["bias"]
    pick = pick.masked_fill(l == -math.inf, -math.inf).double()
    lower = torch.arange(E, device="cuda")

    def winners(v, n):
        """The n best of each row, one after another, the first of equals."""
        v, got = v.clone(), []
        for _ in range(n):
            i = torch.where(v == v.amax(1, keepdim=True), lower[:v.shape[1]], v.shape[1]).amin(1)
            got.append(i)
            v.scatter_(1, i[:, None], -math.inf)
        return torch.stack(got, 1)

    if G > 1:
        per = pick.view(T * G, E // G)
        value = torch.stack([per.gather(1, i[:, None])[:, 0] for i in winners(per, case["best"]).unbind(1)], 1)
        chosen_groups = winners(value.float().sum(1).double().view(T, G), case["top_groups"])
        inside = (lower[None, None, :] // (E // G) == chosen_groups[:, :, None]).any(1)
        pick = pick.masked_fill(~inside, -math.inf)
    ids = winners(pick, k)
    have = pick.gather(1, ids) > -math.inf
    v = p.gather(1, ids) * have
    total = v.sum(1, keepdim=True)
    share = v / total.clamp_min(1e-300)
    out = {"ids": torch.where(have, ids, -1).int(), "weights": share * _route_scale(case)}
    if case["train"]:
        dw = d["dweights"].double()
        # d(weight)/d(logit) along the chosen ones, then through the score.
        ds = _route_scale(case) * (dw - (dw * share).sum(1, keepdim=True)) * have / total.clamp_min(1e-300)
        if case["score"] == "sigmoid":
            dl = torch.zeros((T, E), dtype=torch.float64, device="cuda").scatter_add_(1, ids, ds * v * (1.0 - v))
        else:
            inner = (ds * v).sum(1, keepdim=True)
            dl = -p * inner
            dl.scatter_add_(1, ids, ds * v)
        out["dlogits"] = dl
    return out


def _exact_linear(case, seed):
    if 2.0 * case["tokens"] * case["hidden"] * case["features"] > EXACT_FLOPS:
        return None
    x = _activations(seed, 1, case["tokens"], case["hidden"]).double()
    w, ws = _q8_weights(seed, 2, 1, case["features"], case["hidden"])
    q, step = _exact_q8(x)
    return {"y": (q * step) @ (w[0].double() * ws[0].double()[:, None]).t()}


def _exact_ffn(case, seed):
    if work(case)["flops"] > EXACT_FLOPS:
        return None
    d = _ffn_inputs(case, seed)
    rows = case["tokens"] * case["k"]
    y = torch.zeros((rows, case["hidden"]), dtype=torch.float64, device="cuda")
    off = d["off"].tolist()
    for e in range(case["experts"]):
        lo, hi = off[e], off[e + 1]
        if lo == hi:
            continue
        src = d["row_token"][lo:hi].long() if d["row_token"] is not None else torch.arange(lo, hi, device="cuda")
        x = d["xq"][src].double() * d["xs"][src].double()[:, None]
        g = x @ (d["w1"][e].double() * d["s1"][e].double()[:, None]).t()
        u = x @ (d["w3"][e].double() * d["s3"][e].double()[:, None]).t()
        # The activation is held in 16 bits, then in 8 with a scale for each row.
        q, step = _exact_q8((g * torch.sigmoid(g) * u).to(torch.bfloat16).double())
        y[lo:hi] = (q * step) @ (d["w2"][e].double() * d["s2"][e].double()[:, None]).t()
    return {"y": y}


def exact(case, seed):
    kind = case["kind"]
    if kind == "group":
        return None
    return {"norm": _exact_norm, "route": _exact_route, "linear": _exact_linear, "ffn": _exact_ffn}[kind](case, seed)
