"""What the operators of a dropless MoE layer and its training step are measured on: tokens sorted by expert and back with their
weights (both with their gradients, the router's among them), and the experts' products on the sorted rows with bias, activation
and residual (with their gradients).

``own`` = False runs them in elementary torch operations in 32 bits, ``own`` = True through ``paper_2401_13920_b200.experts``.
"""
import math

import torch

own = False


def listed():
    return [
        # --- tokens sorted by expert: the order from the router's choices, and the rows in it ---
        # a decoding batch, two experts a token: latency
        dict(name="sort_8", op="sort", T=8, H=2560, E=32, K=2, dtype="bf16", pad=0.0),
        # a training step of the full-layer configuration's width, two experts a token, a padded batch (padding is not routed)
        dict(name="sort_65536", op="sort", T=65536, H=2560, E=32, K=2, dtype="bf16", pad=0.06),
        # the way back of the gradient, the router's own gradient added: odd sizes in fp32, three experts a token
        dict(name="sort_grad_odd", op="sort_grad", T=3001, H=777, E=21, K=3, dtype="f32", pad=0.05, bias=True),
        # the same for a training step of the 65536 x 5120 configuration, one expert a token
        dict(name="sort_grad_65536", op="sort_grad", T=65536, H=5120, E=64, K=1, dtype="bf16", pad=0.0, bias=False),
        # --- back to token order: the weighted sum over a token's experts ---
        # a training step: two experts a token, added to the residual stream
        dict(name="unsort_65536", op="unsort", T=65536, H=2560, E=32, K=2, dtype="bf16", pad=0.06, residual=True),
        # its gradient: the experts' rows and the weights
        dict(name="unsort_grad_65536", op="unsort_grad", T=65536, H=2560, E=32, K=2, dtype="bf16", pad=0.06),
        # the tiny configuration in fp32
        dict(name="unsort_grad_f32_4096", op="unsort_grad", T=4096, H=1024, E=8, K=1, dtype="f32", pad=0.0),
        # --- the experts' products on sorted rows ---
        # one token with two experts, the layer's second product (no activation): two matrices' weights, once
        dict(name="linear_2", op="linear", R=2, E=32, IN=10240, OUT=2560, act="none", bias=True, residual=False, want_z=False, lost=0),
        # a decoding batch of 64 tokens with two experts each, the first product: nearly all the weights
        dict(name="linear_128", op="linear", R=128, E=32, IN=2560, OUT=10240, act="gelu", bias=True, residual=False, want_z=False, lost=0),
        # odd sizes: ragged groups, sizes that are no multiple of any tile, rows behind the last group, a residual
        dict(name="linear_1000_odd", op="linear", R=1000, E=24, IN=1560, OUT=4104, act="silu", bias=True, residual=True, want_z=False, lost=37),
        # a training step of the full-layer configuration: the first product, its activation's input kept
        dict(name="linear_65536", op="linear", R=65536, E=32, IN=2560, OUT=10240, act="gelu", bias=True, residual=False, want_z=True, lost=0),
        # the second product's gradient in the same step: towards the first product's output before its activation, the
        # weights and the bias
        dict(name="linear_grad_65536", op="linear_grad", R=65536, E=32, IN=10240, OUT=2560, act="gelu", bias=True, lost=0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sort", "sort_grad", "unsort", "unsort_grad", "linear", "linear", "linear_grad", "linear_grad"])
    E = rng.choice([4, 8, 12, 16, 21, 24, 32, 64])
    if op in ("linear", "linear_grad"):
        R = _log_uniform(rng, 1, 65536)
        IN, OUT = 8 * _log_uniform(rng, 16, 1280), 8 * _log_uniform(rng, 16, 1280)
        while E * IN * OUT > 32 * 2560 * 10240:
            IN, OUT = 8 * max(1, IN // 12), 8 * max(1, OUT // 12)
        c = dict(op=op, R=R, E=E, IN=IN, OUT=OUT, act=rng.choice(["none", "relu", "gelu", "gelu", "silu"]), bias=rng.random() < 0.6,
                 lost=rng.choice([0, 0, R // 20]))
        if op == "linear":
            c.update(residual=rng.random() < 0.3, want_z=c["act"] != "none" and rng.random() < 0.5)
        return c
    T, H, K = _log_uniform(rng, 1, 65536), _log_uniform(rng, 64, 8192), rng.choice([1, 1, 2, 2, 3, 4])
    if rng.random() < 0.75:
        H = 8 * max(1, H // 8)       # three quarters with rows of whole 16-byte vectors, the others odd
    if op == "sort_grad":
        H = E * max(1, H // E)       # the router's groups are equal
    T = max(1, min(T, 65536 * 5120 // (H * K) // 2))
    c = dict(op=op, T=T, H=H, E=E, K=K, dtype=rng.choice(["bf16", "bf16", "f32"]), pad=rng.choice([0.0, 0.0, 0.1]))
    if op == "sort_grad":
        c.update(bias=rng.random() < 0.5)
    if op == "unsort":
        c.update(residual=rng.random() < 0.5)
    return c


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, dtype=torch.float32, std=1.0, mean=0.0):
    return torch.empty(*shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)


def _choices(g, case):
    """K different experts for each token, some experts liked more than others, -1 for the tokens of the padding: [K][T]."""
    T, E, K = case["T"], case["E"], case["K"]
    liked = _normal(g, E, std=0.7)
    score = liked + torch.empty(T, E, device="cuda").exponential_(1.0, generator=g).log().neg()
    idx = score.topk(K, dim=1).indices.t().contiguous().to(torch.int32)
    if case["pad"] > 0.0:
        idx[:, torch.rand(T, generator=g, device="cuda") < case["pad"]] = -1
    return idx


def _order(idx, E):
    """Order of the K * T assignments v = c * T + t by expert, those of one expert in the order of v: where each group begins, the
    row of each assignment (-1: not routed) and the assignment of each row (-1: behind the last group)."""
    flat = idx.reshape(-1).long()
    ok = (flat >= 0) & (flat < E)
    key = torch.where(ok, flat, E)
    by_row = torch.sort(key, stable=True).indices
    n = flat.numel()
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device=idx.device), torch.bincount(key, minlength=E + 1)[:E].cumsum(0)])
    row = torch.empty_like(by_row)
    row[by_row] = torch.arange(n, device=idx.device)
    slot = torch.where(ok, row, -1)
    inv = torch.where(torch.arange(n, device=idx.device) < offsets[E], by_row, -1)
    i32 = torch.int32
    return offsets.to(i32), slot.to(i32).reshape(idx.shape), inv.to(i32)


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] in ("linear", "linear_grad"):
        return _prepare_linear(case, g)
    T, H, E, K = case["T"], case["H"], case["E"], case["K"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = dict(case=case, idx=_choices(g, case))
    if case["op"] == "sort":
        s.update(x=_normal(g, T, H, dtype=dt))
        return s
    offsets, slot, inv = _order(s["idx"], E)
    s.update(offsets=offsets, slot=slot, inv=inv)
    if case["op"] == "sort_grad":
        # the tokens, what comes back from the experts, the gradient of the scores, the balance loss's share per expert
        s.update(x=_normal(g, T, H, dtype=dt), dxs=_normal(g, K * T, H, dtype=dt, std=0.1), dw=_normal(g, K, T, std=0.5),
                 dp=torch.rand(E, generator=g, device="cuda") * 0.02, eps=_normal(g, E, std=0.05) if case["bias"] else None)
    else:
        s.update(y=_normal(g, K * T, H, dtype=dt, std=0.3), w=torch.rand(K, T, generator=g, device="cuda") * 0.9 + 0.05)
        if case["op"] == "unsort_grad":
            s.update(dout=_normal(g, T, H, dtype=dt, std=0.1))
        else:
            s.update(residual=_normal(g, T, H, dtype=dt, std=2.0) if case["residual"] else None)
    return s


def _prepare_linear(case, g):
    R, E, IN, OUT = case["R"], case["E"], case["IN"], case["OUT"]
    bf = torch.bfloat16
    # rows of each expert: some get many, about one in eight none
    share = _normal(g, E, std=0.5).exp() * (torch.rand(E, generator=g, device="cuda") >= 0.125)
    share[0] += 1e-3
    expert = torch.multinomial(share, R - case["lost"], replacement=True, generator=g)
    counts = torch.bincount(expert, minlength=E)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    s = dict(case=case, offsets=offsets, host_offsets=offsets.tolist(), w=_normal(g, E, OUT, IN, dtype=bf, std=IN ** -0.5))
    if case["op"] == "linear":
        s.update(x=_normal(g, R, IN, dtype=bf), bias=_normal(g, E, OUT, std=0.1) if case["bias"] else None,
                 residual=_normal(g, R, OUT, dtype=bf) if case["residual"] else None)
    else:
        z = _normal(g, R, IN, dtype=bf)
        s.update(z=None if case["act"] == "none" else z, dy=_normal(g, R, OUT, dtype=bf, std=0.1),
                 x=_act(z.float(), case["act"]).to(bf))
    return s


# ---- plain forms ----

def _act(v, act):
    if act == "relu":
        return v.clamp_min(0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * 0.7071067811865476))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _act_slope(v, act):
    if act == "relu":
        return (v > 0.0).to(v.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(v * 0.7071067811865476)) + v * torch.exp(-0.5 * v * v) * 0.3989422804014327
    if act == "silu":
        q = 1.0 / (1.0 + torch.exp(-v))
        return q * (1.0 + v * (1.0 - q))
    return torch.ones_like(v)


def _sort_plain(s):
    x, T = s["x"], s["case"]["T"]
    offsets, slot, inv = _order(s["idx"], s["case"]["E"])
    xs = x[inv.clamp_min(0).long() % T] * (inv >= 0)[:, None]
    return dict(offsets=offsets, slot=slot, inv=inv, xs=xs)


def _gather(y, slot):
    """Row of each token for one choice in 32 bits, zero where there is none."""
    return y[slot.clamp_min(0).long()].float() * (slot >= 0)[:, None]


def _sort_grad_plain(s):
    c = s["case"]
    T, H, E, K = c["T"], c["H"], c["E"], c["K"]
    # group means in 64 bits: next to zero their sign decides
    G = torch.cat([x.double().reshape(-1, E, H // E).mean(2) for x in s["x"].split(8192)])
    if s["eps"] is not None:
        G = G + s["eps"]
    on = G > 0.0
    G = torch.where(on, G, 0.0).float()
    p = torch.exp(G - G.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    dp = s["dp"][None, :].expand(T, E).clone()
    for k in range(K):
        dp.scatter_add_(1, s["idx"][k].clamp_min(0).long()[:, None], (s["dw"][k] * (s["idx"][k] >= 0))[:, None])
    dG = p * (dp - (p * dp).sum(1, keepdim=True)) * on
    dx = (dG / (H // E))[:, :, None].expand(T, E, H // E).reshape(T, H).clone()
    for k in range(K):
        dx += _gather(s["dxs"], s["slot"][k])
    return dict(dx=dx.to(s["x"].dtype), deps=dG.double().sum(0).float())


def _unsort_plain(s):
    out = torch.zeros(s["case"]["T"], s["case"]["H"], device="cuda") if s["residual"] is None else s["residual"].float()
    for k in range(s["case"]["K"]):
        out = out + s["w"][k][:, None] * _gather(s["y"], s["slot"][k])
    return dict(out=out.to(s["y"].dtype))


def _unsort_grad_plain(s):
    T, K = s["case"]["T"], s["case"]["K"]
    dout, inv = s["dout"].float(), s["inv"]
    dw = torch.stack([(dout * _gather(s["y"], s["slot"][k])).sum(1) for k in range(K)])
    v = inv.clamp_min(0).long()
    dy = dout[v % T] * (s["w"].reshape(-1)[v] * (inv >= 0))[:, None]
    return dict(dy=dy.to(s["y"].dtype), dw=dw)


def _groups(s):
    o = s["host_offsets"]
    return [(e, o[e], o[e + 1]) for e in range(len(o) - 1) if o[e + 1] > o[e]]


def _linear_plain(s):
    c, bf = s["case"], torch.bfloat16
    y = torch.zeros(c["R"], c["OUT"], dtype=bf, device="cuda")
    z = torch.zeros_like(y) if c["want_z"] else None
    for e, a, b in _groups(s):
        v = torch.matmul(s["x"][a:b].float(), s["w"][e].float().t())
        if s["bias"] is not None:
            v += s["bias"][e]
        if z is not None:
            z[a:b] = v.to(bf)
        v = _act(v, c["act"])
        if s["residual"] is not None:
            v = v + s["residual"][a:b].float()
        y[a:b] = v.to(bf)
    return dict(y=y, z=z) if c["want_z"] else dict(y=y)


def _linear_grad_plain(s):
    c, bf = s["case"], torch.bfloat16
    E, R, IN, OUT = c["E"], c["R"], c["IN"], c["OUT"]
    dx = torch.zeros(R, IN, dtype=bf, device="cuda")
    dw = torch.zeros(E, OUT, IN, dtype=bf, device="cuda")
    db = torch.zeros(E, OUT, device="cuda") if c["bias"] else None
    for e, a, b in _groups(s):
        dy = s["dy"][a:b].float()
        d = torch.matmul(dy, s["w"][e].float())
        if s["z"] is not None:
            d = d * _act_slope(s["z"][a:b].float(), c["act"])
        dx[a:b] = d.to(bf)
        dw[e] = torch.matmul(dy.t(), s["x"][a:b].float()).to(bf)
        if db is not None:
            db[e] = dy.sum(0)
    return dict(dx=dx, dw=dw, db=db) if c["bias"] else dict(dx=dx, dw=dw)


_PLAIN = dict(sort=_sort_plain, sort_grad=_sort_grad_plain, unsort=_unsort_plain, unsort_grad=_unsort_grad_plain, linear=_linear_plain,
              linear_grad=_linear_grad_plain)


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return _PLAIN[op](s)
    from paper_2401_13920_b200 import experts
    if op == "linear":
        y, z = experts.expert_linear(s["x"], s["w"], s["offsets"], bias=s["bias"], act=c["act"], residual=s["residual"], want_z=c["want_z"])
        return dict(y=y, z=z) if c["want_z"] else dict(y=y)
    if op == "linear_grad":
        dx, dw, db = experts.expert_linear_grad(s["dy"], s["x"], s["w"], s["offsets"], z=s["z"], act=c["act"], want_db=c["bias"])
        return dict(dx=dx, dw=dw, db=db) if c["bias"] else dict(dx=dx, dw=dw)
    if op == "sort":
        xs, order = experts.sort_rows(s["x"], s["idx"], c["E"])
        return dict(offsets=order.offsets, slot=order.slot, inv=order.inv, xs=xs)
    order = experts.Order(s["offsets"], s["slot"], s["inv"])
    if op == "sort_grad":
        dx, deps = experts.sort_rows_grad(s["dxs"], order, x=s["x"], idx_k=s["idx"], dw=s["dw"], eps=s["eps"], dp=s["dp"])
        return dict(dx=dx, deps=deps)
    if op == "unsort":
        return dict(out=experts.unsort_rows(s["y"], order, w_k=s["w"], residual=s["residual"]))
    dy, dw = experts.unsort_rows_grad(s["dout"], order, w_k=s["w"], y=s["y"])
    return dict(dy=dy, dw=dw)


def work(case):
    if case["op"] in ("linear", "linear_grad"):
        R, E, IN, OUT = case["R"], case["E"], case["IN"], case["OUT"]
        rows, live = R - case["lost"], 0.875 * E
        hit = live * (1.0 - (1.0 - 1.0 / live) ** rows)               # experts met, on average
        product = 2.0 * rows * IN * OUT
        if case["op"] == "linear":
            out = rows * OUT * 2.0 * (1 + case["want_z"] + case["residual"])
            return {"bytes": hit * IN * OUT * 2.0 + rows * IN * 2.0 + out + (hit * OUT * 4.0 if case["bias"] else 0.0), "flops": product}
        moved = rows * (OUT + IN * (2.0 if case["act"] == "none" else 3.0)) * 2.0
        return {"bytes": hit * IN * OUT * 2.0 + E * IN * OUT * 2.0 + moved + (E * OUT * 4.0 if case["bias"] else 0.0), "flops": 2.0 * product}
    T, H, K = case["T"], case["H"], case["K"]
    el = 2.0 if case["dtype"] == "bf16" else 4.0
    row, kept = H * el, K * T * (1.0 - case["pad"])
    if case["op"] == "sort":
        return {"bytes": T * (1.0 - case["pad"]) * row + K * T * row + 12.0 * K * T + 4.0 * case["E"], "flops": 0.0}
    if case["op"] == "sort_grad":
        return {"bytes": (kept + 2.0 * T) * row + 12.0 * K * T + 12.0 * case["E"], "flops": T * H * (K + 2.0)}
    if case["op"] == "unsort":
        return {"bytes": (kept + T * (1.0 + case["residual"])) * row + 8.0 * K * T, "flops": 2.0 * kept * H}
    return {"bytes": (kept + K * T + T * (1.0 - case["pad"])) * row + 12.0 * K * T, "flops": 3.0 * kept * H}


# ---- the definitions in 64 bits ----

def _exact_sort(s):
    T, H, E = s["case"]["T"], s["case"]["H"], s["case"]["E"]
    flat = s["idx"].flatten()
    rows = torch.cat([torch.nonzero(flat == e).squeeze(1) for e in range(E)])
    xs = torch.zeros(flat.numel(), H, dtype=torch.float64, device="cuda")
    xs[:rows.numel()] = s["x"].double().index_select(0, rows.remainder(T))
    return dict(offsets=None, slot=None, inv=None, xs=xs)


def _exact_sort_grad(s):
    c = s["case"]
    T, H, E, K = c["T"], c["H"], c["E"], c["K"]
    dx = torch.empty(T, H, dtype=torch.float64, device="cuda")
    deps = torch.zeros(E, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // H)
    for a in range(0, T, step):
        b = min(T, a + step)
        x = s["x"][a:b].double()
        logits = torch.stack([x[:, i * (H // E):(i + 1) * (H // E)].sum(1) / (H // E) for i in range(E)], 1)
        if s["eps"] is not None:
            logits = logits + s["eps"].double()
        lp = torch.log_softmax(torch.relu(logits), 1)
        # d loss / d log p_i = p_i * dp_i; the softmax passes q - p * sum(q) on
        q = lp.exp() * s["dp"].double()
        for k in range(K):
            e = s["idx"][k, a:b].long()
            t = torch.nonzero(e >= 0).squeeze(1)
            q[t, e[t]] += lp.exp()[t, e[t]] * s["dw"][k, a:b].double()[t]
        dl = torch.where(logits > 0, q - lp.exp() * q.sum(1, keepdim=True), 0.0)
        deps += dl.sum(0)
        d = torch.repeat_interleave(dl / (H // E), H // E, dim=1)
        for k in range(K):
            at = s["slot"][k, a:b].long()
            t = torch.nonzero(at >= 0).squeeze(1)
            d.index_add_(0, t, s["dxs"][at[t]].double())
        dx[a:b] = d
    return dict(dx=dx, deps=deps)


def _exact_unsort(s):
    T, H, K = s["case"]["T"], s["case"]["H"], s["case"]["K"]
    out = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    if s["residual"] is not None:
        out += s["residual"]
    for r in range(0, K * T, 65536):
        v = s["inv"][r:r + 65536]
        v = v[v >= 0].long()                                          # the rows with an assignment come first
        out.index_add_(0, v % T, s["y"][r:r + v.numel()].double() * s["w"].flatten()[v].double()[:, None])
    return dict(out=out)


def _exact_unsort_grad(s):
    T, H, K = s["case"]["T"], s["case"]["H"], s["case"]["K"]
    dy = torch.zeros(K * T, H, dtype=torch.float64, device="cuda")
    dw = torch.zeros(K * T, dtype=torch.float64, device="cuda")
    for r in range(0, K * T, 65536):
        v = s["inv"][r:r + 65536]
        v = v[v >= 0].long()
        d = s["dout"].index_select(0, v % T).double()
        dw[v] = torch.einsum("rh,rh->r", d, s["y"][r:r + v.numel()].double())
        dy[r:r + v.numel()] = d * s["w"].flatten()[v].double()[:, None]
    return dict(dy=dy, dw=dw.reshape(K, T))


def _exact_linear(s):
    c = s["case"]
    y = torch.zeros(c["R"], c["OUT"], dtype=torch.float64, device="cuda")
    z = torch.zeros_like(y) if c["want_z"] else None
    act = dict(none=lambda v: v, relu=torch.relu, gelu=lambda v: v * torch.special.ndtr(v), silu=lambda v: v * torch.sigmoid(v))[c["act"]]
    for e, (a, b) in enumerate(zip(s["host_offsets"], s["host_offsets"][1:])):
        v = torch.nn.functional.linear(s["x"][a:b].double(), s["w"][e].double(), None if s["bias"] is None else s["bias"][e].double())
        y[a:b] = act(v)
        if z is not None:
            z[a:b] = v
        if s["residual"] is not None:
            y[a:b] += s["residual"][a:b]
    return dict(y=y, z=z) if c["want_z"] else dict(y=y)


def _exact_linear_grad(s):
    c = s["case"]
    E, IN, OUT = c["E"], c["IN"], c["OUT"]
    dx = torch.zeros(c["R"], IN, dtype=torch.float64, device="cuda")
    dw = torch.zeros(E, OUT, IN, dtype=torch.float64, device="cuda")
    db = torch.zeros(E, OUT, dtype=torch.float64, device="cuda")
    for e, (a, b) in enumerate(zip(s["host_offsets"], s["host_offsets"][1:])):
        dy = s["dy"][a:b].double()
        d = dy @ s["w"][e].double()
        if c["act"] == "relu":
            d = torch.where(s["z"][a:b] > 0, d, 0.0)
        elif c["act"] == "gelu":
            z = s["z"][a:b].double()
            d = d * (torch.special.ndtr(z) + z * torch.exp(z.square() / -2.0) / math.sqrt(2.0 * math.pi))
        elif c["act"] == "silu":
            z = s["z"][a:b].double()
            d = d * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        dx[a:b] = d
        torch.mm(dy.t(), s["x"][a:b].double(), out=dw[e])
        db[e] = dy.sum(0)
    return dict(dx=dx, dw=dw, db=db) if c["bias"] else dict(dx=dx, dw=dw)


_EXACT = dict(sort=_exact_sort, sort_grad=_exact_sort_grad, unsort=_exact_unsort, unsort_grad=_exact_unsort_grad, linear=_exact_linear,
              linear_grad=_exact_linear_grad)


def exact(case, seed):
    return _EXACT[case["op"]](prepare(case, seed))
