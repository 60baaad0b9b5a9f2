"""What the operators of one MoE block around the router are measured on: the whole layer for a few tokens, the norms before and
after the block with its gate and residual (forward and gradient), and the same with the activations kept in 8 bits.

``own`` = False runs them in elementary torch operations in 32 bits, ``own`` = True through ``paper_2401_13920_b200.block``.
"""
import math

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # --- the layer for a few tokens: decoding steps of a served model ---
        # one token through a small layer (hidden size and experts of the tiny configuration): launch latency
        dict(name="few_1_small", op="few", T=1, H=1024, F=4096, E=8, K=1, bias=False),
        # one token through the layer of the full-layer configuration: the weights of one expert, once
        dict(name="few_1", op="few", T=1, H=2560, F=10240, E=32, K=1, bias=False),
        # a small decoding batch: most tokens meet an expert of their own
        dict(name="few_8", op="few", T=8, H=2560, F=10240, E=32, K=1, bias=True),
        # a large decoding batch with two experts for each token: nearly all the weights of the layer
        dict(name="few_64_top2", op="few", T=64, H=2560, F=10240, E=32, K=2, bias=False),
        # odd sizes: a prompt's tail of 13 tokens, three choices, sizes that are no multiple of any tile
        dict(name="few_13_odd", op="few", T=13, H=1560, F=4104, E=24, K=3, bias=True),
        # --- norms, forward ---
        # decoding: eight rows, the expert outputs in token order
        dict(name="norm_8", op="norm", T=8, H=2560, dtype="bf16", slots=False, ckpt=False),
        # a training step of the 65536 x 5120 configuration: expert outputs in slot order, some tokens dropped
        dict(name="norm_65536", op="norm", T=65536, H=5120, dtype="bf16", slots=True, ckpt=False),
        # the same pass leaving 8-bit checkpoints behind, on the full-layer configuration
        dict(name="norm_ckpt_65536", op="norm", T=65536, H=2560, dtype="bf16", slots=True, ckpt=True),
        # --- norms, gradient ---
        # the tiny configuration in fp32
        dict(name="grad_f32_4096", op="grad", T=4096, H=1024, dtype="f32", slots=True, ckpt=False),
        # odd sizes: a row length that no 16-byte load divides
        dict(name="grad_odd", op="grad", T=3001, H=777, dtype="bf16", slots=False, ckpt=False),
        # a training step of the 65536 x 5120 configuration, from the stored activations
        dict(name="grad_65536", op="grad", T=65536, H=5120, dtype="bf16", slots=True, ckpt=False),
        # the same from 8-bit checkpoints
        dict(name="grad_ckpt_65536", op="grad", T=65536, H=5120, dtype="bf16", slots=True, ckpt=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["few", "few", "norm", "grad", "grad"])
    if op == "few":
        E = rng.choice([4, 8, 12, 16, 24, 32, 64])
        # H is a multiple of E and of 8; both sizes over their whole range, within the largest listed layer
        unit = E * 8 // math.gcd(E, 8)
        H = unit * max(1, _log_uniform(rng, 256, 5120) // unit)
        F = 8 * _log_uniform(rng, 32, 1280)
        while E * H * F > 32 * 2560 * 10240:
            F = 8 * max(1, F // 16)
        return dict(op="few", T=_log_uniform(rng, 1, 128), H=H, F=F, E=E, K=rng.choice([1, 1, 2, 3]), bias=rng.random() < 0.5)
    T, H = _log_uniform(rng, 1, 65536), _log_uniform(rng, 64, 8192)
    if rng.random() < 0.75:
        H = 8 * max(1, H // 8)      # three quarters with rows of whole 16-byte vectors, the others odd
    T = max(1, min(T, 65536 * 5120 // H // 2))
    return dict(op=op, T=T, H=H, dtype=rng.choice(["bf16", "bf16", "f32"]), slots=rng.random() < 0.6, ckpt=rng.random() < 0.4)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, dtype=torch.float32, std=1.0, mean=0.0):
    return torch.empty(*shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)


def prepare(case, seed):
    g = _gen(seed)
    T, H = case["T"], case["H"]
    if case["op"] == "few":
        E, F = case["E"], case["F"]
        return dict(case=case, x=_normal(g, T, H, dtype=torch.bfloat16),
                    eps=_normal(g, E, std=0.05) if case["bias"] else None,
                    w_in=_normal(g, E, F, H, dtype=torch.bfloat16, std=0.02),
                    w_out=_normal(g, E, H, F, dtype=torch.bfloat16, std=0.02))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = dict(case=case, res_scale=0.9, gate_w=torch.rand(T, generator=g, device="cuda") * 0.9 + 0.05,
             w_post=_normal(g, H, std=0.1, mean=0.5), w_pre=_normal(g, H, std=0.1, mean=1.0), slot=None, inv=None, rows=T)
    if case["slots"]:
        # rows of the dispatch buffer in random order, one in twelve tokens dropped (its row stays empty)
        slot = torch.randperm(T, generator=g, device="cuda").to(torch.int32)
        slot[torch.rand(T, generator=g, device="cuda") < 1.0 / 12.0] = -1
        inv = torch.full((T,), -1, dtype=torch.int32, device="cuda")
        kept = torch.nonzero(slot >= 0).squeeze(1)
        inv[slot[kept].long()] = kept.to(torch.int32)
        s.update(slot=slot, inv=inv)
    if case["op"] == "norm":
        s.update(h=_normal(g, T, H, dtype=dt, std=2.0), y=_normal(g, T, H, dtype=dt, std=0.3))
        return s
    s.update(dh_out=_normal(g, T, H, dtype=dt, std=0.1), dn=_normal(g, T, H, dtype=dt, std=0.1))
    if case["ckpt"]:
        # what the forward pass left: the normalised rows in E4M3 and the reciprocal norms
        s.update(u8=_normal(g, T, H, dtype=torch.bfloat16).to(torch.float8_e4m3fn),
                 x8=_normal(g, T, H, dtype=torch.bfloat16).to(torch.float8_e4m3fn),
                 r_post=torch.rand(T, generator=g, device="cuda") + 2.5, r_pre=torch.rand(T, generator=g, device="cuda") * 0.2 + 0.4)
    else:
        s.update(h_out=_normal(g, T, H, dtype=dt, std=2.0), y=_normal(g, T, H, dtype=dt, std=0.3))
    return s


def _few_plain(s):
    c = s["case"]
    T, H, E, K = c["T"], c["H"], c["E"], c["K"]
    x = s["x"].float()
    G = x.reshape(T, E, H // E).mean(2)
    if s["eps"] is not None:
        G = G + s["eps"]
    G = G.clamp_min(0.0)
    p = torch.exp(G - G.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    order = torch.sort(G, dim=1, descending=True, stable=True).indices[:, :K]     # a tie goes to the lower index
    w = p.gather(1, order)
    share = torch.zeros(T, E, device=x.device).scatter_(1, order, w)
    h = torch.matmul(x, s["w_in"].float().transpose(1, 2))                        # [E][T][F]
    h = 0.5 * h * (1.0 + torch.erf(h * 0.7071067811865476))
    y = torch.matmul(h, s["w_out"].float().transpose(1, 2))                       # [E][T][H]
    out = (share.t()[:, :, None] * y).sum(0)
    return dict(idx=order.t().contiguous().to(torch.int32), w=w.t().contiguous(), out=out.to(torch.bfloat16))


def _rows_of(y, slot):
    """The block's output row of each token, zero for a dropped one."""
    v = y.float()
    if slot is None:
        return v
    return v[slot.clamp_min(0).long()] * (slot >= 0)[:, None]


def _norm_plain(s):
    dt = s["h"].dtype
    v = _rows_of(s["y"], s["slot"])
    r_post = torch.rsqrt((v * v).mean(1) + EPS)
    u = v * r_post[:, None]
    hp = s["res_scale"] * s["h"].float() + s["gate_w"][:, None] * s["w_post"] * u
    r_pre = torch.rsqrt((hp * hp).mean(1) + EPS)
    xh = hp * r_pre[:, None]
    r = dict(h_out=hp.to(dt), n=(xh * s["w_pre"]).to(dt))
    if s["case"]["ckpt"]:
        r.update(u8=u.to(torch.float8_e4m3fn), x8=xh.to(torch.float8_e4m3fn), r_post=r_post, r_pre=r_pre)
    return r


def _grad_plain(s):
    dt, H, slot = s["dn"].dtype, s["case"]["H"], s["slot"]
    if s["case"]["ckpt"]:
        u, xh, r_post, r_pre = s["u8"].float(), s["x8"].float(), s["r_post"], s["r_pre"]
        if slot is not None:
            u = u * (slot >= 0)[:, None]
    else:
        v, hp = _rows_of(s["y"], slot), s["h_out"].float()
        r_post = torch.rsqrt((v * v).mean(1) + EPS)
        r_pre = torch.rsqrt((hp * hp).mean(1) + EPS)
        u, xh = v * r_post[:, None], hp * r_pre[:, None]
    dn = s["dn"].float()
    gp = dn * s["w_pre"]
    D = s["dh_out"].float() + r_pre[:, None] * (gp - xh * (gp * xh).mean(1, keepdim=True))
    Dw = D * s["w_post"]
    k = (Dw * u).sum(1)
    dv = (r_post * s["gate_w"])[:, None] * (Dw - u * (k / H)[:, None])
    if slot is None:
        dy = dv.to(dt)
    else:
        dy = torch.zeros(s["rows"], H, dtype=dt, device=dv.device)
        kept = torch.nonzero(slot >= 0).squeeze(1)
        dy[slot[kept].long()] = dv[kept].to(dt)
    return dict(dh=(s["res_scale"] * D).to(dt), dy=dy, dgate=k, dw_post=(s["gate_w"][:, None] * D * u).sum(0), dw_pre=(dn * xh).sum(0))


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return _few_plain(s) if op == "few" else _norm_plain(s) if op == "norm" else _grad_plain(s)
    from paper_2401_13920_b200 import block
    if op == "few":
        out, idx, w = block.moe_few(s["x"], s["w_in"], s["w_out"], K=s["case"]["K"], eps=s["eps"])
        return dict(idx=idx, w=w, out=out)
    if op == "norm":
        h_out, n, ck = block.block_norm(s["h"], s["y"], slot=s["slot"], gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"],
                                        res_scale=s["res_scale"], eps=EPS, checkpoint=s["case"]["ckpt"])
        r = dict(h_out=h_out, n=n)
        if ck is not None:
            r.update(u8=ck.u8, x8=ck.x8, r_post=ck.r_post, r_pre=ck.r_pre)
        return r
    ck = block.Checkpoint(s["u8"], s["x8"], s["r_post"], s["r_pre"]) if s["case"]["ckpt"] else None
    dh, dy, dgate, dw_post, dw_pre = block.block_norm_grad(
        s["dh_out"], s["dn"], None if ck else s["h_out"], None if ck else s["y"], checkpoint=ck, slot=s["slot"], inv=s["inv"],
        gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"], res_scale=s["res_scale"], eps=EPS)
    return dict(dh=dh, dy=dy, dgate=dgate, dw_post=dw_post, dw_pre=dw_pre)


def work(case):
    T, H = case["T"], case["H"]
    if case["op"] == "few":
        F, E, K = case["F"], case["E"], case["K"]
        hit = E * (1.0 - (1.0 - 1.0 / E) ** (T * K)) if K == 1 else E * (1.0 - (1.0 - K / E) ** T)   # experts met, on average
        return {"bytes": hit * 4.0 * F * H + 4.0 * T * H + 8.0 * T * K, "flops": 4.0 * T * K * F * H}
    el = 2 if case["dtype"] == "bf16" else 4
    kept = 11.0 / 12.0 if case["slots"] else 1.0
    index = 8.0 if case["slots"] else 4.0
    if case["op"] == "norm":
        moved = T * H * el * (3.0 + kept) + (T * H * 2.0 + 8.0 * T if case["ckpt"] else 0.0)
        return {"bytes": moved + index * T + 8.0 * H, "flops": 10.0 * T * H}
    saved = T * H * (1.0 + kept) if case["ckpt"] else T * H * el * (1.0 + kept)
    return {"bytes": T * H * el * 4.0 + saved + (index + 4.0 + (8.0 if case["ckpt"] else 0.0) + (4.0 if case["slots"] else 0.0)) * T + 16.0 * H,
            "flops": 24.0 * T * H}


def _few_exact(s):
    c = s["case"]
    T, H, E, K = c["T"], c["H"], c["E"], c["K"]
    x = s["x"].double()
    G = torch.stack([x[:, i * (H // E):(i + 1) * (H // E)].sum(1) / (H // E) for i in range(E)], 1)
    if s["eps"] is not None:
        G = G + s["eps"].double()[None]
    G = torch.maximum(G, torch.zeros_like(G))
    w_all = (G - torch.logsumexp(G, 1, keepdim=True)).exp()
    left, idx, w = G.clone(), [], []
    for _ in range(K):
        top = left.amax(1, keepdim=True)
        first = (left == top).int().argmax(1)
        at = torch.arange(E, device=x.device)[None].expand(T, E)
        first = torch.where(left == top, at, E).amin(1)
        idx.append(first)
        w.append(w_all.gather(1, first[:, None])[:, 0])
        left.scatter_(1, first[:, None], -1.0)
    out = torch.zeros(T, H, dtype=torch.float64, device=x.device)
    for e in sorted(set(torch.stack(idx).flatten().tolist())):
        wi, wo = s["w_in"][e].double(), s["w_out"][e].double()
        for k in range(K):
            t = torch.nonzero(idx[k] == e).squeeze(1)
            if t.numel():
                a = x[t] @ wi.t()
                a = a * torch.special.ndtr(a)
                out[t] += w[k][t][:, None] * (a @ wo.t())
    return dict(idx=None, w=torch.stack(w), out=out)


def _chunks(T, H):
    step = max(1, (1 << 26) // H)
    return [(a, min(T, a + step)) for a in range(0, T, step)]


def _norm_exact(s):
    T, H = s["case"]["T"], s["case"]["H"]
    names = ["h_out", "n"] + (["u8", "x8", "r_post", "r_pre"] if s["case"]["ckpt"] else [])
    parts = {k: [] for k in names}
    wp, wn = s["w_post"].double(), s["w_pre"].double()
    for a, b in _chunks(T, H):
        at = torch.arange(a, b, device="cuda") if s["slot"] is None else s["slot"][a:b].long()
        v = torch.where((at >= 0)[:, None], s["y"][at.clamp_min(0)].double(), 0.0)
        r1 = 1.0 / (v.pow(2).sum(1) / H + EPS).sqrt()
        hp = s["h"][a:b].double() * s["res_scale"] + (s["gate_w"][a:b].double() * r1)[:, None] * v * wp[None]
        r2 = 1.0 / (hp.pow(2).sum(1) / H + EPS).sqrt()
        for k, t in zip(["h_out", "n", "u8", "x8", "r_post", "r_pre"], [hp, hp * r2[:, None] * wn, v * r1[:, None], hp * r2[:, None], r1, r2]):
            if k in parts:
                parts[k].append(t)
    return {k: torch.cat(v) for k, v in parts.items()}


def _grad_exact(s):
    T, H = s["case"]["T"], s["case"]["H"]
    wp, wn = s["w_post"].double()[None], s["w_pre"].double()[None]
    dh, dg = torch.empty(T, H, dtype=torch.float64, device="cuda"), torch.empty(T, dtype=torch.float64, device="cuda")
    dy = torch.zeros(s["rows"], H, dtype=torch.float64, device="cuda")
    dwp, dwn = torch.zeros(H, dtype=torch.float64, device="cuda"), torch.zeros(H, dtype=torch.float64, device="cuda")
    for a, b in _chunks(T, H):
        at = torch.arange(a, b, device="cuda") if s["slot"] is None else s["slot"][a:b].long()
        have = at >= 0
        if s["case"]["ckpt"]:
            u = torch.where(have[:, None], s["u8"][a:b].double(), 0.0)
            z, r1, r2 = s["x8"][a:b].double(), s["r_post"][a:b].double(), s["r_pre"][a:b].double()
        else:
            v, hp = torch.where(have[:, None], s["y"][at.clamp_min(0)].double(), 0.0), s["h_out"][a:b].double()
            r1, r2 = 1.0 / (v.pow(2).sum(1) / H + EPS).sqrt(), 1.0 / (hp.pow(2).sum(1) / H + EPS).sqrt()
            u, z = v * r1[:, None], hp * r2[:, None]
        q, gate = s["dn"][a:b].double(), s["gate_w"][a:b].double()[:, None]
        dwn += torch.einsum("th,th->h", q, z)
        D = s["dh_out"][a:b].double() + r2[:, None] * (q * wn - z * (torch.einsum("th,th->t", q * wn, z) / H)[:, None])
        dh[a:b] = D * s["res_scale"]
        k = torch.einsum("th,th->t", D * wp, u)
        dg[a:b] = k
        dwp += torch.einsum("th,th->h", D * gate, u)
        dy[at[have]] = (r1[:, None] * gate * (D * wp - u * (k / H)[:, None]))[have]
    return dict(dh=dh, dy=dy, dgate=dg, dw_post=dwp, dw_pre=dwn)


def exact(case, seed):
    s = prepare(case, seed)
    return _few_exact(s) if case["op"] == "few" else _norm_exact(s) if case["op"] == "norm" else _grad_exact(s)
