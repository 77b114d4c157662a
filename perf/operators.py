"""What is measured of the position-wise operators of a BPT layer (arXiv 1911.04070, Algorithm 2): the gated
feed-forward block and the seam between two blocks (norm after a block, gate, scaled residual, norm before the
next block), each forward alone and forward + backward.

``own`` false: plain elementary torch operations in 32 bits, rounded once at the end.  ``own`` true: the calls a
user of this package makes.
"""
import math

import torch

own = False

SQRT_HALF = math.sqrt(0.5)


def listed():
    ff = dict(op="ff", dtype="bf16")
    nm = dict(op="norm", eps=1e-5)
    return [
        # one row through the block of the 6-layer stack (width 512, inner width 2048): a single new token
        dict(ff, name="ff row", rows=1, D=512, F=2048, act="silu", train=False),
        # a decoding step of one sequence of 8192: the new token and its 13 ancestors
        dict(ff, name="ff step", rows=14, D=512, F=2048, act="silu", train=False),
        # a decoding step of 16 sequences
        dict(ff, name="ff step of 16", rows=224, D=512, F=2048, act="gelu", train=False),
        # the whole stack's forward over one sequence of 8192: 16383 nodes
        dict(ff, name="ff prompt", rows=16383, D=512, F=2048, act="silu", train=False),
        # a training step on one short sequence (512 tokens, 1023 nodes); inner width 8/3 of the model's
        dict(ff, name="ff train short", rows=1023, D=512, F=1368, act="gelu", train=True),
        # a training step on the character-LM batch: 4 sequences of 8192, 4 x 16383 nodes
        dict(ff, name="ff train", rows=65532, D=512, F=2048, act="silu", train=True),
        # between two blocks of a decoding step: 14 rows, sandwich norms and a learned gate
        dict(nm, name="norm step", rows=14, D=512, dtype="bf16", norm="layer", post="layer", gate=1, alpha=1.0, keep=True, train=False),
        # Algorithm 2's own norm(H + A) over 16 sequences of 512 (16 x 1023 nodes)
        dict(nm, name="norm infer", rows=16368, D=512, dtype="bf16", norm="layer", post="none", gate=0, alpha=1.0, keep=False, train=False),
        # sandwich norms, gate and residual scale over the character-LM batch, forward + backward
        dict(nm, name="norm train", rows=65532, D=512, dtype="bf16", norm="layer", post="layer", gate=1, alpha=0.5, keep=True, train=True),
        # a gate for each of 32 sequences (conditioning), rms norms, an odd width, 32 bits
        dict(nm, name="norm train gates", rows=32736, D=201, dtype="f32", norm="rms", post="rms", gate=32, alpha=1.0, keep=True, train=True),
        # a wide model's short batch: scaled residual under one norm, forward + backward
        dict(nm, name="norm train wide", rows=4092, D=4096, dtype="bf16", norm="rms", post="none", gate=0, alpha=1.25, keep=False, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        D, F = 8 * _log_int(rng, 4, 160), 8 * _log_int(rng, 4, 512)
        most = min(65532, 65532 * 512 * 2048 // (D * F))
        return dict(op="ff", dtype="bf16", rows=_log_int(rng, 1, most), D=D, F=F, act=rng.choice(["silu", "gelu", "relu"]),
                    train=rng.random() < 0.5)
    D = _log_int(rng, 16, 5000)
    dtype = rng.choice(["bf16", "f32"])
    most = min(65532, 65532 * 512 // (D * (2 if dtype == "f32" else 1)))
    rows = _log_int(rng, 1, most)
    gate = rng.choice([0, 1, 1, 8])                     # no gate, one for all rows, one for each of 8 sequences
    rows = max(8, rows // 8 * 8) if gate == 8 else rows
    norm, post = rng.choice([("layer", "none"), ("layer", "layer"), ("rms", "none"), ("rms", "rms"), ("layer", "rms"), ("none", "layer")])
    return dict(op="norm", rows=rows, D=D, dtype=dtype, norm=norm, post=post, gate=gate, alpha=rng.choice([1.0, 0.5, 1.25]),
                eps=rng.choice([1e-5, 1e-6]), keep=rng.random() < 0.5, train=rng.random() < 0.6)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def rnd(*shape, std=1.0, mean=0.0, dtype=t):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype).requires_grad_(case["train"])

    s = dict(case)
    M, D = case["rows"], case["D"]
    if case["op"] == "ff":
        F = case["F"]
        s.update(x=rnd(M, D), w_gate=rnd(F, D, std=D ** -0.5), w_up=rnd(F, D, std=D ** -0.5), w_down=rnd(D, F, std=F ** -0.5))
        s["d_y"] = rnd(M, D).detach() if case["train"] else None
        return s
    s.update(h=rnd(M, D, mean=0.25), b=rnd(M, D, std=0.5))
    f32 = torch.float32
    for name, kind, par in (("norm", case["norm"], "weight"), ("post", case["post"], "post_weight")):
        s[par] = None if kind == "none" else rnd(D, std=0.2, mean=1.0, dtype=f32)
        s[par.replace("weight", "bias")] = rnd(D, std=0.2, dtype=f32) if kind == "layer" else None
    G = case["gate"]
    s["gate_v"] = None if G == 0 else rnd(D, std=0.2, mean=0.7, dtype=f32) if G == 1 else rnd(G, D, std=0.2, mean=0.7)
    s["with_sum"] = case["keep"] or case["norm"] == "none"
    s["d_y"] = rnd(M, D).detach() if case["train"] and case["norm"] != "none" else None
    s["d_r"] = rnd(M, D).detach() if case["train"] and s["with_sum"] else None
    return s


# ---------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------
def _act(g, act):
    """act(g) and its derivative."""
    if act == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    cdf = 0.5 * (1 + torch.erf(g * SQRT_HALF))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain_ff(s):
    x, wg, wu, wd = (s[n].detach().float() for n in ("x", "w_gate", "w_up", "w_down"))
    t = s["x"].dtype
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(g, s["act"])
    h = a * u
    out = {"y": (h @ wd.T).to(t)}
    if s["train"]:
        dy = s["d_y"].float()
        dh = dy @ wd
        dg, du = dh * u * da, dh * a
        out.update(dx=(dg @ wg + du @ wu).to(t), dw_gate=(dg.T @ x).to(t), dw_up=(du.T @ x).to(t), dw_down=(dy.T @ h).to(t))
    return out


def _plain_norm_fwd(x, kind, w, b, eps):
    """The normalised row, its reciprocal deviation and the scaled and shifted row."""
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    rstd = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    xh = c * rstd
    return xh, rstd, xh * w if b is None else xh * w + b


def _plain_norm_bwd(d, xh, rstd, kind, w):
    dxh = d * w
    c = dxh - dxh.mean(-1, keepdim=True) if kind == "layer" else dxh
    return rstd * (c - xh * (dxh * xh).mean(-1, keepdim=True))


def _plain_norm(s):
    t = s["h"].dtype
    f = lambda n: None if s[n] is None else s[n].detach().float()
    h, b, w, bias, pw, pb, gate = (f(n) for n in ("h", "b", "weight", "bias", "post_weight", "post_bias", "gate_v"))
    M, D, G = s["rows"], s["D"], s["gate"]
    rows = lambda v: v if G < 2 else v.repeat_interleave(M // G, dim=0)
    if s["post"] != "none":
        ph, prstd, n = _plain_norm_fwd(b, s["post"], pw, pb, s["eps"])
    else:
        n = b
    r = s["alpha"] * h + (n if gate is None else rows(gate) * n)
    out = {}
    if s["norm"] != "none":
        xh, rstd, y = _plain_norm_fwd(r, s["norm"], w, bias, s["eps"])
        out["y"] = y.to(t)
    if s["with_sum"]:
        out["r"] = r.to(t)
    if s["train"]:
        dR = torch.zeros_like(r) if s["d_r"] is None else s["d_r"].float()
        if s["norm"] != "none":
            dy = s["d_y"].float()
            dR = dR + _plain_norm_bwd(dy, xh, rstd, s["norm"], w)
            out["d_weight"] = (dy * xh).sum(0)
            if bias is not None:
                out["d_bias"] = dy.sum(0)
        out["dh"] = (s["alpha"] * dR).to(t)
        if gate is not None:
            dg = dR * n
            out["d_gate"] = dg.sum(0) if G == 1 else dg.view(G, M // G, D).sum(1).to(t)
            dn = rows(gate) * dR
        else:
            dn = dR
        if s["post"] != "none":
            out["d_post_weight"] = (dn * ph).sum(0)
            if pb is not None:
                out["d_post_bias"] = dn.sum(0)
            dn = _plain_norm_bwd(dn, ph, prstd, s["post"], pw)
        out["db"] = dn.to(t)
    return out


# ---------------------------------------------------------------------------------------------------------
# the package's calls
# ---------------------------------------------------------------------------------------------------------
def _own_ff(s):
    from paper_1911_04070_b200 import layer
    y = layer.gated_feed_forward(s["x"], s["w_gate"], s["w_up"], s["w_down"], act=s["act"])
    out = {"y": y}
    if s["train"]:
        names = ("x", "w_gate", "w_up", "w_down")
        grads = torch.autograd.grad(y, [s[n] for n in names], s["d_y"])
        out.update(zip(("dx", "dw_gate", "dw_up", "dw_down"), grads))
        out["y"] = y.detach()
    return out


def _own_norm(s):
    from paper_1911_04070_b200 import layer
    kind = lambda n: None if s[n] == "none" else s[n]
    gate = s["gate_v"] if s["gate"] < 2 else s["gate_v"][:, None]
    h, b = ((s[n] if s["gate"] < 2 else s[n].view(s["gate"], -1, s["D"])) for n in ("h", "b"))
    got = layer.residual_norm(h, b, s["weight"], s["bias"], norm=kind("norm"), post_norm=kind("post"), post_weight=s["post_weight"],
                              post_bias=s["post_bias"], gate=gate, alpha=s["alpha"], eps=s["eps"], return_sum=s["with_sum"])
    flat = lambda v: v.detach().view(s["rows"], s["D"])
    if s["norm"] == "none":
        out, tops, ups = {"r": flat(got)}, [got], ["d_r"]
    elif s["with_sum"]:
        out, tops, ups = {"y": flat(got[1]), "r": flat(got[0])}, [got[1], got[0]], ["d_y", "d_r"]
    else:
        out, tops, ups = {"y": flat(got)}, [got], ["d_y"]
    if s["train"]:
        names = [n for n in ("h", "b", "weight", "bias", "gate_v", "post_weight", "post_bias") if s[n] is not None]
        grads = torch.autograd.grad(tops, [s[n] for n in names], [s[n].view(a.shape) for n, a in zip(ups, tops)])
        key = {"h": "dh", "b": "db", "gate_v": "d_gate"}
        out.update((key.get(n, "d_" + n), g) for n, g in zip(names, grads))
    return out


def run(state):
    if own:
        return (_own_ff if state["op"] == "ff" else _own_norm)(state)
    return (_plain_ff if state["op"] == "ff" else _plain_norm)(state)


def work(case):
    M, D = case["rows"], case["D"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "ff":
        F = case["F"]
        if case["train"]:     # reads x, d_y, three weights; writes y, dx, three gradients
            return {"bytes": e * (4 * M * D + 6 * D * F), "flops": 18 * M * D * F}
        return {"bytes": e * (2 * M * D + 3 * D * F), "flops": 6 * M * D * F}
    n_norm, n_sum = int(case["norm"] != "none"), int(case["keep"] or case["norm"] == "none")
    fwd = 2 + n_norm + n_sum                             # h, b, y, r
    bwd = n_norm + n_sum + 2 if case["train"] else 0     # d_y, d_r, dh, db
    small = 4 * D * (case["gate"] + 2) * (2 if case["train"] else 1)
    return {"bytes": e * M * D * (fwd + bwd) + small, "flops": M * D * (40 if case["train"] else 15)}


# ---------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    F = torch.nn.functional
    d = lambda n: None if s.get(n) is None else s[n].detach().double().requires_grad_(case["train"])
    with torch.enable_grad():
        if case["op"] == "ff":
            v = {n: d(n) for n in ("x", "w_gate", "w_up", "w_down")}
            act = {"silu": F.silu, "gelu": F.gelu, "relu": F.relu}[case["act"]]
            y = F.linear(act(F.linear(v["x"], v["w_gate"])) * F.linear(v["x"], v["w_up"]), v["w_down"])
            out = {"y": y.detach()}
            if case["train"]:
                out.update(zip(("dx", "dw_gate", "dw_up", "dw_down"), torch.autograd.grad(y, list(v.values()), d("d_y").detach())))
            return out
        v = {n: d(n) for n in ("h", "b", "weight", "bias", "gate_v", "post_weight", "post_bias")}
        D, G = case["D"], case["gate"]
        norm = {"none": lambda x, w, c: x, "layer": lambda x, w, c: F.layer_norm(x, (D,), w, c, case["eps"]),
                "rms": lambda x, w, c: F.rms_norm(x, (D,), w, case["eps"])}
        n = norm[case["post"]](v["b"], v["post_weight"], v["post_bias"])
        if G == 1:
            n = n * v["gate_v"]
        elif G > 1:
            n = (n.view(G, -1, D) * v["gate_v"].view(G, 1, D)).view(-1, D)
        r = torch.add(n, v["h"], alpha=case["alpha"])
        y = norm[case["norm"]](r, v["weight"], v["bias"])
        has_y = case["norm"] != "none"
        out = {}
        if has_y:
            out["y"] = y.detach()
        if s["with_sum"]:
            out["r"] = r.detach()
        if case["train"]:
            loss = sum((a * d(m).detach()).sum() for a, m in ((y, "d_y"), (r, "d_r")) if s[m] is not None)
            names = [m for m in v if v[m] is not None]
            key = {"h": "dh", "b": "db", "gate_v": "d_gate"}
            out.update((key.get(m, "d_" + m), g) for m, g in zip(names, torch.autograd.grad(loss, [v[m] for m in names])))
        return out
