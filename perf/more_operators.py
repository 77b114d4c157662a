"""What is measured of the operators at the two ends of a BPT language model (arXiv 1911.04070, Sec. 4.2) and around its training
step: token ids to node states with the gradient of the table, the norm over all gradients with clipping, and penalties, biases
and masks on the logits of a decoding step.

``own`` false: plain elementary torch operations in 32 bits (64 for long sums), rounded once at the end.  ``own`` true: the calls a
user of this package makes.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    em = dict(op="embed", ragged=False, pad=False)
    cl = dict(op="clip", norm="2")
    lg = dict(op="logits", prompt=True, per_row=True, empty=False)
    return [
        # a decoding step of 16 sequences: one id each, a table of 32000 words
        dict(em, name="embed step", B=16, n=1, spans=0, V=32000, D=512, weight="bf16", out="bf16", train=False),
        # a prompt of 8192 bytes into the stack: 8192 token rows, 8191 zero rows of the span nodes
        dict(em, name="embed prompt", B=1, n=8192, spans=8191, V=256, D=512, weight="bf16", out="bf16", train=False),
        # a training step on the character-LM batch, forward + backward: few ids, each in thousands of places
        dict(em, name="embed train chars", B=4, n=8192, spans=8191, V=256, D=512, weight="bf16", out="bf16", train=True),
        # 16 padded sentences of up to 512 words, a 32-bit table of an odd size and width, states in bf16
        dict(em, name="embed train words", B=16, n=512, spans=511, V=32001, D=201, weight="f32", out="bf16", train=True, ragged=True, pad=True),
        # a wide model's batch over a large table: most rows of the gradient are zeros
        dict(em, name="embed train wide", B=8, n=8192, spans=0, V=131072, D=2048, weight="bf16", out="bf16", train=True),
        # the gradients of one narrow layer, cut to norm 1 for the optimizer: latency
        dict(cl, name="clip layer", layers=1, D=128, F=512, matrices="f32", vectors="f32", out="f32", most=1.0),
        # the 6-layer stack of width 512 with gated blocks, in place, below the limit (most steps of a training run)
        dict(cl, name="clip stack kept", layers=6, D=512, F=2048, matrices="bf16", vectors="f32", out="none", most=1e6),
        # the same stack above the limit, into 32-bit gradients for the optimizer's master weights
        dict(cl, name="clip stack cut", layers=6, D=512, F=2048, matrices="bf16", vectors="f32", out="f32", most=1.0),
        # a deep stack of odd widths: 0.6 billion values in 432 tensors, clipped by the largest one
        dict(cl, name="clip deep", layers=48, D=1023, F=2729, matrices="bf16", vectors="f32", out="bf16", most=0.05, norm="inf"),
        # one sequence of the character model at its full length: 256 logits, 8192 ids behind it
        dict(lg, name="logits step", B=1, V=256, T=8192, dtype="f32", bias="none", K=0, mask=True),
        # 32 requests with their own settings, ragged histories, a few biased words each and a grammar
        dict(lg, name="logits batch", B=32, V=32000, T=4096, dtype="bf16", bias="none", K=300, mask=True),
        # a full server batch over a large odd vocabulary, one bias for all
        dict(lg, name="logits large", B=256, V=128001, T=2048, dtype="bf16", bias="all", K=0, mask=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "clip", "logits"])
    if op == "embed":
        D, V = _log_int(rng, 16, 2048), _log_int(rng, 30, 131072)
        V = min(V, 131072 * 2048 // (2 * D))
        B, n = rng.choice([1, 2, 4, 16]), _log_int(rng, 1, 8192)
        n = max(1, min(n, 65536 * 2048 // (4 * B * D)))
        weight = rng.choice(["bf16", "f32"])
        return dict(op="embed", B=B, n=n, spans=rng.choice([0, n - 1]), V=V, D=D, weight=weight, out=rng.choice(["bf16", weight]),
                    train=rng.random() < 0.6, ragged=rng.random() < 0.4, pad=rng.random() < 0.4)
    if op == "clip":
        D, F = _log_int(rng, 16, 1023), _log_int(rng, 16, 2729)
        layers = max(1, min(_log_int(rng, 1, 48), 48 * 1023 * 2729 // (2 * D * F)))
        return dict(op="clip", layers=layers, D=D, F=F, matrices=rng.choice(["bf16", "f32"]), vectors=rng.choice(["bf16", "f32"]),
                    out=rng.choice(["none", "bf16", "f32"]), most=1e6 if rng.random() < 0.5 else rng.choice([0.25, 1.0, 5.0]), norm=rng.choice(["2", "2", "inf"]))
    V, B = _log_int(rng, 30, 128001), _log_int(rng, 1, 256)
    B = max(1, min(B, 256 * 128001 // (2 * V)))
    return dict(op="logits", B=B, V=V, T=_log_int(rng, 1, 8192), dtype=rng.choice(["bf16", "f32"]), bias=rng.choice(["none", "all", "each"]),
                K=rng.choice([0, 0, min(V, 17), min(V, 300)]), mask=rng.random() < 0.6, prompt=rng.random() < 0.5, per_row=rng.random() < 0.5,
                empty=rng.random() < 0.3)


def _ids(g, V, *shape):
    """Ids as text has them: a few frequent words, a long tail (about 1 / rank), in no order of their frequency."""
    u = torch.rand(*shape, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1)) - 1).long().clamp(0, V - 1)
    return torch.randperm(V, generator=g, device="cuda")[rank]


def _clip_shapes(case):
    """One layer: four projections, the gated block's three weights, two norms' vectors."""
    D, F = case["D"], case["F"]
    return ([(D, D)] * 4 + [(F, D), (F, D), (D, F)] + [(D,), (D,)]) * case["layers"]


def _name(v):
    return "bf16" if v.dtype == torch.bfloat16 else "f32"


def _in_one_buffer(shapes, kinds):
    """Tensors of these shapes and types as views of one zeroed buffer a type, each on a 128-byte boundary, as buckets of gradients are
    kept.  Returns (views, {type: buffer})."""
    length = lambda shape: -(-math.prod(shape) // 64) * 64
    total = {t: sum(length(s) for s, k in zip(shapes, kinds) if k == t) for t in set(kinds)}
    flat = {t: torch.zeros(k, device="cuda", dtype=TYPES[t]) for t, k in sorted(total.items())}
    at, views = dict.fromkeys(flat, 0), []
    for shape, t in zip(shapes, kinds):
        views.append(flat[t][at[t]:at[t] + math.prod(shape)].view(shape))
        at[t] += length(shape)
    return views, flat


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    ints = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda")
    s = dict(case)
    if case["op"] == "embed":
        B, n, V, D = (case[a] for a in ("B", "n", "V", "D"))
        s["ids"] = _ids(g, V, B, n)
        s["w"] = (rnd(V, D) * D ** -0.5).to(TYPES[case["weight"]]).requires_grad_(case["train"])
        s["scale"] = math.sqrt(D)
        s["lengths"] = ints(0, n + 1, B).to(torch.int32) if case["ragged"] else None
        s["padding"] = int(s["ids"][0, 0]) if case["pad"] else None
        s["d_out"] = rnd(B, n + case["spans"], D).to(TYPES[case["out"]]) if case["train"] else None
    elif case["op"] == "clip":
        shapes = _clip_shapes(case)
        s["grads"], s["flat"] = _in_one_buffer(shapes, [case["matrices" if len(shape) == 2 else "vectors"] for shape in shapes])
        for v in s["grads"]:
            v.copy_(rnd(*v.shape) * 0.02)
        s["into"], s["flat_into"] = (None, None) if case["out"] == "none" else _in_one_buffer(shapes, [case["out"]] * len(shapes))
    else:
        B, V, T, K = (case[a] for a in ("B", "V", "T", "K"))
        t = TYPES[case["dtype"]]
        s["x"] = (rnd(B, V) * 3).to(t)
        s["history"] = _ids(g, V, B, T)
        s["lengths"] = ints(0, T + 1, B).to(torch.int32)
        s["lengths"][0] = T
        s["prompts"] = (s["lengths"].double() * torch.rand(B, generator=g, device="cuda").double()).to(torch.int32) if case["prompt"] else None
        par = lambda lo, hi: torch.rand(B, generator=g, device="cuda") * (hi - lo) + lo
        s["repetition"], s["presence"], s["frequency"] = (par(1.0, 1.5), par(0.0, 1.0), par(0.0, 0.3)) if case["per_row"] else (1.2, 0.5, 0.125)
        s["bias_v"] = None if case["bias"] == "none" else rnd(*((V,) if case["bias"] == "all" else (B, V)))
        start = ints(0, V, B, 1)
        s["bias_ids"] = (start + torch.arange(K, device="cuda")) % V if K else None     # a run of neighbouring words, each once
        s["bias_values"] = rnd(B, K) * 5 if K else None
        s["allowed"] = None
        if case["mask"]:
            words = ints(-2 ** 31, 2 ** 31, B, (V + 31) // 32).to(torch.int32)
            words[::3] = -1                             # these rows are free, the others in the middle of a rule
            if case["empty"]:
                words[0] = 0
            s["allowed"] = words
    return s


# ---------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------
def _real(s):
    """[B, n], true where a token stands."""
    pos = torch.arange(s["n"], device="cuda")[None]
    return (pos < s["n"]).expand(s["B"], -1) if s["lengths"] is None else pos < s["lengths"][:, None]


def _plain_embed(s):
    real = _real(s)[..., None]
    w = s["w"].detach().float()
    rows = torch.where(real, w[s["ids"]] * s["scale"], torch.zeros((), device="cuda"))
    y = torch.zeros(s["B"], s["n"] + s["spans"], s["D"], device="cuda")
    y[:, :s["n"]] = rows
    out = {"y": y.to(TYPES[s["out"]])}
    if s["train"]:
        count = real if s["padding"] is None else real & (s["ids"] != s["padding"])[..., None]
        d = torch.where(count, s["d_out"][:, :s["n"]].float(), torch.zeros((), device="cuda"))
        if s["V"] < 1024:       # thousands of rows for one id
            d = d.double()
        dw = torch.zeros(s["V"], s["D"], device="cuda", dtype=d.dtype).index_add_(0, s["ids"].reshape(-1), d.reshape(-1, s["D"]))
        out["dw"] = (dw * s["scale"]).to(s["w"].dtype)
    return out


def _plain_clip(s):
    f = [v.float() for v in s["grads"]]
    if s["norm"] == "2":
        norm = torch.sqrt(sum((v * v).sum(dtype=torch.float64) for v in f)).float()
    else:
        norm = torch.stack([v.abs().max() for v in f]).max()
    c = torch.clamp(s["most"] / (norm + 1e-6), max=1.0)
    kinds = [_name(g) if s["into"] is None else s["out"] for g in s["grads"]]
    views, flat = _in_one_buffer([v.shape for v in f], kinds)
    for v, g in zip(views, f):
        v.copy_(g * c)
    return {"norm": norm, "grads": flat}


def _plain_logits(s):
    B, V, T = s["B"], s["V"], s["T"]
    x = s["x"].float()
    col = lambda p: p[:, None] if torch.is_tensor(p) else p
    pos = torch.arange(T, device="cuda")[None]
    real = pos < s["lengths"][:, None]
    made = real if s["prompts"] is None else real & (pos >= s["prompts"][:, None])
    count = lambda on: torch.zeros(B, V, device="cuda").scatter_add_(1, s["history"], on.float())
    seen, n = count(real), count(made)
    rep = col(s["repetition"])
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - (col(s["frequency"]) * n + col(s["presence"]) * (n > 0))
    if s["bias_v"] is not None:
        x = x + s["bias_v"]
    if s["K"]:
        x = x.scatter_add(1, s["bias_ids"], s["bias_values"])
    if s["allowed"] is not None:
        bits = (s["allowed"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bits.reshape(B, -1)[:, :V] > 0, x, torch.full((), -math.inf, device="cuda"))
    return {"y": x.to(s["x"].dtype)}


# ---------------------------------------------------------------------------------------------------------
# the package's calls
# ---------------------------------------------------------------------------------------------------------
def _own_embed(s):
    from paper_1911_04070_b200 import layer
    y = layer.token_states(s["ids"], s["w"], scale=s["scale"], span_rows=s["spans"], lengths=s["lengths"], padding_idx=s["padding"],
                           dtype=TYPES[s["out"]])
    if not s["train"]:
        return {"y": y}
    dw, = torch.autograd.grad(y, [s["w"]], s["d_out"])
    return {"y": y.detach(), "dw": dw}


def _own_clip(s):
    from paper_1911_04070_b200 import layer
    norm = layer.clip_gradients(s["grads"], s["most"], norm_type=float(s["norm"]), out=s["into"])
    return {"norm": norm, "grads": s["flat"] if s["into"] is None else s["flat_into"]}


def _own_logits(s):
    from paper_1911_04070_b200 import layer
    return {"y": layer.adjust_logits(s["x"], s["history"], lengths=s["lengths"], prompt_lengths=s["prompts"], repetition=s["repetition"],
                                     presence=s["presence"], frequency=s["frequency"], bias=s["bias_v"], bias_ids=s["bias_ids"],
                                     bias_values=s["bias_values"], allowed=s["allowed"])}


_PLAIN = {"embed": _plain_embed, "clip": _plain_clip, "logits": _plain_logits}
_OWN = {"embed": _own_embed, "clip": _own_clip, "logits": _own_logits}


def run(state):
    return (_OWN if own else _PLAIN)[state["op"]](state)


def work(case):
    size = lambda t: 2 if t == "bf16" else 4
    if case["op"] == "embed":
        B, n, V, D = (case[a] for a in ("B", "n", "V", "D"))
        we, oe = size(case["weight"]), size(case["out"])
        total = 8 * B * n + min(V, B * n) * D * we + B * (n + case["spans"]) * D * oe
        if case["train"]:
            total += B * n * D * oe + V * D * we
        return {"bytes": total, "flops": B * n * D * (3 if case["train"] else 1)}
    if case["op"] == "clip":
        total = flops = 0
        for shape in _clip_shapes(case):
            k = math.prod(shape)
            e = size(case["matrices" if len(shape) == 2 else "vectors"])
            cut = case["most"] < 1e6                      # in place and below the limit nothing is written
            total += k * (e + (size(case["out"]) if case["out"] != "none" else e if cut else 0))
            flops += 3 * k
        return {"bytes": total, "flops": flops}
    B, V, T, K = (case[a] for a in ("B", "V", "T", "K"))
    total = 2 * B * V * size(case["dtype"]) + 8 * B * T + 12 * B * K
    total += {"none": 0, "all": 4 * V, "each": 4 * B * V}[case["bias"]] + (4 * B * ((V + 31) // 32) if case["mask"] else 0)
    return {"bytes": total, "flops": 6 * B * V}


# ---------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------
def _exact_embed(s):
    F = torch.nn.functional
    B, n, D = s["B"], s["n"], s["D"]
    w = s["w"].detach().double()
    keep = torch.ones(B, n, device="cuda", dtype=torch.float64)
    if s["lengths"] is not None:
        for b, m in enumerate(s["lengths"].tolist()):
            keep[b, m:] = 0
    y = F.pad(F.embedding(s["ids"], w) * (s["scale"] * keep)[..., None], (0, 0, 0, s["spans"]))
    out = {"y": y}
    if s["train"]:
        if s["padding"] is not None:
            keep = keep.masked_fill(s["ids"] == s["padding"], 0)
        d = (s["d_out"][:, :n].double() * (s["scale"] * keep)[..., None]).view(-1, D)
        dw = torch.zeros_like(w)
        dw.index_put_((s["ids"].view(-1),), d, accumulate=True)
        out["dw"] = dw
    return out


def _exact_clip(s):
    sizes = [torch.linalg.vector_norm(v.double(), ord=float(s["norm"])) for v in s["grads"]]
    norm = torch.linalg.vector_norm(torch.stack(sizes), ord=float(s["norm"]))
    c = min(1.0, s["most"] / (float(norm) + 1e-6))
    flat = {}
    for v in s["grads"]:        # slot after slot of one buffer a type
        kind = s["out"] if s["into"] is not None else "bf16" if v.dtype == torch.bfloat16 else "f32"
        flat.setdefault(kind, []).append(torch.nn.functional.pad(v.double().reshape(-1) * c, (0, -v.numel() % 64)))
    return {"norm": norm, "grads": {kind: torch.cat(parts) for kind, parts in flat.items()}}


def _exact_logits(s):
    V = s["V"]
    y = s["x"].double()
    number = lambda p, b: float(p[b]) if torch.is_tensor(p) else float(p)
    shift = torch.arange(32, device="cuda", dtype=torch.int64)
    for b, m in enumerate(s["lengths"].tolist()):
        first = 0 if s["prompts"] is None else int(s["prompts"][b])
        words, times = torch.unique(s["history"][b, first:m], return_counts=True)
        known = torch.unique(s["history"][b, :m])
        r = number(s["repetition"], b)
        v = y[b, known]
        y[b, known] = torch.maximum(v, torch.zeros_like(v)) / r + torch.minimum(v, torch.zeros_like(v)) * r
        y[b, words] -= times.double() * number(s["frequency"], b) + number(s["presence"], b)
        if s["bias_v"] is not None:
            y[b] += (s["bias_v"] if s["bias_v"].dim() == 1 else s["bias_v"][b]).double()
        if s["K"]:
            y[b, s["bias_ids"][b]] += s["bias_values"][b].double()
        if s["allowed"] is not None:
            word = s["allowed"][b].long() & 0xffffffff
            free = (word[:, None].bitwise_right_shift(shift) & 1).bool().view(-1)[:V]
            y[b].masked_fill_(~free, -math.inf)
    return {"y": y}


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"embed": _exact_embed, "clip": _exact_clip, "logits": _exact_logits}[case["op"]](s)
