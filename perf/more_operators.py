"""Performance cases of routed layers and of gradient clipping, beside the row operators.

A layer of a radial network is a grouped product with a bias, an activation and perhaps the layer's input added
back (`grouped_layer`). Its weights go by the chemical element or the element pair of a row, or by experts that
the row itself is routed to (`route_rows`), several to a row: then `group_rows` orders the (row, expert) pairs,
the layers run over the pairs, and `mix_rows` joins the results of each row with the router's weights.
`adamw_grad_norm` is what a training step takes between the gradients and `adamw`: the norm of all of them and
the factor that clips it. Widths are those of `paper_2605_15073_amd.inputs`: C * L channels of the benchmark plan
(64 * 7, 128 * 7, 64 * 21), 64 or 128 hidden ones, 8 Gaussians; rows are the 64 nodes, 10,000 nodes, 261,766 and
525,308 edges of its structures. Numbers of experts and of experts a row are generic.

Where `own` is false the operators are computed in elementary torch operations in 32 bits, rounded once at the
end; the keys that experts are chosen by, and sums over whole models, in 64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

MAX_GROUPS = 4005     # unordered pairs of 89 elements
WIDTHS = (8, 16, 64, 128, 448, 896, 1344)   # basis, hidden and C * L widths


# ---------------------------------------------------------------- the cases

def _route(name, rows, experts, top_k, dtype, score, bias=False, blocks=1, keep=1, renorm=True, masked=0.0,
           grad=False):
    return dict(name=name, kind="route", rows=rows, experts=experts, top_k=top_k, dtype=dtype, score=score,
                bias=bias, blocks=blocks, keep=keep, renorm=renorm, masked=masked, grad=grad)


def _layer(name, rows, groups, n_in, n_out, dtype, act, per_row=1, residual=False, keep_z=False, pad=0.0,
           grad=False):
    return dict(name=name, kind="layer", rows=rows, groups=groups, n_in=n_in, n_out=n_out, dtype=dtype, act=act,
                per_row=per_row, residual=residual, keep_z=keep_z, pad=pad, grad=grad)


def _mix(name, rows, per_row, width, dtype, residual=False, weights=True, grad=False):
    return dict(name=name, kind="mix", rows=rows, per_row=per_row, width=width, dtype=dtype, residual=residual,
                weights=weights, grad=grad)


def _norm(name, tensors, elements, dtype):
    return dict(name=name, kind="norm", tensors=tensors, elements=elements, dtype=dtype)


def listed():
    return [
        # the nodes of a small structure to two of eight experts: one launch, latency only
        _route("route_64_e8_k2_f32", 64, 8, 2, "f32", "softmax"),
        # the edges of 10^4 atoms, a balanced model: sigmoid scores, a bias for the choice, four of eight blocks, and
        # experts that a row may not have (those of other elements)
        _route("route_525k_e64_k4_bf16", 525308, 64, 4, "bf16", "sigmoid", bias=True, blocks=8, keep=4,
               masked=0.1),
        # training the router of a large model on part of a batch
        _route("route_grad_131k_e128_k8_f32", 131327, 128, 8, "f32", "softmax", renorm=False, grad=True),
        # an element's own residual layer on the scalars of a small structure: the smallest layer
        _layer("layer_64_g5_64x64_silu_f32", 64, 5, 64, 64, "f32", "silu", residual=True),
        # a hidden layer of the radial network of ten elements in training, which keeps what the gradient needs
        _layer("layer_525k_g55_64x64_silu_bf16", 525308, 55, 64, 64, "bf16", "silu", keep_z=True, pad=0.02),
        # four experts of 32 for each of 131,327 edges: the gather of the inputs, 525,308 pairs
        _layer("layer_131k_k4_e32_128x448_gelu_bf16", 131327, 32, 128, 448, "bf16", "gelu", per_row=4),
        # training the hidden layer of a four-element model in 32 bits
        _layer("layer_grad_525k_g10_64x64_silu_f32", 525308, 10, 64, 64, "f32", "silu", grad=True),
        # training experts: gradients of the inputs that four of them share, and of their weights and biases
        _layer("layer_grad_65k_k4_e32_128x448_silu_bf16", 65441, 32, 128, 448, "bf16", "silu", per_row=4, pad=0.02,
               grad=True),
        # joining the results of four experts at the headline widths, with the input added back
        _mix("mix_131k_k4_896_bf16", 131327, 4, 896, "bf16", residual=True),
        # its gradient for eight experts, an odd width
        _mix("mix_grad_32k_k8_449_f32", 32719, 8, 449, "f32", grad=True),
        # the factors and layers of a deep model: many tensors, most of them small
        _norm("norm_200x5m_f32", 200, 5000000, "f32"),
        # the grouped weights of a many-element model, gradients in 16 bits
        _norm("norm_24x64m_bf16", 24, 64000000, "bf16"),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, hi=1344):
    return rng.choice([w for w in WIDTHS if w <= hi]) if rng.random() < 0.5 else _logu(rng, 8, hi)


def draw(rng):
    largest = [work(c) for c in listed()]
    while True:
        kind = rng.choice(("route", "layer", "layer", "layer", "mix", "norm"))
        rows, grad = _logu(rng, 1, 525308), rng.random() < 0.5
        dtype = rng.choice(("f32", "bf16"))
        if kind == "route":
            per_block, blocks = _logu(rng, 2, 64), rng.choice((1, 1, 2, 4, 8))
            keep = rng.randint(1, blocks)
            c = _route(None, rows, blocks * per_block, rng.randint(1, min(16, keep * per_block)), dtype,
                       rng.choice(("softmax", "sigmoid")), rng.random() < 0.5, blocks, keep, rng.random() < 0.5,
                       rng.choice((0.0, 0.1, 0.6)), grad)
        elif kind == "layer":
            per_row = rng.choice((1, 1, 2, 3, 4, 8))
            groups = _logu(rng, 1, MAX_GROUPS) if per_row == 1 else _logu(rng, per_row, 256)
            c = _layer(None, max(1, rows // per_row), groups, _width(rng), _width(rng), dtype,
                       rng.choice(("silu", "gelu", "relu", "none")), per_row, rng.random() < 0.3,
                       rng.random() < 0.5, rng.choice((0.0, 0.02, 0.3)), grad)
        elif kind == "mix":
            per_row = rng.randint(1, 16)
            c = _mix(None, max(1, rows // per_row), per_row, _width(rng), dtype, rng.random() < 0.5,
                     rng.random() < 0.8, grad)
        else:
            tensors = _logu(rng, 1, 200)
            c = _norm(None, tensors, max(tensors, _logu(rng, 1000, 64000000)), dtype)
        w = work(c)
        weights = c["groups"] * c["n_in"] * c["n_out"] if kind == "layer" else 0
        logits = c["rows"] * c["experts"] if kind == "route" else 0
        if (weights <= 100000000 and logits <= 40000000 and w["bytes"] <= max(v["bytes"] for v in largest)
                and w["flops"] <= max(v["flops"] for v in largest)):
            del c["name"]
            return c


# ---------------------------------------------------------------- inputs

def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device=_device())
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape, scale=1.0):
    return torch.randn(*shape, generator=gen, device=gen.device) * scale


def _ids(case, gen):
    """The group of each row, int32, drawn by an uneven composition, -1 where a row has none; with several a row
    (experts), different ones of each row, [rows, per_row]."""
    dev, n, G, k = gen.device, case["rows"], case["groups"], case["per_row"]
    share = _normal(gen, G, scale=0.5 if k > 1 else 1.0)
    if k > 1:
        ids = torch.topk(share - torch.log(-torch.log(
            torch.rand(n, G, generator=gen, device=dev).clamp(1e-7, 1 - 1e-7))), k, dim=1).indices
    else:
        edges = torch.cumsum(share.exp() / share.exp().sum(), 0)
        ids = torch.searchsorted(edges, torch.rand(n, 1, generator=gen, device=dev)).clamp(max=G - 1)
    ids = torch.where(torch.rand(n, k, generator=gen, device=dev) < case["pad"], -1, ids)
    return ids.to(torch.int32).view(-1)


def _inputs(case, seed):
    gen, c = _generator(seed), case
    dev, dt = gen.device, _dtype(case["dtype"])
    d = {}
    if c["kind"] == "route":
        n, E, k = c["rows"], c["experts"], c["top_k"]
        logits = _normal(gen, n, E, scale=1.2) + _normal(gen, E, scale=0.5)
        if c["masked"]:
            # experts that a row may not have; now and then none is left
            share = torch.where(torch.rand(n, 1, generator=gen, device=dev) < 0.01, 1.0, c["masked"])
            logits[torch.rand(n, E, generator=gen, device=dev) < share] = -math.inf
        d["logits"] = logits.to(dt)
        d["bias"] = _normal(gen, E, scale=0.05) if c["bias"] else None
        if c["grad"]:
            # the choice of a forward call whose bias moved it a little, and the gradient of its weights
            ids = torch.topk(logits + _normal(gen, n, E, scale=0.3), k, dim=1).indices
            gone = torch.isinf(torch.gather(logits, 1, ids))
            d["ids"] = torch.where(gone, -1, ids).to(torch.int32)
            d["dweights"] = _normal(gen, n, k, scale=1e-2)
    elif c["kind"] == "layer":
        n, G, K, N = c["rows"], c["groups"], c["n_in"], c["n_out"]
        d["ids"] = _ids(c, gen)
        x = _normal(gen, n, K)
        d["x"] = (x * torch.sigmoid(x)).to(dt)            # activations of the layer before
        d["w"] = _normal(gen, G, K, N, scale=1.5 * K ** -0.5).to(dt)
        d["bias"] = _normal(gen, G, N, scale=0.2).to(dt)
        pairs = n * c["per_row"]
        if c["grad"]:
            d["dy"] = _normal(gen, pairs, N, scale=1e-2).to(dt)
            d["z"] = None if c["act"] == "none" else _normal(gen, pairs, N).to(dt)  # what the forward call kept
        else:
            d["residual"] = _normal(gen, pairs, N).to(dt) if c["residual"] else None
    elif c["kind"] == "mix":
        n, k, N = c["rows"], c["per_row"], c["width"]
        d["y"] = _normal(gen, n * k, N).to(dt)
        d["weights"] = torch.softmax(_normal(gen, n, k), 1) if c["weights"] else None
        d["residual"] = _normal(gen, n, N).to(dt) if c["residual"] and not c["grad"] else None
        if c["grad"]:
            d["dout"] = _normal(gen, n, N, scale=1e-2).to(dt)
    else:
        # gradients differ in size between tensors
        d["g"] = [(_normal(gen, m) * 10.0 ** (-(i % 4))).to(dt) for i, m in enumerate(_sizes(c))]
        d["grad_scale"] = torch.full((1,), 0.5, device=dev)   # the mean over two batches
    return d


def _sizes(case):
    """Elements of each tensor: uneven, none empty, adding up to the case's."""
    n, total = case["tensors"], case["elements"]
    raw = np.array([(1 + i % 7) ** 2 * (1 + (i * i) % 5) for i in range(n)], dtype=np.float64)
    s = np.maximum(1, np.floor(raw / raw.sum() * total).astype(np.int64))
    s[int(np.argmax(s))] += total - int(s.sum())
    return [int(v) for v in s]


MAX_NORM = 10.0
SCALE = 1.5


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["kind"] == "layer":
        # the rows' order belongs to the graph or the batch: every layer and both directions use it
        if own:
            import paper_2605_15073_amd as cg

            st["offsets"], st["order"] = cg.group_rows(st["ids"], case["groups"])
        else:
            G, ids = case["groups"], st["ids"]
            key = torch.where((ids < 0) | (ids >= G), G, ids)
            st["order"] = torch.argsort(key, stable=True)
            ends = torch.cumsum(torch.bincount(key, minlength=G + 1), 0).tolist()
            st["segments"] = [(g, s, e) for g, (s, e) in enumerate(zip([0] + ends[:-1], ends[:G])) if e > s]
    elif case["kind"] == "norm" and own:
        import paper_2605_15073_amd as cg

        like = lambda: [torch.zeros(g.shape, device=g.device) for g in st["g"]]
        st["tensors"] = cg.AdamWTensors(like(), st["g"], like(), like())
    return st


# ---------------------------------------------------------------- one pass

def run(state):
    case = state["case"]
    name = case["kind"] + ("_grad" if case.get("grad") else "")
    return (_OWN if own else _PLAIN)[name](state, case)


def _own_route(s, c):
    import paper_2605_15073_amd as cg

    return cg.route_rows(s["logits"], c["top_k"], bias=s["bias"], score=c["score"], n_blocks=c["blocks"],
                         keep_blocks=c["keep"], renormalize=c["renorm"], scale=SCALE)


def _own_route_grad(s, c):
    import paper_2605_15073_amd as cg

    return cg.route_rows_grad(s["logits"], s["ids"], s["dweights"], score=c["score"], renormalize=c["renorm"],
                              scale=SCALE)


def _activation(c):
    return None if c["act"] == "none" else c["act"]


def _own_layer(s, c):
    import paper_2605_15073_amd as cg

    return cg.grouped_layer(s["x"], s["w"], s["offsets"], s["order"], bias=s["bias"], activation=_activation(c),
                            residual=s["residual"], per_row=c["per_row"], z=None if c["keep_z"] else False)


def _own_layer_grad(s, c):
    import paper_2605_15073_amd as cg

    return cg.grouped_layer_grad(s["x"], s["w"], s["dy"], s["offsets"], s["order"], z=s["z"],
                                 activation=_activation(c), per_row=c["per_row"])


def _own_mix(s, c):
    import paper_2605_15073_amd as cg

    return cg.mix_rows(s["y"], c["per_row"], weights=s["weights"], residual=s["residual"])


def _own_mix_grad(s, c):
    import paper_2605_15073_amd as cg

    if not c["weights"]:
        return cg.mix_rows_grad(s["dout"], c["per_row"], dweights=False)[0]
    return cg.mix_rows_grad(s["dout"], c["per_row"], weights=s["weights"], y=s["y"])


def _own_norm(s, c):
    import paper_2605_15073_amd as cg

    return cg.adamw_grad_norm(s["tensors"], MAX_NORM, grad_scale=s["grad_scale"])


def _plain_route(s, c):
    l, k, B = s["logits"].double(), c["top_k"], c["blocks"]
    n, E = l.shape
    gone = torch.isinf(l)
    if c["score"] == "softmax":
        top = torch.where(gone, -1e300, l).amax(1, keepdim=True)
        e = torch.where(gone, 0.0, torch.exp(l - top))
        score = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
    key = score if s["bias"] is None else score + s["bias"].double()
    if s["bias"] is None and B == 1:
        key = l                                        # the same order, and ties are ties
    key = torch.where(gone, -math.inf, key)
    if B > 1:
        two = torch.topk(key.view(n, B, E // B), 2, dim=2).values
        of_block = torch.where(torch.isinf(two), 0.0, two).sum(2)
        of_block = torch.where(torch.isinf(two[:, :, 0]), -math.inf, of_block)
        kept = torch.sort(of_block, dim=1, descending=True, stable=True).indices[:, :c["keep"]]
        is_kept = torch.zeros(n, B, dtype=torch.bool, device=l.device).scatter_(1, kept, True)
        key = torch.where(is_kept.repeat_interleave(E // B, dim=1), key, -math.inf)
    ordered = torch.sort(key, dim=1, descending=True, stable=True)
    ids, there = ordered.indices[:, :k], ~torch.isinf(ordered.values[:, :k])
    w = torch.where(there, torch.gather(score, 1, ids), 0.0).float()
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-38)
    return torch.where(there, ids, -1).to(torch.int32), w * SCALE


def _plain_route_grad(s, c):
    l = s["logits"].float()
    ids, u = s["ids"], s["dweights"]
    there = ids >= 0
    at = torch.where(there, ids, 0).long()
    if c["score"] == "softmax":
        top = torch.where(torch.isinf(l), -1e38, l).amax(1, keepdim=True)
        e = torch.where(torch.isinf(l), 0.0, torch.exp(l - top))
        score = e / e.sum(1, keepdim=True).clamp(min=1e-38)
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
    p = torch.where(there, torch.gather(score, 1, at), 0.0)
    u = torch.where(there, u, 0.0) * SCALE
    if c["renorm"]:
        total = p.sum(1, keepdim=True).clamp(min=1e-38)
        u = (u - (u * p).sum(1, keepdim=True) / total) / total
    # u is now the gradient of the chosen scores; of renormalised ones it adds up to nothing with their shares
    dl = torch.zeros_like(l).scatter_add_(1, at, p * u * (1.0 if c["score"] == "softmax" else 1.0 - p))
    if c["score"] == "softmax" and not c["renorm"]:
        dl = dl - score * (p * u).sum(1, keepdim=True)
    return dl.to(s["logits"].dtype)


def _act(z, name):
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return torch.where(z > 0, z, 0.0) if name == "relu" else z


def _act_grad(z, name):
    if name == "silu":
        f = 1.0 / (1.0 + torch.exp(-z))
        return f * (1.0 + z * (1.0 - f))
    if name == "gelu":
        return (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
    return torch.where(z > 0, 1.0, 0.0)


def _plain_layer(s, c):
    order, w, b = s["order"], s["w"], s["bias"]
    xs = s["x"][order // c["per_row"]].float()
    zs = torch.zeros(order.shape[0], c["n_out"], device=xs.device)
    for g, first, end in s["segments"]:
        zs[first:end] = xs[first:end] @ w[g].float() + b[g].float()
    ys = _act(zs, c["act"])
    if s["residual"] is not None:
        ys = ys + s["residual"][order].float()
    y = torch.empty_like(ys, dtype=w.dtype)
    y[order] = ys.to(w.dtype)
    if not c["keep_z"]:
        return y
    z = torch.empty_like(y)
    z[order] = zs.to(w.dtype)
    return y, z


def _plain_layer_grad(s, c):
    order, w, k = s["order"], s["w"], c["per_row"]
    xs, dzs = s["x"][order // k].float(), s["dy"][order].float()
    if s["z"] is not None:
        dzs = dzs * _act_grad(s["z"][order].float(), c["act"])
    dxs = torch.zeros_like(xs)
    dw = torch.zeros(w.shape, device=xs.device)
    db = torch.zeros(c["groups"], c["n_out"], device=xs.device)
    for g, first, end in s["segments"]:
        dxs[first:end] = dzs[first:end] @ w[g].float().t()
        dw[g] = xs[first:end].t() @ dzs[first:end]
        db[g] = dzs[first:end].sum(0)
    dx = torch.empty_like(dxs)
    dx[order] = dxs
    if k > 1:
        dx = dx.view(-1, k, c["n_in"]).sum(1)
    return dx.to(w.dtype), dw.to(w.dtype), db.to(w.dtype)


def _plain_mix(s, c):
    y = s["y"].float().view(c["rows"], c["per_row"], c["width"])
    if s["weights"] is not None:
        y = y * s["weights"][:, :, None]
    out = y.sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return out.to(s["y"].dtype)


def _plain_mix_grad(s, c):
    n, k, N = c["rows"], c["per_row"], c["width"]
    dout = s["dout"].float()[:, None, :]
    if s["weights"] is None:
        return dout.expand(n, k, N).reshape(n * k, N).to(s["y"].dtype)
    dy = (dout * s["weights"][:, :, None]).view(n * k, N).to(s["y"].dtype)
    return dy, (s["y"].float().view(n, k, N) * dout).sum(2)


def _plain_norm(s, c):
    total = torch.zeros(1, dtype=torch.float64, device=_device())
    for g in s["g"]:
        total += g.double().square().sum()
    scale = s["grad_scale"].double()
    norm = torch.sqrt(total) * scale
    return norm.float(), (scale * torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)).float()


_OWN = {"route": _own_route, "route_grad": _own_route_grad, "layer": _own_layer, "layer_grad": _own_layer_grad,
        "mix": _own_mix, "mix_grad": _own_mix_grad, "norm": _own_norm}
_PLAIN = {"route": _plain_route, "route_grad": _plain_route_grad, "layer": _plain_layer,
          "layer_grad": _plain_layer_grad, "mix": _plain_mix, "mix_grad": _plain_mix_grad, "norm": _plain_norm}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c, es = case, 2 if case["dtype"] == "bf16" else 4
    if c["kind"] == "route":
        n, E, k = c["rows"], c["experts"], c["top_k"]
        if not c["grad"]:
            return {"bytes": n * (es * E + 8 * k), "flops": 4 * n * E}
        return {"bytes": n * (2 * es * E + 8 * k), "flops": 6 * n * E}
    if c["kind"] == "layer":
        T, K, N = c["rows"] * c["per_row"], c["n_in"], c["n_out"]
        used, streams = min(c["groups"], T), 2 if c["act"] != "none" else 1
        rows = 4 * T + es * c["rows"] * K + es * T * N * (
            streams if c["grad"] else 1 + c["residual"] + c["keep_z"])
        weights, flops = es * used * (K + 1) * N, 2 * T * K * N
        if c["grad"]:
            return {"bytes": rows + es * c["rows"] * K + weights + es * c["groups"] * (K + 1) * N, "flops": 2 * flops}
        return {"bytes": rows + weights, "flops": flops}
    if c["kind"] == "mix":
        n, k, N = c["rows"], c["per_row"], c["width"]
        wts = 4 * n * k if c["weights"] else 0
        if c["grad"]:
            return {"bytes": es * n * N * (1 + k) + (es * n * k * N + 2 * wts if wts else 0),
                    "flops": (3 if wts else 1) * n * k * N}
        return {"bytes": es * n * N * (k + 1 + c["residual"]) + wts, "flops": 2 * n * k * N}
    return {"bytes": es * c["elements"], "flops": 2 * c["elements"]}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    d = _inputs(case, seed)
    return {"route": _exact_route, "layer": _exact_layer, "mix": _exact_mix, "norm": _exact_norm}[case["kind"]](case, d)


def _exact_route(c, d):
    l = d["logits"].double()
    n, E = l.shape
    score = (torch.softmax(torch.where(torch.isinf(l), -1e9, l), 1) if c["score"] == "softmax"
             else torch.sigmoid(l)).masked_fill(torch.isinf(l), 0.0)
    if c["grad"]:
        chosen = torch.zeros(n, E + 1, dtype=torch.float64, device=l.device)
        at = torch.where(d["ids"] < 0, E, d["ids"]).long()
        u = chosen.clone().scatter_(1, at, d["dweights"].double())[:, :E] * SCALE
        chosen = chosen.scatter_(1, at, 1.0)[:, :E]
        if c["renorm"]:
            # weights share / sum of shares: the derivative by each share, from the quotient
            share = score * chosen
            total = share.sum(1, keepdim=True).clamp(min=1e-300)
            u = chosen * (u * total - (u * share).sum(1, keepdim=True)) / total ** 2
        inner = score * u
        if c["score"] == "softmax":
            return inner - score * inner.sum(1, keepdim=True)
        return inner - inner * score
    # the choice, one expert after the other by the largest key left
    key = score + (0.0 if d["bias"] is None else d["bias"].double())
    if d["bias"] is None and c["blocks"] == 1:
        key = l.clone()
    key[torch.isinf(l)] = -math.inf
    if c["blocks"] > 1:
        by_block = key.view(n, c["blocks"], -1)
        best, second = torch.sort(by_block, dim=2).values[:, :, -1], torch.sort(by_block, dim=2).values[:, :, -2]
        total = best + torch.where(torch.isinf(second), 0.0, second)
        for b in range(c["blocks"]):
            before = torch.arange(c["blocks"], device=l.device) < b
            ahead = (total > total[:, b:b + 1]) | ((total == total[:, b:b + 1]) & before)
            by_block[:, b].masked_fill_((ahead.sum(1) >= c["keep"])[:, None], -math.inf)
    taken = torch.zeros(n, c["top_k"], dtype=torch.float64, device=l.device)
    rows = torch.arange(n, device=l.device)
    for j in range(c["top_k"]):
        value = key.amax(1)
        e = (key == value[:, None]).to(torch.int8).argmax(1)
        taken[:, j] = torch.where(torch.isinf(value), 0.0, score[rows, e])
        key[rows, e] = -math.inf
    if c["renorm"]:
        taken = taken / taken.sum(1, keepdim=True).clamp(min=1e-300)
    return None, taken * SCALE


def _exact_layer(c, d):
    k = c["per_row"]
    x, w, ids = d["x"].double(), d["w"], d["ids"].cpu().numpy()
    by = np.argsort(ids, kind="stable")
    groups, first = np.unique(ids[by], return_index=True)
    rows_of = {int(g): torch.from_numpy(r).to(x.device) for g, r in zip(groups, np.split(by, first[1:])) if g >= 0}

    def normal_cdf(z):
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))

    if not c["grad"]:
        z = x.new_zeros(ids.size, c["n_out"])
        for g, r in rows_of.items():
            z[r] = torch.addmm(d["bias"][g].double()[None], x[r // k], w[g].double())
        y = {"silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * normal_cdf(z), "relu": lambda: z.clamp(min=0),
             "none": lambda: z}[c["act"]]()
        if d["residual"] is not None:
            y = y + d["residual"].double()
        return (y, z) if c["keep_z"] else y
    dz = d["dy"].double()
    if d["z"] is not None:
        z = d["z"].double()
        if c["act"] == "silu":
            slope = torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        elif c["act"] == "gelu":
            slope = normal_cdf(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        else:
            slope = (z > 0).double()
        dz = dz * slope
    dx, dw = torch.zeros_like(x), x.new_zeros(w.shape)
    db = x.new_zeros(w.shape[0], w.shape[2])
    for g, r in rows_of.items():
        dx.index_add_(0, r // k, dz[r] @ w[g].double().t())
        dw[g] = x[r // k].t() @ dz[r]
        db[g] = dz[r].sum(0)
    return dx, dw, db


def _exact_mix(c, d):
    y = d["y"].double().view(c["rows"], c["per_row"], c["width"])
    w = torch.ones(c["rows"], c["per_row"], dtype=torch.float64, device=y.device)
    if d["weights"] is not None:
        w = d["weights"].double()
    if c["grad"]:
        dout = d["dout"].double()
        dy = torch.stack([w[:, j:j + 1] * dout for j in range(c["per_row"])], 1).view(-1, c["width"])
        if d["weights"] is None:
            return dy
        return dy, torch.stack([(y[:, j] * dout).sum(1) for j in range(c["per_row"])], 1)
    out = torch.zeros_like(y[:, 0]) if d["residual"] is None else d["residual"].double()
    for j in range(c["per_row"]):
        out = out + w[:, j:j + 1] * y[:, j]
    return out


def _exact_norm(c, d):
    total = math.fsum(float(torch.dot(g.double(), g.double())) for g in d["g"])
    scale = float(d["grad_scale"])
    norm = scale * math.sqrt(total)
    return [torch.tensor([v], dtype=torch.float64) for v in (norm, scale * min(1.0, MAX_NORM / norm))]
