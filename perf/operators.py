"""Timed cases of the framework's operators on a user's own tensors, their plain forms and their results in 64 bits.

Three operators that a training step outside the built-in one is made of: matrix products grouped by relation (or by
expert) with their gradients, the preference loss over candidate scores with its gradient, and the clipping of many
gradients by their joint norm.  `listed` names the cases, `draw` gives further ones from the same ranges, `prepare`
makes what a program holds before the call, `run` is one pass (the plain form, or with `own` the framework's calls),
`exact` is the operator's definition in float64.
"""

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ----------------------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------------------
def _group(name, **over):
    """n rows in G groups of ragged sizes (skew: the power by which they fall off; tail: rows behind the last group),
    one out_dim x in_dim matrix a group; pad: columns that the rows of x and y are apart beyond their widths."""
    case = {"name": name, "op": "group", "dir": "forward", "type": "f32", "n": 40_000, "G": 64, "in": 128, "out": 128,
            "skew": 1.0, "tail": 0, "pad": 0}
    case.update(over)
    return case


def _pref(name, **over):
    """pairs of sequences with `rows` rows of V candidate scores in all; masked: the share of rows without a label;
    hidden: the share of candidates whose score is -inf."""
    case = {"name": name, "op": "preference", "dir": "train", "type": "f32", "pairs": 64, "rows": 4_096, "V": 2_000,
            "masked": 0.2, "hidden": 0.01, "pad": 0}
    case.update(over)
    return case


def _clip(name, **over):
    """`large` and `small` tensors of about `large_size` and `small_size` values, every `other`-th of a second type;
    bound: the largest norm allowed, of the gradients' own."""
    case = {"name": name, "op": "clip", "type": "f32", "second": "f32", "other": 3, "large": 1, "large_size": 100_000,
            "small": 8, "small_size": 400, "bound": 0.37}
    case.update(over)
    return case


def listed():
    return [
        # the relation matrices of a knowledge graph applied to one step's edges: 1,345 groups, most of them short
        _group("group_relations_f32", n=40_000, G=1_345, **{"in": 400, "out": 400}, skew=1.2),
        # a follower graph's step, the gradients of its linear operator: few relations, one of them most of the edges
        _group("group_follower_backward_f32", dir="backward", n=40_000, G=8, **{"in": 100, "out": 100}, skew=1.2),
        # a layer of 32 experts over a long batch
        _group("group_experts_bf16", type="bf16", n=32_768, G=32, **{"in": 2_048, "out": 4_096}, skew=0.3),
        # the same kind of layer in training: both gradients
        _group("group_experts_backward_bf16", dir="backward", type="bf16", n=16_384, G=32,
               **{"in": 2_048, "out": 2_048}, skew=0.3),
        # serving: single tokens of 24 requests spread over 16 experts; the matrices are what is read
        _group("group_tokens_f16", type="f16", n=24, G=16, **{"in": 2_048, "out": 2_048}, skew=0.0),
        # odd widths, rows apart, rows behind the last group, in half precision
        _group("group_odd_backward_f16", dir="backward", type="f16", n=5_003, G=37, **{"in": 501, "out": 333},
               skew=1.0, tail=61, pad=3),
        # the smallest: two pairs of short paths over a small candidate set
        _pref("preference_small_f32", pairs=2, rows=13, V=200, masked=0.0, hidden=0.0),
        # a step's edges in preferred and other paths, scored against every entity of a knowledge graph
        _pref("preference_entities_bf16", type="bf16", pairs=256, rows=16_384, V=15_000),
        # a reference model's log probabilities: two pairs, few rows, a very wide row with an odd stride
        _pref("preference_wide_f16", dir="forward", type="f16", pairs=2, rows=96, V=131_001, masked=0.3, pad=6),
        # the gradients of a small graph's tables: a few short tensors
        _clip("clip_small_f32"),
        # the gradients of a model in 16 bits with norms and biases in 32
        _clip("clip_mixed_bf16", type="bf16", second="f32", large=24, large_size=2_048 * 1_024, small=32,
              small_size=2_048, bound=0.1),
        # the dense gradient of a social network's table
        _clip("clip_table_f32", large=1, large_size=4_847_571 * 128, small=3, small_size=128, bound=0.6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("group", "group", "preference", "clip"))
    t = rng.choice(("f32", "bf16", "f16"))
    if kind == "group":
        case = {"op": kind, "dir": rng.choice(("forward", "backward")), "type": t,
                "in": rng.choice((100, 128, 400, 1_024, _log(rng, 9, 4_096))),
                "out": rng.choice((100, 128, 400, 1_024, _log(rng, 9, 4_096))), "n": _log(rng, 1, 65_536),
                "skew": rng.choice((0.0, 0.3, 1.0, 1.2)), "tail": rng.choice((0, 0, rng.randint(1, 100))),
                "pad": rng.choice((0, 0, rng.randint(1, 16)))}
        size = case["in"] * case["out"]
        case["G"] = _log(rng, 1, max(1, min(1_500, 200_000_000 // size)))
        passes = 2 if case["dir"] == "backward" else 1
        case["n"] = max(1, min(case["n"], int(2.5e11 / (passes * size))))
        return case
    if kind == "preference":
        rows, V = _log(rng, 4, 20_000), _log(rng, 50, 131_072)
        rows = max(4, min(rows, 240_000_000 // V))
        return {"op": kind, "dir": rng.choice(("train", "train", "forward")), "type": t, "rows": rows, "V": V,
                "pairs": _log(rng, 1, max(1, rows // 4)), "masked": rng.choice((0.0, 0.2, 0.6)),
                "hidden": rng.choice((0.0, 0.01, 0.2)), "pad": rng.choice((0, 0, rng.randint(1, 9)))}
    return {"op": kind, "type": t, "second": rng.choice(("f32", t)), "other": rng.randint(2, 5),
            "large": rng.randint(1, 20), "large_size": _log(rng, 1_000, 12_000_000), "small": rng.randint(0, 38),
            "small_size": _log(rng, 1, 5_000), "bound": rng.choice((rng.uniform(0.05, 0.95), 5.0))}


# ----------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call
# ----------------------------------------------------------------------------------------------------------------
def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _rows(gen, n, width, pad, scale, dtype):
    return _normal(gen, (n, width + pad), scale, dtype)[:, :width]


def _prepare_group(case, gen, rs):
    dt, n, G, k, m = TYPES[case["type"]], case["n"], case["G"], case["in"], case["out"]
    weight = np.arange(1, G + 1, dtype=np.float64) ** -case["skew"]
    counts = rs.multinomial(max(0, n - case["tail"]), rs.permutation(weight / weight.sum()))
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    s = {"op": "group", "dir": case["dir"], "sizes": [int(c) for c in counts] + [int(n - offsets[-1])],
         "offsets": torch.from_numpy(offsets).cuda(), "x": _rows(gen, n, k, case["pad"], 1.0, dt),
         "a": _normal(gen, (G, m, k), k ** -0.5, dt)}
    if case["dir"] == "forward":
        s["y"] = torch.zeros(n, m + case["pad"], dtype=dt, device="cuda")[:, :m]
    else:
        s["dy"] = _rows(gen, n, m, case["pad"], 0.1, dt)
        s["dx"] = torch.zeros(n, k + case["pad"], dtype=dt, device="cuda")[:, :k]
        s["da"] = torch.zeros(G, m, k, dtype=dt, device="cuda")
    return s


def _prepare_pref(case, gen, rs):
    dt, rows, V, Q = TYPES[case["type"]], case["rows"], case["V"], 2 * case["pairs"]
    cuts = np.sort(rs.randint(0, rows + 1, Q - 1))   # paths of every length, none among them
    offsets = np.concatenate([[0], cuts, [rows]]).astype(np.int64)
    labels = rs.randint(0, V, rows).astype(np.int32)
    logits = _rows(gen, rows, V, case["pad"], 3.0, dt)
    if case["hidden"]:
        # known candidates that are left out of the row's distribution, the labels' own never
        hide = torch.rand(rows, V, generator=gen, device="cuda") < case["hidden"]
        hide[torch.arange(rows, device="cuda"), torch.from_numpy(labels).long().cuda()] = False
        logits.masked_fill_(hide, -math.inf)
    labels[rs.rand(rows) < case["masked"]] = -1
    s = {"op": "preference", "dir": case["dir"], "logits": logits, "labels": torch.from_numpy(labels).cuda(),
         "offsets": torch.from_numpy(offsets).cuda(), "beta": 0.1, "smoothing": 0.1}
    # the frozen model's log probabilities lie about the trained one's
    logp = _sequence_logp(s)[0]
    s["ref"] = (logp + 3.0 * torch.randn(Q, generator=gen, device="cuda")).float()
    s["loss"] = torch.zeros(case["pairs"], device="cuda")
    s["logp"], s["dlogp"] = torch.zeros(Q, device="cuda"), torch.zeros(Q, device="cuda")
    s["stats"] = torch.zeros(rows, 2, device="cuda")
    if case["dir"] == "train":
        s["dlogits"] = torch.zeros(rows, V + case["pad"], dtype=dt, device="cuda")[:, :V]
    return s


def _clip_tensors(case):
    """The tensors' sizes (a few percent apart, so odd ones among them) and types."""
    sizes = [case["large_size"]] * case["large"] + [case["small_size"]] * case["small"]
    sizes = [max(1, z - z * (i % 7) // 64) for i, z in enumerate(sizes)]
    other = case["other"]
    return sizes, [case["second"] if i % other == other - 1 else case["type"] for i in range(len(sizes))]


def _prepare_clip(case, gen, rs):
    sizes, types = _clip_tensors(case)
    types = [TYPES[t] for t in types]
    grads = [_normal(gen, (z,), 10.0 ** rs.uniform(-4, -2), t) for z, t in zip(sizes, types)]
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    return {"op": "clip", "grads": grads, "max_norm": case["bound"] * norm,
            "outs": [torch.zeros_like(g) for g in grads]}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 31))
    return {"group": _prepare_group, "preference": _prepare_pref, "clip": _prepare_clip}[case["op"]](case, gen, rs)


# ----------------------------------------------------------------------------------------------------------------
# one pass: the plain forms
# ----------------------------------------------------------------------------------------------------------------
def _plain_group(s):
    """Row blocks and their matrices, product by product; rows behind the last group give nothing (the last block)."""
    dt, sizes = s["x"].dtype, s["sizes"]
    x = s["x"].float().split(sizes)
    if s["dir"] == "forward":
        y = [r @ a.float().t() for r, a in zip(x, s["a"])] + [x[-1].new_zeros(sizes[-1], s["a"].shape[1])]
        return torch.cat(y).to(dt)
    dy = s["dy"].float().split(sizes)
    dx = [r @ a.float() for r, a in zip(dy, s["a"])] + [torch.zeros_like(x[-1])]
    da = [g.t() @ r for g, r in zip(dy[:-1], x)]
    return {"dx": torch.cat(dx).to(dt), "da": torch.stack(da).to(dt)}


def _sequence_logp(s):
    """The sequences' log probabilities (64 bits), each row's largest logit and the logarithm of its sum of
    exponentials behind it, the exponentials and their sums, the rows that count, and the rows' sequences."""
    z, labels, offsets = s["logits"].float(), s["labels"].long(), s["offsets"]
    top = z.amax(1)
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top)[:, None])
    total = e.sum(1)
    counts = (labels >= 0) & (top != -math.inf)
    row = (z.gather(1, labels.clamp(min=0)[:, None])[:, 0] - top).double() - total.double().log()
    sums = torch.cat([row.new_zeros(1), torch.where(counts, row, torch.zeros_like(row)).cumsum(0)])[offsets]
    seq = torch.bucketize(torch.arange(len(labels), device=z.device), offsets[1:], right=True)
    return sums[1:] - sums[:-1], e, total, counts, seq


def _plain_pref(s):
    logp, e, total, counts, seq = _sequence_logp(s)
    ratio = logp - s["ref"].double()
    h = s["beta"] * (ratio[0::2] - ratio[1::2])
    eps = s["smoothing"]
    soft = h.abs().neg().exp().log1p()
    loss = (1 - eps) * (soft + (-h).clamp(min=0)) + eps * (soft + h.clamp(min=0))
    d = s["beta"] * (eps / (1 + torch.exp(-h)) - (1 - eps) / (1 + torch.exp(h)))
    dlogp = torch.stack([d, -d], 1).reshape(-1)
    out = {"loss": loss.float(), "logp": logp.float(), "dlogp": dlogp.float()}
    if s["dir"] == "train":
        g = torch.where(counts, dlogp[seq.clamp(max=len(dlogp) - 1)].float(), torch.zeros_like(total))
        dz = e * (-g / torch.where(counts, total, torch.ones_like(total)))[:, None]
        dz.scatter_add_(1, s["labels"].long().clamp(min=0)[:, None], g[:, None])
        out["dlogits"] = dz.to(s["logits"].dtype)
    return out


def _plain_clip(s):
    total = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    norm = float(total)
    scale = min(1.0, s["max_norm"] / norm) if math.isfinite(norm) and norm > 0 else 1.0
    return {"norm": norm, "outs": [(g.float() * scale).to(g.dtype) for g in s["grads"]]}


# ----------------------------------------------------------------------------------------------------------------
# one pass: the framework's calls
# ----------------------------------------------------------------------------------------------------------------
_kept = {}


def _context():
    """The context that a program creates once and passes to every call."""
    if not _kept:
        from paper_1903_12287_amd import pbg
        _kept["ctx"] = pbg.pbg_bucket_init(1_000, 1, 1, 128, "linear", "dot", "softmax")
    return _kept["ctx"]


def _own_group(s):
    from paper_1903_12287_amd import operators as ops
    if s["dir"] == "forward":
        ops.pbg_group_linear(_context(), s["x"], s["a"], s["offsets"], s["y"])
        return s["y"]
    ops.pbg_group_linear_backward(_context(), s["x"], s["a"], s["offsets"], s["dy"], s["dx"], s["da"])
    return {"dx": s["dx"], "da": s["da"]}


def _own_pref(s):
    from paper_1903_12287_amd import operators as ops
    ops.pbg_preference_loss(_context(), s["logits"], s["labels"], s["offsets"], s["ref"], s["beta"], s["smoothing"],
                            s["loss"], s["logp"], s["dlogp"], s["stats"])
    out = {"loss": s["loss"], "logp": s["logp"], "dlogp": s["dlogp"]}
    if s["dir"] == "train":
        ops.pbg_preference_loss_backward(_context(), s["logits"], s["labels"], s["offsets"], s["stats"], s["dlogp"],
                                         s["dlogits"])
        out["dlogits"] = s["dlogits"]
    return out


def _own_clip(s):
    from paper_1903_12287_amd import operators as ops
    norm = ops.pbg_clip_gradients(_context(), s["grads"], s["max_norm"], s["outs"])
    return {"norm": norm, "outs": s["outs"]}


def run(state):
    if own:
        return {"group": _own_group, "preference": _own_pref, "clip": _own_clip}[state["op"]](state)
    return {"group": _plain_group, "preference": _plain_pref, "clip": _plain_clip}[state["op"]](state)


# ----------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it gives in 64 bits
# ----------------------------------------------------------------------------------------------------------------
def work(case):
    es = SIZE[case["type"]]
    if case["op"] == "group":
        n, G, k, m = max(0, case["n"] - case["tail"]), case["G"], case["in"], case["out"]
        used = min(G, max(n, 1)) * k * m   # matrices that have rows, at most
        if case["dir"] == "forward":
            return {"bytes": es * (n * (k + m) + used), "flops": 2.0 * n * k * m}
        return {"bytes": es * (2 * n * (k + m) + used + G * k * m), "flops": 4.0 * n * k * m}
    if case["op"] == "preference":
        live = case["rows"] * case["V"] * (1.0 - case["masked"])
        if case["dir"] == "forward":
            return {"bytes": es * live, "flops": 4.0 * live}
        return {"bytes": es * (live + case["rows"] * case["V"]), "flops": 8.0 * live}
    values, types = _clip_tensors(case)
    sizes = [SIZE[t] for t in types]
    return {"bytes": 2.0 * sum(v * z for v, z in zip(values, sizes)), "flops": 3.0 * sum(values)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "group":
        return _exact_group(s)
    if case["op"] == "preference":
        return _exact_pref(s)
    squares = sum(float(torch.dot(g.double(), g.double())) for g in s["grads"])
    scale = min(1.0, s["max_norm"] / math.sqrt(squares)) if squares > 0 else 1.0
    return {"norm": math.sqrt(squares), "outs": [g.double() * scale for g in s["grads"]]}


def _exact_group(s):
    bounds = s["offsets"].tolist()
    n, k = s["x"].shape
    G, m = s["a"].shape[:2]
    if s["dir"] == "forward":
        y = torch.zeros(n, m, dtype=torch.float64, device="cuda")
        for g in range(G):
            lo, hi = bounds[g], bounds[g + 1]
            if hi > lo:
                y[lo:hi] = torch.mm(s["x"][lo:hi].double(), s["a"][g].double().t())
        return y
    dx = torch.zeros(n, k, dtype=torch.float64, device="cuda")
    da = torch.zeros(G, m, k, dtype=torch.float64, device="cuda")
    for g in range(G):
        lo, hi = bounds[g], bounds[g + 1]
        if hi > lo:
            dy = s["dy"][lo:hi].double()
            dx[lo:hi] = torch.mm(dy, s["a"][g].double())
            da[g] = torch.mm(dy.t().contiguous(), s["x"][lo:hi].double())
    return {"dx": dx, "da": da}


def _exact_pref(s):
    rows, V = s["logits"].shape
    bounds, labels = s["offsets"].tolist(), s["labels"].long()
    pairs = (len(bounds) - 1) // 2
    lse = torch.cat([torch.logsumexp(b.double(), 1) for b in s["logits"].split(1_024)])
    at = torch.arange(rows, device="cuda")
    picked = s["logits"][at, labels.clamp(min=0)].double() - lse
    picked[labels < 0] = 0.0
    logp = torch.stack([picked[a:b].sum() for a, b in zip(bounds[:-1], bounds[1:])])
    ratio = (logp - s["ref"].double()).view(pairs, 2)
    h = s["beta"] * (ratio[:, 0] - ratio[:, 1])
    eps, F = s["smoothing"], torch.nn.functional
    out = {"loss": -(1 - eps) * F.logsigmoid(h) - eps * F.logsigmoid(-h), "logp": logp}
    slope = s["beta"] * (torch.sigmoid(h) - (1 - eps))   # of the loss, by the first sequence's log probability
    out["dlogp"] = torch.stack([slope, -slope], 1).flatten()
    if s["dir"] == "train":
        dz = torch.zeros(rows, V, dtype=torch.float64, device="cuda")
        for q in range(2 * pairs):
            lo, hi = bounds[q], bounds[q + 1]
            if hi > lo:
                p = torch.exp(s["logits"][lo:hi].double() - lse[lo:hi, None])
                hot = F.one_hot(labels[lo:hi].clamp(min=0), V)
                dz[lo:hi] = out["dlogp"][q] * (hot - p) * (labels[lo:hi] >= 0)[:, None]
        out["dlogits"] = dz
    return out
