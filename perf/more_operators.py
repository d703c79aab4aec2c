"""Performance cases of what stands between and behind the low-bit products of a
decoder: norms of the heads of queries and keys with the position rotation,
the layer of experts on 4-bit weights, and the log probabilities of tokens.

A case is a dict of plain values; `kind` says which operators it goes through:
  heads     dsq_headnorm_fwd: each head of q and k normalised and rotated by its
            token's position, which may have several axes
  headgrad  dsq_headnorm_bwd: gradients of q, k and of the norms' weights
  moe       dsq_moe_route then dsq_moe_group: the router's choice and the chosen
            experts' layers, 4-bit weights with group scales, residual added
  logprob   dsq_logprob_fwd: log probability of a given token, entropy and the
            top alternatives of each row of logits
  logitgrad dsq_logprob_bwd: the logits' gradient where a loss is made of those log
            probabilities and entropies

With `own` false `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token of a decoder: latency only
        dict(name="heads_1x32+8x128_bf16", kind="heads", tokens=1, q=32, k=8, dim=128, rot=128,
             axes=1, interleaved=False, dtype="bf16"),
        # a long prompt, far positions
        dict(name="heads_16384x32+8x128_bf16", kind="heads", tokens=16384, q=32, k=8, dim=128,
             rot=128, axes=1, interleaved=False, dtype="bf16"),
        # the backward pass of a training batch of images: time, height and width
        dict(name="headgrad_8192x16+16x64_bf16_3axes", kind="headgrad", tokens=8192, q=16, k=16,
             dim=64, rot=64, axes=3, interleaved=False, dtype="bf16"),
        # nothing round: odd numbers of tokens and heads, part of a head rotated, neighbours paired
        dict(name="headgrad_1237x10+3x80_f32_2axes", kind="headgrad", tokens=1237, q=10, k=3,
             dim=80, rot=48, axes=2, interleaved=True, dtype="f32"),
        # one token through a layer of small experts: latency and 25 MB of codes
        dict(name="moe_1x2048x1024_e64k8", kind="moe", tokens=1, hidden=2048, width=1024,
             experts=64, top=8, group=128, dtype="bf16"),
        # ragged widths, small groups, few large experts
        dict(name="moe_5x2008x1111_e11k3_f16_g32", kind="moe", tokens=5, hidden=2008, width=1111,
             experts=11, top=3, group=32, dtype="f16"),
        # a few requests at once: most experts have one or two tokens
        dict(name="moe_16x4096x1024_e64k4", kind="moe", tokens=16, hidden=4096, width=1024,
             experts=64, top=4, group=128, dtype="bf16"),
        # a full batch of decoding requests: every expert has several tokens
        dict(name="moe_64x4096x2048_e32k4", kind="moe", tokens=64, hidden=4096, width=2048,
             experts=32, top=4, group=128, dtype="bf16"),
        # one step of one request, alternatives for its user
        dict(name="logprob_1x128000_bf16_top20", kind="logprob", rows=1, vocab=128000, top=20,
             masked=False, dtype="bf16"),
        # a text scored, alternatives of each token
        dict(name="logprob_4096x128000_bf16_top5", kind="logprob", rows=4096, vocab=128000, top=5,
             masked=False, dtype="bf16"),
        # the backward pass of a training batch's loss
        dict(name="logitgrad_2048x128000_bf16", kind="logitgrad", rows=2048, vocab=128000,
             dtype="bf16"),
        # rows that start at odd addresses
        dict(name="logitgrad_777x50261_f32", kind="logitgrad", rows=777, vocab=50261, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "headgrad", "moe", "moe", "logprob", "logitgrad"])
    if kind in ("heads", "headgrad"):
        dim = rng.choice([64, 128, 128, 256, 80, 96, 72, 40])
        rot = dim if rng.random() < 0.7 else dim // 4 * 2
        k = rng.choice([1, 2, 4, 8, 3, 16])
        q = k * rng.choice([1, 2, 4, 7, 8])
        tokens = min(_log_int(rng, 1, 16384), 16384 * 40 * 128 // 4 // ((q + k) * dim))
        return dict(kind=kind, tokens=tokens, q=q, k=k, dim=dim, rot=rot,
                    axes=rng.choice([1, 1, 2, 3]), interleaved=rng.random() < 0.3,
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind == "moe":
        experts = rng.choice([8, 16, 32, 64, 13, 128])
        hidden, top = 8 * _log_int(rng, 64, 512), rng.choice([1, 2, 4, 6, 8])
        most = 32 * 4096 * 2048 // (max(experts, 8 * top) * hidden)
        return dict(kind=kind, tokens=_log_int(rng, 1, 64), hidden=hidden,
                    width=min(_log_int(rng, 128, 2048), most), experts=experts, top=top,
                    group=rng.choice([32, 64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "f16"]))
    vocab = _log_int(rng, 500, 160000)
    if rng.random() < 0.5:
        vocab = (vocab + 7) // 8 * 8
    case = dict(kind=kind, rows=min(_log_int(rng, 1, 4096), 1024 * 128000 // vocab), vocab=vocab,
                dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind == "logprob":
        # answers that have to keep to a grammar: most tokens masked
        case.update(top=rng.choice([0, 1, 5, 20, 32]), masked=rng.random() < 0.3)
    return case


def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _packed(gen, n, k, group):
    """4-bit rows of roughly normal weights (element j in bits 4 j .. 4 j + 3, rows of
    16-byte pitch, spare bits zero) and fp32 scales [groups][n]."""
    pitch = (k + 31) // 32 * 16
    rows = torch.zeros(n, pitch, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // k)
    for at in range(0, n, step):
        m = min(step, n - at)
        c = _normal(gen, m, (k + 1) // 2 * 2).mul_(2.6).floor_().clamp_(-8, 7).to(torch.int8)
        c[:, k:] = 0
        c = c.view(torch.uint8)
        rows[at:at + m, :c.shape[1] // 2] = (c[:, 0::2] & 15) | ((c[:, 1::2] & 15) << 4)
    scales = 0.2 / math.sqrt(k) * (0.5 + torch.rand(-(-k // group), n, device="cuda", generator=gen))
    return rows, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, s = case["kind"], dict(case)
    t = TYPES[case["dtype"]]
    if kind in ("heads", "headgrad"):
        n, dim, half = case["tokens"], case["dim"], case["rot"] // 2
        # q and k as one product leaves them: parts of a row of q, k and v
        heads = case["q"] + 2 * case["k"]
        qkv = (_normal(gen, n, heads, dim) * (0.5 + 2 * torch.rand(heads, 1, device="cuda", generator=gen))).to(t)
        s["x_q"], s["x_k"] = qkv[:, :case["q"]], qkv[:, case["q"]:case["q"] + case["k"]]
        s["w_q"], s["w_k"] = 1.0 + 0.1 * _normal(gen, dim), 1.0 + 0.1 * _normal(gen, dim)
        # frequencies 1 .. 1 / 500000; the axes take pairs in turn
        i = torch.arange(half, device="cuda")
        s["freq"] = torch.pow(500000.0, -i.double() / max(half, 1)).float()
        s["axis"] = (i % case["axes"]).to(torch.uint8) if case["axes"] > 1 else None
        if case["axes"] == 1:
            first = int(torch.randint(0, 1 << 20, (1,), device="cuda", generator=gen))
            s["pos"] = first + torch.arange(n, device="cuda")[None]
        else:
            s["pos"] = torch.randint(0, 4096, (case["axes"], n), device="cuda", generator=gen)
        if kind == "headgrad":
            s["g_q"] = (1e-2 * _normal(gen, n, case["q"], dim)).to(t)
            s["g_k"] = (1e-2 * _normal(gen, n, case["k"], dim)).to(t)
    elif kind == "moe":
        n, h, e, w = case["tokens"], case["hidden"], case["experts"], case["width"]
        x = _normal(gen, n, h)
        # activations of a decoder: a few channels much larger than the rest
        x[:, torch.randint(0, h, (max(1, h // 256),), device="cuda", generator=gen)] *= 8.0
        s["x"] = x.to(t)
        s["residual"] = (2.0 * _normal(gen, n, h)).to(t)
        s["logits"] = 2.0 * _normal(gen, n, e)
        # all experts' rows are one matrix: of each its gate's, then its other half's
        s["w_in"], s["s_in"] = _packed(gen, e * 2 * w, h, case["group"])
        s["w_out"], s["s_out"] = _packed(gen, e * h, w, case["group"])
    else:
        rows, vocab = case["rows"], case["vocab"]
        logits = torch.empty(rows, vocab, dtype=t, device="cuda")
        s["targets"] = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
        lift = 10.0 * torch.rand(rows, device="cuda", generator=gen)
        step = max(1, (1 << 28) // vocab)
        for at in range(0, rows, step):
            z = 2.5 * _normal(gen, min(step, rows - at), vocab)
            here = slice(at, at + z.shape[0])
            # the model mostly expects what comes
            z[torch.arange(z.shape[0], device="cuda"), s["targets"][here]] += lift[here]
            if case.get("masked"):
                allowed = torch.rand(vocab, device="cuda", generator=gen) < 0.02
                allowed[s["targets"][here]] = True
                z[:, ~allowed] = -math.inf
            logits[here] = z.to(t)
        s["logits"] = logits
        if kind == "logitgrad":
            # what the forward pass leaves
            s["lse"], s["entropy"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            for at in range(0, rows, max(1, (1 << 26) // vocab)):
                here = slice(at, at + max(1, (1 << 26) // vocab))
                lp = torch.log_softmax(logits[here].double(), 1)
                s["entropy"][here] = torch.special.entr(lp.exp()).sum(1).float()
                s["lse"][here] = torch.logsumexp(logits[here].double(), 1).float()
            s["g_logp"] = -torch.rand(rows, device="cuda", generator=gen) / rows
            s["g_entropy"] = -1e-2 * torch.rand(rows, device="cuda", generator=gen) / rows
    return s


# ---- the framework's calls -------------------------------------------------------
def _run_own(s):
    import paper_1908_05033_b200 as dsq

    kind = s["kind"]
    if kind == "heads":
        q, k = dsq.dsq_headnorm_fwd(s["x_q"], s["x_k"], s["pos"], s["freq"], s["w_q"], s["w_k"], EPS,
                                    axis=s["axis"], interleaved=s["interleaved"])
        return {"q": q, "k": k}
    if kind == "headgrad":
        gq, gk, gwq, gwk = dsq.dsq_headnorm_bwd(s["g_q"], s["g_k"], s["x_q"], s["x_k"], s["pos"],
                                                s["freq"], s["w_q"], s["w_k"], EPS, axis=s["axis"],
                                                interleaved=s["interleaved"])
        return {"grad_q": gq, "grad_k": gk, "grad_w_q": gwq, "grad_w_k": gwk}
    if kind == "moe":
        ids, weights = dsq.dsq_moe_route(s["logits"], s["top"])
        y = dsq.dsq_moe_group(s["x"], ids, weights, s["w_in"], s["s_in"], s["w_out"], s["s_out"],
                              s["experts"], s["width"], 4, s["group"], residual=s["residual"])
        return {"ids": ids, "weights": weights, "y": y}
    if kind == "logprob":
        logp, entropy, _, top_ids, top_logp = dsq.dsq_logprob_fwd(s["logits"], s["targets"], top=s["top"])
        return {"logp": logp, "entropy": entropy, "top_ids": top_ids, "top_logp": top_logp}
    return dsq.dsq_logprob_bwd(s["logits"], s["targets"], s["lse"], s["g_logp"], entropy=s["entropy"],
                               grad_entropy=s["g_entropy"])


# ---- the plain forms ---------------------------------------------------------------
def _angles(s):
    """cos and sin [tokens][1][rot / 2] of angles formed in 64 bits."""
    pos = s["pos"].double()
    axis = s["axis"].long() if s["axis"] is not None else torch.zeros(len(s["freq"]), dtype=torch.long,
                                                                     device="cuda")
    a = pos[axis].t() * s["freq"].double()
    return a.cos()[:, None], a.sin()[:, None]


def _pairs(x, s):
    """First and second elements of the rotated pairs, and what is not rotated."""
    r = s["rot"]
    if s["interleaved"]:
        return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]
    return x[..., :r // 2], x[..., r // 2:r], x[..., r:]


def _joined(a, b, rest, s):
    both = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([both, rest], -1)


def _plain_heads(x, w, c, d, s):
    x = x.float()
    n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    a, b, rest = _pairs(n, s)
    return _joined(a * c - b * d, b * c + a * d, rest, s)


def _plain_headgrad(g, x, w, c, d, s):
    a, b, rest = _pairs(g.float(), s)
    g = _joined(a * c + b * d, b * c - a * d, rest, s)
    x = x.float()
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    n, gw = x * rstd, g * w
    return rstd * (gw - n * (gw * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


def _plain_weights(codes, scales, first, n, k, group):
    """fp32 values [n][k] of the packed rows `first` and on."""
    b = codes[first:first + n]
    c = torch.stack([b & 15, b >> 4], 2).view(n, -1)[:, :k].float()
    c = torch.where(c > 7, c - 16, c)                       # signed codes
    scale = scales[:, first:first + n].t().repeat_interleave(group, 1)[:, :k]
    return (2.0 * c + 1.0) * scale


def _largest(z, k):
    """Indices of the k largest of a row, ties to the lowest index."""
    bits = (z.float() + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)             # ordered as the values are
    key = key * (1 << 32) - torch.arange(z.shape[1], device=z.device)
    return torch.topk(key, k, 1).indices


def _row_parts(rows, vocab):
    step = max(1, (1 << 27) // vocab)
    return [slice(at, min(at + step, rows)) for at in range(0, rows, step)]


def _run_plain(s):
    kind, t = s["kind"], TYPES[s["dtype"]]
    if kind in ("heads", "headgrad"):
        c, d = (v.float() for v in _angles(s))
        if kind == "heads":
            return {"q": _plain_heads(s["x_q"], s["w_q"], c, d, s).to(t),
                    "k": _plain_heads(s["x_k"], s["w_k"], c, d, s).to(t)}
        gq, gwq = _plain_headgrad(s["g_q"], s["x_q"], s["w_q"], c, d, s)
        gk, gwk = _plain_headgrad(s["g_k"], s["x_k"], s["w_k"], c, d, s)
        return {"grad_q": gq.to(t), "grad_k": gk.to(t), "grad_w_q": gwq, "grad_w_k": gwk}
    if kind == "moe":
        ids = _largest(s["logits"], s["top"])
        weights = torch.softmax(torch.gather(s["logits"], 1, ids), 1)
        x, h, w, group = s["x"].float(), s["hidden"], s["width"], s["group"]
        y = s["residual"].float()
        for e in range(s["experts"]):
            both = x @ _plain_weights(s["w_in"], s["s_in"], e * 2 * w, 2 * w, h, group).t()
            mid = both[:, :w] * torch.sigmoid(both[:, :w]) * both[:, w:]
            out = mid @ _plain_weights(s["w_out"], s["s_out"], e * h, h, w, group).t()
            y = y + (weights * (ids == e)).sum(1, keepdim=True) * out
        return {"ids": ids.int(), "weights": weights, "y": y.to(t)}
    logits, targets = s["logits"], s["targets"]
    rows, vocab = logits.shape
    if kind == "logitgrad":
        grad = torch.empty_like(logits)
        for part in _row_parts(rows, vocab):
            lp = logits[part].float() - s["lse"][part, None]
            p = lp.exp()
            gl, ge, h = (s[i][part, None] for i in ("g_logp", "g_entropy", "entropy"))
            g = -gl * p - ge * torch.where(p > 0, p * (lp + h), 0.0)
            grad[part] = g.scatter_add_(1, targets[part, None], gl).to(t)
        return grad
    logp, entropy = (torch.empty(rows, device="cuda") for _ in range(2))
    top_ids = torch.empty(rows, s["top"], dtype=torch.long, device="cuda")
    top_logp = torch.empty(rows, s["top"], device="cuda")
    for part in _row_parts(rows, vocab):
        z = logits[part].float()
        d = z - z.amax(1, keepdim=True)
        e = d.exp()
        total = e.sum(1, keepdim=True)
        lp = d - total.log()
        p = e / total
        logp[part] = torch.gather(lp, 1, targets[part, None])[:, 0]
        entropy[part] = -torch.where(p > 0, p * lp, 0.0).sum(1)
        if s["top"]:
            top_ids[part] = _largest(z, s["top"])
            top_logp[part] = torch.gather(lp, 1, top_ids[part])
    if not s["top"]:
        top_ids = top_logp = None
    return {"logp": logp, "entropy": entropy, "top_ids": top_ids, "top_logp": top_logp}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- bytes and operations ------------------------------------------------------------
def work(case):
    kind, t = case["kind"], SIZE[case["dtype"]]
    if kind in ("heads", "headgrad"):
        n, heads = case["tokens"], case["q"] + case["k"]
        elements = n * heads * case["dim"]
        # positions, frequencies and weights in (and the weights' gradients out)
        small = 8 * n * case["axes"] + 2 * case["rot"] + 8 * case["dim"]
        if kind == "heads":
            return {"bytes": 2 * elements * t + small, "flops": 8 * elements}
        return {"bytes": 3 * elements * t + small + 8 * case["dim"], "flops": 18 * elements}
    if kind == "moe":
        n, h, w, e, k = (case[i] for i in ("tokens", "hidden", "width", "experts", "top"))
        # experts that anything goes to, every choice as likely as another
        used = e * (1.0 - (1.0 - k / e) ** n)
        weights = used * (3 * h * w / 2 + 4 * 2 * w * -(-h // case["group"]) + 4 * h * -(-w // case["group"]))
        return {"bytes": int(weights) + 3 * n * h * t + 4 * n * e, "flops": 6 * n * k * h * w}
    rows, vocab = case["rows"], case["vocab"]
    if kind == "logprob":
        return {"bytes": rows * vocab * t + rows * (8 + 8 + 12 * case["top"]), "flops": 6 * rows * vocab}
    return {"bytes": 2 * rows * vocab * t + 24 * rows, "flops": 8 * rows * vocab}


# ---- the definitions in 64 bits ---------------------------------------------------------
def _exact_turns(s):
    """The rotation of each token as complex numbers [tokens][rot / 2]."""
    n, half = s["tokens"], s["rot"] // 2
    angle = torch.empty(n, half, dtype=torch.float64, device="cuda")
    for i in range(half):
        a = int(s["axis"][i]) if s["axis"] is not None else 0
        angle[:, i] = s["pos"][a].double() * s["freq"][i].double()
    return torch.polar(torch.ones_like(angle), angle)


def _turn(v, turns, s):
    """Rotated heads [tokens][heads][dim]."""
    out, r = v.clone(), s["rot"]
    i = torch.arange(r // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + r // 2)
    z = torch.complex(v[..., first], v[..., second]) * turns[:, None]
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_weights(codes, scales, rows, k, group):
    b = codes[rows].long()
    half_bytes = torch.empty(b.shape[0], 2 * b.shape[1], dtype=torch.int64, device="cuda")
    half_bytes[:, 0::2] = torch.remainder(b, 16)
    half_bytes[:, 1::2] = torch.div(b, 16, rounding_mode="floor")
    v = (2 * (torch.remainder(half_bytes + 8, 16) - 8) + 1)[:, :k].double()
    for g in range(scales.shape[0]):
        v[:, g * group:(g + 1) * group] *= scales[g, rows].double()[:, None]
    return v


def _exact_moe(s):
    n, h, w = s["tokens"], s["hidden"], s["width"]
    order = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    ids = order.indices[:, :s["top"]]
    z = torch.exp(order.values[:, :s["top"]].double() - order.values[:, :1].double())
    weights = z / z.sum(1, keepdim=True)
    y = s["residual"].double()
    chosen = ids.cpu().tolist()
    for e in range(s["experts"]):
        where = [(t, j) for t in range(n) for j in range(s["top"]) if chosen[t][j] == e]
        if not where:
            continue
        t, j = (torch.tensor(v, device="cuda") for v in zip(*where))
        x = s["x"][t].double()
        both = torch.einsum("th,oh->to", x, _exact_weights(s["w_in"], s["s_in"],
                                                           slice(e * 2 * w, (e + 1) * 2 * w), h, s["group"]))
        gate, up = both[:, :w], both[:, w:]
        mid = gate / (1.0 + torch.exp(-gate)) * up
        out = torch.einsum("tw,hw->th", mid, _exact_weights(s["w_out"], s["s_out"],
                                                            slice(e * h, (e + 1) * h), w, s["group"]))
        y.index_add_(0, t, weights[t, j, None] * out)
    return {"ids": ids.int(), "weights": weights, "y": y}


def _exact_logits(s):
    rows, vocab = s["logits"].shape
    k = s["top"]
    out = {i: torch.empty(rows, dtype=torch.float64, device="cuda") for i in ("logp", "entropy")}
    out["top_ids"] = torch.empty(rows, k, dtype=torch.long, device="cuda") if k else None
    out["top_logp"] = torch.empty(rows, k, dtype=torch.float64, device="cuda") if k else None
    for at in range(0, rows, max(1, (1 << 26) // vocab)):
        here = slice(at, at + max(1, (1 << 26) // vocab))
        z, t = s["logits"][here].double(), s["targets"][here]
        r = torch.arange(z.shape[0], device="cuda")
        lp = z - torch.logsumexp(z, 1)[:, None]
        out["logp"][here], out["entropy"][here] = lp[r, t], torch.special.entr(torch.exp(lp)).sum(1)
        left = z.clone()
        for i in range(k):
            # the first of equal largest values (what is taken is NaN: neither equal nor larger)
            best = left.nan_to_num(nan=-math.inf).amax(1, keepdim=True)
            first = (left == best).byte().argmax(1)
            out["top_ids"][here, i], out["top_logp"][here, i] = first, lp[r, first]
            left[r, first] = math.nan
    return out


def _exact_logit_grad(s):
    grad = torch.empty(s["logits"].shape, dtype=torch.float64, device="cuda")
    for row in range(len(grad)):
        p = torch.exp(s["logits"][row].double() - s["lse"][row].double())
        gl, ge = s["g_logp"][row].double(), s["g_entropy"][row].double()
        # d H / d z_j = -p_j (log p_j + H) = entr(p_j) - p_j H
        grad[row] = ge * (torch.special.entr(p) - p * s["entropy"][row].double()) - gl * p
        grad[row, s["targets"][row]] += gl
    return grad


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "moe":
        return _exact_moe(s)
    if kind == "logprob":
        return _exact_logits(s)
    if kind == "logitgrad":
        return _exact_logit_grad(s)
    turns = _exact_turns(s)
    out = {}
    for name in ("q", "k"):
        x, w = s["x_" + name].double(), s["w_" + name].double()
        mean = torch.linalg.vector_norm(x, dim=2) ** 2 / case["dim"]
        r = 1.0 / torch.sqrt(mean + EPS)
        if kind == "heads":
            out[name] = _turn(torch.einsum("thd,th,d->thd", x, r, w), turns, s)
            continue
        g = _turn(s["g_" + name].double(), torch.conj(turns), s)
        # d/dx_j of sum_i g_i w_i x_i r(x): r g_j w_j - r^3 x_j / dim sum_i g_i w_i x_i
        dot = torch.einsum("thd,d,thd->th", g, w, x)
        out["grad_" + name] = (torch.einsum("thd,d,th->thd", g, w, r)
                               - torch.einsum("thd,th->thd", x, r ** 3 * dot / case["dim"]))
        out["grad_w_" + name] = torch.einsum("thd,thd,th->d", g, x, r)
    return out
