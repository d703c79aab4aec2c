"""Performance cases of the operators around a low-bit linear layer of a
decoder: root-mean-square norm with the residual's addition and 8-bit output,
its backward pass, 4-bit weights with a scale per group, and products of few
rows with them.

A case is a dict of plain values; `kind` says which operators it goes through:
  norm    dsq_rmsnorm_fwd: h = x + residual, then the norm; `quant`: its
          output goes through 8 bits with a scale per row (the forward pass of
          quantisation-aware training)
  grad    dsq_rmsnorm_bwd: gradients of the input and of the norm's weight
  groups  dsq_quantize_groups then dsq_dequantize_groups: weights to 4-bit
          codes with group scales and the values those stand for
  linear  dsq_wgemm_group on bf16 or fp16 rows
  step    dsq_rmsnorm_fwd to 8-bit codes, then dsq_wgemm_group on those: the
          front of a decoder layer when it serves

With `own` false `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token of a decoder at width 4096: the smallest call there is, latency only
        dict(name="norm_1x4096_bf16", kind="norm", rows=1, k=4096, dtype="bf16", quant=False),
        # a training batch, the linear layers' inputs quantised to 8 bits in the loop
        dict(name="norm_8192x4096_bf16_quant", kind="norm", rows=8192, k=4096, dtype="bf16",
             quant=True),
        # the backward pass of such a batch
        dict(name="grad_8192x4096_bf16", kind="grad", rows=8192, k=4096, dtype="bf16"),
        # nothing a multiple of a vector: rows start at odd addresses
        dict(name="grad_1111x1777_f16", kind="grad", rows=1111, k=1777, dtype="f16"),
        # weights of a wide linear layer prepared for serving
        dict(name="groups_16384x4096_bf16_g128", kind="groups", n=16384, k=4096, group=128,
             dtype="bf16"),
        # ragged, the last group a short one, small groups
        dict(name="groups_1111x1777_f32_g32", kind="groups", n=1111, k=1777, group=32,
             dtype="f32"),
        # one token through a square layer: latency and 8 MiB of codes
        dict(name="linear_1x4096x4096_bf16_g128", kind="linear", m=1, n=4096, k=4096, group=128,
             dtype="bf16", out="bf16"),
        # one token through the widest layer: the rate at which weights are read
        dict(name="linear_1x16384x8192_bf16_g128", kind="linear", m=1, n=16384, k=8192, group=128,
             dtype="bf16", out="bf16"),
        # a few requests together, ragged widths
        dict(name="linear_7x2777x5000_f16_g64", kind="linear", m=7, n=2777, k=5000, group=64,
             dtype="f16", out="f32"),
        # a full batch of decoding requests: the most arithmetic
        dict(name="linear_64x8192x8192_bf16_g128", kind="linear", m=64, n=8192, k=8192, group=128,
             dtype="bf16", out="f32"),
        # one token, norm and 8-bit product one after the other
        dict(name="step_1x8192x8192_g128", kind="step", m=1, n=8192, k=8192, group=128,
             dtype="bf16"),
        # the same for a batch, groups of 64
        dict(name="step_24x6144x2048_g64", kind="step", m=24, n=6144, k=2048, group=64,
             dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "grad", "groups", "linear", "linear", "step"])
    if kind in ("norm", "grad"):
        k = _log_int(rng, 64, 16384)
        if rng.random() < 0.6:
            k = (k + 7) // 8 * 8
        rows = min(_log_int(rng, 1, 8192), (8192 * 4096 // 2) // k)
        case = dict(kind=kind, rows=rows, k=k, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
        if kind == "norm":
            # (training quantises what it holds in 16 bits)
            case["quant"] = case["dtype"] != "f32" and rng.random() < 0.6
        return case
    group = rng.choice([32, 64, 128, 128, 256])
    if kind == "groups":
        return dict(kind=kind, n=_log_int(rng, 256, 9000), k=_log_int(rng, 256, 5000), group=group,
                    dtype=rng.choice(["bf16", "f16", "f32"]))
    # rows of activations start on 16-byte boundaries: k is a multiple of 8, of 16 in 8 bits
    if kind == "linear":
        return dict(kind=kind, m=_log_int(rng, 1, 64), n=_log_int(rng, 512, 8192),
                    k=8 * _log_int(rng, 64, 1024), group=group, dtype=rng.choice(["bf16", "f16"]),
                    out=rng.choice(["bf16", "f16", "f32"]))
    return dict(kind=kind, m=_log_int(rng, 1, 64), n=_log_int(rng, 512, 8192),
                k=16 * _log_int(rng, 32, 512), group=group, dtype="bf16")


def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _acts(gen, rows, k, dtype):
    """Activations of a decoder: near normal, a few channels much larger than the rest."""
    x = _normal(gen, rows, k)
    x[:, torch.randint(0, k, (max(1, k // 256),), device="cuda", generator=gen)] *= 12.0
    return x.to(dtype)


def _packed(gen, n, k, group):
    """4-bit rows of roughly normal weights (element j in bits 4 j .. 4 j + 3, rows of
    16-byte pitch, spare bits zero) and fp32 scales [groups][n]."""
    pitch = (k + 31) // 32 * 16
    rows = torch.zeros(n, pitch, dtype=torch.uint8, device="cuda")
    c = torch.randn(n, (k + 1) // 2 * 2, device="cuda", generator=gen).mul_(2.6).floor_()
    c = c.clamp_(-8, 7).to(torch.int8)
    c[:, k:] = 0
    c = c.view(torch.uint8)
    rows[:, :c.shape[1] // 2] = (c[:, 0::2] & 15) | ((c[:, 1::2] & 15) << 4)
    groups = -(-k // group)
    scales = 0.02 / math.sqrt(k) * (0.5 + torch.rand(groups, n, device="cuda", generator=gen))
    return rows, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, s = case["kind"], dict(case)
    if kind in ("norm", "grad", "step"):
        rows, k, t = case.get("rows", case.get("m")), case["k"], TYPES[case["dtype"]]
        s["weight"] = 1.0 + 0.1 * _normal(gen, k)
        s["x"] = _acts(gen, rows, k, t)
        if kind == "grad":
            # h and rstd as the forward pass leaves them
            s["rstd"] = torch.rsqrt(s["x"].double().square().mean(1) + EPS).float()
            s["grad_y"] = (1e-2 * _normal(gen, rows, k)).to(t)
            s["grad_h"] = (1e-2 * _normal(gen, rows, k)).to(t)
        else:
            s["residual"] = (2.0 * _normal(gen, rows, k)).to(t)
    if kind in ("linear", "step"):
        s["codes"], s["scales"] = _packed(gen, case["n"], case["k"], case["group"])
        s["bias"] = 0.1 * _normal(gen, case["n"])
        if kind == "linear":
            s["x"] = _acts(gen, case["m"], case["k"], TYPES[case["dtype"]])
    if kind == "groups":
        s["w"] = (0.02 * _normal(gen, case["n"], case["k"])).to(TYPES[case["dtype"]])
    return s


# ---- the framework's calls -------------------------------------------------------
def _run_own(s):
    import paper_1908_05033_b200 as dsq

    kind = s["kind"]
    if kind == "norm":
        h, y, _, scale, rstd = dsq.dsq_rmsnorm_fwd(s["x"], s["weight"], EPS,
                                                   residual=s["residual"], quantised=s["quant"],
                                                   want_rstd=True)
        return {"h": h, "y": y, "scale": scale, "rstd": rstd}
    if kind == "grad":
        gx, gw = dsq.dsq_rmsnorm_bwd(s["grad_y"], s["x"], s["weight"], s["rstd"],
                                     grad_h=s["grad_h"])
        return {"grad_x": gx, "grad_weight": gw}
    if kind == "groups":
        codes, scales = dsq.dsq_quantize_groups(s["w"], 4, s["group"])
        values = dsq.dsq_dequantize_groups(codes, scales, s["n"], s["k"], 4, s["group"],
                                           out_dtype=torch.bfloat16)
        return {"scales": scales, "values": values}
    if kind == "linear":
        return dsq.dsq_wgemm_group(s["x"], s["codes"], s["m"], s["n"], s["k"], 4, s["group"],
                                   s["scales"], bias=s["bias"], out_dtype=TYPES[s["out"]])
    h, _, q, row_scale, _ = dsq.dsq_rmsnorm_fwd(s["x"], s["weight"], EPS, residual=s["residual"],
                                                quantised=True, want_y=False, want_codes=True)
    y = dsq.dsq_wgemm_group(q, s["codes"], s["m"], s["n"], s["k"], 4, s["group"], s["scales"],
                            bias=s["bias"], row_scale=row_scale, out_dtype=torch.bfloat16)
    return {"h": h, "y": y}


# ---- the plain forms ---------------------------------------------------------------
def _plain_norm(s, quant):
    """h, y, codes, scale, rstd before any rounding to fewer bits."""
    h = s["x"].float() + s["residual"].float()
    rstd = torch.rsqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None] * s["weight"]
    if not quant:
        return h, y, None, None, rstd
    # which side of a border a value lies on is decided in 64 bits
    h64 = s["x"].double() + s["residual"].double()
    y64 = h64 * torch.rsqrt(h64.square().mean(1, keepdim=True) + EPS) * s["weight"].double()
    scale = y64.abs().amax(1) / 127.0
    q = torch.floor(y64 / scale[:, None] + 0.5).clamp(-127, 127).float()
    scale = scale.float()
    return h, q * scale[:, None], q, scale, rstd


def _plain_weights(s):
    """fp32 values [n][k] of the packed rows."""
    b = s["codes"]
    c = torch.stack([b & 15, b >> 4], 2).view(s["n"], -1)[:, :s["k"]].float()
    c = torch.where(c > 7, c - 16, c)                       # signed codes
    scale = s["scales"].t().repeat_interleave(s["group"], 1)[:, :s["k"]]
    return (2.0 * c + 1.0) * scale


def _run_plain(s):
    kind = s["kind"]
    t = TYPES.get(s.get("dtype"))
    if kind == "norm":
        h, y, _, scale, rstd = _plain_norm(s, s["quant"])
        return {"h": h.to(t), "y": y.to(t), "scale": scale, "rstd": rstd}
    if kind == "grad":
        gy, h, rstd = s["grad_y"].float(), s["x"].float(), s["rstd"][:, None]
        g, n = gy * s["weight"], h * rstd
        gx = rstd * (g - n * (g * n).mean(1, keepdim=True)) + s["grad_h"].float()
        return {"grad_x": gx.to(t), "grad_weight": (gy * n).sum(0)}
    if kind == "groups":
        n, k, group = s["n"], s["k"], s["group"]
        groups = -(-k // group)
        w = torch.zeros(n, groups * group, device="cuda")
        w[:, :k] = s["w"]
        w = w.view(n, groups, group)
        a = w.abs().amax(2, keepdim=True)
        # (w + a) 15 / (2 a) + 1/2 as one quotient of numbers that are exact in 64 bits: bf16
        # weights often lie on a border, which belongs to the code above it
        q = torch.floor((15.0 * w.double() + 16.0 * a.double()) / (2.0 * a.double()))
        q = q.clamp(0, 15).float()
        values = (2.0 * q - 15.0) * (a / 15.0)
        values = values.view(n, groups * group)[:, :k]
        return {"scales": (a[:, :, 0] / 15.0).t().contiguous(), "values": values.to(torch.bfloat16)}
    if kind == "linear":
        y = s["x"].float() @ _plain_weights(s).t() + s["bias"]
        return y.to(TYPES[s["out"]])
    h, x, _, _, _ = _plain_norm(s, True)
    y = x @ _plain_weights(s).t() + s["bias"]
    return {"h": h.to(t), "y": y.to(torch.bfloat16)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- bytes and operations ------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "norm":
        m, k, t = case["rows"], case["k"], SIZE[case["dtype"]]
        # x, residual, weight in; h, y, rstd (and scales) out
        return {"bytes": 4 * m * k * t + 4 * k + 4 * m * (2 if case["quant"] else 1),
                "flops": m * k * (8 if case["quant"] else 5)}
    if kind == "grad":
        m, k, t = case["rows"], case["k"], SIZE[case["dtype"]]
        # grad_y, h, grad_h, weight, rstd in; grad_x, grad_weight out
        return {"bytes": 4 * m * k * t + 8 * k + 4 * m, "flops": 11 * m * k}
    n, k, groups = case["n"], case["k"], -(-case["k"] // case["group"])
    if kind == "groups":
        # weights in, codes out and in again, scales, bf16 values out
        return {"bytes": n * k * (SIZE[case["dtype"]] + 2) + 2 * (n * k // 2) + 8 * n * groups,
                "flops": 6 * n * k}
    m = case["m"]
    weights = n * k // 2 + 4 * n * groups + 4 * n
    if kind == "linear":
        return {"bytes": weights + m * k * SIZE[case["dtype"]] + m * n * SIZE[case["out"]],
                "flops": 2 * m * n * k}
    # x, residual in, h out, codes out and in again
    return {"bytes": weights + m * k * (3 * SIZE[case["dtype"]] + 2) + 4 * k + 2 * m * n,
            "flops": 2 * m * n * k + 8 * m * k}


# ---- the definitions in 64 bits ---------------------------------------------------------
def _exact_norm(s):
    h = torch.add(s["x"].to(torch.float64), s["residual"].to(torch.float64))
    mean = torch.linalg.vector_norm(h, dim=1) ** 2 / h.shape[1]
    rstd = 1.0 / torch.sqrt(mean + EPS)
    return h, torch.einsum("mk,m,k->mk", h, rstd, s["weight"].double()), rstd


def _exact_eight_bits(y):
    """s q and s: 127 steps to the largest magnitude of a row, midpoints upwards."""
    step = y.abs().max(dim=1).values / 127.0
    return torch.einsum("mk,m->mk", torch.floor(y / step[:, None] + 0.5), step), step


def _exact_weights(s):
    n, k, group = s["n"], s["k"], s["group"]
    half_bytes = torch.empty(n, 2 * s["codes"].shape[1], dtype=torch.int64, device="cuda")
    half_bytes[:, 0::2] = torch.remainder(s["codes"].long(), 16)
    half_bytes[:, 1::2] = torch.div(s["codes"].long(), 16, rounding_mode="floor")
    # two's complement c = ((b + 8) mod 16) - 8, value 2 c + 1
    v = (2 * (torch.remainder(half_bytes + 8, 16) - 8) + 1)[:, :k].double()
    for g in range(s["scales"].shape[0]):
        v[:, g * group:(g + 1) * group] *= s["scales"][g].double()[:, None]
    return v


def exact(case, seed):
    if case["kind"] in ("linear", "step") and case["n"] * case["k"] > 1 << 28:
        return None
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h, y, rstd = _exact_norm(s)
        step = None
        if case["quant"]:
            y, step = _exact_eight_bits(y)
        return {"h": h, "y": y, "scale": step, "rstd": rstd}
    if kind == "grad":
        k = case["k"]
        gy, h, r = s["grad_y"].double(), s["x"].double(), s["rstd"].double()
        w = s["weight"].double()
        # d/dh_j of sum_i gy_i w_i h_i r(h): r gy_j w_j - r^3 h_j / k sum_i gy_i w_i h_i
        dot = torch.einsum("mk,k,mk->m", gy, w, h)
        gx = torch.einsum("mk,k,m->mk", gy, w, r) - torch.einsum("mk,m->mk", h, r ** 3 * dot / k)
        return {"grad_x": gx + s["grad_h"].double(),
                "grad_weight": torch.einsum("mk,mk,m->k", gy, h, r)}
    if kind == "groups":
        n, k, group = case["n"], case["k"], case["group"]
        w = s["w"].double()
        scales = torch.empty(-(-k // group), n, dtype=torch.float64, device="cuda")
        values = torch.empty_like(w)
        for g in range(scales.shape[0]):
            part = w[:, g * group:(g + 1) * group]
            half_step = part.abs().max(dim=1).values / 15.0
            # codes of the grid -a + 2 a q / 15: q = floor((w + a) 15 / (2 a) + 1/2), a quotient
            # of numbers that are exact in 64 bits
            a = part.abs().max(dim=1).values[:, None]
            q = torch.floor((15.0 * part + 16.0 * a) / (2.0 * a)).clamp(0, 15)
            scales[g] = half_step
            values[:, g * group:(g + 1) * group] = (2 * q - 15) * half_step[:, None]
        return {"scales": scales, "values": values}
    if kind == "linear":
        return torch.einsum("mk,nk->mn", s["x"].double(), _exact_weights(s)) + s["bias"].double()
    h, y, _ = _exact_norm(s)
    y, _ = _exact_eight_bits(y)
    return {"h": h, "y": torch.einsum("mk,nk->mn", y, _exact_weights(s)) + s["bias"].double()}
