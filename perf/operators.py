"""Measured cases of the layer-norm, top-logits and distillation operators, through the
public entry points (paper_2509_26092_amd.binding).

Four kinds of case:
  ln_fwd   layer norm over the channels of [rows][width]: y, mean, rstd
  ln_bwd   its backward pass: dx and the gradients of gamma and beta
  topk     the K largest logits of every row with their classes, ties to the lowest class:
           what a teacher keeps of a batch
  distill  the distillation loss of a batch against a teacher's top logits, mixed with
           the labels' cross-entropy, and the gradient of the logits

Sizes are those of the training configurations (the NHWC tensors of ResNet-18 at batch
256 and 224 pixels, 512 pooled features, 1000 classes, batches 64 and 256) and generic
ones: wide rows, large class counts, odd sizes, rows inside wider buffers.

`own` is False: the operators in plain torch operations, in 32 bits, rounded once at the
end. `own` is True: the library's operators.
"""
import math

import torch

own = False

EPS = 1e-5
TYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
MAX_BYTES = 16384 * 8192 * 6          # of the largest listed case


# ---------------------------------------------------------------- the cases
def _ln(name, kind, prec, rows, width, pad=0):
    return {"name": name, "kind": kind, "prec": prec, "rows": rows, "width": width, "pad": pad}


def _topk(name, prec, rows, classes, k, pad=0):
    return {"name": name, "kind": "topk", "prec": prec, "rows": rows, "classes": classes, "k": k, "pad": pad}


def _distill(name, prec, rows, classes, k, temperature, alpha, masked=False, pad=0):
    return {"name": name, "kind": "distill", "prec": prec, "rows": rows, "classes": classes, "k": k,
            "temperature": temperature, "alpha": alpha, "masked": masked, "pad": pad}


def listed():
    return [
        # the pooled features of a small worker's batch before its classifier: latency
        _ln("ln_fwd_fp32_64x512", "ln_fwd", "fp32", 64, 512),
        # in place of a stage-1 batch norm of the large worker: every pixel of 256 x 56 x 56, 64 channels
        _ln("ln_fwd_bf16_802816x64", "ln_fwd", "bf16", 802816, 64),
        # odd rows of a wider buffer: a slice of a concatenation, ragged token count
        _ln("ln_fwd_fp16_16385x2050_strided", "ln_fwd", "fp16", 16385, 2050, 7),
        # the backward passes of the first two
        _ln("ln_bwd_fp32_64x512", "ln_bwd", "fp32", 64, 512),
        _ln("ln_bwd_bf16_802816x64", "ln_bwd", "bf16", 802816, 64),
        # wide rows of a large model's token batch
        _ln("ln_bwd_bf16_16384x8192", "ln_bwd", "bf16", 16384, 8192),
        # a teacher's logits of the headline batch over 1000 classes
        _topk("topk_fp32_256x1000_k10", "fp32", 256, 1000, 10),
        # a teacher over a large class set or vocabulary: 4096 tokens
        _topk("topk_bf16_4096x32768_k64", "bf16", 4096, 32768, 64),
        # few long odd rows: an interactive request
        _topk("topk_fp16_7x131071_k20", "fp16", 7, 131071, 20),
        # the small worker's step: 1000 classes, temperature 4, mostly the teacher's word
        _distill("distill_fp32_64x1000_k10", "fp32", 64, 1000, 10, 4.0, 0.9),
        # a large batch of tokens, teacher only
        _distill("distill_bf16_8192x32768_k64", "bf16", 8192, 32768, 64, 2.0, 1.0),
        # odd class count, padded rows, masked classes, short and empty lists, unlabelled and switched-off rows
        _distill("distill_fp16_1023x50001_masked", "fp16", 1023, 50001, 32, 1.5, 0.5, True, 3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ln_fwd", "ln_bwd", "topk", "distill"])
    prec = rng.choice(["fp32", "bf16", "fp16"])
    pad = rng.choice([0, 0, 0, rng.randint(1, 64)])
    if kind in ("ln_fwd", "ln_bwd"):
        width = _log(rng, 16, 16384)
        if rng.random() < 0.5:
            width = (width + 7) // 8 * 8
        most = MAX_BYTES // (width * SIZE[prec] * 3)
        c = _ln("", kind, prec, _log(rng, 1, min(most, 1 << 20)), width, pad)
    else:
        classes = _log(rng, 10, 131072)
        if rng.random() < 0.3:
            classes = (classes + 7) // 8 * 8
        k = min(classes, _log(rng, 1, 64))
        # the plain form sorts: rows x classes as in the listed cases
        most = (4096 * 32768 if kind == "topk" else MAX_BYTES // (2 * SIZE[prec])) // classes
        rows = _log(rng, 1, min(most, 1 << 14))
        if kind == "topk":
            c = _topk("", prec, rows, classes, k, pad)
        else:
            c = _distill("", prec, rows, classes, k, round(rng.uniform(1.0, 6.0), 2),
                         rng.choice([1.0, round(rng.uniform(0.1, 0.95), 2)]), rng.random() < 0.4, pad)
    del c["name"]
    return c


def work(case):
    es, rows = SIZE[case["prec"]], case["rows"]
    if case["kind"] == "ln_fwd":
        n = rows * case["width"]
        return {"bytes": 2 * n * es + 8 * case["width"] + 8 * rows, "flops": 8 * n}
    if case["kind"] == "ln_bwd":
        n = rows * case["width"]
        return {"bytes": 3 * n * es + 12 * case["width"] + 8 * rows, "flops": 14 * n}
    n, k = rows * case["classes"], rows * case["k"]
    if case["kind"] == "topk":
        return {"bytes": n * es + 8 * k, "flops": n}
    return {"bytes": 2 * n * es + 8 * k + 12 * rows + 4, "flops": (6 if case["alpha"] == 1.0 else 12) * n}


# ---------------------------------------------------------------- inputs
def _rows(g, rows, width, pad, dtype, scale, shift=0.0):
    """A [rows][width] view of a buffer `width + pad` wide."""
    b = torch.empty((rows, width + pad), dtype=dtype, device="cuda").normal_(shift, scale, generator=g)
    return b[:, :width]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, rows, pad = TYPE[case["prec"]], case["rows"], case["pad"]
    f32 = dict(dtype=torch.float32, device="cuda")
    s = dict(case)
    if case["kind"] in ("ln_fwd", "ln_bwd"):
        w = case["width"]
        s["x"] = _rows(g, rows, w, pad, dt, 1.5, 0.4)
        s["gamma"] = 1.0 + 0.2 * torch.randn(w, generator=g, **f32)
        s["mean"], s["rstd"] = torch.empty(rows, **f32), torch.empty(rows, **f32)
        if case["kind"] == "ln_fwd":
            s["beta"] = 0.2 * torch.randn(w, generator=g, **f32)
            s["y"] = torch.empty((rows, w), dtype=dt, device="cuda")
        else:
            s["dy"] = _rows(g, rows, w, pad, dt, 0.7)
            step = max(1, (1 << 26) // w)
            for r in range(0, rows, step):     # what the forward pass left
                v, m = torch.var_mean(s["x"][r:r + step].float(), dim=1, unbiased=False)
                s["mean"][r:r + step], s["rstd"][r:r + step] = m, torch.rsqrt(v + EPS)
            s["dx"] = torch.empty((rows, w), dtype=dt, device="cuda")
            s["dgamma"], s["dbeta"] = torch.empty(w, **f32), torch.empty(w, **f32)
        return s
    c, k = case["classes"], case["k"]
    s["z"] = _rows(g, rows, c, pad, dt, 2.5)
    if case["kind"] == "topk":
        s["vals"] = torch.empty((rows, k), **f32)
        s["idx"] = torch.empty((rows, k), dtype=torch.int32, device="cuda")
        return s
    # the teacher: the student's logits moved by noise, its k largest
    s["t_vals"] = torch.empty((rows, k), **f32)
    s["t_idx"] = torch.empty((rows, k), dtype=torch.int32, device="cuda")
    step = max(1, (1 << 26) // c)
    for r in range(0, rows, step):
        t = s["z"][r:r + step].float()
        v, i = (t + torch.randn(t.shape, generator=g, device="cuda")).topk(k, dim=1)
        s["t_vals"][r:r + step], s["t_idx"][r:r + step] = v, i
    s["labels"] = torch.randint(0, c, (rows,), generator=g, device="cuda", dtype=torch.int32)
    s["weight"] = None
    if case["masked"]:
        u = torch.rand((4, rows), generator=g, device="cuda")
        s["t_idx"].masked_fill_(torch.rand((rows, k), generator=g, device="cuda") < 0.2, -1)  # short lists
        s["t_idx"].masked_fill_((u[0] < 0.05)[:, None], -1)                                   # empty lists
        s["labels"].masked_fill_(u[1] < 0.2, -1)                                              # no label
        hidden = torch.randint(0, c, (max(1, c // 50),), generator=g, device="cuda")          # masked classes
        hidden = hidden[~torch.isin(hidden, torch.cat([s["labels"], s["t_idx"].reshape(-1)]).long().clamp_(min=0))]
        s["z"][:, hidden] = -math.inf
        s["weight"] = torch.where(u[2] < 0.1, 0.0, 0.5 + u[3])                                # switched-off rows ...
        s["z"].masked_fill_((u[2] < 0.1)[:, None], math.nan)                                  # ... hold anything
    s["scale"] = (1024.0 if case["prec"] == "fp16" else 1.0) / rows      # the batch's mean, fp16 with a loss scale
    s["dz"] = torch.empty((rows, c), dtype=dt, device="cuda")
    s["row_loss"], s["loss"] = torch.empty(rows, **f32), torch.empty(1, **f32)
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    return globals()[("_own_" if own else "_plain_") + state["kind"]](state)


def _plain_ln_fwd(s):
    x = s["x"].float()
    mean = x.mean(dim=1)
    d = x - mean[:, None]
    rstd = torch.rsqrt((d * d).mean(dim=1) + EPS)
    y = d * rstd[:, None] * s["gamma"] + s["beta"]
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_ln_bwd(s):
    dy = s["dy"].float()
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["gamma"]
    dx = s["rstd"][:, None] * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(dim=0), "dbeta": dy.sum(dim=0)}


def _plain_topk(s):
    v, i = torch.sort(s["z"].float(), dim=1, descending=True, stable=True)
    return {"vals": v[:, :s["k"]].contiguous(), "idx": i[:, :s["k"]].to(torch.int32)}


def _softmax(x):
    """(probabilities, log of the sum of exponentials, whether the row has any) of every row."""
    m = x.amax(dim=1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(x - m)
    t = e.sum(dim=1, keepdim=True)
    some = t != 0
    return e / torch.where(some, t, torch.ones_like(t)), (m + torch.log(t))[:, 0], some


def _plain_distill(s):
    z, c, temp, alpha = s["z"].float(), s["classes"], s["temperature"], s["alpha"]
    w = s["weight"] if s["weight"] is not None else torch.ones_like(s["row_loss"])
    on = (w != 0)[:, None]
    z = torch.where(on, z, torch.zeros_like(z)) if s["weight"] is not None else z
    idx = s["t_idx"].long()
    valid = (idx >= 0) & (idx < c)
    at = torch.where(valid, idx, torch.zeros_like(idx))
    q, lse_t, some_t = _softmax(torch.where(valid, s["t_vals"] / temp, torch.full_like(s["t_vals"], -math.inf)))
    p, lse, some = _softmax(z / temp)
    some_t = some_t & some & on
    zero = torch.zeros_like(q)
    terms = torch.where(q > 0, q * (s["t_vals"] / temp - lse_t[:, None] - z.gather(1, at) / temp + lse[:, None]), zero)
    loss = alpha * temp * temp * torch.where(some_t[:, 0], terms.sum(dim=1), torch.zeros_like(lse))
    dz = alpha * temp * torch.where(some_t, p, torch.zeros_like(p))
    dz.scatter_add_(1, at, -alpha * temp * torch.where(some_t, q, zero))
    if alpha != 1.0:
        y = s["labels"].long()[:, None]
        p, lse, some = _softmax(z)
        some_y = (y >= 0) & (y < c) & some & on
        y = torch.where(some_y, y, torch.zeros_like(y))
        loss = loss + (1 - alpha) * torch.where(some_y[:, 0], lse - z.gather(1, y)[:, 0], torch.zeros_like(lse))
        dz = dz + (1 - alpha) * torch.where(some_y, p, torch.zeros_like(p))
        dz.scatter_add_(1, y, (alpha - 1) * some_y.float())
    loss = w * loss
    return {"dz": (dz * (s["scale"] * w)[:, None]).to(s["z"].dtype), "row_loss": loss,
            "loss": s["scale"] * loss.sum(dim=0, keepdim=True)}


def _binding():
    from paper_2509_26092_amd import binding
    return binding


def _own_ln_fwd(s):
    B = _binding()
    x, y = s["x"], s["y"]
    B.rn18op_layernorm_fwd(B.PREC_IDS[s["prec"]], x, s["gamma"], s["beta"], y, s["mean"], s["rstd"], s["rows"],
                           s["width"], x.stride(0), y.stride(0), EPS)
    return {"y": y, "mean": s["mean"], "rstd": s["rstd"]}


def _workspace(s, need):
    """The program's workspace: made on the first pass, kept with its other buffers."""
    if "ws" not in s:
        n = need()
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return s["ws"]


def _own_ln_bwd(s):
    B = _binding()
    p, x, dy, dx = B.PREC_IDS[s["prec"]], s["x"], s["dy"], s["dx"]
    ws = _workspace(s, lambda: B.rn18op_layernorm_bwd_workspace(p, s["rows"], s["width"]))
    B.rn18op_layernorm_bwd(p, dy, x, s["gamma"], s["mean"], s["rstd"], dx, s["dgamma"], s["dbeta"], s["rows"],
                           s["width"], dy.stride(0), x.stride(0), dx.stride(0), ws)
    return {"dx": dx, "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _own_topk(s):
    B = _binding()
    p, z = B.PREC_IDS[s["prec"]], s["z"]
    ws = _workspace(s, lambda: B.rn18op_topk_logits_workspace(p, s["rows"], s["classes"], s["k"]))
    B.rn18op_topk_logits(p, z, s["vals"], s["idx"], s["rows"], s["classes"], z.stride(0), s["k"], ws)
    return {"vals": s["vals"], "idx": s["idx"]}


def _own_distill(s):
    B = _binding()
    p, z, dz = B.PREC_IDS[s["prec"]], s["z"], s["dz"]
    ws = _workspace(s, lambda: B.rn18op_distill_loss_workspace(p, s["rows"], s["classes"], s["k"]))
    B.rn18op_distill_loss(p, z, s["t_vals"], s["t_idx"], s["labels"], s["weight"], dz, s["row_loss"], s["loss"],
                          s["rows"], s["classes"], z.stride(0), dz.stride(0), s["k"], s["temperature"], s["alpha"],
                          s["scale"], ws)
    return {"dz": dz, "row_loss": s["row_loss"], "loss": s["loss"]}


# ---------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    rows, step = case["rows"], max(1, (1 << 25) // case.get("width", case.get("classes")))
    parts = [globals()["_exact_" + case["kind"].split("_")[0]](s, slice(r, min(r + step, rows)))
             for r in range(0, rows, step)]
    out = {}
    for name in parts[0]:
        v = [p[name] for p in parts]
        out[name] = sum(v[1:], v[0]) if name in ("dgamma", "dbeta", "loss") else torch.cat(v)
    return out


def _exact_ln(s, r):
    x, gamma, d = s["x"][r].double(), s["gamma"].double(), s["width"]
    if s["kind"] == "ln_fwd":
        mean = x.sum(dim=1) / d
        rstd = 1.0 / torch.sqrt(((x * x).sum(dim=1) / d - mean * mean).clamp_(min=0.0) + EPS)
        return {"y": (x * rstd[:, None] - (mean * rstd)[:, None]) * gamma + s["beta"].double(), "mean": mean,
                "rstd": rstd}
    dy, mean, rstd = s["dy"][r].double(), s["mean"][r].double(), s["rstd"][r].double()
    xh = (x - mean[:, None]) * rstd[:, None]
    a = (dy * gamma).sum(dim=1) / d
    b = (dy * gamma * xh).sum(dim=1) / d
    return {"dx": (dy * gamma - a[:, None] - xh * b[:, None]) * rstd[:, None], "dgamma": (dy * xh).sum(dim=0),
            "dbeta": dy.sum(dim=0)}


def _exact_topk(s, r):
    # distinct keys: the value's order in the high half, the class from the last to the first in the low one
    z, c = s["z"][r].float().add(0.0), s["classes"]
    bits = z.view(torch.int32).long()
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
    key = (order << 32) + (c - 1 - torch.arange(c, device=z.device))
    idx = c - 1 - (key.topk(s["k"], dim=1).values & 0xFFFFFFFF)
    return {"vals": z.gather(1, idx).double(), "idx": idx}


def _exact_distill(s, r):
    z, t, i = s["z"][r].double(), s["t_vals"][r].double() / s["temperature"], s["t_idx"][r].long()
    temp, alpha, c = s["temperature"], s["alpha"], s["classes"]
    w = s["weight"][r].double() if s["weight"] is not None else torch.ones(len(z), dtype=torch.float64, device=z.device)
    z = torch.nan_to_num(z, nan=0.0, neginf=-math.inf) if s["weight"] is not None else z
    ok = (i >= 0) & (i < c)
    q = torch.zeros((len(z), c + 1), dtype=torch.float64, device=z.device)   # the teacher over all classes
    soft = torch.exp(t - t.amax(dim=1, keepdim=True)) * ok
    mass = soft.sum(dim=1, keepdim=True)
    q.scatter_add_(1, torch.where(ok, i, c), soft / torch.where(mass > 0, mass, 1.0))
    q = q[:, :c]
    has = (mass[:, 0] > 0).double()
    logp = torch.log_softmax(z / temp, dim=1)
    logq = torch.log(soft / torch.where(mass > 0, mass, 1.0))
    gap = (soft / torch.where(mass > 0, mass, 1.0)) * (logq - logp.gather(1, torch.where(ok, i, 0)))
    loss = alpha * temp ** 2 * torch.where(ok, gap, 0.0).sum(dim=1) * has
    dz = alpha * temp * (torch.exp(logp) * has[:, None] - q)
    if alpha != 1.0:
        y = s["labels"][r].long()
        known = (y >= 0) & (y < c)
        logp = torch.log_softmax(z, dim=1)
        hard = torch.zeros_like(z).scatter_(1, torch.where(known, y, 0)[:, None], 1.0) * known[:, None]
        loss = loss - (1 - alpha) * torch.where(known, logp.gather(1, torch.where(known, y, 0)[:, None])[:, 0], 0.0)
        dz = dz + (1 - alpha) * (torch.exp(logp) * known[:, None] - hard)
    loss = torch.where(w == 0, 0.0, w * loss)
    dz = torch.where((w == 0)[:, None], 0.0, dz * (s["scale"] * w)[:, None])
    return {"dz": dz, "row_loss": loss, "loss": s["scale"] * loss.sum(dim=0, keepdim=True)}
