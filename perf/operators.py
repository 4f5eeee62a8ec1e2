"""The measured cases of the operators around a token table's optimizer step:
what stands between the last layer's output and the step, and the quantised
head that serves the trained table.

Five kinds of pass, each one call (or, where 8-bit values have to come back
as what they stand for, a call and its dequantisation):
  norm      `Ops.rmsnorm` / `Ops.rmsnorm_quant`: the residual's addition and
            the root-mean-square norm, with an output in the input's type or
            in 8 bits with a scale per token;
  normback  `Ops.rmsnorm_backward`: the norm's gradients, the residual's own
            gradient added;
  head      `Ops.matmul_quant`: logits from 8-bit hidden states and an 8-bit
            table, with scales per token and per vocabulary entry;
  loss      `Ops.softmax_loss`: cross-entropy over the vocabulary with the
            gradient of the logits, which `Ember.step_lmhead` takes;
  clip      `Ops.clip_grads`: the global norm over many gradients and their
            clipping.

Inputs have the values of training and serving: hidden states of unit scale
with a few channels that are ten times larger, gains near one, logits with a
raised target and a masked padding of the vocabulary, gradients whose scale
differs from tensor to tensor.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
CLIP_EPS = 1e-6
IGNORE = -100
MAX_NORM_ELEMS = 8192 * 8192
MAX_HEAD_WORK = 4096 * 32000 * 4096
MAX_HEAD_ELEMS = 128256 * 8192
MAX_LOSS_ELEMS = 4096 * 128256
MAX_CLIP_ELEMS = 400_000_000
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(T, D, x, res="none", out="same", pad=0, gain="f32", **kw):
    return dict(kind="norm", T=T, D=D, x=x, res=res, out=out, pad=pad, gain=gain, **kw)


def _normback(T, D, x, dres=True, gain="f32", **kw):
    return dict(kind="normback", T=T, D=D, x=x, dres=dres, gain=gain, **kw)


def _head(T, V, K, out="bf16", **kw):
    return dict(kind="head", T=T, V=V, K=K, out=out, **kw)


def _loss(T, V, x, d="bf16", pad=0, masked=0, weighted=False, **kw):
    return dict(kind="loss", T=T, V=V, x=x, d=d, pad=pad, masked=masked, weighted=weighted, **kw)


def _clip(n, total, g, mix, clipped=True, **kw):
    return dict(kind="clip", n=n, total=total, g=g, mix=mix, clipped=clipped, **kw)


def listed():
    return [
        # one token of one sequence being generated: all latency
        _norm(1, 4096, "bf16", res="bf16", gain="bf16", name="norm_1x4096_bf16"),
        # two sequences of 4096 tokens in training, the residual stream kept in 32 bits
        _norm(8192, 4096, "bf16", res="f32", name="norm_8192x4096_bf16_res_f32"),
        # hidden states of a prompt, quantised for the 8-bit head; an odd count of tokens
        _norm(4095, 8192, "bf16", res="bf16", out="int8", gain="bf16", name="norm_int8_4095x8192_bf16"),
        # the norm's backward pass of the widest model here
        _normback(8192, 8192, "bf16", gain="bf16", name="normback_8192x8192_bf16"),
        # the same in 32 bits at a width that no vector access divides
        _normback(2051, 1003, "f32", name="normback_2051x1003_f32"),
        # the 8-bit head for one token: the table is read once
        _head(1, 128256, 8192, name="head_1x128256x8192"),
        # the 8-bit head of a narrow model for a batch of sequences being generated, logits in 32 bits
        _head(49, 151936, 896, out="f32", name="head_49x151936x896_f32"),
        # the 8-bit head over a prompt that is scored token by token: matrix products
        _head(2048, 32000, 4096, name="head_2048x32000x4096"),
        # a short batch over a small, odd vocabulary in 32 bits, weighted by advantages as in policy gradients
        _loss(127, 50257, "f32", d="f32", weighted=True, name="loss_127x50257_f32"),
        # a training batch over the largest vocabulary
        _loss(4096, 128256, "bf16", masked=256, name="loss_4096x128256_bf16"),
        # a few small tensors (a table of 1024 x 64 and its neighbours): all latency
        _clip(12, 100_000, "f32", 1, name="clip_12_tensors_100k_f32"),
        # the gradients of a model of 400 million parameters, most in 32 bits, some in bf16
        _clip(48, MAX_CLIP_ELEMS, "mixed", 2, name="clip_48_tensors_400m_mixed"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "normback", "head", "head", "loss", "loss", "clip"])
    gain = rng.choice(["bf16", "f32"])
    x = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("norm", "normback"):
        D = _log(rng, 64, 16384)
        if rng.random() < 0.8:  # most widths are multiples of 16, some are any number
            D = D // 16 * 16
        T = _log(rng, 1, min(32768, MAX_NORM_ELEMS // D))
        if kind == "normback":
            return _normback(T, D, x, dres=rng.random() < 0.75, gain=gain)
        return _norm(T, D, x, res=rng.choice(["none", "bf16", "f32"]), out=rng.choice(["same", "int8"]),
                     pad=rng.choice([0, 0, 64]), gain=gain)
    if kind == "head":
        K = _log(rng, 64, 8192)
        if rng.random() < 0.8:
            K = K // 16 * 16
        V = _log(rng, 1000, min(200000, MAX_HEAD_ELEMS // K))
        T = _log(rng, 1, min(4096, MAX_HEAD_WORK // (V * K), MAX_LOSS_ELEMS // V))
        return _head(T, V, K, out=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "loss":
        V = _log(rng, 1000, 262144)
        T = _log(rng, 1, min(16384, MAX_LOSS_ELEMS // (2 * V) if x == "f32" else MAX_LOSS_ELEMS // V))
        return _loss(T, V, x, d=rng.choice(["bf16", "f32"]) if x == "f32" else "bf16",
                     pad=(-V) % 64 if rng.random() < 0.5 else 0, masked=rng.choice([0, 0, V // 50]),
                     weighted=rng.random() < 0.5)
    n = rng.randint(1, 60)
    total = _log(rng, 1000 * n, MAX_CLIP_ELEMS)
    return _clip(n, total, rng.choice(["f32", "bf16", "mixed"]), rng.randint(1, 1 << 20), clipped=rng.random() < 0.75)


# ---- inputs, from the seed alone ----

def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed) * 1_000_003 + 29)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device=DEVICE)


def _hidden(g, T, D, dtype, pad=0):
    """T hidden states of width D, a hundredth of the channels ten times larger, as a slice of rows of D + pad."""
    h = _randn(g, T, D + pad)
    big = torch.randperm(D, generator=g, device=DEVICE)[:max(1, D // 100)]
    h[:, big] *= 10.0
    return h.to(dtype)[:, :D]


def _gain(g, D, kind):
    return (1.0 + 0.1 * _randn(g, D)).to(TYPES[kind])


def _sizes(case):
    """The tensors' sizes: cuts of `total` by weights over a range of a thousand, a third of them a vector's."""
    rng = random.Random(case["mix"])
    w = [math.exp(rng.uniform(0, math.log(1000))) / (300.0 if rng.random() < 0.33 else 1.0) for _ in range(case["n"])]
    return [max(1, int(case["total"] * x / sum(w))) for x in w]


def _clip_types(case):
    rng = random.Random(case["mix"] + 1)
    return [case["g"] if case["g"] != "mixed" else rng.choice(["f32", "f32", "bf16"]) for _ in range(case["n"])]


def _inputs(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    if kind == "norm":
        T, D = case["T"], case["D"]
        x = {"x": _hidden(g, T, D, TYPES[case["x"]], case["pad"]), "gain": _gain(g, D, case["gain"]), "res": None}
        if case["res"] != "none":
            x["res"] = _hidden(g, T, D, TYPES[case["res"]])
        return x
    if kind == "normback":
        T, D, t = case["T"], case["D"], TYPES[case["x"]]
        return {"h": _hidden(g, T, D, t), "gain": _gain(g, D, case["gain"]), "dy": (_randn(g, T, D) * 1e-3).to(t),
                "dres": (_randn(g, T, D) * 1e-3).to(t) if case["dres"] else None}
    if kind == "head":
        T, V, K = case["T"], case["V"], case["K"]
        ld = -(-K // 16) * 16  # rows of 8-bit tables start on 16 bytes
        wq = torch.empty(V, ld, device=DEVICE, dtype=torch.int8)
        for v in range(0, V, 16384):
            n = min(16384, V - v)
            wq[v:v + n] = (_randn(g, n, ld) * 30.0).round_().clamp_(-127, 127)
        xq = (_randn(g, T, ld) * 20.0).round_().clamp_(-127, 127).to(torch.int8)
        return {"xq": xq[:, :K], "wq": wq[:, :K], "xs": (0.5 + _rand(g, T)) * 0.05, "ws": (0.5 + _rand(g, V)) * 6e-4}
    if kind == "loss":
        T, V = case["T"], case["V"]
        z = torch.empty(T, V + case["pad"], device=DEVICE, dtype=TYPES[case["x"]])
        y = (_rand(g, T) ** 3 * (V - case["masked"])).long().clamp_(max=V - case["masked"] - 1)
        for t in range(0, T, 1024):
            b = _randn(g, min(1024, T - t), V + case["pad"]) * 2.0
            b.scatter_add_(1, y[t:t + 1024, None], 8.0 * _rand(g, b.shape[0], 1))
            z[t:t + 1024] = b
        if case["masked"]:  # the vocabulary's padding, masked out by the model
            z[:, V - case["masked"]:] = -math.inf
        y[_rand(g, T) < 0.1] = IGNORE  # prompt tokens
        y[0] = min(5, V - case["masked"] - 1)  # one counted token at least
        return {"logits": z[:, :V], "targets": y, "weights": _randn(g, T) if case["weighted"] else None}
    grads, sq = [], 0.0
    for n, t in zip(_sizes(case), _clip_types(case)):
        std = 10.0 ** (-4.0 + 2.0 * float(torch.rand(1, generator=g, device=DEVICE)))
        grads.append((_randn(g, n) * std).to(TYPES[t]))
        sq += n * std * std
    return {"grads": grads, "max_norm": math.sqrt(sq) * (0.5 if case["clipped"] else 2.0)}


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed), "ops": None}
    if case["kind"] == "clip":
        s["out"] = [torch.empty_like(t) for t in s["grads"]]
    if own:  # the operators' handle: a user's program keeps one
        from paper_2607_01455_gb300 import Ops
        s["ops"] = Ops(device=DEVICE)
    return s


# ---- one pass ----

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    case, ops = s["case"], s["ops"]
    kind = case["kind"]
    if kind == "norm" and case["out"] == "int8":
        q, scales, h = ops.rmsnorm_quant(s["x"], s["gain"], residual=s["res"], eps=EPS)
        return {"y": ops.dequantize_rows(q, scales, dtype=torch.bfloat16), "scales": scales, "h": h}
    if kind == "norm":
        y, h = ops.rmsnorm(s["x"], s["gain"], residual=s["res"], eps=EPS)
        return {"y": y, "h": h}
    if kind == "normback":
        dx, dgain = ops.rmsnorm_backward(s["dy"], s["h"], s["gain"], eps=EPS, dres=s["dres"])
        return {"dx": dx, "dgain": dgain}
    if kind == "head":
        return {"logits": ops.matmul_quant(s["xq"], s["xs"], s["wq"], s["ws"], dtype=TYPES[case["out"]])}
    if kind == "loss":
        loss, nll, d = ops.softmax_loss(s["logits"], s["targets"], weights=s["weights"], ignore_index=IGNORE,
                                        grad_dtype=TYPES[case["d"]])
        return {"loss": loss, "nll": nll, "dlogits": d}
    norm = ops.clip_grads(s["grads"], s["max_norm"], out=s["out"], eps=CLIP_EPS)
    return {"norm": norm, "grads": s["out"]}


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].float()
        if s["res"] is not None:
            h = h + s["res"].float()
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["gain"].float()
        out = {"h": None if s["res"] is None else h.to(s["res"].dtype)}
        if case["out"] == "int8":
            scales = y.abs().amax(1) / 127.0
            q = torch.round(y / scales.clamp(min=1e-38)[:, None])
            return {"y": (q * scales[:, None]).to(torch.bfloat16), "scales": scales, **out}
        return {"y": y.to(s["x"].dtype), **out}
    if kind == "normback":
        h, dy = s["h"].float(), s["dy"].float()
        r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        xh = h * r
        gy = dy * s["gain"].float()
        dx = r * (gy - xh * (gy * xh).mean(1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return {"dx": dx.to(s["h"].dtype), "dgain": (dy * xh).sum(0)}
    if kind == "head":
        z = torch.mm(s["xq"].float(), s["wq"].float().T)
        return {"logits": (z * s["xs"][:, None] * s["ws"][None, :]).to(TYPES[case["out"]])}
    if kind == "loss":
        z, y = s["logits"].float(), s["targets"]
        valid = y != IGNORE
        at = torch.where(valid, y, 0)[:, None]
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(1, keepdim=True)
        nll = torch.where(valid, (torch.log(total) + m - z.gather(1, at))[:, 0], 0.0)
        w = valid.float() if s["weights"] is None else torch.where(valid, s["weights"], 0.0)
        g = (w / valid.sum())[:, None]
        d = e.mul_(g / total)
        d.scatter_add_(1, at, -g)
        return {"loss": (w * nll).sum() / valid.sum(), "nll": nll, "dlogits": d.to(TYPES[case["d"]])}
    norm = torch.sqrt(torch.stack([t.float().square().sum() for t in s["grads"]]).sum())
    scale = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0)
    [o.copy_(t.float() * scale) for o, t in zip(s["out"], s["grads"])]
    return {"norm": norm, "grads": s["out"]}


def _bytes(t):
    return 2 if t == "bf16" else 4


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n = case["T"] * case["D"]
        b = n * _bytes(case["x"]) + case["D"] * _bytes(case["gain"])
        if case["res"] != "none":
            b += 2 * n * _bytes(case["res"])  # read, and the sum written
        b += n + 4 * case["T"] if case["out"] == "int8" else n * _bytes(case["x"])
        return {"bytes": b, "flops": 6 * n}
    if kind == "normback":
        n = case["T"] * case["D"]
        return {"bytes": n * _bytes(case["x"]) * (4 if case["dres"] else 3) + case["D"] * (_bytes(case["gain"]) + 4),
                "flops": 12 * n}
    if kind == "head":
        T, V, K = case["T"], case["V"], case["K"]
        return {"bytes": (T + V) * (K + 4) + T * V * _bytes(case["out"]), "flops": 2 * T * V * K}
    if kind == "loss":
        T, V = case["T"], case["V"]
        return {"bytes": T * V * (_bytes(case["x"]) + _bytes(case["d"])) + T * (12 + 4 * case["weighted"]),
                "flops": 6 * T * V}
    n = sum(s * _bytes(t) for s, t in zip(_sizes(case), _clip_types(case)))
    return {"bytes": 2 * n, "flops": 3 * sum(_sizes(case))}


def exact(case, seed):
    """The same outputs from the operators' definitions in 64 bits."""
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        v = s["x"].double()
        if s["res"] is not None:
            v += s["res"].double()
        y = v / torch.sqrt(v.pow(2).sum(1) / case["D"] + EPS).unsqueeze(1) * s["gain"].double()
        h = v if s["res"] is not None else None
        if case["out"] == "same":
            return {"y": y, "h": h}
        top = torch.linalg.vector_norm(y, ord=math.inf, dim=1)
        step = top / 127
        return {"y": torch.round(y * (127 / top.clamp(min=1e-300)).unsqueeze(1)) * step.unsqueeze(1), "scales": step, "h": h}
    if kind == "normback":  # by the quotient rule on y_j = gain_j h_j / n, n = sqrt(sum h^2 / D + eps)
        h, dy = s["h"].double(), s["dy"].double()
        n = torch.sqrt(h.pow(2).sum(1, keepdim=True) / case["D"] + EPS)
        a = dy * s["gain"].double()
        dn = -(a * h).sum(1, keepdim=True) / n.pow(2)  # of the loss with respect to n
        dx = a / n + dn * h / (case["D"] * n)
        if s["dres"] is not None:
            dx += s["dres"].double()
        return {"dx": dx, "dgain": torch.einsum("td,td->d", dy, h / n)}
    if kind == "head":
        x = s["xq"].double() * s["xs"].double().unsqueeze(1)
        out = torch.empty(case["T"], case["V"], device=DEVICE, dtype=torch.float64)
        for v in range(0, case["V"], 16384):
            w = s["wq"][v:v + 16384].double() * s["ws"][v:v + 16384].double().unsqueeze(1)
            out[:, v:v + 16384] = x @ w.T
        return {"logits": out}
    if kind == "loss":
        T, V = case["T"], case["V"]
        rows = torch.nonzero(s["targets"] != IGNORE).squeeze(1)
        n = rows.numel()
        w = torch.ones(T, device=DEVICE, dtype=torch.float64) if s["weights"] is None else s["weights"].double()
        nll = torch.zeros(T, device=DEVICE, dtype=torch.float64)
        d = torch.zeros(T, V, device=DEVICE, dtype=torch.float64)
        for k in range(0, n, 512):
            at = rows[k:k + 512]
            lp = torch.log_softmax(s["logits"][at].double(), dim=1)
            y = s["targets"][at].unsqueeze(1)
            nll[at] = -lp.gather(1, y).squeeze(1)
            p = lp.exp()
            p.scatter_add_(1, y, torch.full(y.shape, -1.0, device=DEVICE, dtype=torch.float64))
            d[at] = p * (w[at] / n).unsqueeze(1)
        return {"loss": (w * nll).sum() / n, "nll": nll, "dlogits": d}
    sq = [torch.dot(t.double(), t.double()) for t in s["grads"]]
    norm = torch.stack(sq).sum().sqrt()
    scale = min(1.0, s["max_norm"] / (float(norm) + CLIP_EPS))
    return {"norm": norm, "grads": [t.double() * scale for t in s["grads"]]}
