"""Workloads of the operators that multiply by SQuant's codes.

A layer whose weights are codes with one scale for each output channel: the product with bias,
activation and residual, its gradient through the frozen codes with the pre-activation kept in 8 bits
or in full, and the cross entropy over a vocabulary whose output embedding is codes, with its gradient.
``run`` computes them in elementary torch operations, or (``own``) through this package's entry points.
"""
import math

import torch

own = False

_DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
_GROUP = 64  # columns of a row that share a scale of the kept pre-activation


def _linear(name, m, k, n, dtype, codes, act="none", bias=True, residual=False, pad=0):
    return {"name": name, "op": "linear", "m": m, "k": k, "n": n, "dtype": dtype, "codes": codes, "act": act,
            "bias": bias, "residual": residual, "pad": pad}


def _step(name, m, k, n, dtype, codes, act, keep, residual=False, pad=0):
    return {"name": name, "op": "step", "m": m, "k": k, "n": n, "dtype": dtype, "codes": codes, "act": act,
            "keep": keep, "bias": True, "residual": residual, "pad": pad}


def _loss(name, t, d, v, dtype, codes, grad, pad=0):
    return {"name": name, "op": "loss", "m": t, "k": d, "n": v, "dtype": dtype, "codes": codes, "grad": grad,
            "pad": pad}


def listed():
    return [
        # one new token through a square projection with 4-bit codes, added to the residual stream
        _linear("one_token_int4", 1, 4096, 4096, "bf16", "int4", bias=False, residual=True),
        # a small batch of features through ResNet-50's classifier
        _linear("classifier_fp32", 32, 2048, 1000, "fp32", "int8"),
        # one new token each of 13 sequences through a wide layer
        _linear("token_batch_int8", 13, 8192, 8192, "fp16", "int8", act="gelu"),
        # a ragged prompt through a layer with odd sizes on both sides
        _linear("ragged_int4", 333, 5003, 1283, "fp16", "int4", act="silu", residual=True, pad=5),
        # a prompt in full precision
        _linear("prompt_fp32_int4", 1024, 2048, 4096, "fp32", "int4", act="silu"),
        # long prompts through the first product of a feed-forward block
        _linear("prompts_bf16", 4096, 4096, 8192, "bf16", "int8", act="gelu", residual=True),
        # fine-tuning around MobileNetV2's classifier
        _step("step_classifier", 200, 1280, 1000, "bf16", "int8", "gelu", "int8"),
        # a training step of a layer with odd sizes, pre-activations kept in full
        _step("step_odd_int4", 777, 2049, 2559, "fp16", "int4", "silu", "full", residual=True, pad=3),
        # a training step of a square layer on long sequences
        _step("step_bf16", 4096, 4096, 4096, "bf16", "int8", "silu", "int8"),
        # scoring a few tokens against a large vocabulary
        _loss("score_few", 7, 2048, 50001, "bf16", "int8", False),
        # a short batch in full precision, odd everywhere
        _loss("loss_fp32_odd", 301, 1030, 10007, "fp32", "int8", True, pad=2),
        # a training step's loss over a large vocabulary
        _loss("loss_bf16", 2048, 2048, 32768, "bf16", "int8", True),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    top = 2.0 * 4096 * 4096 * 8192
    while True:
        op = rng.choice(["linear", "linear", "step", "loss"])
        dtype, codes = rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.choice(["int8", "int4"])
        pad = rng.choice([0, 0, rng.randint(1, 40)])
        act = rng.choice(["none", "gelu", "silu"])
        if op == "linear":
            c = _linear("", _spread(rng, 1, 4096), _spread(rng, 256, 8192), _spread(rng, 256, 8192), dtype, codes,
                        rng.choice([act, "relu"]), rng.random() < 0.7, rng.random() < 0.5, pad)
        elif op == "step":
            c = _step("", _spread(rng, 16, 4096), _spread(rng, 256, 4096), _spread(rng, 256, 4096), dtype, codes,
                      act, "full" if dtype == "fp32" else rng.choice(["int8", "full"]), rng.random() < 0.5, pad)
        else:
            c = _loss("", _spread(rng, 1, 2048), _spread(rng, 256, 2048), _spread(rng, 2000, 60000), dtype, codes,
                      rng.random() < 0.7, pad)
        for d in ("m", "k", "n"):  # half of the sizes are multiples of 64, as most models have them
            if c[d] > 64 and rng.random() < 0.5:
                c[d] = c[d] // 64 * 64
        flops = work(c)["flops"]
        if flops > top or (flops > top / 8 and dtype == "fp32"):
            continue
        del c["name"]
        return c


def _strided(rows, cols, pad, dtype, gen, scale=1.0):
    buf = torch.randn(rows, cols + pad, device="cuda", generator=gen) * scale
    return buf.to(dtype)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, k, n, dtype = case["m"], case["k"], case["n"], _DTYPES[case["dtype"]]
    loss = case["op"] == "loss"
    # trained-like weights rounded to codes of the full range, one scale a row
    w = torch.randn(n, k, device="cuda", generator=gen) * math.sqrt((1.0 if loss else 2.0) / k)
    qmax = 7 if case["codes"] == "int4" else 127
    scales = w.abs().amax(1) / qmax
    codes = torch.round(w / scales[:, None]).to(torch.int8)
    del w
    if case["codes"] == "int4":
        c = torch.nn.functional.pad(codes, (0, k & 1)).view(torch.uint8)
        codes = ((c[:, 0::2] & 15) | (c[:, 1::2] << 4)).contiguous()
    s = dict(case, codes_format=case["codes"], codes=codes, scales=scales)
    s["x"] = _strided(m, k, case["pad"], dtype, gen)
    if loss:
        # hidden states of different lengths: flat rows and peaked ones; some labels are ignored
        s["x"].mul_((torch.rand(m, 1, device="cuda", generator=gen) * 4).to(dtype))
        labels = torch.randint(0, n, (m,), device="cuda", generator=gen)
        if m > 1:
            labels[torch.rand(m, device="cuda", generator=gen) < 0.05] = -100
        s["labels"] = labels
        s["dloss"] = torch.where(labels >= 0, 1.0, 0.0) / max(1, m)
        return s
    s["bias_v"] = (torch.randn(n, device="cuda", generator=gen) * 0.1).to(dtype) if case["bias"] else None
    s["res"] = _strided(m, n, case["pad"], dtype, gen) if case["residual"] else None
    if case["op"] == "step":
        s["dy"] = _strided(m, n, case["pad"], dtype, gen, 1e-3)
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2202_07471_amd as sq

    if s["op"] == "loss":
        loss, lse = sq.squant_cross_entropy(s["x"], s["codes"], s["scales"], s["labels"])
        if not s["grad"]:
            return loss, lse
        dh = sq.squant_cross_entropy_backward(s["x"], s["codes"], s["scales"], s["labels"], lse, s["dloss"])
        return loss, lse, dh
    act = sq.ACTS[s["act"]]
    if s["op"] == "linear":
        return sq.squant_linear(s["x"], s["codes"], s["scales"], s["bias_v"], act, s["res"])
    keep = sq.KEEPS[s["keep"] if s["act"] != "none" else "none"]
    y, kept = sq.squant_linear(s["x"], s["codes"], s["scales"], s["bias_v"], act, s["res"], keep=keep)
    dx, dbias = sq.squant_linear_backward(s["dy"], s["codes"], s["scales"], s["k"], act, kept)
    return y, dx, dbias


def _plain_codes(s):
    """The codes as binary32 [n, k]."""
    if s["codes_format"] == "int8":
        return s["codes"].float()
    c = s["codes"]
    pair = torch.stack((c & 15, c >> 4), 2).flatten(1)[:, :s["k"]]
    return ((pair ^ 8).to(torch.int16) - 8).float()


def _plain_act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _plain_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _plain_kept(z, keep, dtype):
    """z as the backward pass finds it."""
    if keep == "full":
        return z.to(dtype).float()
    m, n = z.shape
    g = torch.nn.functional.pad(z, (0, -n % _GROUP)).view(m, -1, _GROUP)
    scale = g.abs().amax(2, keepdim=True) / 127
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    return (torch.round(g / scale) * scale).reshape(m, -1)[:, :n]


def _run_plain(s):
    dtype = s["x"].dtype
    x = s["x"].float()
    c = _plain_codes(s)
    if s["op"] == "loss":
        logits = (x @ c.t()) * s["scales"]
        top = logits.amax(1, keepdim=True)
        e = torch.exp(logits - top)
        total = e.sum(1, keepdim=True)
        lse = (top + torch.log(total))[:, 0]
        valid = s["labels"] >= 0
        label = torch.where(valid, s["labels"], torch.zeros_like(s["labels"]))
        loss = torch.where(valid, lse - logits.gather(1, label[:, None])[:, 0], torch.zeros_like(lse))
        if not s["grad"]:
            return loss, lse
        e /= total
        e.scatter_add_(1, label[:, None], torch.full_like(lse[:, None], -1.0))
        dh = (e * s["scales"]) @ c
        return loss, lse, (dh * torch.where(valid, s["dloss"], torch.zeros_like(lse))[:, None]).to(dtype)
    z = (x @ c.t()) * s["scales"]
    if s["bias_v"] is not None:
        z = z + s["bias_v"].float()
    y = _plain_act(z, s["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    if s["op"] == "linear":
        return y.to(dtype)
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _plain_slope(_plain_kept(z, s["keep"], dtype), s["act"])
    return y.to(dtype), ((dz * s["scales"]) @ c).to(dtype), dz.sum(0).to(dtype)


def work(case):
    m, k, n = case["m"], case["k"], case["n"]
    e = _DTYPES[case["dtype"]].itemsize
    weights = n * ((k + 1) // 2 if case["codes"] == "int4" else k) + 4 * n
    if case["op"] == "loss":
        # the logits once, and their probabilities' product where the gradient is asked for
        return {"bytes": weights + m * k * e * (2 if case["grad"] else 1) + m * (8 + 4 + 4),
                "flops": 2.0 * m * n * k * (2 if case["grad"] else 1)}
    bytes_ = weights + m * k * e + m * n * e * (2 if case["residual"] else 1) + (n * e if case["bias"] else 0)
    if case["op"] == "step":
        return {"bytes": bytes_ + m * n * e + m * k * e + n * e, "flops": 4.0 * m * n * k}
    return {"bytes": bytes_, "flops": 2.0 * m * n * k}


def exact(case, seed):
    s = prepare(case, seed)
    m, k, n, dtype = case["m"], case["k"], case["n"], s["x"].dtype
    f64 = torch.float64
    codes = s["codes"]
    if case["codes"] == "int4":
        wide = torch.empty(n, 2 * codes.shape[1], dtype=f64, device=codes.device)
        low, high = (codes % 16).to(f64), (codes // 16).to(f64)
        wide[:, 0::2] = low - 16 * (low > 7)
        wide[:, 1::2] = high - 16 * (high > 7)
        wide = wide[:, :k]
    else:
        wide = codes.to(f64)
    w = wide * s["scales"].to(f64).unsqueeze(1)
    x = s["x"].to(f64)
    parts = []
    step = max(1, (1 << 26) // n)  # rows at a time: half a GiB for each intermediate
    for a in range(0, m, step):
        rows = slice(a, min(m, a + step))
        pre = torch.mm(x[rows], w.T)
        if case["op"] == "loss":
            lse = torch.logsumexp(pre, 1)
            y = s["labels"][rows]
            keep = y != -100
            hit = torch.zeros_like(pre)
            hit[torch.nonzero(keep)[:, 0], y[keep]] = 1.0
            out = [torch.where(keep, lse - (pre * hit).sum(1), 0.0), lse]
            if case["grad"]:
                g = s["dloss"][rows].to(f64) * keep
                out.append(torch.mm(torch.softmax(pre, 1) - hit, w) * g.unsqueeze(1))
            parts.append(out)
            continue
        if case["bias"]:
            pre += s["bias_v"].to(f64)
        act = case["act"]
        normal = 0.5 * torch.erfc(-pre / 2 ** 0.5) if act == "gelu" else None
        y = {"none": lambda: pre, "relu": lambda: pre.relu(), "gelu": lambda: pre * normal,
             "silu": lambda: pre / (1 + torch.exp(-pre))}[act]()
        if case["residual"]:
            y = y + s["res"][rows].to(f64)
        if case["op"] == "linear":
            parts.append([y])
            continue
        z = pre
        if act != "none" and case["keep"] == "full":
            z = pre.to(dtype).to(f64)
        elif act != "none":
            z = pre.clone()
            for b in range(0, n, 64):
                block = pre[:, b:b + 64]
                unit = block.abs().max(1, keepdim=True).values / 127
                unit[unit == 0] = 1.0
                z[:, b:b + 64] = torch.round(block / unit) * unit
        if act == "gelu":
            slope = 0.5 * torch.erfc(-z / 2 ** 0.5) + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
        elif act == "silu":
            sig = 1 / (1 + torch.exp(-z))
            slope = sig + z * sig * (1 - sig)
        else:
            slope = torch.ones_like(z) if act == "none" else (z > 0).to(f64)
        dz = s["dy"][rows].to(f64) * slope
        parts.append([y, torch.mm(dz, w), dz.sum(0, keepdim=True)])
    out = [torch.cat([p[i] for p in parts]) for i in range(len(parts[0]))]
    if case["op"] == "linear":
        return out[0]
    if case["op"] == "step":
        out[2] = out[2].sum(0)
    return tuple(out)
