"""Workloads of attention and of a cache of keys and values in 4 or 8 bits.

New tokens' keys and values quantised into a paged cache and read back, one or a few new tokens of each sequence
attending over such a cache, and attention over whole prompts packed one after the other, with its gradients.
``run`` computes them in elementary torch operations, or (``own``) through this package's entry points.

A cache holds, for each page, head and slot, D codes (4 bits: two a byte, the low half first) and a bfloat16 scale for
each 32 of them: scale = max|x| / qmax in binary32, rounded to bfloat16, code = round(x / scale), ties to even, at most qmax.
"""
import math
import random

import torch

own = False

_DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
_GROUP = 32  # elements of a head that share a scale


def _cache(name, op, batch, longest, new, heads, kv_heads, dim, page, dtype, codes, mix):
    """`new` tokens of each sequence are written, read or attend; 0: all of them."""
    return {"name": name, "op": op, "batch": batch, "longest": longest, "new": new, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "page": page, "dtype": dtype, "codes": codes, "mix": mix}


def _prompt(name, op, batch, longest, heads, kv_heads, dim, dtype, causal, fused, mix, prefix=0):
    return {"name": name, "op": op, "batch": batch, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "causal": causal, "fused": fused, "mix": mix, "prefix": prefix}


def listed():
    return [
        # one new token of each of a few dozen sequences goes into the cache
        _cache("store_tokens_int4", "store", 48, 4000, 1, 32, 8, 128, 16, "bf16", "int4", 1),
        # the prompts of a batch go into the cache
        _cache("store_prompts_int8", "store", 9, 4096, 0, 32, 8, 128, 64, "fp16", "int8", 2),
        # a few short sequences read back in full precision
        _cache("read_short_int8", "read", 3, 700, 0, 6, 6, 64, 24, "fp32", "int8", 3),
        # a server's cache read back whole
        _cache("read_int4", "read", 24, 8192, 0, 32, 8, 128, 32, "bf16", "int4", 4),
        # one user's next token after a long text
        _cache("decode_one_int4", "decode", 1, 8192, 1, 32, 8, 128, 16, "bf16", "int4", 0),
        # full precision, a key head for each query head, odd pages and lengths
        _cache("decode_fp32_odd", "decode", 13, 3001, 1, 12, 12, 64, 24, "fp32", "int4", 5),
        # five drafted tokens of each sequence are checked in one pass
        _cache("decode_drafts_int8", "decode", 11, 6007, 5, 28, 4, 128, 64, "fp16", "int8", 6),
        # a server's batch, one token each
        _cache("decode_batch_int4", "decode", 96, 16384, 1, 32, 8, 128, 32, "bf16", "int4", 7),
        # a handful of short prompts
        _prompt("prompt_short", "prompt", 5, 200, 16, 4, 64, "fp16", True, True, 8),
        # a long text
        _prompt("prompt_long", "prompt", 1, 16384, 32, 8, 128, "bf16", True, False, 0),
        # a training step on packed texts
        _prompt("step_packed", "step", 7, 4096, 32, 8, 128, "bf16", True, True, 9),
        # a training step in full precision, sizes odd everywhere
        _prompt("step_fp32_odd", "step", 6, 515, 6, 2, 96, "fp32", True, False, 10),
    ]


def _lengths(case):
    """Tokens of each sequence: from the case alone, the first one the longest; mix 0: all the same."""
    rng = random.Random(case["mix"])
    top = case["longest"]
    rest = [top if case["mix"] == 0 else _spread(rng, max(1, top // 16), top) for _ in range(case["batch"] - 1)]
    return [top] + rest


def _new(case, lengths):
    return [min(case["new"], n) if case["new"] else n for n in lengths]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {c["op"]: work(c) for c in sorted(listed(), key=lambda c: work(c)["flops"] + work(c)["bytes"])}
    while True:
        op = rng.choice(["store", "read", "decode", "decode", "prompt", "step"])
        dtype, mix = rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.randint(1, 10 ** 6)
        kv_heads, group = rng.choice([1, 2, 3, 4, 6, 8, 12, 16]), rng.choice([1, 2, 3, 4, 7, 8])
        dim = rng.choice([32, 64, 64, 96, 128, 128, 128, 192, 256])
        if op in ("prompt", "step"):
            c = _prompt("", op, _spread(rng, 1, 16), _spread(rng, 16, 8192), kv_heads * group, kv_heads, dim, dtype,
                        rng.random() < 0.8, rng.random() < 0.5, mix, rng.choice([0, 0, rng.randint(1, 600)]))
        else:
            new = 0 if op == "read" else rng.choice([0, 1]) if op == "store" else rng.choice([1, 1, rng.randint(2, 8)])
            c = _cache("", op, _spread(rng, 1, 128), _spread(rng, 16, 16384), new, kv_heads * group, kv_heads, dim,
                       rng.choice([16, 32, 64, 128, rng.randint(8, 100)]), dtype, rng.choice(["int4", "int4", "int8"]), mix)
        if rng.random() < 0.5 and c["longest"] > 128:  # half of the lengths are multiples of 64, as most configurations have them
            c["longest"] = c["longest"] // 64 * 64
        w = work(c)
        slow = 8 if dtype == "fp32" and op in ("prompt", "step") else 1
        if w["flops"] * slow > most[op]["flops"] or w["bytes"] > most[op]["bytes"]:
            continue
        del c["name"]
        return c


def _starts(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return s


def _quantise(x, codes):
    """Codes (as integers) and bfloat16 scales of x [..., D]."""
    qmax = 7 if codes == "int4" else 127
    g = x.float().unflatten(-1, (-1, _GROUP))
    scale = (g.abs().amax(-1, keepdim=True) / qmax).to(torch.bfloat16)
    wide = scale.float()
    c = torch.where(wide > 0, torch.clamp(torch.round(g / wide), -qmax, qmax), torch.zeros_like(g))
    return c.flatten(-2).to(torch.int8), scale[..., 0]


def _pack(c):
    c = c.view(torch.uint8)
    return (c[..., 0::2] & 15) | (c[..., 1::2] << 4)


def _values(codes, scales):
    """What codes and scales stand for, in binary32."""
    if codes.dtype == torch.uint8:
        pair = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
        codes = (pair ^ 8).to(torch.int16) - 8
    return (codes.float().unflatten(-1, (-1, _GROUP)) * scales.float()[..., None]).flatten(-2)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, heads, kv_heads, dim = _DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"]
    lengths = _lengths(case)
    s = dict(case, lengths=lengths, scale=dim ** -0.5)

    def randn(*shape, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=gen) * scale).to(dtype)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    if case["op"] in ("prompt", "step"):
        longer = [n + case["prefix"] for n in lengths]
        rows, keys = sum(lengths), sum(longer)
        s.update(k_lengths=longer, starts=ints(_starts(lengths)), k_starts=ints(_starts(longer)))
        if case["fused"] and not case["prefix"]:
            # queries, keys and values as one projection writes them
            x = randn(rows, heads + 2 * kv_heads, dim)
            s["q"], s["k"], s["v"] = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
        else:
            s["q"], s["k"], s["v"] = randn(rows, heads, dim), randn(keys, kv_heads, dim), randn(keys, kv_heads, dim)
        # peaked rows and flat ones
        s["q"].mul_((torch.rand(rows, 1, 1, device="cuda", generator=gen) * 3).to(dtype))
        if case["op"] == "step":
            s["dout"] = randn(rows, heads, dim, scale=1e-2)
        return s
    new, page = _new(case, lengths), case["page"]
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 3
    order = torch.randperm(pages, device="cuda", generator=gen, dtype=torch.int64).to(torch.int32)
    table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s.update(new_lengths=new, table=table, table_long=table.long(), lens=ints(lengths), starts=ints(_starts(new)))
    shape = (pages, kv_heads, page, dim)
    bytes_ = shape[:-1] + (dim // 2 if case["codes"] == "int4" else dim,)
    if case["op"] == "store":
        code_type = torch.uint8 if case["codes"] == "int4" else torch.int8
        s["cache"] = [torch.zeros(b, dtype=t, device="cuda") for _ in range(2)
                      for b, t in ((bytes_, code_type), (shape[:-1] + (dim // _GROUP,), torch.bfloat16))]
        # keys and values beside each other, as a projection writes them; some elements stand out
        x = randn(sum(new), 2 * kv_heads, dim)
        x.mul_(1 + 9 * (torch.rand(1, 2 * kv_heads, dim, device="cuda", generator=gen) < 0.02).to(dtype))
        s["k"], s["v"] = x[:, :kv_heads], x[:, kv_heads:]
    else:
        cache = []
        for _ in range(2):
            codes = torch.empty(bytes_, dtype=torch.uint8 if case["codes"] == "int4" else torch.int8, device="cuda")
            scales = torch.empty(shape[:-1] + (dim // _GROUP,), dtype=torch.bfloat16, device="cuda")
            step = max(1, (1 << 27) // (kv_heads * page * dim))
            for a in range(0, pages, step):
                c, sc = _quantise(torch.randn((min(step, pages - a),) + shape[1:], device="cuda", generator=gen), case["codes"])
                codes[a:a + step] = _pack(c) if case["codes"] == "int4" else c
                scales[a:a + step] = sc
            cache += [codes, scales]
        s["cache"] = cache
        if case["op"] == "decode":
            s["q"] = randn(sum(new), heads, dim)
            s["q"].mul_((torch.rand(sum(new), 1, 1, device="cuda", generator=gen) * 3).to(dtype))
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2202_07471_amd as sq

    if s["op"] == "prompt":
        return sq.squant_attention(s["q"], s["k"], s["v"], s["starts"], s["k_starts"], s["scale"], s["causal"])
    if s["op"] == "step":
        out, lse = sq.squant_attention(s["q"], s["k"], s["v"], s["starts"], s["k_starts"], s["scale"], s["causal"])
        return (out,) + sq.squant_attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, s["starts"], s["k_starts"],
                                                     s["scale"], s["causal"])
    cache = sq.QuantizedCache(*s["cache"])
    if s["op"] == "store":
        sq.squant_cache_write(s["k"], s["v"], cache, s["table"], s["lens"], s["starts"])
    if s["op"] != "decode":
        return sq.squant_cache_read(cache, s["table"], s["lens"], s["starts"], sum(s["new_lengths"]), _DTYPES[s["dtype"]])
    one_each = s["new"] == 1
    return sq.squant_cache_attention(s["q"], cache, s["table"], s["lens"], None if one_each else s["starts"], s["scale"])


def _slots(s, b, first, last):
    """Pages and slots in them of a sequence's tokens."""
    t = torch.arange(first, last, device="cuda")
    return s["table_long"][b, t // s["page"]], t % s["page"]


def _plain_attention(q, k, v, scale, causal):
    """Output and log-sum-exp, [kv head, query head of it, row]; q and k, v [row, head, D] in binary32."""
    n, m, kv = q.shape[0], k.shape[0], k.shape[1]
    q = q.unflatten(1, (kv, -1)).permute(1, 2, 0, 3)
    g = q.shape[1]
    kt, vt = k.permute(1, 2, 0).contiguous(), v.permute(1, 0, 2).contiguous()
    x = torch.bmm(q.reshape(kv, g * n, -1), kt).view(kv, g, n, m).mul_(scale)
    if causal and n > 1:
        hidden = torch.arange(m, device=x.device) > (torch.arange(n, device=x.device) + (m - n))[:, None]
        x.masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p.view(kv, g * n, m), vt).view(kv, g, n, -1) / total
    return out, (top + torch.log(total))[..., 0], p, total


def _run_plain(s):
    dtype, op = _DTYPES[s["dtype"]], s["op"]
    if op in ("prompt", "step"):
        q, k, v = s["q"], s["k"], s["v"]
        group = s["heads"] // s["kv_heads"]
        out = torch.empty(q.shape, dtype=dtype, device="cuda")
        lse = torch.empty(q.shape[1], q.shape[0], device="cuda")
        if op == "step":
            dq, dk, dv = torch.empty_like(out), torch.empty(k.shape, dtype=dtype, device="cuda"), torch.empty(v.shape, dtype=dtype, device="cuda")
        a = c = 0
        for n, m in zip(s["lengths"], s["k_lengths"]):
            some = max(1, min(s["kv_heads"], (1 << 28) // (group * n * m)))  # heads at a time: about a GiB of scores
            for h in range(0, s["kv_heads"], some):
                hk, hq = slice(h, min(h + some, s["kv_heads"])), slice(h * group, min(h + some, s["kv_heads"]) * group)
                qf, kf, vf = q[a:a + n, hq].float(), k[c:c + m, hk].float(), v[c:c + m, hk].float()
                o, l, p, total = _plain_attention(qf, kf, vf, s["scale"], s["causal"])
                out[a:a + n, hq] = o.permute(2, 0, 1, 3).flatten(1, 2).to(dtype)
                lse[hq, a:a + n] = l.flatten(0, 1)
                if op == "prompt":
                    continue
                kv = kf.shape[1]
                do = s["dout"][a:a + n, hq].float().unflatten(1, (kv, group)).permute(1, 2, 0, 3).reshape(kv, group * n, -1)
                p = (p / total).view(kv, group * n, m)
                pt = p.transpose(1, 2).contiguous()
                dv[c:c + m, hk] = torch.bmm(pt, do).transpose(0, 1).to(dtype)
                delta = (do * o.reshape(kv, group * n, -1)).sum(-1, keepdim=True)
                ds = torch.bmm(do, vf.permute(1, 2, 0).contiguous()).sub_(delta).mul_(p).mul_(s["scale"])
                dq[a:a + n, hq] = torch.bmm(ds, kf.transpose(0, 1).contiguous()).view(kv, group, n, -1).permute(2, 0, 1, 3).flatten(1, 2).to(dtype)
                qh = qf.unflatten(1, (kv, group)).permute(1, 2, 0, 3).reshape(kv, group * n, -1)
                dk[c:c + m, hk] = torch.bmm(ds.transpose(1, 2).contiguous(), qh).transpose(0, 1).to(dtype)
            a, c = a + n, c + m
        return (out, lse) if op == "prompt" else (out, dq, dk, dv)
    kc, ks, vc, vs = s["cache"]
    outs, a = [], 0
    for b, (n, m) in enumerate(zip(s["new_lengths"], s["lengths"])):
        if op == "store":
            pages, slots = _slots(s, b, m - n, m)
            for x, codes, scales in ((s["k"], kc, ks), (s["v"], vc, vs)):
                c, sc = _quantise(x[a:a + n], s["codes"])
                codes[pages, :, slots] = _pack(c) if s["codes"] == "int4" else c
                scales[pages, :, slots] = sc
            a += n
        if op != "decode":
            pages, slots = _slots(s, b, m - n, m)
            outs.append([_values(c[pages, :, slots], sc[pages, :, slots]).to(dtype) for c, sc in ((kc, ks), (vc, vs))])
            continue
        pages, slots = _slots(s, b, 0, m)
        o = _plain_attention(s["q"][a:a + n].float(), _values(kc[pages, :, slots], ks[pages, :, slots]),
                             _values(vc[pages, :, slots], vs[pages, :, slots]), s["scale"], True)[0]
        outs.append([o.permute(2, 0, 1, 3).flatten(1, 2).to(dtype)])
        a += n
    outs = tuple(torch.cat([o[i] for o in outs]) for i in range(len(outs[0])))
    return outs if len(outs) > 1 else outs[0]


def work(case):
    lengths = _lengths(case)
    e, heads, kv_heads, dim = _DTYPES[case["dtype"]].itemsize, case["heads"], case["kv_heads"], case["dim"]
    if case["op"] in ("prompt", "step"):
        pairs, p = 0, case["prefix"]
        for n in lengths:
            pairs += n * (n + 1) // 2 + n * p if case["causal"] else n * (n + p)
        rows, keys = sum(lengths), sum(lengths) + p * len(lengths)
        q, kv, lse = rows * heads * dim * e, keys * kv_heads * dim * e, rows * heads * 4
        if case["op"] == "prompt":
            return {"bytes": 2 * q + 2 * kv + lse, "flops": 4.0 * pairs * heads * dim}
        # forward; its backward reads them and the output's gradient again and multiplies five times
        return {"bytes": 2 * q + 2 * kv + 3 * q + 2 * kv + q + 2 * kv + 2 * lse, "flops": 14.0 * pairs * heads * dim}
    new = _new(case, lengths)
    token = 2 * kv_heads * (dim // 2 if case["codes"] == "int4" else dim) + 2 * kv_heads * dim // _GROUP * 2
    wide = 2 * kv_heads * dim * e
    if case["op"] == "read":
        return {"bytes": sum(new) * (token + wide), "flops": 2.0 * sum(new) * kv_heads * dim}
    if case["op"] == "store":
        return {"bytes": sum(new) * 2 * (token + wide), "flops": 8.0 * sum(new) * kv_heads * dim}
    pairs = sum(n * m - n * (n - 1) // 2 for n, m in zip(new, lengths))
    return {"bytes": sum(lengths) * token + 2 * sum(new) * heads * dim * e, "flops": 4.0 * pairs * heads * dim}


def exact(case, seed):
    s = prepare(case, seed)
    f64, dev = torch.float64, "cuda"
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group = heads // kv_heads
    scale = 1.0 / math.sqrt(dim)
    if case["op"] in ("prompt", "step"):
        out = torch.zeros(sum(s["lengths"]), heads, dim, dtype=f64, device=dev)
        lse = torch.zeros(heads, out.shape[0], dtype=f64, device=dev)
        step = case["op"] == "step"
        if step:
            dq = torch.zeros_like(out)
            dk = torch.zeros(sum(s["k_lengths"]), kv_heads, dim, dtype=f64, device=dev)
            dv = torch.zeros_like(dk)
        a = c = 0
        for n, m in zip(s["lengths"], s["k_lengths"]):
            for h in range(heads):
                k, v = s["k"][c:c + m, h // group].to(f64), s["v"][c:c + m, h // group].to(f64)
                size = max(1, (1 << 27) // m)  # rows at a time
                for r in range(0, n, size):
                    last = min(n, r + size)
                    rows = slice(a + r, a + last)
                    seen = m - n + last if case["causal"] else m
                    q, kk, vv = s["q"][rows, h].to(f64), k[:seen], v[:seen]
                    x = torch.mm(q, kk.T) * scale
                    if case["causal"]:
                        x = x.masked_fill(torch.ones_like(x, dtype=torch.bool).triu(m - n + r + 1), -math.inf)
                    lse[h, rows] = torch.logsumexp(x, 1)
                    p = torch.exp(x - lse[h, rows, None])
                    out[rows, h] = torch.mm(p, vv)
                    if step:
                        do = s["dout"][rows, h].to(f64)
                        dp = torch.mm(do, vv.T)
                        ds = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
                        dq[rows, h] = torch.mm(ds, kk)
                        dk[c:c + seen, h // group] += torch.mm(ds.T, q)
                        dv[c:c + seen, h // group] += torch.mm(p.T, do)
            a, c = a + n, c + m
        return (out, dq, dk, dv) if step else (out, lse)
    top = 7.0 if case["codes"] == "int4" else 127.0
    if case["op"] == "store":
        outs = []
        for x in (s["k"], s["v"]):
            blocks = x.to(f64).reshape(x.shape[0], kv_heads, dim // 32, 32)
            unit = (blocks.abs().amax(3).float() / top).to(torch.bfloat16).to(f64).unsqueeze(3)
            whole = torch.where(unit > 0, (blocks / unit).round().clamp(-top, top), 0.0)
            outs.append((whole * unit).reshape(x.shape[0], kv_heads, dim))
        return tuple(outs)
    kc, ks, vc, vs = s["cache"]

    def wide(codes, scales, b, first, last):
        where = torch.arange(first, last, device=dev)
        page, slot = s["table"][b].long()[torch.div(where, case["page"], rounding_mode="floor")], where % case["page"]
        codes, scales = codes[page, :, slot], scales[page, :, slot].to(f64)
        if case["codes"] == "int4":
            both = torch.empty(codes.shape[:-1] + (dim,), dtype=f64, device=dev)
            low, high = (codes % 16).to(f64), torch.div(codes, 16, rounding_mode="floor").to(f64)
            both[..., 0::2], both[..., 1::2] = low - 16 * (low > 7), high - 16 * (high > 7)
        else:
            both = codes.to(f64)
        return both * scales.repeat_interleave(32, dim=-1)

    parts, a = [], 0
    for b, (n, m) in enumerate(zip(s["new_lengths"], s["lengths"])):
        if case["op"] == "read":
            parts.append((wide(kc, ks, b, m - n, m), wide(vc, vs, b, m - n, m)))
            continue
        k, v = wide(kc, ks, b, 0, m), wide(vc, vs, b, 0, m)
        o = torch.empty(n, heads, dim, dtype=f64, device=dev)
        for h in range(heads):
            x = torch.mm(s["q"][a:a + n, h].to(f64), k[:, h // group].T) * scale
            x = x.masked_fill(torch.ones_like(x, dtype=torch.bool).triu(m - n + 1), -math.inf)
            o[:, h] = torch.mm(torch.softmax(x, 1), v[:, h // group])
        parts.append((o,))
        a += n
    outs = tuple(torch.cat([p[i] for p in parts]) for i in range(len(parts[0])))
    return outs if len(outs) > 1 else outs[0]
