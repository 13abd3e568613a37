"""64-bit definitions of attention and of the quantised cache, on the CPU, seeded inputs, and error bounds.

Bounds.  Half a step is U (bfloat16 2^-8, binary16 2^-11, binary32 2^-24), relative.  A score is a binary32 sum of D products: off by
at most e = (D / 8 + 16) 2^-23 of scale * sum |q k|, a step of the running sum for each group the matrix units add; its
exponential by 2 e + 2^-21 relative (softmax's sum has the same terms).  A weight is rounded once to the element
type before it is multiplied by a value: U of sum p |v|.  The output is rounded once: U of itself.
"""
import math

import torch

from lin_reference import TINY, U

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
GROUP = 32


def starts_of(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32)


def quantise(x, bits):
    """(integer codes, bfloat16 scales) of x [..., D] by the definition; quotients in 64 bits."""
    top = 7 if bits == 4 else 127
    g = x.double().unflatten(-1, (-1, GROUP))
    most = g.abs().amax(-1)
    scale = (most.float() / top).to(BF16)
    scale = torch.where(most.isfinite(), scale, torch.full_like(scale, math.nan))
    wide = scale.double()[..., None]
    q = g / wide
    code = torch.where((wide > 0) & q.isfinite(), torch.clamp(torch.round(q), -top, top), torch.zeros_like(q))
    return code.flatten(-2).to(torch.int8), scale


def pack4(c):
    u = c.view(torch.uint8)
    return (u[..., 0::2] & 15) | (u[..., 1::2] << 4)


def values(codes, scales):
    """code * scale in 64 bits; codes integers or packed."""
    if codes.dtype == torch.uint8:
        both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).to(torch.int16)
        codes = (both ^ 8) - 8
    return (codes.double().unflatten(-1, (-1, GROUP)) * scales.double()[..., None]).flatten(-2)


def visible(n, m, causal):
    """[n, m]: which keys each row sees; the last row all."""
    if not causal:
        return torch.ones(n, m, dtype=torch.bool)
    return torch.arange(m)[None, :] <= torch.arange(n)[:, None] + (m - n)


def attention64(q, k, v, scale, causal, dtype, dout=None, key_error=0.0, value_error=0.0, floor=0.0):
    """One sequence: q [n, H, D], k and v [m, KV, D] in 64 bits.  A dict of out, lse and, with dout, dq, dk, dv, and of a bound
    for each (`out_tol` and so on) of an implementation in `dtype`.  key_error, value_error: relative rounding of an
    element of k, v (independent ones); floor: what a weight may be off by whatever its size."""
    n, heads, dim = q.shape
    m, kv = k.shape[:2]
    group = heads // kv
    u = U[dtype]
    up = u if dtype != F32 else 0.0
    see = visible(n, m, causal)
    r = {name: torch.zeros(*shape, dtype=torch.float64) for name, shape in
         (("out", q.shape), ("out_tol", q.shape), ("lse", (heads, n)), ("lse_tol", (heads, n)), ("dq", q.shape), ("dq_tol", q.shape),
          ("dk", k.shape), ("dk_tol", k.shape), ("dv", v.shape), ("dv_tol", v.shape))}
    e32 = (dim / 8 + 16) * 2.0 ** -23
    for h in range(heads):
        qh, kh, vh = q[:, h], k[:, h // group], v[:, h // group]
        s = torch.where(see, scale * (qh @ kh.T), torch.full((n, m), -math.inf, dtype=torch.float64))
        lse = torch.logsumexp(s, 1) if m else torch.full((n,), -math.inf, dtype=torch.float64)
        p = torch.where(see, torch.exp(s - torch.where(lse.isfinite(), lse, torch.zeros_like(lse))[:, None]), torch.zeros_like(s))
        out = p @ vh
        size = scale * (qh.abs() @ kh.abs().T)
        es = e32 * size + key_error * 4 * scale * ((qh * qh) @ (kh * kh).T).sqrt() + 2.0 ** -23 * torch.where(see, s.abs(), torch.zeros_like(s))
        worst = torch.where(see, es, torch.zeros_like(es)).amax(1, keepdim=True) if m else torch.zeros(n, 1, dtype=torch.float64)
        rel = 2 * worst + 2.0 ** -20 + m * 2.0 ** -26
        out_tol = (up + rel) * (p @ vh.abs()) + 4 * value_error * ((p * p) @ (vh * vh)).sqrt()
        out_tol = out_tol + floor * (see.double() @ vh.abs())
        r["out"][:, h], r["lse"][h] = out, lse
        r["out_tol"][:, h] = out_tol + u * out.abs() + TINY[dtype]
        r["lse_tol"][h] = (worst[:, 0] + 2.0 ** -20 + 2.0 ** -22 * lse.abs())
        if dout is None or n == 0 or m == 0:
            continue
        do = dout[:, h]
        delta = (do * out).sum(1, keepdim=True)
        dp = do @ vh.T
        ds = p * (dp - delta)
        # the row's own dot product is taken of the rounded output
        err = p * (u * (do.abs() * out.abs()).sum(1, keepdim=True) + (do.abs() * out_tol).sum(1, keepdim=True) + e32 * (do.abs() @ vh.abs().T))
        err = err + (up + rel) * ds.abs() + 2.0 ** -38 * ds.abs().amax()
        r["dq"][:, h] = scale * (ds @ kh)
        r["dq_tol"][:, h] = scale * (err @ kh.abs()) + (m / 8 + 16) * 2.0 ** -23 * scale * (ds.abs() @ kh.abs())
        r["dk"][:, h // group] += scale * (ds.T @ qh)
        r["dk_tol"][:, h // group] += scale * (err.T @ qh.abs()) + (n / 8 + 16) * 2.0 ** -23 * scale * (ds.T.abs() @ qh.abs())
        r["dv"][:, h // group] += p.T @ do
        r["dv_tol"][:, h // group] += (up + rel.amax() + (n / 8 + 16) * 2.0 ** -23) * (p.T @ do.abs())
    for name in ("dq", "dk", "dv"):
        r[name + "_tol"] += u * r[name].abs() + TINY[dtype]
    return r


def packed64(q, k, v, q_counts, k_counts, scale, causal, dtype, dout=None):
    """attention64 over packed sequences; rows behind the last one are 0."""
    total = None
    a = c = 0
    for n, m in zip(q_counts, k_counts):
        one = attention64(q[a:a + n], k[c:c + m], v[c:c + m], scale, causal, dtype, None if dout is None else dout[a:a + n])
        if total is None:
            total = {x: torch.zeros((t.shape[0], q.shape[0]) if x.startswith("lse") else (q if x[:2] in ("ou", "dq") else k).shape,
                                    dtype=torch.float64) for x, t in one.items()}
            total["lse"].fill_(-math.inf)
        for x, t in one.items():
            if x.startswith("lse"):
                total[x][:, a:a + n] = t
            elif x[:2] in ("ou", "dq"):
                total[x][a:a + n] = t
            else:
                total[x][c:c + m] = t
        a, c = a + n, c + m
    return total


def close(got, r, name, what=""):
    """Asserts that `got` is within r's bound of r's value, and equal where that is infinite."""
    got, want, tol = got.double().cpu(), r[name], r[name + "_tol"]
    assert got.shape == want.shape, f"{what} {name}: {tuple(got.shape)} for {tuple(want.shape)}"
    same = torch.where(want.isfinite(), (got - want).abs() <= tol, got == want)
    if not same.all():
        at = (~same).nonzero()[0].tolist()
        raise AssertionError(f"{what} {name}: {(~same).sum().item()} of {same.numel()} off, first at {at}: {got[tuple(at)].item()} for "
                             f"{want[tuple(at)].item()}, bound {tol[tuple(at)].item()}")
