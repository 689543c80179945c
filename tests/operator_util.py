"""Plain 64-bit forms of the operators around the sparse layer, and how far a kernel may be from them.

A rounding to a type is off by at most HALF[type] relative to the value.  Every bound below is a sum of such terms: the final rounding of
the result, the roundings of what a product takes in (weights and their gradients in bfloat16), and float32 sums, whose error is at most
(number of terms) * 2^-24 times the sum of the terms' magnitudes."""
from __future__ import annotations

import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float8_e4m3fn: 2.0 ** -4}
F32 = 2.0 ** -24


def normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def within(name, got, ref, bound):
    """got and ref agree to `bound` element by element, and not finite values are the same ones."""
    got, ref, bound = got.double(), ref.double(), torch.as_tensor(bound, dtype=torch.float64, device=ref.device).expand(ref.shape)
    fine = ref.isfinite()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert torch.equal(fine, got.isfinite()), (name, "other values are not finite", int((fine != got.isfinite()).sum()))
    same = (got == ref) | (got.isnan() & ref.isnan())
    assert bool(same[~fine].all()), (name, "infinities or NaNs differ")
    over = (got - ref).abs()[fine] / bound[fine].clamp_min(1e-300)
    worst = float(over.max()) if over.numel() else 0.0
    print(f"   {name}: worst error {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, (name, worst)


def ranges(B, Sq, Sk, doc_off=None, prefix=None, causal=False, q_pos=None, q_first=0):
    """Key ranges by the definition, one query at a time: lists [B][Sq] of (lo, hi)."""
    out = []
    for b in range(B):
        rows = []
        for r in range(Sq):
            p = q_pos[b][r] if q_pos is not None else q_first + r
            docs = [(0, Sk)] if doc_off is None else list(zip(doc_off[b % len(doc_off)][:-1], doc_off[b % len(doc_off)][1:]))
            lo, hi = 0, 0
            for d, (s, e) in enumerate(docs):
                if doc_off is None or s <= p < e:
                    lo, hi = s, e
                    if causal:
                        hi = min(e, max(p + 1, s + (prefix[b % len(prefix)][d] if prefix is not None else 0)))
            lo, hi = max(0, min(lo, Sk)), max(0, min(hi, Sk))
            rows.append((lo, hi) if lo < hi else (0, 0))
        out.append(rows)
    return out


def attention(Q, K, V, lo, hi, pos, scale, cap=0.0, slopes=None, dO=None):
    """Reference results and bounds of dense attention: dict name -> (value, bound).  lo, hi, pos: [B, Sq] integers.  Pairs outside a range are left out
    by selection, so what stands there never counts."""
    dt = Q.dtype
    half = HALF[dt]
    B, Sq, Hq, D = Q.shape
    Sk, Hkv = K.shape[1], K.shape[2]
    G = Hq // Hkv
    q, k, v = (t.double().permute(0, 2, 1, 3) for t in (Q, K, V))                            # [B, h, s, D]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    key = torch.arange(Sk, device=Q.device)
    seen = ((key >= lo[..., None]) & (key < hi[..., None]))[:, None].expand(B, Hq, Sq, Sk)
    z = torch.where(seen, scale * (q @ k.transpose(2, 3)), 0.0)
    size = torch.where(seen, abs(scale) * (q.abs() @ k.abs().transpose(2, 3)), 0.0)
    score_err = (D + 8) * F32 * size + 4 * F32 * z.abs()
    slope = torch.ones_like(z)
    if cap:
        t = torch.tanh(z / cap)
        slope, z = 1 - t * t, cap * t
        score_err = score_err + 16 * F32 * cap                                             # exponential and reciprocal of 2 ulp, two roundings
    if slopes is not None:
        dist = (pos[:, None, :, None] - key).abs().double()
        z = z - slopes.double().view(1, Hq, 1, 1) * dist
        score_err = score_err + 4 * F32 * slopes.double().abs().view(1, Hq, 1, 1) * dist
    score_err = torch.where(seen, score_err + 4 * F32 * z.abs(), 0.0)
    z = torch.where(seen, z, -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    l = e.sum(-1, keepdim=True)
    lse = (m + l.log())[..., 0]
    A = torch.where(l > 0, e / l, 0.0)
    worst = score_err.nan_to_num(0.0, 0.0, 0.0).amax(-1, keepdim=True)                      # of a row's scores
    rel = 2 * worst + (Sk + 64) * F32                                                       # relative error of a weight in float32
    if dt == torch.bfloat16:
        rel = rel + half                                                                    # and its rounding
    back = lambda x: x.permute(0, 2, 1, 3)                                                  # noqa: E731
    shared = lambda x: x.view(B, Hkv, G, Sk, D).sum(2)                                      # noqa: E731
    vz, kz = v, k
    dot = lambda w, x: _select_matmul(w, x, seen)                                           # noqa: E731
    O = dot(A, vz)
    out = {"O": (back(O), back(rel * dot(A, vz.abs()) + half * O.abs())), "LSE": (lse, worst[..., 0] + (Sk + 64) * F32 + 4 * F32 * lse.abs())}
    if dO is None:
        return out
    g = dO.double().permute(0, 2, 1, 3)
    ones = seen.transpose(2, 3)
    dV = _select_matmul(A.transpose(2, 3), g, ones)
    dP = torch.where(seen, g @ v.transpose(2, 3), 0.0)
    delta = torch.where(l > 0, (g * O).sum(-1, keepdim=True), 0.0)
    # what the kernel subtracts is the sum over the stored O, rounded to the inputs' type; dP and the sum are float32
    delta_err = half * (g.abs() * O.abs()).sum(-1, keepdim=True) + (D + 8) * F32 * torch.where(seen, g.abs() @ v.abs().transpose(2, 3), 0.0).amax(-1, keepdim=True)
    if dt == torch.float32:
        delta_err = delta_err + ((rel * dot(A, vz.abs()) + half * O.abs()) * g.abs()).sum(-1, keepdim=True)
    else:
        delta_err = delta_err + (rel * dot(A, vz.abs()) * g.abs()).sum(-1, keepdim=True)
    W = A * slope
    dz = W * torch.where(seen, dP - delta, 0.0)
    dz_err = dz.abs() * (rel + (16 * F32 if not cap else 64 * F32 + 4 * worst)) + W * delta_err
    if cap:
        dz_err = dz_err + A * 64 * F32 * torch.where(seen, (dP - delta).abs(), 0.0)         # 4 r (1 - r) close to 0
    n = (Sk + Sq * G + 64) * F32
    rel_q = dz_err + n * dz.abs()
    s = abs(scale)
    dQ = scale * dot(dz, kz)
    out["dQ"] = (back(dQ), back(s * dot(rel_q, kz.abs()) + half * dQ.abs()))
    dK = scale * shared(_select_matmul(dz.transpose(2, 3), q, ones))
    out["dK"] = (back(dK), back(s * shared(_select_matmul(rel_q.transpose(2, 3), q.abs(), ones)) + half * dK.abs()))
    dVs = shared(dV)
    dv_err = shared(_select_matmul(((rel + n) * A).transpose(2, 3), g.abs(), ones))
    out["dV"] = (back(dVs), back(dv_err + half * dVs.abs()))
    return out


def _select_matmul(w, x, seen):
    """w @ x over the pairs that are seen: values of x that are not finite count where they are, and nowhere else."""
    clean = x.nan_to_num(0.0, 0.0, 0.0)
    y = torch.where(seen, w, 0.0) @ clean
    bad = (~x.isfinite()).any(-1) & seen.any(-2)
    if not bool(bad.any()):
        return y
    B, H, N, _ = x.shape
    for b, h, j in bad.nonzero().tolist():
        rows = seen[b, h, :, j]
        extra = torch.where(x[b, h, j].isfinite(), 0.0, x[b, h, j])
        y[b, h, rows] += torch.where(x[b, h, j].isfinite(), 0.0, w[b, h, rows, j][:, None] * extra)
    return y
