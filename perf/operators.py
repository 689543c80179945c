"""What the operators around an attention layer are measured on: rotary positions, root-mean-square norms, and dense attention
with a score cap, a distance bias and key ranges, as calls that a user's program makes, and in a plain form.

A case says which operator runs ("rope", "norm", "attn") and which of its forms: "fwd", or "bwd" (the gradient), for rotary
positions; "infer" or "train" (forward and backward) for the others.  Sizes are those of this repository's latent grids, or
generic.  Inputs are drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------------------------ the cases
def _rope(name, what, batch, S, Hq, Hkv, D, dims, *, layout="half", scaling="plain", factor=1.0, train_len=0, base=10000.0, grid="", first=0,
          scattered=False, dtype="bf16"):
    return {"name": name, "op": "rope", "what": what, "batch": batch, "S": S, "Hq": Hq, "Hkv": Hkv, "D": D, "dims": dims, "layout": layout,
            "scaling": scaling, "factor": factor, "train_len": train_len, "base": base, "grid": grid, "first": first, "scattered": scattered,
            "dtype": dtype}


def _norm(name, what, batch, S, Hh, D, *, residual=True, out8=False, dtype="bf16", wtype="f32"):
    return {"name": name, "op": "norm", "what": what, "batch": batch, "S": S, "Hh": Hh, "D": D, "residual": residual, "out8": out8,
            "dtype": dtype, "wtype": wtype}


def _attn(name, what, batch, Hq, Hkv, Sq, Sk, D, *, cap=0.0, slopes=False, docs="", prefix=0, causal=False, lens=False, dtype="bf16"):
    return {"name": name, "op": "attn", "what": what, "batch": batch, "Hq": Hq, "Hkv": Hkv, "Sq": Sq, "Sk": Sk, "D": D, "cap": cap,
            "slopes": slopes, "docs": docs, "prefix": prefix, "causal": causal, "lens": lens, "dtype": dtype}


def listed():
    return [
        # the queries and keys of a 480p layer, positions on the latent grid, three axes
        _rope("rope_480p_grid", "fwd", 1, 32760, 12, 12, 128, "44,42,42", layout="interleaved", grid="21,30,52"),
        # gradient of a long text-like sequence with shared key heads: half of the channels, frequencies scaled beyond the trained
        # length, positions far from 0
        _rope("rope_far_yarn_bwd", "bwd", 2, 9001, 16, 4, 128, "64", scaling="yarn", factor=16.0, train_len=8192, first=120000),
        # one new token for each of eight sequences, each at its own position
        _rope("rope_token", "fwd", 8, 1, 16, 4, 64, "64", scattered=True),
        # the residual stream of a 480p layer, forward and backward: latent tokens x (12 heads x 128)
        _norm("norm_480p_train", "train", 1, 32760, 1, 1536),
        # the same stream on its way into an 8-bit projection
        _norm("norm_480p_8bit", "infer", 1, 32760, 1, 1536, out8=True, wtype="bf16"),
        # queries normalised head by head, float32, a short clip
        _norm("norm_heads_f32_train", "train", 1, 14040, 12, 128, residual=False, dtype="f32"),
        # eight new tokens: latency
        _norm("norm_token", "infer", 8, 1, 1, 1536, wtype="bf16"),
        # one new token against caches of up to 32 760 keys, sixteen heads on four key heads
        _attn("attn_token", "infer", 8, 16, 4, 1, 32760, 128, slopes=True, lens=True),
        # one latent frame (an image) behind a prefix of text, frames in order
        _attn("attn_image_prefix", "infer", 1, 12, 12, 1637, 1637, 128, prefix=77, causal=True, cap=30.0),
        # a training step on three clips packed into one row of 14 040 tokens, the last places empty
        _attn("attn_packed_train", "train", 1, 12, 12, 14040, 14040, 128, cap=50.0, docs="0.31,0.08,0.58"),
        # float32, shared key heads, 64 channels, odd length, a bias that falls with the distance
        _attn("attn_prefix_f32_train", "train", 2, 16, 4, 2001, 2001, 64, slopes=True, prefix=300, causal=True, dtype="f32"),
        # the dense attention of the first sampling steps at 480p
        _attn("attn_480p_infer", "infer", 1, 12, 12, 32760, 32760, 128),
    ]


def _log(rng, a, b):
    """A whole number between a and b, spread over its logarithm."""
    return max(a, min(b, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))


def draw(rng):
    c = {"rope": _draw_rope, "norm": _draw_norm, "attn": _draw_attn}[rng.choice(["rope", "norm", "attn", "attn"])](rng)
    del c["name"]
    return c


def _draw_rope(rng):
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 12])
    Hq = Hkv * rng.choice([1, 2, 4]) if Hkv < 12 else 12
    batch, dtype, layout, what = rng.choice([1, 1, 2, 5]), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["half", "interleaved"]), rng.choice(["fwd", "bwd"])
    if rng.random() < 0.4:
        T, H, W = _log(rng, 1, 21), rng.randint(3, 30), rng.randint(3, 52)
        dims = {64: ["24,20,20", "20,20,20", "16,24,24"], 128: ["44,42,42", "32,48,48", "40,40,40"]}[D]
        return _rope("", what, 1, T * H * W, Hq, Hkv, D, rng.choice(dims), layout=layout, grid="%d,%d,%d" % (T, H, W), dtype=dtype)
    S = _log(rng, 1, 32760 // batch)
    scaling = rng.choice(["plain", "linear", "ntk", "yarn"])
    return _rope("", what, batch, S, Hq, Hkv, D, str(rng.choice([D, D // 2, D // 4, D - 6])), layout=layout, scaling=scaling,
                 factor=1.0 if scaling == "plain" else rng.choice([2.0, 8.0, 32.0]), train_len=rng.choice([2048, 8192]), base=rng.choice([1e4, 5e5]),
                 first=_log(rng, 1, 1000000) - 1, scattered=rng.random() < 0.3, dtype=dtype)


def _draw_norm(rng):
    Hh, D = rng.choice([(1, 1536), (12, 128), (1, 5120), (16, 64), (1, 96), (1, 1000), (1, 2047), (1, 4104), (3, 33)])
    batch = rng.choice([1, 1, 2, 8])
    S = _log(rng, 1, max(1, 32760 * 1536 // (Hh * D * batch)))
    what = rng.choice(["infer", "train"])
    return _norm("", what, batch, S, Hh, D, residual=rng.random() < 0.6, out8=what == "infer" and rng.random() < 0.5,
                 dtype=rng.choice(["bf16", "bf16", "f32"]), wtype=rng.choice(["f32", "bf16"]))


def _draw_attn(rng):
    D, dtype, batch = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice([1, 1, 2, 3])
    Hkv, G = rng.choice([1, 2, 4, 12]), rng.choice([1, 1, 2, 4, 5])
    G = 1 if Hkv == 12 else G
    Hq = Hkv * G
    cap, slopes = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.4
    form = rng.choice(["token", "infer", "infer", "train", "train"])
    if form == "token":
        return _attn("", "infer", rng.choice([1, 2, 8, 16]), Hq, Hkv, _log(rng, 1, 8), _log(rng, 8, 32760), D, cap=cap, slopes=slopes, lens=True, dtype=dtype)
    most = math.sqrt((12 * 32760.0 ** 2 if form == "infer" else 12 * 14040.0 ** 2) / (Hq * batch) * (1.0 if dtype == "bf16" else 0.1))
    S = _log(rng, 17, min(32760, int(most)))
    mask = rng.choice(["none", "docs", "prefix", "docs+prefix"])
    return _attn("", form, batch, Hq, Hkv, S, S, D, cap=cap, slopes=slopes, dtype=dtype, causal="prefix" in mask,
                 docs=rng.choice(["0.31,0.08,0.58", "0.5,0.5", "0.05,0.9"]) if "docs" in mask else "",
                 prefix=rng.randint(0, max(1, S // 4)) if "prefix" in mask else 0)


# ------------------------------------------------------------------------------------------------------------------ their inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _doc_offsets(c):
    """[batch or 1][documents + 1] first positions of the documents, as lists; None: all positions are one document."""
    if c["lens"]:      # sequences of a batch, each of its own length
        return [[0, max(1, int(c["Sk"] * (1.0 - 0.07 * (b % 7))))] for b in range(c["batch"])]
    if not c["docs"]:
        return None
    off, at = [0], 0.0
    for share in c["docs"].split(","):
        at += float(share)
        off.append(min(c["Sk"], int(at * c["Sk"] + 1e-6)))
    return [off]


def _query_positions(c):
    """[batch][Sq] position of every query among the keys."""
    if c["lens"]:      # the last positions of each sequence
        return [[max(0, o[1] - c["Sq"] + r) for r in range(c["Sq"])] for o in _doc_offsets(c)]
    return [[c["Sk"] - c["Sq"] + r for r in range(c["Sq"])]] * c["batch"]


def _packed(g, batch, S, heads, D, dtype):
    """Tensors [batch, S, h, D] for each h of `heads`, as views of one packed projection."""
    x = _normal(g, (batch, S, sum(heads), D), dtype)
    return list(x.split(heads, dim=2))


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = DT[c["dtype"]]
    s = {"case": c}
    if c["op"] == "rope":
        B, S, D = c["batch"], c["S"], c["D"]
        s["ins"] = _packed(g, B, S, [c["Hq"], c["Hkv"]], D, dt)
        s["outs"] = [torch.empty(B, S, h, D, dtype=dt, device="cuda") for h in (c["Hq"], c["Hkv"])]
        s["positions"] = torch.randint(0, 32768, (B, S, 1), generator=g, device="cuda", dtype=torch.int32) if c["scattered"] else None
        if own:       # the handle that a program keeps: frequencies, laid out once
            from paper_2506_23858_amd import binding as vb
            scaling = {"plain": vb.ROPE_PLAIN, "linear": vb.ROPE_LINEAR, "ntk": vb.ROPE_NTK, "yarn": vb.ROPE_YARN}[c["scaling"]]
            freqs, s["mscale"] = vb.vmoba_rope_freqs(_ints(c["dims"]), c["base"], scaling, c["factor"], c["train_len"])
            s["freqs"] = freqs.cuda()
    elif c["op"] == "norm":
        shape, wdt = (c["batch"], c["S"], c["Hh"], c["D"]), DT[c["wtype"]]
        s["x"] = _normal(g, shape, dt, 1.5)
        s["residual"] = _normal(g, shape, dt) if c["residual"] else None
        s["weight"] = (1.0 + 0.2 * torch.randn(c["D"], generator=g, device="cuda")).to(wdt)
        s["y"] = torch.empty(shape, dtype=torch.float8_e4m3fn if c["out8"] else dt, device="cuda")
        s["y_scale"] = torch.empty(shape[:3], device="cuda") if c["out8"] else None
        s["total"] = torch.empty(shape, dtype=dt, device="cuda") if c["residual"] else None
        s["inv_rms"] = torch.empty(shape[:3], device="cuda")
        if c["what"] == "train":
            s["dy"] = _normal(g, shape, dt)
            s["dtotal"] = _normal(g, shape, dt) if c["residual"] else None
            s["dx"] = torch.empty(shape, dtype=dt, device="cuda")
            s["dweight"] = torch.empty(c["D"], device="cuda")
            if own:   # the workspace that a program keeps
                from paper_2506_23858_amd import binding as vb
                s["workspace"] = torch.empty(vb.vmoba_rmsnorm_workspace_bytes(c["batch"], c["Hh"], c["S"], c["D"]), dtype=torch.uint8, device="cuda")
    else:
        B, Hq, Hkv, Sq, Sk, D = (c[k] for k in ("batch", "Hq", "Hkv", "Sq", "Sk", "D"))
        if Sq == Sk:
            s["q"], s["k"], s["v"] = _packed(g, B, Sq, [Hq, Hkv, Hkv], D, dt)
        else:
            s["q"], s["k"], s["v"] = (_normal(g, (B, n, h, D), dt) for n, h in ((Sq, Hq), (Sk, Hkv), (Sk, Hkv)))
        off, masked = _doc_offsets(c), bool(c["docs"] or c["causal"] or c["lens"])
        s["doc_off"] = torch.tensor(off, dtype=torch.int32, device="cuda") if off else None
        s["prefix"] = torch.full((len(off) if off else 1, len(off[0]) - 1 if off else 1), c["prefix"], dtype=torch.int32, device="cuda") if c["prefix"] else None
        s["q_pos"] = torch.tensor(_query_positions(c), dtype=torch.int32, device="cuda") if c["lens"] else None
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], device="cuda") if c["slopes"] else None
        s["key_lo"], s["key_hi"] = (torch.empty(B, Sq, dtype=torch.int32, device="cuda") if masked else None for _ in range(2))
        s["o"], s["lse"] = torch.empty(B, Sq, Hq, D, dtype=dt, device="cuda"), torch.empty(B, Hq, Sq, device="cuda")
        if c["what"] == "train":
            s["do"] = _normal(g, (B, Sq, Hq, D), dt)
            s["dq"], s["dk"], s["dv"] = (torch.empty(t.shape, dtype=dt, device="cuda") for t in (s["q"], s["k"], s["v"]))
        if own:       # the workspace that a program keeps, one for both directions
            from paper_2506_23858_amd import binding as vb
            code, ops = vb.VMOBA_BF16 if dt == torch.bfloat16 else vb.VMOBA_F32, [vb.OP_ATTN_FWD] + [vb.OP_ATTN_BWD] * (c["what"] == "train")
            s["workspace"] = torch.empty(max(vb.vmoba_dense_workspace_bytes(op, B, Hq, Hkv, Sq, Sk, D, code) for op in ops), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------------------ the framework's calls
def run(state):
    c = state["case"]
    if own:
        from paper_2506_23858_amd import binding as vb
        return {"rope": _own_rope, "norm": _own_norm, "attn": _own_attn}[c["op"]](vb, state, c)
    return {"rope": _plain_rope, "norm": _plain_norm, "attn": _plain_attn}[c["op"]](state, c)


def _own_rope(vb, s, c):
    vb.vmoba_rope(c["batch"], c["S"], c["D"], s["ins"], s["outs"], s["freqs"], _ints(c["dims"]),
                  layout=vb.ROPE_INTERLEAVED if c["layout"] == "interleaved" else vb.ROPE_HALF, inverse=c["what"] == "bwd", mscale=s["mscale"],
                  grid=_ints(c["grid"]) if c["grid"] else None, first=c["first"], positions=s["positions"])
    return s["outs"]


def _own_norm(vb, s, c):
    size = (c["batch"], c["Hh"], c["S"], c["D"])
    vb.vmoba_rmsnorm_fwd(*size, s["x"], s["residual"], s["weight"], 1e-6, s["total"], s["y"], s["y_scale"], s["inv_rms"])
    out = {k: s[k] for k in ("total", "y", "y_scale", "inv_rms") if s[k] is not None}
    if c["what"] == "train":
        vb.vmoba_rmsnorm_bwd(*size, s["x"] if s["total"] is None else s["total"], s["weight"], s["inv_rms"], s["dy"], s["dtotal"], s["dx"], s["dweight"],
                             s["workspace"])
        out.update(dx=s["dx"], dweight=s["dweight"])
    return out


def _own_attn(vb, s, c):
    size = tuple(c[k] for k in ("batch", "Hq", "Hkv", "Sq", "Sk", "D"))
    if s["key_lo"] is not None:
        vb.vmoba_key_ranges(c["batch"], c["Sq"], c["Sk"], s["key_lo"], s["key_hi"], doc_off=s["doc_off"], prefix=s["prefix"], causal=c["causal"],
                            q_pos=s["q_pos"], q_first=c["Sk"] - c["Sq"])
    how = dict(softmax_scale=1.0 / math.sqrt(c["D"]), cap=c["cap"], slopes=s["slopes"], key_lo=s["key_lo"], key_hi=s["key_hi"], q_pos=s["q_pos"],
               q_first=c["Sk"] - c["Sq"])
    vb.vmoba_dense_fwd(*size, s["q"], s["k"], s["v"], s["o"], s["lse"], s["workspace"], **how)
    if c["what"] != "train":
        return {"o": s["o"], "lse": s["lse"]}
    vb.vmoba_dense_bwd(*size, s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"], s["workspace"], **how)
    return {k: s[k] for k in ("o", "lse", "dq", "dk", "dv")}


# ------------------------------------------------------------------------------------------------------------------ the plain form
def _plain_freqs(c):
    """(radians per position of every rotated pair, axis of every pair, factor of the rotated values), 64 bits."""
    dims, freqs, axis = _ints(c["dims"]), [], []
    for a, d in enumerate(dims):
        base = c["base"]
        if c["scaling"] == "ntk":
            base = base * c["factor"] ** (d / (d - 2.0))
        f = base ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
        if c["scaling"] == "linear":
            f = f / c["factor"]
        if c["scaling"] == "yarn":       # pairs that turn often over the trained length keep their frequency, slow ones are stretched
            keep = ((c["train_len"] * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
            f = f * keep + f / c["factor"] * (1.0 - keep)
        freqs.append(f)
        axis += [a] * (d // 2)
    mscale = 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "yarn" else 1.0
    return torch.cat(freqs), torch.tensor(axis, device="cuda"), mscale


def _plain_positions(s, c):
    """[batch or 1, S, axes] in 64 bits."""
    if s["positions"] is not None:
        return s["positions"].double() + c["first"]
    at = torch.arange(c["S"], device="cuda")
    if not c["grid"]:
        return (at + c["first"]).double()[None, :, None]
    _, H, W = _ints(c["grid"])
    return torch.stack([at // (H * W) + c["first"], at // W % H, at % W], -1).double()[None]


def _plain_rope(s, c):
    f, axis, mscale = _plain_freqs(c)
    angle = _plain_positions(s, c)[:, :, axis] * f                       # [batch or 1, S, pairs]
    cos, sin = (t.float()[:, :, None] for t in (angle.cos() * mscale, angle.sin() * (-mscale if c["what"] == "bwd" else mscale)))
    R = 2 * f.numel()

    def turned(x):
        x = x.float()
        a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["layout"] == "interleaved" else (x[..., :R // 2], x[..., R // 2:R])
        u, v = a * cos - b * sin, a * sin + b * cos
        r = torch.stack([u, v], -1).flatten(-2) if c["layout"] == "interleaved" else torch.cat([u, v], -1)
        return torch.cat([r, x[..., R:]], -1).to(DT[c["dtype"]])

    return [turned(s["ins"][0]), turned(s["ins"][1])]


def _plain_norm(s, c):
    dt = DT[c["dtype"]]
    x, out = s["x"], {}
    if s["residual"] is not None:
        x = out["total"] = (x.float() + s["residual"].float()).to(dt)
    x, w = x.float(), s["weight"].float()
    inv = (x.square().mean(-1) + 1e-6).rsqrt()
    normed = x * inv[..., None]
    y = normed * w
    if c["out8"]:
        amax = y.abs().amax(-1)
        out["y_scale"] = torch.where(amax > 0, amax / 448.0, 1.0)
        out["y"] = (y / out["y_scale"][..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    else:
        out["y"] = y.to(dt)
    out["inv_rms"] = inv
    if c["what"] == "train":
        dy = s["dy"].float()
        g = dy * w
        dx = (g - normed * (g * normed).mean(-1, keepdim=True)) * inv[..., None]
        if s["dtotal"] is not None:
            dx = dx + s["dtotal"].float()
        out["dx"] = dx.to(dt)
        out["dweight"] = (dy * normed).double().sum((0, 1, 2)).float()
    return out


def _plain_ranges(s, c):
    """First key and one past the last key of every query, [batch or 1, Sq]; the queries' positions, the same."""
    pos = s["q_pos"].long() if s["q_pos"] is not None else torch.arange(c["Sq"], device="cuda")[None] + (c["Sk"] - c["Sq"])
    lo, hi = torch.zeros_like(pos), torch.full_like(pos, c["Sk"])
    if s["doc_off"] is not None:
        off = s["doc_off"].long()
        doc = (pos[..., None] >= off[:, None, :]).sum(-1) - 1
        inside = (doc >= 0) & (doc < off.shape[1] - 1)
        at = doc.clamp(0, off.shape[1] - 2).expand(max(pos.shape[0], off.shape[0]), -1)
        lo = torch.gather(off.expand(at.shape[0], -1), 1, at)
        hi = torch.where(inside, torch.gather(off.expand(at.shape[0], -1), 1, at + 1), lo)
    if c["causal"]:
        hi = torch.minimum(hi, torch.maximum(pos + 1, lo + c["prefix"]))
    return lo, hi, pos


def _plain_attn(s, c):
    dt, B, Hq, Hkv, Sq, Sk, D = (c[k] if k != "dtype" else DT[c[k]] for k in ("dtype", "batch", "Hq", "Hkv", "Sq", "Sk", "D"))
    G, scale = Hq // Hkv, 1.0 / math.sqrt(D)
    rows = lambda x, h: x.float().permute(0, 2, 1, 3).reshape(B, Hkv, h * x.shape[1], D)                # noqa: E731
    back = lambda x, n, h: x.reshape(B, Hkv * h, n, D).permute(0, 2, 1, 3).contiguous().to(dt)         # noqa: E731
    q, k, v = rows(s["q"], G), rows(s["k"], 1), rows(s["v"], 1)
    t = torch.matmul(q, k.transpose(2, 3)).view(B, Hkv, G, Sq, Sk).mul_(scale)
    if c["cap"]:
        t = t.div_(c["cap"]).tanh_()
        p = t * c["cap"]
    else:
        p = t
    lo, hi, pos = _plain_ranges(s, c)
    at = torch.arange(Sk, device="cuda")
    if s["slopes"] is not None:
        p = p - s["slopes"].view(Hkv, G, 1, 1) * (pos[..., None] - at).abs().float()[:, None, None]
    if s["key_lo"] is not None:
        p = p.masked_fill(~((at >= lo[..., None]) & (at < hi[..., None]))[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = (p - m).exp_()
    l = p.sum(-1, keepdim=True)
    lse = (m + l.log()).reshape(B, Hq, Sq)
    p.div_(torch.where(l > 0, l, 1.0))
    flat = p.view(B, Hkv, G * Sq, Sk)
    out = {"o": back(torch.matmul(flat, v), Sq, G), "lse": lse}
    if c["what"] == "train":
        do = rows(s["do"], G)
        out["dv"] = back(torch.matmul(flat.transpose(2, 3), do), Sk, 1)
        ds = torch.matmul(do, v.transpose(2, 3))
        ds = ds.sub_((flat * ds).sum(-1, keepdim=True)).mul_(flat)
        if c["cap"]:
            ds = ds.mul_(t.square_().neg_().add_(1.0).view(ds.shape))
        ds.mul_(scale)
        out["dq"] = back(torch.matmul(ds, k), Sq, G)
        out["dk"] = back(torch.matmul(ds.transpose(2, 3), q), Sk, 1)
    return out


# ------------------------------------------------------------------------------------------------------------------ what a pass cannot do without
def _pairs(c):
    """Number of (query, key) pairs of one head, over the batch."""
    n, off = 0, _doc_offsets(c)
    for b, positions in enumerate(_query_positions(c)):
        starts = [0, c["Sk"]] if off is None else off[b % len(off)]
        for p in positions:
            for lo, hi in zip(starts[:-1], starts[1:]):
                if lo <= p < hi:
                    n += (min(hi, max(p + 1, lo + c["prefix"])) if c["causal"] else hi) - lo
    return n


def _keys_read(c):
    """Number of keys that some query reads, over the batch."""
    off = _doc_offsets(c)
    return c["batch"] * c["Sk"] if off is None else sum(o[-1] for o in off) * (c["batch"] if len(off) == 1 else 1)


def work(case):
    c = case
    if c["op"] == "rope":
        n = c["batch"] * c["S"] * (c["Hq"] + c["Hkv"]) * c["D"]
        return {"bytes": 2 * n * ES[c["dtype"]], "flops": 3 * n}
    if c["op"] == "norm":
        n, es = c["batch"] * c["S"] * c["Hh"] * c["D"], ES[c["dtype"]]
        moved = (es + (1 if c["out8"] else es)) + (2 * es if c["residual"] else 0)            # x and y; the residual and the sum
        flops = 5 * n
        if c["what"] == "train":
            moved += 3 * es + (es if c["residual"] else 0)                                     # x again, dy, dx; the sum's gradient
            flops += 9 * n
        return {"bytes": n * moved, "flops": flops}
    es, D = ES[c["dtype"]], c["D"]
    row_q, row_k = c["batch"] * c["Sq"] * c["Hq"] * D * es, _keys_read(c) * c["Hkv"] * D * es
    products = 2 + (5 if c["what"] == "train" else 0)
    moved = 2 * row_q + 2 * row_k + c["batch"] * c["Hq"] * c["Sq"] * 4
    if c["what"] == "train":      # backward: Q, O, dO, K, V and LSE again; dQ, dK, dV
        moved += 4 * row_q + 4 * row_k + c["batch"] * c["Hq"] * c["Sq"] * 4
    return {"bytes": moved, "flops": products * 2 * D * _pairs(c) * c["Hq"]}


# ------------------------------------------------------------------------------------------------------------------ the definitions, 64 bits
def exact(case, seed):
    """From the definitions: a rotation by position x frequency as a complex product; the norm's gradient as that of
    x / sqrt(mean x^2 + eps); the attention head by head, rows of weights from their logarithms."""
    c, s = case, prepare(case, seed)
    return {"rope": _exact_rope, "norm": _exact_norm, "attn": _exact_attn}[c["op"]](c, s)


def _exact_rope(c, s):
    turns, axes = [], []
    for a, d in enumerate(_ints(c["dims"])):
        for i in range(d // 2):
            theta = c["base"]
            if c["scaling"] == "ntk":
                theta *= math.pow(c["factor"], d / (d - 2))
            w = math.pow(theta, -2.0 * i / d)
            if c["scaling"] == "linear":
                w /= c["factor"]
            elif c["scaling"] == "yarn":
                gamma = min(1.0, max(0.0, (c["train_len"] * w / (2.0 * math.pi) - 1.0) / 31.0))
                w = (1.0 - gamma) * w / c["factor"] + gamma * w
            turns.append(w)
            axes.append(a)
    B, S = c["batch"], c["S"]
    if s["positions"] is not None:
        at = s["positions"].to(torch.float64)
    else:
        _, H, W = _ints(c["grid"]) if c["grid"] else (0, 1, 1)
        n = torch.arange(S, device="cuda", dtype=torch.float64)
        at = torch.stack([torch.div(n, H * W, rounding_mode="floor"), torch.div(n, W, rounding_mode="floor") % H, n % W][:len(set(axes))], 1).expand(B, S, -1).clone()
    at[..., 0] += c["first"]
    phase = torch.stack([at[..., a] * w for a, w in zip(axes, turns)], -1)
    size = 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "yarn" else 1.0
    z = torch.polar(torch.full_like(phase, size), -phase if c["what"] == "bwd" else phase)[:, :, None]
    P, got = len(turns), []
    first = [2 * i if c["layout"] == "interleaved" else i for i in range(P)]
    second = [i + (1 if c["layout"] == "interleaved" else P) for i in first]
    for x in s["ins"]:
        y = x.to(torch.float64)
        r = torch.complex(y[..., first], y[..., second]) * z
        y = y.clone()
        y[..., first], y[..., second] = r.real, r.imag
        got.append(y)
    return got


def _exact_norm(c, s):
    got = {}
    x = s["x"].to(torch.float64)
    if s["residual"] is not None:      # the sum is stored in the inputs' type, and what is stored is normalised
        got["total"] = x = (x + s["residual"].to(torch.float64)).to(DT[c["dtype"]]).to(torch.float64)
    w = s["weight"].to(torch.float64)
    n, power = c["D"], (x * x).sum(-1, keepdim=True)
    rms = torch.sqrt(power / n + 1e-6)
    y = x / rms * w
    got["inv_rms"] = 1.0 / rms[..., 0]
    if c["out8"]:
        top = y.abs().max(-1, keepdim=True).values
        step = torch.where(top == 0, torch.ones_like(top), top / 448.0)
        got["y"], got["y_scale"] = y / step, step[..., 0]
    else:
        got["y"] = y
    if c["what"] == "train":
        dy = s["dy"].to(torch.float64)
        got["dx"] = dy * w / rms - x * (dy * w * x).sum(-1, keepdim=True) / (n * rms ** 3)
        if s["dtotal"] is not None:
            got["dx"] = got["dx"] + s["dtotal"].to(torch.float64)
        got["dweight"] = (dy * x / rms).flatten(0, 2).sum(0)
    return got


def _exact_attn(c, s):
    B, Hq, Hkv, Sq, Sk, D = (c[k] for k in ("batch", "Hq", "Hkv", "Sq", "Sk", "D"))
    G, train, d64 = Hq // Hkv, c["what"] == "train", dict(dtype=torch.float64, device="cuda")
    got = {"o": torch.zeros(B, Sq, Hq, D, **d64), "lse": torch.zeros(B, Hq, Sq, **d64)}
    if train:
        got.update(dq=torch.zeros(B, Sq, Hq, D, **d64), dk=torch.zeros(B, Sk, Hkv, D, **d64), dv=torch.zeros(B, Sk, Hkv, D, **d64))
    offsets, positions = _doc_offsets(c), _query_positions(c)
    key = torch.arange(Sk, device="cuda")
    for b in range(B):
        where = torch.tensor(positions[b], device="cuda")
        begin, end = torch.zeros(Sq, dtype=torch.int64, device="cuda"), torch.zeros(Sq, dtype=torch.int64, device="cuda")
        bounds = [0, Sk] if offsets is None else offsets[b % len(offsets)]
        for lo, hi in zip(bounds[:-1], bounds[1:]):
            mine = (where >= lo) & (where < hi)
            begin[mine] = lo
            end[mine] = torch.clamp(where[mine] + 1, min=min(hi, lo + c["prefix"])) if c["causal"] else hi
        seen = (key[None] >= begin[:, None]) & (key[None] < end[:, None])
        for h in range(Hq):
            q, k, v = s["q"][b, :, h].double(), s["k"][b, :, h // G].double(), s["v"][b, :, h // G].double()
            z = q @ k.T / math.sqrt(D)
            slope = 1.0
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
                slope = 1.0 - (z / c["cap"]) ** 2 if train else 1.0
            if c["slopes"]:
                z = z - 2.0 ** (-8.0 * (h + 1) / Hq) * (where[:, None] - key[None]).abs()
            z = torch.where(seen, z, -math.inf)
            lse = torch.logsumexp(z, 1)
            a = torch.where(seen, torch.exp(z - lse[:, None]), 0.0)
            del z
            got["lse"][b, h] = lse
            got["o"][b, :, h] = o = a @ v
            if train:
                do = s["do"][b, :, h].double()
                got["dv"][b, :, h // G] += a.T @ do
                dz = a * (do @ v.T - (do * o).sum(1, keepdim=True)) * slope / math.sqrt(D)
                got["dq"][b, :, h] = dz @ k
                got["dk"][b, :, h // G] += dz.T @ q
    return got
