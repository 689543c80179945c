"""Rotary positions, root-mean-square norms and dense attention against plain 64-bit forms, at the sizes and masks where they can go wrong."""
import math

import pytest
import torch

from paper_2506_23858_amd import binding as vb
from tests import operator_util as ou

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


# ---------------------------------------------------------------------------------------------------------------- rotary positions
def rope_reference(x, freqs, axis, at, layout, inverse, mscale):
    """Value and bound.  at: [B or 1, S, axes] float64.  The angle's sine and cosine are float32 (angle in turns rounded to float32: 2^-25 of a
    turn; two ulp of the functions), as are the products and their sum."""
    angle = at[:, :, axis] * freqs * (-1.0 if inverse else 1.0)
    c, s = angle.cos()[:, :, None] * mscale, angle.sin()[:, :, None] * mscale
    P = freqs.numel()
    y = x.double()
    first = torch.arange(P, device=x.device) * (2 if layout == vb.ROPE_INTERLEAVED else 1)
    second = first + (1 if layout == vb.ROPE_INTERLEAVED else P)
    a, b = y[..., first], y[..., second]
    out, err = y.clone(), torch.zeros_like(y)
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    arithmetic = 2.0 ** -21 * mscale * (a.abs() + b.abs())
    err[..., first], err[..., second] = (arithmetic + ou.HALF[x.dtype] * out[..., i].abs() for i in (first, second))
    return out, err


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", [vb.ROPE_HALF, vb.ROPE_INTERLEAVED])
@pytest.mark.parametrize("B,S,heads,D,dims,scaling", [
    (1, 1, [1], 64, [64], vb.ROPE_PLAIN), (2, 37, [4, 2], 128, [64], vb.ROPE_YARN), (1, 300, [3, 1, 1], 64, [58], vb.ROPE_NTK),
    (3, 5, [2], 128, [122], vb.ROPE_LINEAR), (1, 64, [2, 2], 32, [2], vb.ROPE_PLAIN), (1, 9, [1, 5], 64, [16], vb.ROPE_PLAIN), (1, 3, [1], 1024, [1000], vb.ROPE_PLAIN)])
def test_rope_on_sequences(dtype, layout, B, S, heads, D, dims, scaling):
    packed = ou.normal(1, (B, S, sum(heads), D), dtype)
    ins = list(packed.split(heads, 2))
    outs = [torch.full((B, h, S, D), 7.0, dtype=dtype, device="cuda").permute(0, 2, 1, 3) for h in heads]
    freqs, mscale = vb.vmoba_rope_freqs(dims, 1e4, scaling, 1.0 if scaling == vb.ROPE_PLAIN else 8.0, 2048)
    freqs = freqs.cuda()
    pos = torch.randint(-5, 100000, (B, S, 1), device="cuda", dtype=torch.int32)
    for positions, first, inverse in ((None, 0, False), (None, 999983, True), (pos, 17, False), (pos[:1].contiguous(), 0, True)):
        vb.vmoba_rope(B, S, D, ins, outs, freqs, dims, layout, inverse, mscale, first=first, positions=positions)
        at = (positions.double() if positions is not None else torch.arange(S, device="cuda").double()[None, :, None]) + first
        for x, y in zip(ins, outs):
            ref, err = rope_reference(x, freqs, torch.zeros(freqs.numel(), dtype=torch.long, device="cuda"), at, layout, inverse, mscale)
            ou.within("rope", y, ref, err)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("grid,dims,D", [((1, 1, 1), [2, 4, 6], 64), ((3, 5, 7), [44, 42, 42], 128), ((4, 1, 9), [20, 20, 20], 64)])
def test_rope_on_a_grid_and_in_place(dtype, grid, dims, D):
    T, H, W = grid
    S = T * H * W
    x = ou.normal(2, (2, S, 3, D), dtype)
    freqs, mscale = vb.vmoba_rope_freqs(dims)
    freqs = freqs.cuda()
    at = torch.stack(torch.meshgrid(*[torch.arange(n, device="cuda") for n in grid], indexing="ij"), -1).reshape(1, S, 3).double()
    at[..., 0] += 40
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor([d // 2 for d in dims], device="cuda"))
    ref, err = rope_reference(x, freqs, axis, at, vb.ROPE_INTERLEAVED, False, mscale)
    y = torch.empty_like(x)
    vb.vmoba_rope(2, S, D, [x], [y], freqs, dims, vb.ROPE_INTERLEAVED, grid=grid, first=40)
    ou.within("rope", y, ref, err)
    z = x.clone()
    vb.vmoba_rope(2, S, D, [z], [z], freqs, dims, vb.ROPE_INTERLEAVED, grid=grid, first=40)
    assert torch.equal(y, z)
    # positions given one by one are the grid's
    vb.vmoba_rope(2, S, D, [x], [z], freqs, dims, vb.ROPE_INTERLEAVED, first=40, positions=(at - torch.tensor([40.0, 0, 0], device="cuda")).int().contiguous())
    assert torch.equal(y, z)


def test_rope_gradient_by_differences():
    """<dy, d rope(x)> = <inverse rope(dy), dx>: the call is linear, so the difference quotient is exact up to roundings (float32)."""
    freqs, m = vb.vmoba_rope_freqs([40], 1e4, vb.ROPE_YARN, 4.0, 512)
    x, dy, e = (ou.normal(i, (1, 50, 2, 64), F32) for i in (3, 4, 5))
    out = [torch.empty_like(x) for _ in range(3)]
    for src, dst, inv in ((x, out[0], False), (x + e, out[1], False), (dy, out[2], True)):
        vb.vmoba_rope(1, 50, 64, [src], [dst], freqs.cuda(), [40], inverse=inv, mscale=m)
    left, right = (dy.double() * (out[1].double() - out[0].double())).sum(), (out[2].double() * e.double()).sum()
    terms = (dy.double().abs() * (out[1].abs() + out[0].abs()).double()).sum()
    assert abs(float(left - right)) <= 2.0 ** -20 * float(terms)


# ---------------------------------------------------------------------------------------------------------------- norms
def norm_case(B, S, Hh, D, dtype, wdtype, residual, strided):
    def make(seed, scale=1.0):
        if strided:      # rows of odd distance: no 16-byte access is aligned
            return ou.normal(seed, (B, S, Hh, D + 3), dtype, scale)[..., 1:1 + D]
        return ou.normal(seed, (B, S, Hh, D), dtype, scale)
    return make(1, 2.0), make(2) if residual else None, (1 + 0.3 * ou.normal(3, (D,), F32)).to(wdtype), make(4), make(5) if residual else None, make


SIZES = [(1, 1, 1, 1), (2, 3, 5, 7), (1, 70, 12, 128), (3, 11, 1, 64), (1, 33, 1, 1536), (1, 5, 2, 1000), (2, 4, 1, 2047), (1, 3, 1, 5120), (1, 2, 1, 16384)]


@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("B,S,Hh,D", SIZES)
@pytest.mark.parametrize("residual,strided", [(False, False), (True, False), (True, True)])
def test_norm(B, S, Hh, D, dtype, wdtype, residual, strided):
    x, r, w, dy, dt, make = norm_case(B, S, Hh, D, dtype, wdtype, residual, strided)
    total, y, dx = (make(9).zero_() for _ in range(3))
    inv = torch.empty(B, S, Hh, device="cuda")
    vb.vmoba_rmsnorm_fwd(B, Hh, S, D, x, r, w, 1e-5, total if residual else None, y, None, inv)
    t = x
    if residual:
        assert torch.equal(total, (x.float() + r.float()).to(dtype))
        t = total
    t64, w64, g64 = t.double(), w.double(), dy.double()
    inv64 = (t64.square().mean(-1, keepdim=True) + 1e-5).rsqrt()
    half, sums = ou.HALF[dtype], 80 * ou.F32                       # a lane sums at most 64 squares, then 8 levels
    ou.within("inv_rms", inv, inv64[..., 0], sums * inv64[..., 0])
    ref = t64 * inv64 * w64
    ou.within("y", y, ref, (half + sums + 4 * ou.F32) * ref.abs())
    # the 8-bit form of the same
    y8, scale = make(9).to(torch.float8_e4m3fn), torch.empty(B, S, Hh, device="cuda")
    vb.vmoba_rmsnorm_fwd(B, Hh, S, D, x, r, w, 1e-5, total if residual else None, y8, scale, None)
    top = ref.abs().amax(-1)
    ou.within("scale", scale, top / 448, (sums + 8 * ou.F32) * top / 448)
    q = ref / scale.double()[..., None]
    ou.within("y8", y8.float(), q, (2.0 ** -4 + 2 * sums) * q.abs() + 2.0 ** -10)
    # gradient
    n = t64 * inv64
    gw = g64 * w64
    mean = (gw * n).mean(-1, keepdim=True)
    ref = inv64 * (gw - n * mean) + (dt.double() if residual else 0.0)
    err = inv64 * 4 * sums * (gw.abs() + n.abs() * (gw * n).abs().mean(-1, keepdim=True)) + (dt.double().abs() * 4 * ou.F32 if residual else 0.0)
    dw, ws = torch.empty(D, device="cuda"), torch.empty(max(1, vb.vmoba_rmsnorm_workspace_bytes(B, Hh, S, D)), dtype=torch.uint8, device="cuda")
    vb.vmoba_rmsnorm_bwd(B, Hh, S, D, t, w, inv, dy, dt, dx, dw, ws)
    ou.within("dx", dx, ref, err + half * ref.abs())
    terms = (g64 * n).flatten(0, 2)
    ou.within("dweight", dw, terms.sum(0), (sums + (B * S * Hh + 64) * ou.F32) * terms.abs().sum(0) + 1e-30)
    again = torch.empty_like(dw)
    vb.vmoba_rmsnorm_bwd(B, Hh, S, D, t, w, inv, dy, dt, dx, again, ws)
    assert torch.equal(dw, again)
    if strided:                                                     # what lies between the rows stays
        assert all(float(z._base[..., 0].abs().min()) > 0 for z in (x, r, dy))


def test_norm_of_many_rows_and_in_place():
    """More rows than workgroups: every group walks several."""
    B, S, Hh, D = 1, 40000, 1, 96
    x, dy, w = ou.normal(1, (B, S, Hh, D), F32), ou.normal(2, (B, S, Hh, D), F32), 1 + 0.1 * ou.normal(3, (D,), F32)
    y, dx, inv, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(B, S, Hh, device="cuda"), torch.empty(D, device="cuda")
    ws = torch.empty(vb.vmoba_rmsnorm_workspace_bytes(B, Hh, S, D), dtype=torch.uint8, device="cuda")
    vb.vmoba_rmsnorm_fwd(B, Hh, S, D, x, None, w, 0.0, None, y, None, inv)
    vb.vmoba_rmsnorm_bwd(B, Hh, S, D, x, w, inv, dy, None, dx, dw, ws)
    n = x.double() * x.double().square().mean(-1, keepdim=True).rsqrt()
    ou.within("y", y, n * w.double(), 90 * ou.F32 * (n * w.double()).abs())
    terms = (dy.double() * n).flatten(0, 2)
    ou.within("dweight", dw, terms.sum(0), (80 + S + 64) * ou.F32 * terms.abs().sum(0))
    z, e = x.clone(), dy.clone()
    vb.vmoba_rmsnorm_bwd(B, Hh, S, D, x, w, inv, e, None, e, None, None)
    vb.vmoba_rmsnorm_fwd(B, Hh, S, D, z, None, w, 0.0, None, z, None, None)
    assert torch.equal(z, y) and torch.equal(e, dx)


def test_norm_rows_of_zeros_infinities_and_nan():
    x = ou.normal(1, (1, 6, 1, 128), BF16)
    x[0, 1], x[0, 2, 0, 5], x[0, 4, 0, 7] = 0.0, math.inf, math.nan
    y, y8, s = torch.empty_like(x), torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(1, 6, 1, device="cuda")
    vb.vmoba_rmsnorm_fwd(1, 1, 6, 128, x, None, None, 1e-6, None, y, None, None)
    vb.vmoba_rmsnorm_fwd(1, 1, 6, 128, x, None, None, 1e-6, None, y8, s, None)
    assert bool((y[0, 1] == 0).all()) and bool((y8[0, 1].float() == 0).all()) and float(s[0, 1]) == 1.0
    assert bool(y[0, 2].isnan().any()) and bool(y[0, 4].isnan().all()) and bool(s[0, 2].isnan()) and bool(s[0, 4].isnan())
    assert bool(y8[0, 4].float().isnan().all())
    for r in (0, 3, 5):
        assert bool(y[0, r].isfinite().all()) and bool(y8[0, r].float().isfinite().all())
        assert float(y8[0, r].float().abs().max()) == 448.0


def test_calls_without_rows():
    """The binding hands out no address for an empty tensor; the library takes any and launches nothing but the clearing of dweight."""
    assert vb.vmoba_rmsnorm_workspace_bytes(1, 1, 0, 64) == 0
    some, dw = torch.empty(64, dtype=BF16, device="cuda"), torch.full((64,), 3.0, device="cuda")
    d = vb._desc(some.view(1, 1, 1, 64))
    L, st = vb.lib(), torch.cuda.current_stream().cuda_stream
    assert L.vmoba_rmsnorm_fwd(1, 1, 0, 64, d, None, None, 0, 1e-6, None, d, None, None, st) == 0
    assert L.vmoba_rmsnorm_bwd(1, 1, 0, 64, d, None, 0, dw.data_ptr(), d, None, d, dw.data_ptr(), None, 0, st) == 0
    assert bool((dw == 0).all())


# ---------------------------------------------------------------------------------------------------------------- dense attention
def tensors(B, Hq, Hkv, Sq, Sk, D, dtype, seed=1, scale=1.3):
    if Sq == Sk:
        Q, K, V = ou.normal(seed, (B, Sq, Hq + 2 * Hkv, D), dtype, scale).split([Hq, Hkv, Hkv], 2)
    else:
        Q, K, V = (ou.normal(seed + i, (B, n, h, D), dtype, scale) for i, (n, h) in enumerate(((Sq, Hq), (Sk, Hkv), (Sk, Hkv))))
    return Q, K, V, ou.normal(seed + 7, (B, Sq, Hq, D), dtype)


def run(Q, K, V, dO, lo=None, hi=None, scale=None, cap=0.0, slopes=None, q_pos=None, q_first=0, bwd=True):
    B, Sq, Hq, D = Q.shape
    Sk, Hkv = K.shape[1], K.shape[2]
    code = vb.VMOBA_BF16 if Q.dtype == BF16 else vb.VMOBA_F32
    n = max(vb.vmoba_dense_workspace_bytes(op, B, Hq, Hkv, Sq, Sk, D, code) for op in (vb.OP_ATTN_FWD, vb.OP_ATTN_BWD))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
    out = {"O": torch.full((B, Sq, Hq, D), 7.0, dtype=Q.dtype, device="cuda"), "LSE": torch.full((B, Hq, Sq), 7.0, device="cuda")}
    how = dict(softmax_scale=1 / math.sqrt(D) if scale is None else scale, cap=cap, slopes=slopes, key_lo=lo, key_hi=hi, q_pos=q_pos, q_first=q_first)
    size = (B, Hq, Hkv, Sq, Sk, D)
    vb.vmoba_dense_fwd(*size, Q, K, V, out["O"], out["LSE"], ws, **how)
    if bwd:
        ws.fill_(255)
        out.update((name, torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda")) for name, t in (("dQ", Q), ("dK", K), ("dV", V)))
        vb.vmoba_dense_bwd(*size, Q, K, V, out["O"], out["LSE"], dO, out["dQ"], out["dK"], out["dV"], ws, **how)
    return out


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(Q, K, V, dO, lo=None, hi=None, scale=None, cap=0.0, slopes=None, q_pos=None, q_first=0, bwd=True):
    B, Sq, _, D = Q.shape
    Sk = K.shape[1]
    got = run(Q, K, V, dO, lo, hi, scale, cap, slopes, q_pos, q_first, bwd)
    l, h = (torch.zeros(B, Sq, device="cuda") if lo is None else lo), (torch.full((B, Sq), Sk, device="cuda") if hi is None else hi)
    pos = q_pos if q_pos is not None else (torch.arange(Sq, device="cuda") + q_first).expand(B, Sq)
    ref = ou.attention(Q, K, V, l, h, pos, 1 / math.sqrt(D) if scale is None else scale, cap, slopes, dO if bwd else None)
    for name, (value, bound) in ref.items():
        ou.within(name, got[name], value, bound + 1e-12)
    return got


SHAPES = [(1, 1, 1, 1, 1), (2, 4, 2, 1, 37), (1, 3, 3, 33, 65), (1, 5, 1, 77, 77), (2, 4, 2, 40, 300), (1, 2, 2, 257, 257), (3, 8, 8, 2, 515), (1, 2, 1, 700, 129)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk", SHAPES)
@pytest.mark.parametrize("cap,bias", [(0.0, False), (5.0, True)])
def test_dense_without_ranges(B, Hq, Hkv, Sq, Sk, D, dtype, cap, bias):
    slopes = torch.linspace(0.02, 0.3, Hq, device="cuda") if bias else None
    check(*tensors(B, Hq, Hkv, Sq, Sk, D, dtype), cap=cap, slopes=slopes, q_first=Sk - Sq)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (8.0, False), (0.0, True)])
@pytest.mark.parametrize("mask", ["causal", "docs", "prefix", "lens", "any"])
@pytest.mark.parametrize("D,B,Hq,Hkv,S", [(128, 2, 3, 3, 301), (64, 2, 6, 2, 190)])
def test_dense_with_ranges(D, B, Hq, Hkv, S, mask, cap, bias, dtype):
    Q, K, V, dO = tensors(B, Hq, Hkv, S, S, D, dtype)
    lo, hi = torch.empty(B, S, dtype=torch.int32, device="cuda"), torch.empty(B, S, dtype=torch.int32, device="cuda")
    spec = {"causal": dict(causal=True), "docs": dict(doc_off=[[0, 33, 33, 34, 150, S - 20], [5, 64, 128, 128, 160, S]]),
            "prefix": dict(doc_off=[[0, 70, S - 9]], prefix=[[20, 100]], causal=True), "lens": dict(doc_off=[[0, S - 77], [0, 1]], causal=True)}.get(mask)
    if spec:
        given = {k: int32(v) if k in ("doc_off", "prefix") else v for k, v in spec.items()}
        vb.vmoba_key_ranges(B, S, S, lo, hi, **given)
        want = ou.ranges(B, S, S, **spec)
        assert [list(zip(a, b)) for a, b in zip(lo.tolist(), hi.tolist())] == want
    else:      # ranges of every kind: empty ones, reversed ones, beyond both ends
        g = torch.Generator().manual_seed(5)
        lo.copy_(torch.randint(-50, S, (B, S), generator=g))
        hi.copy_(lo.cpu() + torch.randint(-30, S, (B, S), generator=g))
        hi[:, ::7] = 2 ** 31 - 1
        lo[:, ::11] = -2 ** 31
    check(Q, K, V, dO, lo, hi, cap=cap, slopes=torch.linspace(0.01, 0.2, Hq, device="cuda") if bias else None)


def test_key_ranges_of_single_queries_and_bad_offsets():
    B, S = 3, 50
    q_pos = [[49], [7], [0]]
    spec = dict(doc_off=[[0, 50], [0, 8], [3, 9]], q_pos=q_pos, causal=True)
    lo, hi = (torch.empty(B, 1, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(B, 1, S, lo, hi, doc_off=int32(spec["doc_off"]), q_pos=int32(q_pos), causal=True)
    assert [list(zip(a, b)) for a, b in zip(lo.tolist(), hi.tolist())] == ou.ranges(B, 1, S, **spec) == [[(0, 50)], [(0, 8)], [(0, 0)]]
    # whatever the arrays hold, ranges stay inside the keys
    lo, hi = (torch.empty(1, S, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(1, S, S, lo, hi, doc_off=int32([[9, -4, 2 ** 31 - 1, 3]]), prefix=int32([[2 ** 31 - 1, -2 ** 31, 5]]), causal=True, q_first=-20)
    assert int(lo.min()) >= 0 and int(hi.max()) <= S and bool((lo <= hi).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale,cap", [(-0.2, 0.0), (0.0, 0.0), (-0.2, 3.0), (0.0, 3.0), (40.0, 0.0), (0.2, 4096.0), (0.2, 1e-30)])
def test_dense_scales_of_any_sign(dtype, scale, cap):
    Q, K, V, dO = tensors(1, 2, 1, 70, 70, 64, dtype, scale=0.5)
    lo, hi = (torch.empty(1, 70, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(1, 70, 70, lo, hi, causal=True)
    check(Q, K, V, dO, lo, hi, scale=scale, cap=cap)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_dense_large_scores_and_late_maxima(dtype):
    """Scores up to some hundreds whose maximum comes late, early, and in the middle of a row."""
    Q, K, V, dO = tensors(1, 1, 1, 96, 400, 128, dtype, scale=1.0)
    ramp = torch.linspace(0.01, 6.0, 400, device="cuda")
    K = (K.float() * ramp.view(1, 400, 1, 1)).to(dtype)
    check(Q, K, V, dO)
    check(Q, K.flip(1), V, dO)


@pytest.mark.parametrize("Sq,Hq,Hkv,Sk", [(1, 16, 4, 5000), (3, 5, 1, 2049), (1, 1, 1, 33), (8, 12, 12, 4000)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_dense_single_queries_over_a_cache(Sq, Hq, Hkv, Sk, dtype):
    B = 3
    Q, K, V, _ = tensors(B, Hq, Hkv, Sq, Sk, 128, dtype)
    lens = [Sk, max(1, Sk // 3), 0]
    for b in range(B):      # what lies behind a sequence's end is never read into a result
        K[b, lens[b]:], V[b, lens[b]:] = math.nan, math.inf
    q_pos = int32([[max(0, n - Sq + r) for r in range(Sq)] for n in lens])
    lo, hi = (torch.empty(B, Sq, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(B, Sq, Sk, lo, hi, doc_off=int32([[0, n] for n in lens]), causal=True, q_pos=q_pos)
    got = check(Q, K, V, None, lo, hi, slopes=torch.linspace(0.001, 0.1, Hq, device="cuda"), q_pos=q_pos, bwd=False)
    assert bool((got["O"][2] == 0).all()) and bool((got["LSE"][2] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (6.0, True)])
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_dense_masked_places_do_not_reach_results(dtype, poison, cap, bias):
    """Two documents that share tiles, a causal mask, and empty places at the end: what stands in the second document, in keys that a query may not see
    yet, and in the empty places changes no bit of the first document's results."""
    B, H, S, D, cut, end = 1, 2, 200, 64, 91, 170
    Q, K, V, dO = (t.clone() for t in tensors(B, H, H, S, S, D, dtype))
    slopes = torch.tensor([0.1, 0.01], device="cuda") if bias else None
    lo, hi = (torch.empty(B, S, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(B, S, S, lo, hi, doc_off=int32([[0, cut, end]]), causal=True)
    clean = run(Q, K, V, dO, lo, hi, cap=cap, slopes=slopes)
    for t in (Q, K, V, dO):
        t[:, cut + 40:] = poison
        t[:, end:, :, ::2] = math.nan
    got = run(Q, K, V, dO, lo, hi, cap=cap, slopes=slopes)
    for name in ("O", "dQ"):
        assert torch.equal(got[name][:, :cut + 40], clean[name][:, :cut + 40]), name        # a later key never reaches an earlier query
        assert bool((got[name][:, end:] == 0).all()), name
    assert torch.equal(got["LSE"][:, :, :cut + 40], clean["LSE"][:, :, :cut + 40])
    for name in ("dK", "dV"):
        assert torch.equal(got[name][:, :cut], clean[name][:, :cut]), name
        assert bool((got[name][:, end:] == 0).all()), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Sq,Sk", [(60, 60), (1, 3000)])
def test_dense_values_that_are_not_finite_reach_their_readers(dtype, Sq, Sk):
    Q, K, V, _ = (t.clone() for t in tensors(1, 2, 2, Sq, Sk, 64, dtype))
    V[0, 20, 0, 3], V[0, 31, 1, 40], V[0, Sk - 2, 0, 7] = math.inf, math.nan, -math.inf
    lo, hi = (torch.empty(1, Sq, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(1, Sq, Sk, lo, hi, causal=True, q_first=Sk - Sq)
    check(Q, K, V, None, lo, hi, bwd=False)
    check(Q, K, V, None, bwd=False)


def test_dense_gradient_by_differences():
    """Directional derivatives of <O, dO> in float32 with cap, bias and ranges, by central differences of a 64-bit reference."""
    Q, K, V, dO = tensors(1, 4, 2, 45, 45, 64, F32)
    slopes = torch.tensor([0.3, 0.1, 0.03, 0.01], device="cuda")
    lo, hi = (torch.empty(1, 45, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(1, 45, 45, lo, hi, doc_off=int32([[0, 20, 40]]), prefix=int32([[4, 3]]), causal=True)
    got = run(Q, K, V, dO, lo, hi, cap=4.0, slopes=slopes)
    pos = torch.arange(45, device="cuda").expand(1, 45)
    value = lambda q, k, v: (ou.attention(q, k, v, lo, hi, pos, 0.125, 4.0, slopes)["O"][0] * dO.double()).sum()      # noqa: E731
    ou.HALF[torch.float64] = 2.0 ** -53
    for i, name in enumerate(("dQ", "dK", "dV")):
        step = ou.normal(40 + i, (Q, K, V)[i].shape, F32).double()
        moved = [[t.double() + (h * step if j == i else 0.0) for j, t in enumerate((Q, K, V))] for h in (1e-4, -1e-4)]
        numeric = (value(*moved[0]) - value(*moved[1])) / 2e-4
        exact = (got[name].double() * step).sum()
        terms = (got[name].double().abs() * step.abs()).sum()
        assert abs(float(numeric - exact)) <= 1e-5 * float(terms), name      # 1e-8 of the quotient's own error, some hundred float32 roundings


def test_dense_streams_graphs_and_repeats():
    Q, K, V, dO = tensors(1, 4, 2, 300, 300, 128, BF16)
    every = int32([[0] * 300]), int32([[300] * 300])
    first = run(Q, K, V, dO, *every)
    again = run(Q, K, V, dO, *every)
    assert all(torch.equal(first[k], again[k]) for k in first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run(Q, K, V, dO, *every)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(first[k], other[k]) for k in first)
    B, Sq, Hq, D = Q.shape
    n = max(vb.vmoba_dense_workspace_bytes(op, 1, 4, 2, 300, 300, 128, vb.VMOBA_BF16) for op in (vb.OP_ATTN_FWD, vb.OP_ATTN_BWD))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = {k: torch.zeros_like(v) for k, v in first.items()}
    lo, hi = (torch.empty(1, 300, dtype=torch.int32, device="cuda") for _ in range(2))
    args = (1, 4, 2, 300, 300, 128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.vmoba_key_ranges(1, 300, 300, lo, hi)
        how = dict(softmax_scale=1 / math.sqrt(128), key_lo=lo, key_hi=hi)
        vb.vmoba_dense_fwd(*args, Q, K, V, out["O"], out["LSE"], ws, **how)
        vb.vmoba_dense_bwd(*args, Q, K, V, out["O"], out["LSE"], dO, out["dQ"], out["dK"], out["dV"], ws, **how)
    for _ in range(3):
        for t in out.values():
            t.zero_()
        lo.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(first[k], out[k]) for k in first)
        assert torch.equal(run(Q, K, V, dO, *every)["dK"], first["dK"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hq,Sq", [(300, 1), (300, 3), (255, 2)])
def test_dense_many_heads_on_one_key_head(Hq, Sq, dtype):
    check(*tensors(1, Hq, 1, Sq, 70, 64, dtype), slopes=torch.linspace(0.0, 0.1, Hq, device="cuda"), q_first=70 - Sq)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_dense_strides_and_orders(dtype):
    """Head-major tensors, tensors with rows further apart than they are long, keys and values that all batch elements share."""
    B, Hq, Hkv, Sq, Sk, D = 2, 4, 2, 50, 90, 64
    Q = ou.normal(1, (B, Hq, Sq, D), dtype).transpose(1, 2)
    K = ou.normal(2, (1, Sk, Hkv, D), dtype).expand(B, -1, -1, -1)
    V = ou.normal(3, (1, Hkv, Sk, 2 * D), dtype).transpose(1, 2)[..., :D].expand(B, -1, -1, -1)
    dO = ou.normal(4, (B, Sq, D // 8, Hq, 16), dtype)[:, :, 2:6].reshape(B, Sq, Hq, D)
    check(Q, K, V, dO)


def test_dense_cache_beyond_32_bit_offsets():
    """Three caches of 2 GiB each for keys and for values: the last keys of the last one."""
    B, H, S, D, n = 3, 8, 1 << 20, 128, 300
    K, V = (torch.empty(B, S, H, D, dtype=BF16, device="cuda") for _ in range(2))
    tail = ou.normal(1, (2, n, H, D), BF16)
    K[2, S - n:], V[2, S - n:] = tail[0], tail[1]
    Q = ou.normal(2, (B, 1, H, D), BF16)
    lo, hi = int32([[0], [0], [S - n]]), int32([[0], [0], [S]])
    got = run(Q, K, V, None, lo, hi, bwd=False)
    ref = ou.attention(Q[2:], tail[:1], tail[1:], int32([[0]]), int32([[n]]), None, 1 / math.sqrt(D))
    ou.within("O", got["O"][2:], *ref["O"])
    ou.within("LSE", got["LSE"][2:], *ref["LSE"])
    assert bool((got["O"][:2] == 0).all())


# float32 calls of 3e8 multiply-adds and more multiply operands split into bfloat16 terms.  The bound of a product holds for them, too: a term left out is below
# 2^-25 of it, and its sum is rounded once per matrix instruction, 6 times in 16 channels, where the bound counts every channel.
MANY = [(64, 1, 6, 2, 901, 901), (128, 2, 3, 3, 641, 641), (128, 1, 5, 1, 333, 1511), (64, 3, 4, 4, 700, 613)]


@pytest.mark.parametrize("D,B,Hq,Hkv,Sq,Sk", MANY)
@pytest.mark.parametrize("mask,cap,bias,scale", [("none", 0.0, False, None), ("none", 7.0, True, -0.1), ("causal", 0.0, True, None), ("docs", 9.0, False, None), ("any", 0.0, False, -0.2)])
def test_dense_float32_calls_of_many_pairs(D, B, Hq, Hkv, Sq, Sk, mask, cap, bias, scale):
    Q, K, V, dO = tensors(B, Hq, Hkv, Sq, Sk, D, F32)
    lo = hi = None
    if mask != "none":
        lo, hi = (torch.empty(B, Sq, dtype=torch.int32, device="cuda") for _ in range(2))
    if mask == "any":      # empty ones, reversed ones, beyond both ends
        g = torch.Generator().manual_seed(6)
        lo.copy_(torch.randint(-50, Sk, (B, Sq), generator=g))
        hi.copy_(lo.cpu() + torch.randint(-30, Sk, (B, Sq), generator=g))
    elif mask != "none":
        docs = dict(doc_off=int32([[0, 65, 65, 301, Sk - 120]]), prefix=int32([[10, 0, 100, 7]])) if mask == "docs" else {}
        vb.vmoba_key_ranges(B, Sq, Sk, lo, hi, causal=True, q_first=Sk - Sq, **docs)
    check(Q, K, V, dO, lo, hi, scale=scale, cap=cap, slopes=torch.linspace(0.001, 0.05, Hq, device="cuda") if bias else None, q_first=Sk - Sq)


@pytest.mark.parametrize("where", ["masked NaN", "masked infinity", "large", "small"])
def test_dense_float32_values_that_terms_do_not_hold(where):
    """Such a call gives what the float32 instruction gives, and the next one, in the same workspace or a replay of the same graph, split operands again."""
    B, H, S, D, end = 1, 6, 901, 64, 850
    Q, K, V, dO = (t.clone() for t in tensors(B, H, H, S, S, D, F32))
    lo, hi = (torch.empty(B, S, dtype=torch.int32, device="cuda") for _ in range(2))
    vb.vmoba_key_ranges(B, S, S, lo, hi, doc_off=int32([[0, end]]), causal=True)
    for t in (Q, K, V, dO):
        t[:, end:] = 0.0
    plain = [t.clone() for t in (Q, K, V, dO)]
    clean = check(Q, K, V, dO, lo, hi)
    if "masked" in where:
        for t in (Q, K, V, dO):
            t[:, end:] = math.nan if "NaN" in where else -math.inf
    else:      # values that are read: scores stay moderate
        V[0, 3, 0, 5], dO[0, 700, 1, 2] = (3e9, -2e8) if where == "large" else (1e-36, -1e-33)
    other = check(Q, K, V, dO, lo, hi)
    if "masked" in where:      # off by the rounding of the sums alone, and nothing where there is nothing
        assert all(bool((other[n][:, end:] == 0).all()) for n in ("O", "dQ", "dK", "dV"))
    # a graph whose inputs change between such values and others
    size, ws = (B, H, H, S, S, D), torch.empty(max(vb.vmoba_dense_workspace_bytes(op, B, H, H, S, S, D, vb.VMOBA_F32) for op in (vb.OP_ATTN_FWD, vb.OP_ATTN_BWD)),
                                               dtype=torch.uint8, device="cuda")
    ins, odd = [t.clone() for t in plain], [t.clone() for t in (Q, K, V, dO)]
    out = {n: torch.empty_like(t) for n, t in clean.items()}
    how = dict(softmax_scale=1 / math.sqrt(D), key_lo=lo, key_hi=hi)

    def step():
        vb.vmoba_dense_fwd(*size, *ins[:3], out["O"], out["LSE"], ws, **how)
        vb.vmoba_dense_bwd(*size, *ins[:3], out["O"], out["LSE"], ins[3], out["dQ"], out["dK"], out["dV"], ws, **how)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for values, want in ((odd, other), (plain, clean), (odd, other), (plain, clean)):
        for t, v in zip(ins, values):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n].view(torch.int32), want[n].view(torch.int32)), n


# ---------------------------------------------------------------------------------------------------------------- together
def layer_reference(Q, K, V, wq, wk, dims, grid, norm, dO, cap):
    """Norm, rotation, dense attention in 64 bits, and their gradients by automatic differentiation."""
    leaves = [t.double().detach().requires_grad_() for t in (Q, K, V, wq, wk)]
    q, k, v, a, b = leaves

    def prepared(x, w):
        y = x if norm == "head" else x.flatten(2)
        y = (y * (y.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w).view(x.shape)
        freqs = torch.cat([1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d) for d in dims])
        axis = torch.repeat_interleave(torch.arange(len(dims), device="cuda"), torch.tensor([d // 2 for d in dims], device="cuda"))
        at = torch.stack(torch.meshgrid(*[torch.arange(n, device="cuda") for n in grid], indexing="ij"), -1).reshape(-1, 3).double()
        z = torch.view_as_complex(y[..., :sum(dims)].reshape(*y.shape[:-1], -1, 2)) * torch.polar(torch.ones_like(at[:, axis]), at[:, axis] * freqs)[:, None]
        return torch.cat([torch.view_as_real(z).flatten(-2), y[..., sum(dims):]], -1)

    G = Q.shape[2] // K.shape[2]
    s = torch.einsum("bqhd,bkhd->bhqk", prepared(q, a), prepared(k, b).repeat_interleave(G, 2)) / math.sqrt(Q.shape[3])
    s = cap * torch.tanh(s / cap) if cap else s
    o = torch.einsum("bhqk,bkhd->bqhd", s.softmax(-1), v.repeat_interleave(G, 2))
    (o * dO.double()).sum().backward()
    return o.detach(), [t.grad for t in leaves]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("kind", ["dense", "sparse"])
def test_a_layer_with_norms_and_positions(kind, norm, dtype):
    """QueryKeyPlan in front of a dense plan, and of a sparse plan that keeps every pair (tau = 1), forward and backward."""
    grid, dims, B, Hq, D = (3, 5, 7), [24, 20, 20], 1, 4, 64
    Hkv = 2 if kind == "dense" else 4
    S, cap = 105, 20.0 if kind == "dense" else 0.0
    Q, K, V = ou.normal(1, (B, S, Hq + 2 * Hkv, D), dtype).split([Hq, Hkv, Hkv], 2)
    dO = ou.normal(2, (B, S, Hq, D), dtype)
    wq, wk = (1 + 0.1 * ou.normal(3 + i, (D if norm == "head" else h * D,), F32) for i, h in enumerate((Hq, Hkv)))
    prepare = vb.QueryKeyPlan(B, Hq, Hkv, S, D, dims, grid, vb.ROPE_INTERLEAVED, norm=norm, wq=wq, wk=wk, dtype=dtype)
    if kind == "dense":
        plan = vb.DensePlan(B, Hq, Hkv, S, S, D, dtype, cap=cap, prepare=prepare)
    else:
        plan = vb.LayerPlan(B, Hq, D, grid, (3, 5, 3), tau=1.0, dtype=dtype, q_in_place=True, prepare=prepare)
    O = plan.forward(Q, K, V).clone()
    grads = [*(t.clone() for t in plan.backward(dO)), prepare.dwq, prepare.dwk]
    ref, want = layer_reference(Q, K, V, wq, wk, dims, grid, norm, dO, cap)
    # The outputs of norm and rotation are rounded to the type (twice), weights, dz, O and the gradients once more each: six roundings, whose
    # relative errors add up in the 2-norm at worst
    bound = 6 * ou.HALF[dtype] if dtype == BF16 else 2e-5
    for name, got, value in zip(("O", "dQ", "dK", "dV", "dwq", "dwk"), [O] + grads, [ref] + want):
        rel = float((got.double() - value).norm() / value.norm())
        print(f"   {name}: relative error {rel:.2e} of {bound:.2e}", flush=True)
        assert rel <= bound, name


def test_a_token_against_a_cache_with_positions():
    """A step of serving: the new token's query and key are normalised and turned at its own position, the key joins the cache, and the query
    reads the cache as far as its sequence goes -- the same as the last row of the whole sequence."""
    B, Hq, Hkv, S, D = 2, 8, 2, 150, 64
    Q, K, V = ou.normal(1, (B, S, Hq + 2 * Hkv, D), BF16).split([Hq, Hkv, Hkv], 2)
    w = 1 + 0.1 * ou.normal(2, (D,), F32)
    args = dict(dims=[32], scaling=vb.ROPE_YARN, factor=4.0, train_len=64, wq=w, wk=w, need_bwd=False)
    whole = vb.QueryKeyPlan(B, Hq, Hkv, S, D, **args)
    q, k = whole.forward(Q, K)
    full = vb.DensePlan(B, Hq, Hkv, S, S, D, causal=True, need_bwd=False).forward(q, k, V)
    step = vb.QueryKeyPlan(B, Hq, Hkv, 1, D, **args)
    lens = [S, 83]
    at = int32([[n - 1] for n in lens])
    cache_k, cache_v = (torch.full((B, 256, Hkv, D), math.nan, dtype=BF16, device="cuda") for _ in range(2))
    for b, n in enumerate(lens):
        cache_k[b, :n], cache_v[b, :n] = k[b, :n], V[b, :n]
    qt, kt = step.forward(torch.stack([Q[b, n - 1:n] for b, n in enumerate(lens)]), torch.stack([K[b, n - 1:n] for b, n in enumerate(lens)]),
                          positions=at[:, :, None].contiguous())
    for b, n in enumerate(lens):
        assert torch.equal(kt[b, 0], k[b, n - 1])
        assert torch.equal(qt[b, 0], q[b, n - 1])
    plan = vb.DensePlan(B, Hq, Hkv, 1, 256, D, doc_off=int32([[0, n] for n in lens]), causal=True, need_bwd=False)
    got = plan.forward(qt, cache_k, cache_v, q_pos=at)
    for b, n in enumerate(lens):
        ref = ou.attention(q[b:b + 1, n - 1:n], k[b:b + 1, :n], V[b:b + 1, :n], int32([[0]]), int32([[n]]), None, 0.125)["O"]
        ou.within("token", got[b:b + 1], *ref)
        ou.within("row of the whole", full[b:b + 1, n - 1:n], *ref)


def test_rows_behind_the_last_sequence_stay_as_they_are():
    """Calls on a part of a larger buffer touch nothing outside it."""
    B, S, H, D, n = 1, 96, 2, 64, 61
    big = {k: torch.full((B, S, H, D), 7.0, dtype=BF16, device="cuda") for k in ("O", "dQ", "dK", "dV", "y", "r")}
    Q, K, V, dO = (ou.normal(i, (B, S, H, D), BF16) for i in range(4))
    part = {k: v[:, :n] for k, v in big.items()}
    lse = torch.empty(B, H, n, device="cuda")
    ws = torch.empty(max(vb.vmoba_dense_workspace_bytes(op, B, H, H, n, n, D, vb.VMOBA_BF16) for op in (2, 3)), dtype=torch.uint8, device="cuda")
    vb.vmoba_dense_fwd(B, H, H, n, n, D, Q[:, :n], K[:, :n], V[:, :n], part["O"], lse, ws, 0.125)
    vb.vmoba_dense_bwd(B, H, H, n, n, D, Q[:, :n], K[:, :n], V[:, :n], part["O"], lse, dO[:, :n], part["dQ"], part["dK"], part["dV"], ws, 0.125)
    vb.vmoba_rmsnorm_fwd(B, H, n, D, Q[:, :n], None, None, 1e-6, None, part["y"], None, None)
    freqs, _ = vb.vmoba_rope_freqs([64])
    vb.vmoba_rope(B, n, D, [Q[:, :n]], [part["r"]], freqs.cuda(), [64])
    for k, v in big.items():
        assert bool((v[:, n:] == 7.0).all()), k
        assert not bool((v[:, :n] == 7.0).all()), k
