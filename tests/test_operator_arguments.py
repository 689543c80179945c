"""What the calls around the sparse layer refuse, on the CPU: nothing is launched."""
import ctypes as C
import math

import pytest
import torch

from paper_2506_23858_amd import binding as vb

OK, INVALID, UNSUPPORTED, WORKSPACE = vb.VMOBA_OK, vb.VMOBA_ERR_INVALID_ARG, vb.VMOBA_ERR_UNSUPPORTED, vb.VMOBA_ERR_WORKSPACE
P = 4096                                    # an aligned address that nothing reads


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(vb.LIB_PATH):
        from paper_2506_23858_amd import build
        build.build_lib(verbose=False)
    return vb.lib()


def desc(ptr=P, dtype=vb.VMOBA_BF16, b=1 << 20, s=1024, h=64):
    return bytes(vb.vmoba_tensor(ptr, dtype, b, s, h))


def ints(*v):
    return (C.c_int32 * max(1, len(v)))(*v)


# ------------------------------------------------------------------------------------------------------------------ frequencies
def test_frequencies_follow_their_definitions():
    f, m = vb.vmoba_rope_freqs([8, 4], base=100.0)
    assert m == 1.0 and f.tolist() == pytest.approx([100.0 ** (-i / 4) for i in range(4)] + [1.0, 0.1], rel=1e-15)
    assert vb.vmoba_rope_freqs([8], 100.0, vb.ROPE_LINEAR, 4.0)[0].tolist() == pytest.approx([x / 4 for x in f[:4].tolist()], rel=1e-15)
    assert vb.vmoba_rope_freqs([8], 100.0, vb.ROPE_NTK, 4.0)[0].tolist() == pytest.approx([(100.0 * 4.0 ** (8 / 6)) ** (-i / 4) for i in range(4)], rel=1e-14)
    y, m = vb.vmoba_rope_freqs([64], 1e4, vb.ROPE_YARN, 8.0, 4096)
    plain = vb.vmoba_rope_freqs([64], 1e4)[0]
    assert m == pytest.approx(0.1 * math.log(8.0) + 1.0, rel=1e-7)
    for i in range(32):
        turns = 4096 * float(plain[i]) / (2 * math.pi)
        g = min(1.0, max(0.0, (turns - 1.0) / 31.0))
        assert float(y[i]) == pytest.approx(float(plain[i]) * (g + (1 - g) / 8.0), rel=1e-14)
    assert float(y[0]) == float(plain[0]) and float(y[31]) == float(plain[31]) / 8.0


@pytest.mark.parametrize("dims,base,scaling,factor,train,want", [
    ([], 1e4, 0, 1.0, 0, INVALID), ([2, 2, 2, 2], 1e4, 0, 1.0, 0, INVALID), ([3], 1e4, 0, 1.0, 0, INVALID), ([0], 1e4, 0, 1.0, 0, INVALID), ([-2], 1e4, 0, 1.0, 0, INVALID),
    ([2000], 1e4, 0, 1.0, 0, INVALID), ([8], 0.0, 0, 1.0, 0, INVALID), ([8], math.inf, 0, 1.0, 0, INVALID), ([8], 1e4, 1, 0.5, 0, INVALID), ([8], 1e4, 1, math.nan, 0, INVALID),
    ([8], 1e4, 4, 1.0, 0, UNSUPPORTED), ([8], 1e4, 3, 2.0, 0, INVALID), ([8, 2], 1e4, 2, 2.0, 0, INVALID)])
def test_frequencies_refuse(dims, base, scaling, factor, train, want):
    with pytest.raises(vb.VmobaError) as e:
        vb.vmoba_rope_freqs(dims, base, scaling, factor, train)
    assert e.value.code == want


# ------------------------------------------------------------------------------------------------------------------ rotary positions
ROPE = dict(B=1, S=8, D=64, n=1, heads=(2,), ins=None, outs=None, freqs=P, axes=1, dims=(64,), layout=0, inverse=0, mscale=1.0, grid=None, first=0, pos=None)


def rope(L, **change):
    a = dict(ROPE, **change)
    ins, outs = (b"".join(a[k] or [desc()] * a["n"]) for k in ("ins", "outs"))
    return L.vmoba_rope(a["B"], a["S"], a["D"], a["n"], ints(*a["heads"]) if a["heads"] else None, ins, outs, a["freqs"], a["axes"], ints(*a["dims"]),
                        a["layout"], a["inverse"], a["mscale"], a["grid"], a["first"], a["pos"], 0, None)


@pytest.mark.parametrize("change,want", [
    (dict(S=0), OK), (dict(B=0), OK), (dict(B=-1), INVALID), (dict(S=-1), INVALID), (dict(n=0), INVALID), (dict(n=9, heads=(1,) * 9), INVALID), (dict(heads=None), INVALID),
    (dict(heads=(0,)), INVALID), (dict(freqs=None), INVALID), (dict(D=63), UNSUPPORTED), (dict(D=0), UNSUPPORTED), (dict(D=2048), UNSUPPORTED), (dict(dims=(66,)), INVALID),
    (dict(dims=(63,)), INVALID), (dict(axes=0), INVALID), (dict(axes=4, dims=(2, 2, 2, 2)), INVALID), (dict(axes=2, dims=(2, 2)), INVALID), (dict(layout=2), UNSUPPORTED),
    (dict(inverse=2), INVALID), (dict(mscale=math.nan), INVALID), (dict(ins=[desc(P + 8)]), INVALID), (dict(ins=[desc(dtype=vb.VMOBA_F8E4M3)]), INVALID),
    (dict(ins=[desc(dtype=vb.VMOBA_F32)]), UNSUPPORTED), (dict(outs=[desc(s=1028)]), INVALID), (dict(outs=[desc(s=2048)]), INVALID), (dict(ins=[desc(None)]), INVALID),
    (dict(axes=3, dims=(2, 2, 2)), INVALID), (dict(axes=3, dims=(2, 2, 2), grid=vb.make_grid(2, 2, 3)), INVALID),
    (dict(axes=3, dims=(2, 2, 2), grid=vb.make_grid(2, 0, 3)), INVALID)])
def test_rope_refuses(L, change, want):
    assert rope(L, **change) == want


# ------------------------------------------------------------------------------------------------------------------ norms
FWD = dict(B=1, Hh=2, S=4, D=64, x=desc(), residual=None, weight=P, wtype=vb.VMOBA_F32, eps=1e-6, total=None, y=desc(), y_scale=None, inv=None)


@pytest.mark.parametrize("change,want", [
    (dict(S=0), OK), (dict(B=0), OK), (dict(B=-1), INVALID), (dict(Hh=0), INVALID), (dict(D=0), INVALID), (dict(D=16385), UNSUPPORTED), (dict(S=1 << 31), UNSUPPORTED),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(x=desc(None)), INVALID), (dict(x=desc(P + 1)), INVALID), (dict(x=desc(dtype=5)), INVALID),
    (dict(x=desc(dtype=vb.VMOBA_F8E4M3)), INVALID), (dict(y=desc(dtype=vb.VMOBA_F32)), UNSUPPORTED), (dict(residual=desc()), INVALID), (dict(total=desc()), INVALID),
    (dict(residual=desc(), total=desc(dtype=vb.VMOBA_F32)), INVALID), (dict(y=desc(dtype=vb.VMOBA_F8E4M3)), INVALID), (dict(y_scale=P), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=math.nan), INVALID), (dict(weight=P + 2), INVALID), (dict(wtype=vb.VMOBA_F8E4M3), INVALID)])
def test_norm_refuses(L, change, want):
    a = dict(FWD, **change)
    assert L.vmoba_rmsnorm_fwd(a["B"], a["Hh"], a["S"], a["D"], a["x"], a["residual"], a["weight"], a["wtype"], a["eps"], a["total"], a["y"], a["y_scale"],
                               a["inv"], None) == want


BWD = dict(B=1, Hh=2, S=4, D=64, x=desc(), weight=P, wtype=vb.VMOBA_F32, inv=P, dy=desc(), dtotal=None, dx=desc(), dweight=P, ws=P, size=1 << 20)


@pytest.mark.parametrize("change,want", [
    (dict(S=0, dweight=None), OK), (dict(D=0), INVALID), (dict(x=None), INVALID), (dict(dy=None), INVALID), (dict(dx=None), INVALID), (dict(inv=None), INVALID),
    (dict(dy=desc(dtype=vb.VMOBA_F32)), INVALID), (dict(dtotal=desc(dtype=vb.VMOBA_F32)), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 4), INVALID),
    (dict(size=8 * 64 * 4 - 1), WORKSPACE), (dict(weight=P + 1), INVALID)])
def test_norm_gradient_refuses(L, change, want):
    a = dict(BWD, **change)
    assert L.vmoba_rmsnorm_bwd(a["B"], a["Hh"], a["S"], a["D"], a["x"], a["weight"], a["wtype"], a["inv"], a["dy"], a["dtotal"], a["dx"], a["dweight"], a["ws"],
                               a["size"], None) == want


# ------------------------------------------------------------------------------------------------------------------ dense attention
@pytest.mark.parametrize("change,want", [
    (dict(B=0), INVALID), (dict(Sq=0), INVALID), (dict(Sk=-1), INVALID), (dict(lo=None), INVALID), (dict(hi=None), INVALID), (dict(hi=P), INVALID), (dict(causal=2), INVALID),
    (dict(docs=0), INVALID), (dict(docs=2), INVALID), (dict(doc=P, docs=0), INVALID), (dict(doc=P, stride=-1), INVALID), (dict(prefix=P, causal=0), INVALID),
    (dict(first=1 << 31), INVALID), (dict(Sq=1 << 31), UNSUPPORTED)])
def test_key_ranges_refuse(L, change, want):
    a = dict(dict(B=1, Sq=4, Sk=4, doc=None, stride=0, docs=1, prefix=None, causal=1, q_pos=None, first=0, lo=P, hi=2 * P), **change)
    assert L.vmoba_key_ranges(a["B"], a["Sq"], a["Sk"], a["doc"], a["stride"], a["docs"], a["prefix"], 0, a["causal"], a["q_pos"], a["first"], a["lo"], a["hi"], None) == want


DENSE = dict(B=1, Hq=4, Hkv=2, Sq=8, Sk=8, D=64, Q=desc(), K=desc(), V=desc(), scale=0.125, cap=0.0, lo=None, hi=None, first=0, O=desc(), LSE=P, dO=desc(), dQ=desc(),
             dK=desc(), dV=desc(), ws=P, size=1 << 30)
BOTH = [
    (dict(B=0), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID), (dict(Hkv=3), INVALID), (dict(Sq=0), INVALID), (dict(Sk=0), INVALID), (dict(D=96), UNSUPPORTED),
    (dict(Sk=1 << 24), UNSUPPORTED), (dict(Sq=1 << 23), UNSUPPORTED), (dict(Q=None), INVALID), (dict(K=desc(P + 8)), INVALID), (dict(V=desc(s=1001)), INVALID),
    (dict(K=desc(dtype=vb.VMOBA_F32)), UNSUPPORTED), (dict(O=desc(dtype=vb.VMOBA_F32)), UNSUPPORTED), (dict(Q=desc(dtype=vb.VMOBA_F8E4M3)), INVALID), (dict(K=desc(s=-1024)), UNSUPPORTED),
    (dict(K=desc(s=1 << 22)), UNSUPPORTED), (dict(Sk=1 << 22, K=desc(s=1 << 10)), UNSUPPORTED), (dict(scale=math.nan), INVALID), (dict(cap=-1.0), INVALID), (dict(cap=math.inf), INVALID), (dict(cap=4097.0), UNSUPPORTED),
    (dict(lo=P), INVALID), (dict(hi=P), INVALID), (dict(first=1 << 31), INVALID), (dict(LSE=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 16), INVALID), (dict(size=255), WORKSPACE)]


def scores(a):
    return vb.vmoba_scores(a["scale"], a["cap"], None, a["lo"], a["hi"], None, a["first"])


@pytest.mark.parametrize("change,want", BOTH)
def test_dense_forward_refuses(L, change, want):
    a = dict(DENSE, **change)
    size = tuple(a[k] for k in ("B", "Hq", "Hkv", "Sq", "Sk", "D"))
    assert L.vmoba_dense_fwd(*size, a["Q"], a["K"], a["V"], scores(a), a["O"], a["LSE"], a["ws"], a["size"], None) == want


@pytest.mark.parametrize("change,want", BOTH + [
    (dict(dO=None), INVALID), (dict(dQ=desc(dtype=vb.VMOBA_F32)), UNSUPPORTED), (dict(dK=desc(P + 2)), INVALID), (dict(dO=desc(h=-64)), UNSUPPORTED), (dict(Q=desc(s=-64)), UNSUPPORTED)])
def test_dense_gradient_refuses(L, change, want):
    a = dict(DENSE, **change)
    size = tuple(a[k] for k in ("B", "Hq", "Hkv", "Sq", "Sk", "D"))
    assert L.vmoba_dense_bwd(*size, a["Q"], a["K"], a["V"], scores(a), a["O"], a["LSE"], a["dO"], a["dQ"], a["dK"], a["dV"], a["ws"], a["size"], None) == want


def test_workspace_sizes(L):
    size = vb.vmoba_dense_workspace_bytes
    assert size(vb.OP_ATTN_FWD, 1, 4, 3, 8, 8, 64, 1) == size(vb.OP_ATTN_FWD, 1, 4, 2, 8, 8, 65, 1) == size(vb.OP_SELECT, 1, 4, 2, 8, 8, 64, 1) == size(vb.OP_ATTN_FWD, 1, 4, 2, 8, 8, 64, 7) == 0
    # one query against a long cache is split; a whole sequence of many tiles is not
    assert size(vb.OP_ATTN_FWD, 1, 4, 2, 1, 8192, 64, 1) > 4 * 64 * 4 * 2
    assert size(vb.OP_ATTN_FWD, 1, 16, 16, 8192, 8192, 64, 1) < 1 << 20
    # 1 KB of row information per 32 rows
    assert size(vb.OP_ATTN_BWD, 1, 16, 16, 8192, 8192, 64, 1) >= 16 * 256 * 1024
    assert vb.vmoba_rmsnorm_workspace_bytes(1, 1, 5, 128) == 5 * 128 * 4 and vb.vmoba_rmsnorm_workspace_bytes(1, 1, 5, 0) == 0
    assert vb.vmoba_rmsnorm_workspace_bytes(1, 12, 1 << 20, 128) <= 1024 * 128 * 4


def test_the_binding_checks_shapes_devices_and_types():
    x = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: vb.vmoba_rope(1, 4, 64, [x], [x], torch.zeros(32, dtype=torch.float64), [64]),
                 lambda: vb.vmoba_rmsnorm_fwd(1, 2, 4, 64, x, None, None, 1e-6, None, x, None, None),
                 lambda: vb.vmoba_rmsnorm_bwd(1, 2, 4, 64, x, None, torch.zeros(1, 4, 2), x, None, x, None, None),
                 lambda: vb.vmoba_key_ranges(1, 4, 4, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)),
                 lambda: vb.vmoba_dense_fwd(1, 2, 2, 4, 4, 64, x, x, x, x, torch.zeros(1, 2, 4), torch.zeros(256, dtype=torch.uint8), 0.125)):
        with pytest.raises(ValueError, match="not on the current GPU"):
            call()
    with pytest.raises(ValueError, match="shape"):
        vb._shaped("x", x, (1, 4, 2, 32))
    with pytest.raises(ValueError, match="contiguous"):
        vb._packed_array(torch.zeros(4, 4)[:, 0], "lse", torch.float32)
    with pytest.raises(ValueError, match="contiguous"):
        vb._packed_array(torch.zeros(4, dtype=torch.float64), "lse", torch.float32)
    assert vb._packed_array(None, "lse", torch.float32) is None
