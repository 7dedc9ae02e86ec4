"""What the calls of the int8 layers and of the routing by scores refuse, before anything is launched."""
import ctypes

import pytest

import paper_2405_18832_amd as moe

FAKE = 0x10000      # a non-null, 256-aligned address that is never dereferenced on these paths
ARG, UNS, WS = moe.MOE_ERR_INVALID_ARG, moe.MOE_ERR_UNSUPPORTED, moe.MOE_ERR_WORKSPACE
BIG = 1 << 40


def layer(**kw):
    a = dict(T=8, d_model=64, d_ff=64, E=16, k=4, dtype="bf16", renormalize=True)
    a.update(kw)
    return moe.make_shape(**a)


def refused(status, call, *args, **kw):
    with pytest.raises(moe.MoEError) as e:
        call(*args, stream=0, **kw)
    assert e.value.status == status


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(x=None)), (ARG, dict(w=None)), (ARG, dict(out=None)), (ARG, dict(x=FAKE + 1)), (ARG, dict(w=FAKE + 1)), (ARG, dict(bias=FAKE + 2)),
    (ARG, dict(out=FAKE + 2)), (ARG, dict(T=-1)), (ARG, dict(E=0)), (ARG, dict(d_model=0)), (ARG, dict(dtype=5)), (UNS, dict(E=1025)),
    (UNS, dict(d_model=40)), (UNS, dict(T=1 << 30)), (ARG, dict(dtype="f32", x=FAKE + 2)),
])
def test_gate_logits(status, kw):
    p = dict(x=FAKE, w=FAKE, bias=None, out=FAKE)
    p.update({k: kw.pop(k) for k in list(kw) if k in p})
    refused(status, moe.moe_gate_logits, layer(**kw), p["x"], p["w"], p["bias"], p["out"])


def test_gate_logits_of_no_tokens():
    moe.moe_gate_logits(layer(T=0), None, None, None, None, stream=0)


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(score=2)), (ARG, dict(score=-1)), (ARG, dict(groups=0)), (ARG, dict(groups=3)), (ARG, dict(groups=4, kept=0)),
    (ARG, dict(groups=4, kept=5)), (ARG, dict(groups=8, kept=1)),                  # two experts for k = 4
    (ARG, dict(top=0)), (ARG, dict(top=3)), (ARG, dict(groups=16, kept=16, top=2)),     # groups of one
    (ARG, dict(scale=float("nan"))), (ARG, dict(scale=float("inf"))), (UNS, dict(E=1024, groups=128, kept=128)),
    (ARG, dict(ldtype="e4m3")), (ARG, dict(ldtype="i8")), (ARG, dict(logits=None)), (ARG, dict(idx=None)), (ARG, dict(w=None)),
    (ARG, dict(counts=None)), (ARG, dict(offsets=None)), (ARG, dict(H=3)), (ARG, dict(logits=FAKE + 2)), (ARG, dict(ldtype="bf16", logits=FAKE + 1)),
    (ARG, dict(balance=FAKE + 2)), (ARG, dict(idx=FAKE + 2)), (ARG, dict(w=FAKE + 1)), (ARG, dict(counts=FAKE + 1)), (ARG, dict(offsets=FAKE + 2)),
    (WS, dict(ws=None)), (WS, dict(ws=FAKE + 128)), (WS, dict(ws_bytes=1)),
    (ARG, dict(k=17)), (UNS, dict(k=9)), (ARG, dict(k=0)), (ARG, dict(T=-1)), (UNS, dict(E=1025)), (UNS, dict(T=1 << 29)),
])
def test_route_logits(status, kw):
    p = dict(score=1, groups=1, kept=1, top=1, scale=1.0, ldtype="f32", logits=FAKE, balance=None, idx=FAKE, w=FAKE, counts=FAKE, offsets=FAKE, H=-1,
             hot=None, ws=FAKE, ws_bytes=BIG)
    p.update({k: kw.pop(k) for k in list(kw) if k in p})
    s, r = layer(**kw), moe.make_routing(p["score"], p["groups"], p["kept"], p["top"], p["scale"])
    lib = moe.load()
    assert lib.moe_route_logits(ctypes.byref(s), ctypes.byref(r), moe._DTYPE_NAMES[p["ldtype"]], p["logits"], p["balance"], p["idx"], p["w"], p["counts"],
                                p["offsets"], p["H"], p["hot"], p["ws"], p["ws_bytes"], None) == status
    assert lib.moe_route_logits(ctypes.byref(s), None, 0, FAKE, None, FAKE, FAKE, FAKE, FAKE, -1, None, FAKE, BIG, None) != moe.MOE_OK


@pytest.mark.parametrize("status,args", [
    (ARG, (0, 8, 8, "f32", FAKE, FAKE + 256, FAKE)), (ARG, (1, 0, 8, "f32", FAKE, FAKE + 256, FAKE)), (ARG, (1, 8, 0, "f32", FAKE, FAKE + 256, FAKE)),
    (UNS, (1025, 8, 8, "f32", FAKE, FAKE + 256, FAKE)), (UNS, (1, (1 << 24) + 1, 8, "f32", FAKE, FAKE + 256, FAKE)),
    (UNS, (1, 8, moe.MOE_INT_MAX_K + 1, "i8", FAKE, FAKE + 256, None)), (ARG, (1, 8, 8, "e4m3", FAKE, FAKE + 256, FAKE)),
    (ARG, (1, 8, 8, "f32", None, FAKE, FAKE)), (ARG, (1, 8, 8, "f32", FAKE, None, FAKE)), (ARG, (1, 8, 8, "bf16", FAKE, FAKE + 256, None)),
    (ARG, (1, 8, 8, "i8", FAKE, FAKE, None)), (ARG, (1, 8, 8, "i8", FAKE, FAKE + 8, None)), (ARG, (1, 8, 8, "f32", FAKE + 2, FAKE + 256, FAKE)),
    (ARG, (1, 8, 8, "f32", FAKE, FAKE + 256, FAKE + 2)),
])
def test_weights(status, args):
    refused(status, moe.moe_quantize_weights_int, *args)


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(rows=-1)), (ARG, dict(d=0)), (ARG, dict(dtype="i8")), (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))), (ARG, dict(eps=float("inf"))),
    (UNS, dict(d=(1 << 24) + 1)), (UNS, dict(rows=1 << 30)), (ARG, dict(x=None)), (ARG, dict(q=None)), (ARG, dict(scales=None)), (ARG, dict(x=FAKE + 1)),
    (ARG, dict(residual=FAKE + 1)), (ARG, dict(weight=FAKE + 2)), (ARG, dict(sum_out=FAKE + 1)), (ARG, dict(norm_out=FAKE + 1)), (ARG, dict(q=FAKE + 8)),
    (ARG, dict(scales=FAKE + 2)),
])
def test_norm(status, kw):
    a = dict(rows=4, d=64, dtype="bf16", x=FAKE, residual=None, weight=None, eps=1e-6, sum_out=None, norm_out=None, q=FAKE, scales=FAKE)
    a.update(kw)
    refused(status, moe.moe_norm_quantize_int, *a.values())


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(rows=-1)), (ARG, dict(f=0)), (ARG, dict(dtype="e4m3")), (ARG, dict(gated=2)), (ARG, dict(gated=-1)), (UNS, dict(act=3)), (UNS, dict(act=-2)),
    (UNS, dict(f=(1 << 24) + 1)), (UNS, dict(rows=1 << 30)), (ARG, dict(h=None)), (ARG, dict(q=None)), (ARG, dict(scales=None)), (ARG, dict(h=FAKE + 1)),
    (ARG, dict(q=FAKE + 4)), (ARG, dict(h=FAKE, q=FAKE)), (ARG, dict(scales=FAKE + 1)), (ARG, dict(mask=FAKE)), (ARG, dict(offsets=FAKE)),
    (UNS, dict(offsets=FAKE, E=1025)), (ARG, dict(offsets=FAKE + 1, E=4)),
])
def test_act(status, kw):
    a = dict(rows=4, f=64, dtype="bf16", h=FAKE + 4096, gated=0, act="silu", E=0, offsets=None, mask=None, q=FAKE, scales=FAKE)
    a.update(kw)
    refused(status, moe.moe_act_quantize_int, *a.values())


def product_args(**kw):
    a = dict(rows=8, N=64, K=64, E=4, k=2, act="none", out_dtype="bf16", a=FAKE, sa=FAKE, perm=None, offsets=FAKE, mask=None, w=FAKE, sw=FAKE, bias=None,
             out=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    return a


@pytest.mark.parametrize("status,kw", [
    (ARG, dict(rows=-2)), (ARG, dict(N=0)), (ARG, dict(K=0)), (ARG, dict(E=0)), (ARG, dict(k=0)), (ARG, dict(k=3)), (UNS, dict(k=9, rows=18)),
    (UNS, dict(E=1025)), (UNS, dict(K=moe.MOE_INT_MAX_K + 1)), (UNS, dict(N=(1 << 24) + 1)), (UNS, dict(rows=1 << 30)), (UNS, dict(rows=1 << 28, N=1 << 20)),
    (UNS, dict(act=5)), (ARG, dict(out_dtype="e4m3")), (ARG, dict(out_dtype="i8")), (ARG, dict(out_dtype=moe.MOE_BF16 | moe.MOE_QUANT_UNIT_SUMS)),
    (ARG, dict(a=None)), (ARG, dict(sa=None)), (ARG, dict(offsets=None)), (ARG, dict(w=None)), (ARG, dict(sw=None)), (ARG, dict(out=None)),
    (ARG, dict(a=FAKE + 8)), (ARG, dict(w=FAKE + 4)), (ARG, dict(out=FAKE + 1)), (ARG, dict(out_dtype="f32", out=FAKE + 2)), (ARG, dict(sa=FAKE + 1)),
    (ARG, dict(sw=FAKE + 2)), (ARG, dict(bias=FAKE + 2)), (ARG, dict(perm=FAKE + 2)), (ARG, dict(offsets=FAKE + 1)), (WS, dict(ws=None)),
    (WS, dict(ws=FAKE + 64)), (WS, dict(ws_bytes=0)),
])
def test_products(status, kw):
    a = product_args(**kw)
    s = moe.make_quant_shape(a["rows"], a["N"], a["K"], a["E"], a["k"], a["act"], a["out_dtype"])
    lib = moe.load()
    assert lib.moe_int_expert_linear(ctypes.byref(s), a["a"], a["sa"], a["perm"], a["offsets"], a["mask"], a["w"], a["sw"], a["bias"], a["out"], a["ws"],
                                     a["ws_bytes"], None) == status
    if not {"perm", "offsets", "E", "k"} & set(kw):
        s.E = s.k = 1
        assert lib.moe_int_linear(ctypes.byref(s), a["a"], a["sa"], a["w"], a["sw"], a["bias"], a["out"], a["ws"], a["ws_bytes"], None) == status
    if status == UNS or set(kw) & {"rows", "N", "K", "E", "k", "act", "out_dtype"} and "out" not in kw:
        assert moe.moe_int_workspace_bytes(moe.make_quant_shape(a["rows"], a["N"], a["K"], a["E"], a["k"], a["act"], a["out_dtype"])) == 0


def test_linear_takes_one_matrix():
    lib = moe.load()
    for kw in (dict(E=2), dict(k=2)):
        s = moe.make_quant_shape(8, 64, 64, **kw)
        assert lib.moe_int_linear(ctypes.byref(s), FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, BIG, None) == ARG
    assert lib.moe_int_linear(None, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, BIG, None) == ARG and lib.moe_int_workspace_bytes(None) == 0


def test_no_rows_and_workspaces():
    moe.moe_int_linear(moe.make_quant_shape(0, 64, 64), None, None, None, None, None, None, None, stream=0)
    moe.moe_int_expert_linear(moe.make_quant_shape(0, 64, 64, 4, 2), None, None, None, None, None, None, None, None, None, None, stream=0)
    moe.moe_norm_quantize_int(0, 64, "bf16", None, None, None, 0.0, None, None, None, None, stream=0)
    moe.moe_act_quantize_int(0, 64, "bf16", None, 1, "silu", 0, None, None, None, None, stream=0)
    for rows in (0, 1, 64, 65, 100000):
        n = moe.moe_int_workspace_bytes(moe.make_quant_shape(rows, 2048, 8192))
        assert n >= 256 and n % 256 == 0
