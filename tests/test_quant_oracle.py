"""The reference of the 8-bit layers against values worked out by hand, and the host side of their C ABI."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2405_18832_amd as moe
from oracle import quant_oracle as qo

FAKE = 0x1000      # a non-null, 256-aligned address that is never dereferenced on these paths


def test_code_values():
    v = qo.code_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6
    assert v[0x38] == 1.0 and v[0x39] == 1.125 and v[0x7e] == 448.0 and np.isnan(v[0x7f]) and v[0xb8] == -1.0
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, t, equal_nan=True)


def test_nearest():
    # between 1 and 1.125 the middle goes to the even mantissa (1), between 1.125 and 1.25 to 1.25; subnormal steps are 2^-9
    assert qo.nearest(np.array([1.0625, 1.1875, 1.07, 448.0, 460.0, -0.3])).tolist() == [1.0, 1.25, 1.125, 448.0, 448.0, -0.3125]
    assert qo.nearest(np.array([2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 0.0])).tolist() == [0.0, 2.0 ** -8, 0.0, 0.0]
    v = np.random.default_rng(1).standard_normal(10000) * 100
    v = np.clip(v, -448, 448)
    assert np.array_equal(qo.nearest(v), torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy())


def test_rows_by_hand():
    v = np.zeros((2, 130))
    v[0, 0], v[0, 1], v[0, 128], v[0, 129] = 896.0, 3.0, -1.0, 0.5
    q, s = qo.quantize_rows(v)
    assert s[0].tolist() == [2.0, 1 / 448] and s[1].tolist() == [qo.TINY] * 2
    assert q[0, :2].tolist() == [448.0, 1.5] and q[0, 128:].tolist() == [-448.0, 224.0] and not q[1].any()
    assert qo.dequantize_rows(q, s)[0, 129] == 0.5
    v[1, 5] = np.inf
    q, s = qo.quantize_rows(v)
    assert np.isnan(s[1, 0]) and np.isnan(q[1, :128]).all() and s[1, 1] == qo.TINY and not q[1, 128:].any()


def test_product_and_norm_by_hand():
    y, size = qo.linear(np.array([[1.0, -2.0]]), np.array([[3.0, 4.0], [1.0, 0.25]]), np.array([1.0, 0.0]), "relu")
    assert y.tolist() == [[0.0, 0.5]] and size.tolist() == [[12.0, 1.5]]
    assert np.allclose(qo.activate(np.array([1.0]), "gelu"), 0.8413447460685429)
    n = qo.norm(np.array([[3.0, 4.0]]), np.array([1.0, 2.0]), 0.0)
    assert np.allclose(n, [[3 / 12.5 ** 0.5, 8 / 12.5 ** 0.5]])


def test_pack_layout_by_hand():
    codes = np.arange(17 * 200, dtype=np.int64).reshape(17, 200).astype(np.uint8)
    p = qo.pack(codes)
    assert p.size == moe.moe_quant_weight_bytes(1, 17, 200) == 128 * 256
    # row 16, column 128 + 64 + 5 -> fragment (nb = 1, kb = 1), h = 1, g = 0, r = 0
    assert p[((1 * 2) + 1) * 2048 + 1024 + 5] == codes[16, 197]
    # row 3, column 37 -> fragment (0, 0), h = 0, g = 2
    assert p[16 * (2 * 16 + 3) + 5] == codes[3, 37]


def test_sizes():
    assert [moe.moe_quant_pitch(n) for n in (-1, 0, 1, 128, 129)] == [0, 0, 128, 128, 256]
    assert moe.moe_quant_weight_bytes(3, 128, 256) == 3 * 128 * 256
    assert moe.moe_quant_weight_bytes(0, 1, 1) == moe.moe_quant_weight_bytes(1025, 1, 1) == moe.moe_quant_weight_bytes(1, 1, 0) == 0
    assert moe.moe_quant_weight_bytes(1024, 1 << 24, 1 << 20) == 1 << 54          # 64-bit arithmetic
    s = moe.make_quant_shape(64, 128, 256, 8, 2, "relu", "e4m3")
    n = moe.moe_quant_workspace_bytes(s)
    assert n >= 256 and n % 256 == 0
    assert moe.moe_quant_workspace_bytes(moe.make_quant_shape(63, 128, 256, 8, 2)) == 0


def status(call, *args):
    return getattr(moe.load(), call)(*args)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), moe.MOE_ERR_INVALID_ARG), (dict(N=0), moe.MOE_ERR_INVALID_ARG), (dict(K=0), moe.MOE_ERR_INVALID_ARG),
    (dict(E=0), moe.MOE_ERR_INVALID_ARG), (dict(k=0), moe.MOE_ERR_INVALID_ARG), (dict(rows=5, k=2), moe.MOE_ERR_INVALID_ARG),
    (dict(out_dtype=3), moe.MOE_ERR_INVALID_ARG), (dict(activation=2), moe.MOE_ERR_UNSUPPORTED), (dict(E=1025), moe.MOE_ERR_UNSUPPORTED),
    (dict(k=9, rows=9), moe.MOE_ERR_UNSUPPORTED), (dict(N=(1 << 24) + 1), moe.MOE_ERR_UNSUPPORTED),
    (dict(K=(1 << 24) + 1), moe.MOE_ERR_UNSUPPORTED), (dict(rows=1 << 30), moe.MOE_ERR_UNSUPPORTED),
    (dict(rows=1 << 24, N=1 << 20), moe.MOE_ERR_UNSUPPORTED),
])
def test_bad_product_shapes(kw, want):
    base = dict(rows=4, N=128, K=128, E=2, k=1, activation="none", out_dtype="bf16")
    base.update(kw)
    s = moe.make_quant_shape(**base)
    assert moe.moe_quant_workspace_bytes(s) == 0
    assert status("moe_quant_expert_linear", ctypes.byref(s), FAKE, FAKE, None, FAKE, None, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 40, None) == want


def test_bad_product_arguments():
    s = moe.make_quant_shape(4, 128, 128, 2, 1, "none", "bf16")
    n = moe.moe_quant_workspace_bytes(s)
    good = dict(a=FAKE, sa=FAKE, perm=None, off=FAKE, mask=None, w=FAKE, sw=FAKE, bias=None, out=FAKE, so=None, ws=FAKE, n=n)

    def call(shape=s, **kw):
        v = dict(good, **kw)
        return status("moe_quant_expert_linear", ctypes.byref(shape) if shape is not None else None, *[v[k] for k in good], None)

    for name in ("a", "sa", "off", "w", "sw", "out"):
        assert call(**{name: None}) == moe.MOE_ERR_INVALID_ARG, name
    for name, by in (("a", 8), ("w", 8), ("out", 1), ("sa", 2), ("sw", 2), ("bias", 2), ("perm", 2), ("off", 2)):
        assert call(**{name: FAKE + by}) == moe.MOE_ERR_INVALID_ARG, name
    assert call(so=FAKE) == moe.MOE_ERR_INVALID_ARG                       # scales belong to a quantised output only
    assert call(shape=moe.make_quant_shape(4, 128, 128, 2, 1, "none", "e4m3")) == moe.MOE_ERR_INVALID_ARG      # which needs them
    assert call(ws=None) == moe.MOE_ERR_WORKSPACE and call(ws=FAKE + 16) == moe.MOE_ERR_WORKSPACE
    assert call(n=n - 1) == moe.MOE_ERR_WORKSPACE
    assert call(shape=None) == moe.MOE_ERR_INVALID_ARG
    # rows == 0: a no-op that needs no buffers
    empty = moe.make_quant_shape(0, 128, 128, 2, 1, "none", "bf16")
    assert call(shape=empty, a=None, sa=None, off=None, w=None, sw=None, out=None, ws=None, n=0) == moe.MOE_OK
    # the single product has one matrix and no assignments
    for E, k in ((2, 1), (1, 2)):
        t = moe.make_quant_shape(4, 128, 128, E, k)
        assert status("moe_quant_linear", ctypes.byref(t), FAKE, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 30, None) == moe.MOE_ERR_INVALID_ARG


def test_bad_norm_and_weight_arguments():
    def norm(rows=2, d=64, dtype=moe.MOE_BF16, x=FAKE, res=None, w=None, eps=1e-6, s=None, n=None, q=FAKE, sc=FAKE):
        return status("moe_norm_quantize", rows, d, dtype, x, res, w, eps, s, n, q, sc, None)

    for kw in (dict(rows=-1), dict(d=0), dict(dtype=2), dict(dtype=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(x=None), dict(q=None), dict(sc=None), dict(x=FAKE + 1), dict(res=FAKE + 1), dict(s=FAKE + 1), dict(n=FAKE + 1),
               dict(w=FAKE + 2), dict(q=FAKE + 8), dict(sc=FAKE + 2), dict(dtype=moe.MOE_F32, x=FAKE + 2)):
        assert norm(**kw) == moe.MOE_ERR_INVALID_ARG, kw
    assert norm(d=(1 << 24) + 1) == moe.MOE_ERR_UNSUPPORTED
    assert norm(rows=0, x=None, q=None, sc=None) == moe.MOE_OK

    def weights(E=1, N=8, K=8, dtype=moe.MOE_F32, src=FAKE, dst=2 * FAKE, sc=FAKE):
        return status("moe_quantize_weights", E, N, K, dtype, src, dst, sc, None)

    for kw in (dict(E=0), dict(N=0), dict(K=-1), dict(dtype=3), dict(src=None), dict(dst=None), dict(dst=FAKE), dict(sc=None),
               dict(dst=2 * FAKE + 8), dict(src=FAKE + 2), dict(sc=FAKE + 2)):
        assert weights(**kw) == moe.MOE_ERR_INVALID_ARG, kw
    assert weights(E=1025) == moe.MOE_ERR_UNSUPPORTED


def test_binding_refuses_other_layouts():
    t = torch.zeros((4, 128))
    with pytest.raises(ValueError, match="CUDA"):
        moe.moe_norm_quantize(4, 128, "f32", t, None, None, 1e-6, None, None, t, t)


def test_sums_are_the_callers_choice():
    """fp32 unless MOE_QUANT_UNIT_SUMS is asked for, which fp32 outputs refuse."""
    assert moe.make_quant_shape(4, 128, 128, out_dtype="e4m3").out_dtype == moe.MOE_E4M3
    for out, value in (("bf16", moe.MOE_BF16), ("e4m3", moe.MOE_E4M3)):
        s = moe.make_quant_shape(4, 128, 128, out_dtype=out, sums="units")
        assert s.out_dtype == value | moe.MOE_QUANT_UNIT_SUMS
        assert moe.moe_quant_workspace_bytes(s) == moe.moe_quant_workspace_bytes(moe.make_quant_shape(4, 128, 128, out_dtype=out)) > 0
    s = moe.make_quant_shape(4, 128, 128, out_dtype="f32", sums="units")
    assert moe.moe_quant_workspace_bytes(s) == 0
    assert status("moe_quant_linear", ctypes.byref(s), FAKE, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 30, None) == moe.MOE_ERR_INVALID_ARG
    # a quantised output still needs its scales, a bf16 one takes none
    for out, scales in (("e4m3", None), ("bf16", FAKE)):
        s = moe.make_quant_shape(4, 128, 128, out_dtype=out, sums="units")
        assert status("moe_quant_linear", ctypes.byref(s), FAKE, FAKE, FAKE, FAKE, None, FAKE, scales, FAKE, 1 << 30, None) == moe.MOE_ERR_INVALID_ARG
    with pytest.raises(KeyError):
        moe.make_quant_shape(4, 128, 128, sums="bf16")


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("E", [1, 2, 1024])
@pytest.mark.parametrize("N,K", [(1, 1), (256, 256), (2048, 8192)])
def test_workspace_of_no_rows(N, K, E, out):
    """A call without rows is a no-op, and its size query answers."""
    s = moe.make_quant_shape(0, N, K, E, 1, "none", out)
    assert moe.moe_quant_workspace_bytes(s) == 256
    assert status("moe_quant_expert_linear", ctypes.byref(s), None, None, None, None, None, None, None, None, None, None, None, 0, None) == moe.MOE_OK
