"""The 4-bit page format and the norm and rotation, without a GPU: the oracle's
parts against independent statements of the rules, and the refusals of the
entry points (all made on the host, before any HIP call)."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

from oracle import kv4, rope
from paper_2510_15330_amd import _binding as B
from tests.test_abi import ERR_INVALID, ERR_UNSUPPORTED, FAKE, t


def test_every_code_and_scale():
    vals = [0, .5, 1, 1.5, 2, 3, 4, 6]
    assert [kv4.code_value(c) for c in range(16)] == vals + [-v for v in vals]
    assert kv4.scale_value(127) == 1 and kv4.scale_value(0) == 2.0 ** -127 and kv4.scale_value(254) == 2.0 ** 127
    assert np.isnan(kv4.scale_value(255))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["k", "v"])
def test_every_nibble_of_a_tile_is_one_value(D, kind):
    byte, nib, sc = kv4.offsets(D, kind)
    assert sorted((2 * byte + nib).ravel()) == list(range(16 * D))
    assert sorted(set(sc.ravel())) == list(range(8 * D, 8 * D + D // 2))
    # one scale byte for each (slot, 32 dims)
    assert all(len(set(sc[s, 32 * b:32 * b + 32])) == 1 for s in range(16) for b in range(D // 32))


def test_quantisation_rule():
    def block(*v):
        return np.array(list(v) + [0.0] * (32 - len(v)))
    c, e = kv4.quantize(block(6, 5, 2.5, 3.5, .25, .75, 1.25, 1.75, -0.0, -5))
    assert list(e) == [127]
    # ties to the even code: 5 -> 4, 2.5 -> 2, 3.5 -> 4, .25 -> 0, .75 -> 1, 1.25 -> 1, 1.75 -> 2
    assert list(c[:10]) == [7, 6, 4, 6, 0, 2, 2, 4, 8, 14]
    assert list(kv4.quantize(block(7.0))[1]) == [127] and kv4.quantize(block(7.0))[0][0] == 7      # saturates to 6
    assert list(kv4.quantize(block(7.0625))[1]) == [128] and kv4.quantize(block(7.0625))[0][0] == 6  # 4 * 2
    assert list(kv4.quantize(block(4.0))[1]) == [127] and list(kv4.quantize(block(3.96875))[1]) == [127]
    assert list(kv4.quantize(block())[1]) == [0]
    big = float(torch.finfo(torch.bfloat16).max)
    c, e = kv4.quantize(block(big))
    assert list(e) == [252] and c[0] == 7
    for bad in (np.nan, np.inf, -np.inf):
        c, e = kv4.quantize(block(1.0, bad))
        assert list(e) == [255] and not c.any()
    tiny = 2.0 ** -133
    assert list(kv4.quantize(block(tiny))[1]) == [0]


def test_quantisation_error_is_half_a_step():
    x = np.random.default_rng(0).standard_normal((500, 64)) * 10.0 ** np.random.default_rng(1).uniform(-20, 20, (500, 1))
    c, e = kv4.quantize(x)
    y = kv4.dequantize(c, e)
    unit = np.repeat(kv4.scale_value(e), 32, -1)
    mag = np.abs(x) / unit
    step = np.where(mag < 2, .5, np.where(mag < 4, 1, 2))
    assert (np.abs(x - y) <= 0.5 * step * unit).all()
    assert (mag <= 7).all()


@pytest.mark.parametrize("D", [64, 128])
def test_rows_written_are_rows_read(D):
    rng = np.random.default_rng(D)
    pools = [rng.integers(0, 256, (5, 3, 17, D // 2), dtype=np.uint8) for _ in range(2)]
    before = [p.copy() for p in pools]
    table = np.array([[3, 1], [4, 0]], dtype=np.int32)
    lens = np.array([10, 0], dtype=np.int32)
    rows = [rng.standard_normal((12 + 7, 3, D)) for _ in range(2)]
    kv4.write(*pools, *rows, table, lens, [12, 7])
    assert list(lens) == [22, 7]
    for pool, old, x, kind in zip(pools, before, rows, "kv"):
        want = kv4.dequantize(*kv4.quantize(x))
        with np.errstate(all="ignore"):
            got0, got1 = kv4.read_pages(pool, table[0], kind), kv4.read_pages(pool, table[1, :1], kind)
            was = kv4.read_pages(old, table[0], kind)
        assert np.array_equal(got0[10:22], want[:12]) and np.array_equal(got1[:7], want[12:])
        assert np.array_equal(got0[:10], was[:10], equal_nan=True) and np.array_equal(got0[22:], was[22:], equal_nan=True)
        assert np.array_equal(pool[2], old[2]) and np.array_equal(pool[0], old[0])


def test_oracle_attention_is_the_dense_softmax():
    from tests._dense import dense_attention
    rng = np.random.default_rng(5)
    D, H, G = 64, 2, 3
    pools = [np.zeros((4, H, 17, D // 2), dtype=np.uint8) for _ in range(2)]
    table, lens = np.array([[2, 0]], dtype=np.int32), np.array([0], dtype=np.int32)
    k, v = rng.standard_normal((21, H, D)), rng.standard_normal((21, H, D))
    kv4.write(*pools, k, v, table, lens, [21])
    q = rng.standard_normal((4, H * G, D))
    out, mag, dot = kv4.attention(q, *pools, table, lens, [4], 0.125)
    kd, vd = (kv4.dequantize(*kv4.quantize(x)) for x in (k, v))
    for i in range(4):
        ref = dense_attention(q[i], kd[:18 + i], vd[:18 + i], 0.125)
        assert np.abs(out[i] - ref).max() < 1e-12
    assert (mag >= np.abs(out) - 1e-12).all() and (dot > 0).all()


def test_oracle_rotation_against_complex_numbers():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((5, 2, 64))
    inv = 10.0 ** rng.uniform(-4, 0, 16)
    pos = rng.integers(0, 1000, (2, 5))
    for inter in (False, True):
        y = rope.rotate(x, pos, inv, (6, 10), inter)
        a = np.concatenate([pos[0][:, None] * inv[:6], pos[1][:, None] * inv[6:]], 1)[:, None]
        i, j = (np.arange(0, 32, 2), np.arange(1, 32, 2)) if inter else (np.arange(16), np.arange(16, 32))
        z = (x[..., i] + 1j * x[..., j]) * np.exp(1j * a)
        assert np.abs(y[..., i] - z.real).max() < 1e-12 and np.abs(y[..., j] - z.imag).max() < 1e-12
        assert np.array_equal(y[..., 32:], x[..., 32:])


# --------------------------------------------------------------- refusals --

def good4(Bsz=4, D=128, Hq=32, H=8, T=20):
    g = dict(q=t(B.BF16, [Bsz, Hq, D]), k=t(B.FP4_E2M1, [100, H, 17, D // 2]), v=t(B.FP4_E2M1, [100, H, 17, D // 2]),
             bt=t(B.INT32, [Bsz, 10]), sl=t(B.INT32, [Bsz]), out=t(B.BF16, [Bsz, Hq, D]),
             kn=t(B.BF16, [Bsz, H, D]), vn=t(B.BF16, [Bsz, H, D]), qs=t(B.INT32, [Bsz + 1]),
             kt=t(B.BF16, [T, H, D]), vt=t(B.BF16, [T, H, D]), qt=t(B.BF16, [T, Hq, D]), ot=t(B.BF16, [T, Hq, D]))
    return g


def opts(**kw):
    o = B.AttnOpts()
    for k, v in kw.items():
        setattr(o, k, v)
    return ctypes.byref(o)


CALLS = {
    "append": lambda L, g: L.bellman_kv_append(g["kn"], g["vn"], g["k"], g["v"], g["bt"], g["sl"], None),
    "write": lambda L, g: L.bellman_kv_write(g["kt"], g["vt"], g["k"], g["v"], g["bt"], g["sl"], g["qs"], None),
    "read": lambda L, g: L.bellman_kv_read(g["k"], g["v"], g["bt"], g["sl"], g["qs"], g["kt"], g["vt"], None),
    "decode": lambda L, g: L.bellman_decode_attention_opts(g["q"], g["k"], g["v"], g["bt"], g["sl"], 0.1, g["out"],
                                                           g.get("opts"), None),
    "step": lambda L, g: L.bellman_decode_step(g["kn"], g["vn"], g["q"], g["k"], g["v"], g["bt"], g["sl"], 0.1,
                                               g["out"], g.get("opts"), None),
    "prefill": lambda L, g: L.bellman_prefill_attention(g["qt"], g["k"], g["v"], g["bt"], g["sl"], g["qs"], 0.1,
                                                        g["ot"], None),
}
EVERY = list(CALLS)
REFUSED = [
    (EVERY, "16 rows", dict(k=t(B.FP4_E2M1, [100, 8, 16, 64])), ERR_INVALID, "rows a tile"),
    (EVERY, "V differs", dict(v=t(B.FP4_E2M1, [100, 4, 17, 64])), ERR_INVALID, "v_pages"),
    (EVERY, "V of fp8", dict(v=t(B.FP8_E4M3FN, [100, 8, 17, 64])), ERR_INVALID, "v_pages: dtype"),
    (EVERY, "head_dim 96", dict(k=t(B.FP4_E2M1, [100, 8, 17, 48]), v=t(B.FP4_E2M1, [100, 8, 17, 48])),
     ERR_UNSUPPORTED, "head_dim 96"),
    (EVERY, "no pages", dict(k=t(B.FP4_E2M1, [0, 8, 17, 64]), v=t(B.FP4_E2M1, [0, 8, 17, 64])), ERR_INVALID, "no pages"),
    (EVERY, "five dims", dict(k=t(B.FP4_E2M1, [100, 8, 4, 16, 16])), ERR_INVALID, "expected 4 dims"),
    (EVERY, "strided pool", dict(k=t(B.FP4_E2M1, [100, 8, 17, 64], [20000, 1088, 64, 1])), ERR_UNSUPPORTED, "contiguous"),
    (EVERY, "unaligned pool", dict(v=t(B.FP4_E2M1, [100, 8, 17, 64], data=FAKE + 8)), ERR_UNSUPPORTED, "16-byte"),
    (EVERY, "scales given", dict(k=t(B.FP4_E2M1, [100, 8, 17, 64], scale=FAKE)), ERR_INVALID, "dequant_scale"),
    (["append", "step"], "packed rows", dict(kn=t(B.FP4_E2M1, [4, 8, 128])), ERR_INVALID, "k_new: dtype"),
    (["append", "step"], "head mismatch", dict(vn=t(B.BF16, [4, 4, 128])), ERR_INVALID, "v_new: shape"),
    (["write"], "fp8 rows", dict(kt=t(B.FP8_E4M3FN, [20, 8, 128])), ERR_INVALID, "k_new: dtype"),
    (["read"], "fp32 rows", dict(kt=t(B.FP32, [20, 8, 128])), ERR_INVALID, "k_out: dtype"),
    (["read"], "unaligned rows", dict(vt=t(B.BF16, [20, 8, 128], data=FAKE + 8)), ERR_UNSUPPORTED, "v_out"),
    (["read", "write"], "q_start", dict(qs=t(B.INT32, [4])), ERR_INVALID, "q_start"),
    (["decode", "step"], "one page a step", dict(opts=opts(pages_per_step=1)), ERR_UNSUPPORTED, "pages_per_step"),
    (["decode", "step"], "eight pages a step", dict(opts=opts(pages_per_step=8)), ERR_UNSUPPORTED, "pages_per_step"),
    (["decode", "step"], "two steps ahead", dict(opts=opts(pipeline_depth=2)), ERR_UNSUPPORTED, "pipeline_depth"),
    (EVERY, "too many heads", dict(k=t(B.FP4_E2M1, [1, 70000, 17, 64]), v=t(B.FP4_E2M1, [1, 70000, 17, 64])),
     ERR_UNSUPPORTED, "65535"),
    (["decode", "step"], "queries of 4 bits", dict(q=t(B.FP4_E2M1, [4, 32, 128])), ERR_INVALID, "q: dtype"),
    (["decode", "step"], "group of 32", dict(q=t(B.BF16, [4, 256, 128]), out=t(B.BF16, [4, 256, 128])), ERR_UNSUPPORTED,
     "group"),
]


@pytest.mark.parametrize("call,change,code,text",
                         [(c, ch, code, text) for cs, _, ch, code, text in REFUSED for c in cs],
                         ids=[f"{c}-{n}" for cs, n, *_ in REFUSED for c in cs])
def test_refusals(call, change, code, text):
    L = B.library()
    assert CALLS[call](L, {**good4(), **change}) == code
    assert text in B.last_error(), B.last_error()


def test_empty_batches_are_nothing():
    L = B.library()
    g = good4(Bsz=0, T=0)
    for name in EVERY:
        assert CALLS[name](L, g) == 0, (name, B.last_error())


def test_fp8_read_needs_scales():
    g = good4()
    g.update(k=t(B.FP8_E4M3FN, [100, 8, 8, 16, 16]), v=t(B.FP8_E4M3FN, [100, 8, 128, 16]))
    assert CALLS["read"](B.library(), g) == ERR_INVALID and "dequant_scale" in B.last_error()


def rope_args(T=6, Hq=4, H=2, D=128, F=64, axes=1):
    return dict(q=t(B.BF16, [T, Hq, D]), k=t(B.BF16, [T, H, D]), qw=t(B.BF16, [D]), kw=t(B.FP32, [D]),
                pos=t(B.INT32, [T] if axes == 1 else [axes, T]), inv=t(B.FP32, [F]), qo=t(B.BF16, [T, Hq, D]),
                ko=t(B.BF16, [T, H, D]), o=B.RopeOpts(1e-6, 0.0, 0, axes))


def call_rope(a):
    return B.library().bellman_qk_norm_rope(a["q"], a["k"], a["qw"], a["kw"], a["pos"], a["inv"], a["qo"], a["ko"],
                                            None if a["o"] is None else ctypes.byref(a["o"]), None)


def sect(*s, axes=None, **kw):
    o = B.RopeOpts(1e-6, 0.0, 0, axes or len(s))
    for i, n in enumerate(s):
        o.sections[i] = n
    for k, v in kw.items():
        setattr(o, k, v)
    return o


@pytest.mark.parametrize("change,code,text", [
    (dict(q=None), ERR_INVALID, "q: null"),
    (dict(k=None), ERR_INVALID, "k: null"),
    (dict(q=t(B.FP32, [6, 4, 128])), ERR_INVALID, "q: dtype"),
    (dict(q=t(B.BF16, [6, 4, 96])), ERR_UNSUPPORTED, "head_dim 96"),
    (dict(k=t(B.BF16, [6, 2, 64])), ERR_INVALID, "k: shape"),
    (dict(k=t(B.BF16, [5, 2, 128])), ERR_INVALID, "k: shape"),
    (dict(qo=t(B.BF16, [6, 2, 128])), ERR_INVALID, "q_out: shape"),
    (dict(ko=t(B.BF16, [6, 2, 128], data=FAKE + 4)), ERR_UNSUPPORTED, "k_out: rows"),
    (dict(q=t(B.BF16, [6, 4, 128], [512, 128, 2])), ERR_UNSUPPORTED, "q: innermost"),
    (dict(qw=t(B.INT32, [128])), ERR_INVALID, "q_weight: dtype"),
    (dict(kw=t(B.FP32, [64])), ERR_INVALID, "k_weight: 64"),
    (dict(kw=t(B.FP32, [128], [2])), ERR_UNSUPPORTED, "k_weight: must be contiguous"),
    (dict(inv=t(B.FP32, [72])), ERR_INVALID, "frequencies"),
    (dict(inv=t(B.FP32, [0])), ERR_INVALID, "frequencies"),
    (dict(inv=t(B.FP32, [20])), ERR_UNSUPPORTED, "multiple of 8"),
    (dict(inv=t(B.BF16, [64])), ERR_INVALID, "inv_freq: dtype"),
    (dict(pos=t(B.INT32, [5])), ERR_INVALID, "positions"),
    (dict(pos=t(B.INT32, [1, 6])), ERR_INVALID, "positions"),
    (dict(pos=t(B.FP32, [6])), ERR_INVALID, "positions: dtype"),
    (dict(pos=t(B.INT32, [6], [2])), ERR_UNSUPPORTED, "positions"),
    (dict(o=sect(axes=5)), ERR_UNSUPPORTED, "axes"),
    (dict(o=sect(32, 32, axes=3), pos=t(B.INT32, [2, 6])), ERR_INVALID, "positions"),
    (dict(o=sect(32, 30), pos=t(B.INT32, [2, 6])), ERR_INVALID, "sections sum"),
    (dict(o=sect(70, -6), pos=t(B.INT32, [2, 6])), ERR_INVALID, "sections[1]"),
    (dict(o=B.RopeOpts(-1.0, 0.0, 0, 1)), ERR_INVALID, "eps"),
    (dict(o=B.RopeOpts(float("nan"), 0.0, 0, 1)), ERR_INVALID, "eps"),
    (dict(o=B.RopeOpts(1e-6, float("inf"), 0, 1)), ERR_INVALID, "weight_offset"),
    (dict(o=B.RopeOpts(1e-6, 0.0, 2, 1)), ERR_INVALID, "interleaved"),
    (rope_args(T=1 << 26), ERR_UNSUPPORTED, "2^26 tokens"),
])
def test_rope_refusals(change, code, text):
    assert call_rope({**rope_args(), **change}) == code
    assert text in B.last_error(), B.last_error()


def test_rope_of_no_tokens():
    for o in (None, B.RopeOpts()):
        assert call_rope({**rope_args(T=0), "o": o}) == 0, B.last_error()
    assert call_rope({**rope_args(T=0, axes=3), "o": sect(0, 64, 0)}) == 0, B.last_error()


def test_binding_refuses_host_tensors_and_sections():
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    pos, inv = torch.zeros(2, dtype=torch.int32), torch.ones(32)
    with pytest.raises(ValueError, match="device tensors"):
        B.qk_norm_rope(x, x, pos, inv, x, x)
    for s in ((32,), (8, 8, 8, 4, 4)):
        with pytest.raises(ValueError, match="axes"):
            B.qk_norm_rope(x, x, pos, inv, x, x, sections=s)
    pool = torch.zeros((2, 2, 17, 32), dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        B.kv_read(pool, pool, i[None], i, i.repeat(2), x, x)


def test_descriptor_of_a_4_bit_pool():
    pool = torch.zeros((3, 2, 17, 64), dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    d = B.desc(pool)
    assert (d.dtype, d.ndim, list(d.shape)[:4], list(d.stride)[:4]) == (B.FP4_E2M1, 4, [3, 2, 17, 64], [2176, 1088, 64, 1])


@pytest.mark.parametrize("form,tensors,opts,optional", [("_READ", 7, False, ()), ("_ROPE", 8, True, (2, 3))])
def test_native_forms_hand_over_the_same_descriptors(form, tensors, opts, optional):
    """As the marshalling of the other calls is checked, without a device: a
    recorder in the library's place, tensors that say they are on one."""
    B.library()
    if B._native is None:
        pytest.skip("_marshal is not built for this Python")
    n = getattr(B, form)
    P, TP = ctypes.c_void_p, ctypes.POINTER(B.Tensor)

    def never(*a):
        raise AssertionError("called")
    fn = ctypes.CFUNCTYPE(ctypes.c_int, *([TP] * tensors), *([P] if opts else []), P)(never)
    addr = ctypes.cast(fn, P).value
    host = torch.zeros(2, 2)
    for ts in ([host] * tensors, [None] * tensors):
        assert B._native(addr, n, 0, 0.0, 0, None, None, *ts) is None
    with pytest.raises(TypeError):
        B._native(addr, n, 0, 0.0, 0, None, None, *([host] * (tensors - 1)))


def wide4(Bsz, T):
    """Descriptors whose sizes a launch just holds, or just does not; the last
    argument checked after the sizes is wrong, so no call gets past the checks."""
    g = good4(Bsz=Bsz, D=64, Hq=1, H=1, T=T)
    g.update(qs=t(B.INT32, [Bsz + 2]), sl=t(B.INT32, [Bsz]), bt=t(B.INT32, [Bsz, 1]))
    return g


@pytest.mark.parametrize("call,held,refused,later,text", [
    # workgroups of 256 (append: 512 over other pools) threads, fewer than 2^32 in all
    ("append", ((1 << 23) - 1, 1), (1 << 23, 1), "seq_lens", "2^23 requests"),
    ("write", (1, (1 << 28) - 49), (1, (1 << 28) - 48), "q_start", "tokens or requests"),
    ("write", ((1 << 23) - 2, 47), ((1 << 23) - 2, 48), "q_start", "tokens or requests"),
    ("read", (1, (1 << 28) - 49), (1, (1 << 28) - 48), "q_start", "tokens or requests"),
    ("prefill", (1, ((1 << 24) - 9) * 128 + 127), (1, ((1 << 24) - 9) * 128 + 128), "q_start", "KV heads"),
])
def test_sizes_that_a_launch_does_not_hold(call, held, refused, later, text):
    L = B.library()
    for size, word in ((held, later), (refused, text)):
        g = wide4(*size)
        if call == "append":
            g["sl"] = t(B.INT32, [size[0] + 1])
        if call == "prefill":       # (2^30 tokens and more are refused before: a wider group has as many rows)
            g.update(qt=t(B.BF16, [size[1] // 16, 16, 64]), ot=t(B.BF16, [size[1] // 16, 16, 64]))
        assert CALLS[call](L, g) in (ERR_INVALID, ERR_UNSUPPORTED)
        assert word in B.last_error(), B.last_error()


def test_rope_tokens_that_a_launch_does_not_hold():
    for T, text in (((1 << 26) - 4, "sections sum"), ((1 << 26) - 3, "2^26 tokens"), ((1 << 26) - 1, "2^26 tokens")):
        a = {**rope_args(T=T), "o": sect(32, 30), "pos": t(B.INT32, [2, T])}
        assert call_rope(a) in (ERR_INVALID, ERR_UNSUPPORTED) and text in B.last_error(), B.last_error()


@pytest.mark.parametrize("call", ["decode", "step"])
def test_no_traced_kernel_over_4_bit_pools(call):
    for change in ({}, dict(q=t(B.BF16, [4, 32, 64]), out=t(B.BF16, [4, 32, 64]), kn=t(B.BF16, [4, 8, 64]),
                            vn=t(B.BF16, [4, 8, 64]), k=t(B.FP4_E2M1, [100, 8, 17, 32]), v=t(B.FP4_E2M1, [100, 8, 17, 32]))):
        g = {**good4(), **change, "opts": opts(wave_times=FAKE)}
        assert CALLS[call](B.library(), g) == ERR_UNSUPPORTED
        assert "4-bit pools" in B.last_error(), B.last_error()
