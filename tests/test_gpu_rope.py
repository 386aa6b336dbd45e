"""Norm and rotation of queries and keys on the GPU, against binary64: element
by element |got - ref| <= 2^-8 |ref| + 2^-18 M, M the larger of the pair's
magnitudes before the turn: the output's rounding to bf16, and sines and cosines
within 1.3e-7, a position of 2^31 within 4e-7 turns, some binary32 roundings."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import rope

pytestmark = pytest.mark.gpu

bl = pytest.importorskip("paper_2510_15330_amd")


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def run(rng, T, H_q, H, D, F, pos, sections=None, inter=False, qw=None, kw=None, eps=1e-6, offset=0.0, scale=1.0,
        theta=10000.0, in_place=False):
    x = (torch.from_numpy(rng.standard_normal((T, H_q + H + 2, D)).astype(np.float32)) * scale).to(torch.bfloat16).cuda()
    q, k = x[:, :H_q], x[:, H_q + 1:H_q + 1 + H]
    inv = (theta ** (-np.arange(F) / F)).astype(np.float32)
    w = []
    for kind in (qw, kw):
        w.append(None if kind is None else torch.from_numpy((1 - offset + 0.3 * rng.standard_normal(D)).astype(np.float32))
                 .to(kind).cuda())
    want = [rope.rotate(rope.norm(t.double().cpu().numpy(), None if u is None else u.double().cpu().numpy(), eps, offset),
                        pos, inv, sections, inter) for t, u in zip((q, k), w)]
    flat = [rope.norm(t.double().cpu().numpy(), None if u is None else u.double().cpu().numpy(), eps, offset)
            for t, u in zip((q, k), w)]
    between = x[:, H_q].clone(), x[:, -1].clone()
    if in_place:
        qo, ko = q, k
    else:
        buf = torch.full((T, H_q + H + 1, D + 8), 3.0, dtype=torch.bfloat16, device="cuda")
        qo, ko = buf[:, :H_q, :D], buf[:, H_q + 1:, 8:]
    bl.qk_norm_rope(q, k, torch.from_numpy(np.ascontiguousarray(pos, dtype=np.int32)).cuda(), torch.from_numpy(inv).cuda(),
                    qo, ko, q_weight=w[0], k_weight=w[1], eps=eps, weight_offset=offset, sections=sections,
                    interleaved=inter)
    torch.cuda.synchronize()
    for got, ref, f in zip((qo, ko), want, flat):
        got = got.double().cpu().numpy()
        i, j = (np.arange(0, 2 * F, 2), np.arange(1, 2 * F, 2)) if inter else (np.arange(F), np.arange(F, 2 * F))
        M = np.abs(f)
        M[..., i] = M[..., j] = np.maximum(M[..., i], M[..., j])
        off = np.abs(got - ref) - 2.0 ** -8 * np.abs(ref) - 2.0 ** -18 * M
        assert off.size == 0 or off.max() <= 0, off.max()
    assert torch.equal(x[:, H_q], between[0]) and torch.equal(x[:, -1], between[1])
    if not in_place:
        assert (buf[:, H_q] == 3).all() and (buf[:, :H_q, D:] == 3).all() and (buf[:, H_q + 1:, :8] == 3).all()


@pytest.mark.parametrize("D,F", [(64, 32), (64, 16), (64, 8), (128, 64), (128, 32), (128, 48), (128, 8)])
@pytest.mark.parametrize("inter", [False, True])
def test_rotation_alone(D, F, inter):
    rng = np.random.default_rng(D + F)
    run(rng, 37, 5, 3, D, F, rng.integers(0, 5000, 37), inter=inter)


@pytest.mark.parametrize("qw,kw", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16),
                                   (None, torch.float32), (torch.bfloat16, None)])
@pytest.mark.parametrize("H_q,H,D", [(32, 8, 128), (28, 4, 128), (1, 1, 64), (40, 5, 64), (7, 9, 128)])
def test_norm_and_rotation(qw, kw, H_q, H, D):
    rng = np.random.default_rng(H_q)
    run(rng, 50, H_q, H, D, D // 2, rng.integers(0, 40000, 50), qw=qw, kw=kw, offset=0.0 if H_q < 30 else 1.0)


@pytest.mark.parametrize("T", [1, 2, 3, 5000, 8191, 8192, 9001])
def test_token_counts(T):
    rng = np.random.default_rng(T)
    run(rng, T, 3, 1, 128, 64, rng.integers(0, 131072, T), qw=torch.bfloat16, kw=torch.bfloat16)


@pytest.mark.parametrize("sections", [(16, 24, 24), (64, 0, 0), (0, 0, 64), (1, 62, 1), (30, 34), (16, 16, 16, 16), (0, 7, 9, 48)])
@pytest.mark.parametrize("inter", [False, True])
def test_several_axes(sections, inter):
    rng = np.random.default_rng(len(sections))
    run(rng, 21, 4, 2, 128, 64, rng.integers(0, 3000, (len(sections), 21)), sections=sections, inter=inter, qw=torch.bfloat16)


def test_axes_in_a_wider_tensor():
    rng = np.random.default_rng(1)
    pos = torch.from_numpy(rng.integers(0, 500, (3, 40)).astype(np.int32)).cuda()
    x = torch.randn((20, 2, 64), device="cuda").to(torch.bfloat16)
    inv = torch.logspace(0, -3, 32, device="cuda")
    a, b, c, d = (torch.empty_like(x) for _ in range(4))
    bl.qk_norm_rope(x, x, pos[:, 11:31], inv, a, b, sections=(8, 12, 12))
    bl.qk_norm_rope(x, x, pos[:, 11:31].contiguous(), inv, c, d, sections=(8, 12, 12))
    assert torch.equal(a, c) and torch.equal(b, d) and torch.equal(a, b)


def test_far_and_negative_positions():
    rng = np.random.default_rng(2)
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1048576, 10 ** 9 + 7, -65537])
    for theta in (10000.0, 1.0, 1e6):
        run(rng, 8, 4, 2, 128, 64, pos, theta=theta)


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 1e15])
def test_sizes_of_values_and_eps(scale):
    rng = np.random.default_rng(3)
    for eps in (1e-6, 1e-5, 0.0):
        if scale == 1e-20 and eps == 0.0:
            continue                             # squares below binary32's smallest
        run(rng, 9, 4, 2, 64, 32, rng.integers(0, 99, 9), qw=torch.float32, kw=torch.bfloat16, eps=eps, scale=scale)


def test_in_place():
    rng = np.random.default_rng(4)
    for inter in (False, True):
        run(rng, 300, 12, 4, 128, 32, rng.integers(0, 999, 300), inter=inter, qw=torch.bfloat16, kw=torch.bfloat16, in_place=True)


@pytest.mark.parametrize("T,H_q,H,D,F,inter", [(36001, 32, 8, 128, 64, False), (17000, 32, 8, 128, 48, False),
                                               (17000, 32, 8, 128, 64, True), (30011, 40, 8, 64, 32, False),
                                               (30011, 40, 8, 64, 16, True)])
def test_many_tokens_are_as_few(T, H_q, H, D, F, inter):
    """Rows past the memory-side cache (streamed), and the same in parts that fit, bit for bit."""
    g = torch.Generator("cuda").manual_seed(T + D)
    x = torch.randn((T, H_q + H, D), generator=g, device="cuda").to(torch.bfloat16)
    q, k = x[:, :H_q], x[:, H_q:]
    pos = torch.randint(0, 100000, (T,), generator=g, device="cuda", dtype=torch.int32)
    inv, w = torch.logspace(0, -4, F, device="cuda"), torch.rand(D, generator=g, device="cuda").to(torch.bfloat16)
    outs = []
    for step in (T, 5001):
        qo, ko = torch.full((T, H_q, D), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, H, D), 3.0, dtype=torch.bfloat16, device="cuda")
        for i in range(0, T, step):
            s = slice(i, min(i + step, T))
            bl.qk_norm_rope(q[s], k[s], pos[s], inv, qo[s], ko[s], q_weight=w, k_weight=w, interleaved=inter)
        outs.append((qo, ko))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    bl.qk_norm_rope(q, k, pos, inv, q, k, q_weight=w, k_weight=w, interleaved=inter)      # in place
    assert torch.equal(q, outs[0][0]) and torch.equal(k, outs[0][1])


def test_rows_past_binary32_are_zero():
    x = torch.randn((5, 2, 128), device="cuda").to(torch.bfloat16)
    x[2, 1, 3] = 1e25                                 # its square is infinite
    w = torch.ones(128, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    bl.qk_norm_rope(x, x, torch.arange(5, dtype=torch.int32, device="cuda"), torch.logspace(0, -3, 64, device="cuda"), a, b,
                    q_weight=w)
    assert not a[2, 1].any() and a[2, 0].all() and not torch.isnan(a).any()
    assert b[2, 1].abs().max() > 1e24                 # no norm, no squares


def test_nan_and_zero_rows_stay_their_own():
    x = torch.randn((6, 3, 64), device="cuda").to(torch.bfloat16)
    x[2, 1, 5] = float("nan")
    x[3, 0] = 0
    w = torch.ones(64, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    bl.qk_norm_rope(x, x, pos, torch.logspace(0, -3, 32, device="cuda"), a, b, q_weight=w, k_weight=w)
    bad = torch.isnan(a).any(-1)
    assert bad[2, 1] and int(bad.sum()) == 1 and not a[3, 0].any()
    # without a norm only the NaN's pair is
    bl.qk_norm_rope(x, x, pos, torch.logspace(0, -3, 32, device="cuda"), a, b)
    assert torch.isnan(a).sum() == 2 and torch.isnan(a[2, 1, [5, 37]]).all()


@pytest.mark.parametrize("D,inter", [(64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("scale", [1e-20, 2.0 ** -54, 2.0 ** -66, 2.0 ** -100, 2.0 ** -128])
def test_rows_whose_squares_are_below_binary32(D, inter, scale):
    """With an eps of the rows' own size or none; other rows of the call as ever."""
    rng = np.random.default_rng(D)
    for eps in (0.0, 1e-40, 1e-32):
        run(rng, 9, 4, 2, D, D // 2, rng.integers(0, 99, 9), qw=torch.float32, kw=torch.bfloat16, eps=eps, scale=scale, inter=inter)
        mixed = np.exp2(rng.integers(-130, 10, (9, 4 + 2 + 2, 1))).astype(np.float32)
        run(rng, 9, 4, 2, D, D // 2, rng.integers(0, 99, 9), qw=torch.float32, kw=torch.bfloat16, eps=eps, scale=torch.from_numpy(mixed),
            inter=inter)
