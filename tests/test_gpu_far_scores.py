"""Prompt and decode attention on finite scores of any size, over every kind of pool.

Two tokens of a request hold the same key, along the query's signs and six
times as long as the others': from queries of 2^14 on, every row is the mean of
the two tokens' values, whatever the scores' size, as the two scores are equal
and the others' weights vanish.  The values of successive 64-key steps differ
by 2^3 (their copies have scales that differ).

|got - ref| <= 2^-8 |ref| + (2^-11 + 2^-12 S) A against binary64 over the values
that the pool holds, A the weighted sum of |values|: the output's rounding to
bf16, the weights' to fp16 (decode: less) and the exponents' roundings; S, the sum of |products|
of a row's largest score, counts below 2^14 alone, where weights depend on the
scores' own error (2^-13 S over 4-bit pools, less over the others).
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

bl = pytest.importorskip("paper_2510_15330_amd")

POWERS = [-100, -20, -3, 14, 15, 16, 18, 21, 25, 28, 32, 60]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bl.device_errors()
    yield
    torch.cuda.synchronize()


def pools(kv, pages, D):
    if kv == "fp4":
        z = torch.zeros((pages, 1, 17, D // 2), dtype=torch.uint8, device="cuda")
        return z.view(torch.float4_e2m1fn_x2), z.clone().view(torch.float4_e2m1fn_x2)
    x = 8 if kv == "bf16" else 16
    dt = torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn
    return (torch.zeros((pages, 1, D // x, 16, x), device="cuda").to(dt),
            torch.zeros((pages, 1, D, 16), device="cuda").to(dt))


@pytest.mark.parametrize("kv", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("call", ["prompt", "decode"])
@pytest.mark.parametrize("shift", [0, -110, 50])      # queries 2^shift, the softmax scale 2^-shift times as large
@pytest.mark.parametrize("L,twins", [(340, (70, 200)), (2540, (100, 1700))], ids=["whole", "keys-shared-out"])
def test_finite_scores_of_any_size(kv, D, L, twins, shift, call):
    rng = np.random.default_rng(D + L)
    n, G, scale = 40, len(POWERS), 0.1 * 2.0 ** -shift
    u = rng.choice([-1.0, 1.0], D)
    k = rng.choice([-1.0, -0.5, 0.5, 1.0], (L, D))
    k[list(twins)] = 6 * u
    v = rng.standard_normal((L, D)) * np.exp2(-3.0 * (np.arange(L) // 64 % 3))[:, None]
    dt = torch.float8_e4m3fn if kv == "fp8" else torch.bfloat16
    rows = [torch.from_numpy(x[:, None].astype(np.float32)).cuda().to(dt) for x in (k, v)]
    P = (L + 15) // 16
    kp, vp = pools(kv, P + 2, D)
    table = torch.from_numpy(rng.permutation(P + 2)[:P].astype(np.int32)).cuda()[None].contiguous()
    lens, start = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, L], dtype=torch.int32, device="cuda")
    bl.kv_write(*rows, kp, vp, table, lens, start)
    one = torch.ones((1, 1), device="cuda") if kv == "fp8" else None
    held = [torch.empty((L, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bl.kv_read(kp, vp, table, lens, start, *held, k_scale=one, v_scale=one)
    kh, vh = (t[:, 0].double().cpu().numpy() for t in held)
    assert np.array_equal(kh, k)                       # 4 bits and 8 hold these keys

    q = torch.from_numpy((np.exp2(np.add(POWERS, shift))[None, :, None] * u * np.ones((n, 1, 1))).astype(np.float32)).to(torch.bfloat16).cuda()
    qs = torch.tensor([0, n], dtype=torch.int32, device="cuda")

    def attend(q, scale, out):
        if call == "prompt":
            bl.prefill_attention(q, kp, vp, table, lens, qs, scale, out, k_scale=one, v_scale=one)
        else:                       # the same rows, a request each of its own length
            ones = None if one is None else one.expand(n, 1).contiguous()
            bl.decode_attention(q, kp, vp, table.expand(n, P).contiguous(), lens - torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda"),
                                scale, out, k_scale=ones, v_scale=ones)
    out, neg = (torch.full((n, G, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    attend(q, scale, out)
    attend(-q, -scale, neg)
    assert bl.device_errors() == 0

    seen = np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]
    for i, p in enumerate(POWERS):
        s = np.where(seen, 2.0 ** (p + shift) * (k @ u) * float(np.float32(scale)), -np.inf)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        if p >= 14:
            assert np.array_equal(w > 0, np.isin(np.arange(L), twins)[None] & seen)
        ref, mag = w @ vh, w @ np.abs(vh)
        S = 6 * D * 2.0 ** (p + shift) * scale if p < 14 else 0.0
        got = out[:, i].double().cpu().numpy()
        assert np.isfinite(got).all(), f"queries of 2^{p}"
        off = (np.abs(got - ref) - 2.0 ** -8 * np.abs(ref) - (2.0 ** -11 + 2.0 ** -12 * S) * mag).max()
        assert off <= 0, f"queries of 2^{p}: over the bound by {off:.3e}"
    same = torch.equal(out, neg)
    assert same, "a negative scale and the queries' other sign"
