"""4-bit pages on the GPU, against the numpy oracle (oracle/kv4.py).

Writes: bytes of the whole pools, equal.  Reads: values, equal.  Attention:
element by element |got - ref| <= 2^-8 |ref| + (c + 2^-12 S) A, A the oracle's
sum of weights times |values|, S its largest sum of |query * key| products of the
row's scores (scaled): the output's own rounding (bf16, half a step), and what
weights and scores are off by.
  c      decode 2^-12: weights as hi + lo of truncated bf16, 2^-14, and the
         exponent's binary32 roundings; prompt 2^-11: rounded to fp16, 2^-12,
         and the same
  2^-12  a score is off by at most 2^-13 of its sum of |products| (the scaled
         matrix instructions align the products of a few neighbouring dims,
         keeping 13 bits below the largest); a weight by that and its sum's
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import kv4, rope

pytestmark = pytest.mark.gpu

bl = pytest.importorskip("paper_2510_15330_amd")
from paper_2510_15330_amd import _binding  # noqa: E402

F4 = torch.float4_e2m1fn_x2
DECODE, PROMPT = 2.0 ** -12, 2.0 ** -11


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bl.library()
    bl.device_errors()
    yield
    torch.cuda.synchronize()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(x):
    """Nearest bf16 of each value, as float64 and as a device tensor."""
    t = torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)
    return t.double().numpy(), t.cuda()


class Cache:
    """Pools of random bytes (any code, any scale byte: what a tail slot may
    hold) with scattered pages, `lens` real tokens a request."""

    def __init__(self, rng, lens, H, D, room=0, spare=3, fill=None):
        lens = np.asarray(lens, dtype=np.int32)
        need = (lens + room + 15) // 16
        self.H, self.D, self.B = H, D, len(lens)
        NP = int(need.sum()) + spare
        self.pools = [rng.integers(0, 256, (NP, H, 17, D // 2), dtype=np.uint8) for _ in range(2)]
        self.table = np.full((len(lens), max(1, int(need.max(initial=0)))), -1, dtype=np.int32)
        perm, at = rng.permutation(NP).astype(np.int32), 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.spare = [int(p) for p in perm[at:]]
        # real rows, a page at a time; slots past the length keep their random bytes
        byte = {k: kv4.offsets(D, k) for k in "kv"}
        for pool, kind in zip(self.pools, "kv"):
            for b, L in enumerate(lens):
                for i in range((L + 15) // 16):
                    n = min(16, L - 16 * i)
                    x = rng.standard_normal((H, n, D)) if fill is None else fill(kind, b, i, (H, n, D))
                    codes, scales = kv4.quantize(x)
                    t = pool[self.table[b, i]].reshape(H, -1)
                    at_, nib, sc = (a[:n] for a in byte[kind])
                    for v in (0, 1):
                        m = nib == v
                        t[:, at_[m]] = (t[:, at_[m]] & (0xF0 if v == 0 else 0x0F)) | (codes[:, m] << (4 * v))
                    t[:, sc[:, ::32]] = scales
                    pool[self.table[b, i]] = t.reshape(H, 17, D // 2)
        self.lens = lens.copy()

    def to_device(self):
        self.k, self.v = (dev(p).view(F4) for p in self.pools)
        self.bt, self.sl = dev(self.table), dev(self.lens)
        return self

    def bytes(self):
        return [p.view(torch.uint8).cpu().numpy() for p in (self.k, self.v)]


def close(got, ref, mag, dot, c, what=""):
    got = got.detach().float().cpu().double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN where none belongs, or none where one does"
    ok = ~np.isnan(ref)
    off = np.abs(got - ref)[ok] - 2.0 ** -8 * np.abs(ref)[ok] - ((c + 2.0 ** -12 * dot) * mag)[ok]
    assert not off.size or off.max() <= 0, f"{what}: over the bound by {off.max():.3e}"


def decode(c, q, scale, **kw):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    bl.decode_attention(q, c.k, c.v, c.bt, c.sl, scale, out, **kw)
    return out


# ----------------------------------------------------------------- writes --

def _magnitudes(rng, shape):
    """bf16 values of all magnitudes, subnormal and largest among them."""
    x = torch.from_numpy(rng.integers(0, 1 << 16, shape, dtype=np.uint16).view(np.int16)).view(torch.bfloat16)
    # values of one row near each other in size, so that all codes appear
    y = torch.from_numpy(rng.standard_normal(shape).astype(np.float32) *
                         np.exp2(rng.uniform(-130, 120, shape[:-1] + (1,))).astype(np.float32)).to(torch.bfloat16)
    pick = torch.from_numpy(rng.random(shape[:-1] + (1,)) < 0.2)
    return torch.where(pick, x, y)


def test_every_bf16_pattern_is_quantised_as_the_rule_says():
    rng = np.random.default_rng(0)
    pat = np.arange(1 << 16, dtype=np.uint16)
    alone = np.zeros((1 << 16, 32), dtype=np.uint16)
    alone[np.arange(1 << 16), rng.integers(0, 32, 1 << 16)] = pat
    # and every finite pattern below a maximum of 1 to 64 times it
    fin = pat[(pat & 0x7F80) < 0x7C00]
    pairs = np.zeros((len(fin), 32), dtype=np.uint16)
    pairs[:, 0], pairs[:, 17] = fin, (fin & 0x7FFF) + (rng.integers(0, 6 * 128, len(fin))).astype(np.uint16)
    bits = np.concatenate([alone, pairs])
    H, D = 8, 128
    bits = np.resize(bits, (-(-bits.size // (H * D)) * H * D)).reshape(-1, H, D)
    rows = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16)
    T = rows.shape[0]
    c = Cache(rng, [0], H, D, room=T).to_device()
    qs = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    bl.kv_write(rows.cuda(), rows.cuda(), c.k, c.v, c.bt, c.sl, qs)
    codes, scales = kv4.quantize(rows.double().numpy())
    for pool, kind in zip(c.bytes(), "kv"):
        at, nib, sc = kv4.offsets(D, kind)
        t = pool[c.table[0, :(T + 15) // 16]].reshape(-1, H, 17 * D // 2)
        got_s = t[:, :, sc[:, ::32]].transpose(0, 2, 1, 3).reshape(-1, H, D // 32)[:T]
        got_c = ((t[:, :, at] >> (4 * nib).astype(np.uint8)) & 15).transpose(0, 2, 1, 3).reshape(-1, H, D)[:T]
        assert np.array_equal(got_s, scales)
        assert np.array_equal(got_c, codes)


@pytest.mark.parametrize("D,H", [(64, 1), (64, 5), (128, 2), (128, 8), (128, 9)])
def test_append_bytes(D, H):
    rng = np.random.default_rng(D + H)
    lens = list(range(0, 34)) + [200, 511]
    c = Cache(rng, lens, H, D, room=1).to_device()
    rows = [_magnitudes(rng, (len(lens), H, D)) for _ in range(2)]
    bl.kv_append(rows[0].cuda(), rows[1].cuda(), c.k, c.v, c.bt, c.sl)
    kv4.write(*c.pools, *(r.double().numpy() for r in rows), c.table, c.lens, [1] * len(lens))
    assert all(np.array_equal(a, b) for a, b in zip(c.bytes(), c.pools))
    assert np.array_equal(c.sl.cpu().numpy(), c.lens) and bl.device_errors() == 0


def test_append_strided_rows_and_refused_slots():
    rng = np.random.default_rng(3)
    H, D = 3, 128
    c = Cache(rng, [5, 16, 31, 40], H, D, room=1)
    c.table[1, 1] = -1                       # the slot's page is not there
    c.table[2, 1] = c.pools[0].shape[0]      # outside the pool
    c.lens[3] = -2
    c.to_device()
    both = _magnitudes(rng, (4, 2 * H + 1, D)).cuda()
    k, v = both[:, 1:1 + H], both[:, 1 + H:]
    bl.kv_append(k, v, c.k, c.v, c.bt, c.sl)
    assert bl.device_errors() == 1
    want = c.lens.copy()
    one = c.lens[:1].copy()
    kv4.write(*c.pools, k[:1].double().cpu().numpy(), v[:1].double().cpu().numpy(), c.table[:1], one, [1])
    want[0] += 1
    assert all(np.array_equal(a, b) for a, b in zip(c.bytes(), c.pools))
    assert np.array_equal(c.sl.cpu().numpy(), want)


@pytest.mark.parametrize("D,H", [(64, 2), (64, 7), (128, 1), (128, 8)])
@pytest.mark.parametrize("many", [False, True])
def test_prompt_write_bytes_and_read_back(D, H, many):
    rng = np.random.default_rng(10 * D + H + many)
    if many:
        cached, new = rng.integers(0, 40, 70), rng.integers(0, 40, 70)
        new[:3] = 0, 1, 0
    else:
        cached, new = np.array([0, 3, 16, 17, 0, 100, 15]), np.array([16, 5, 1, 64, 0, 33, 1])
    c = Cache(rng, cached, H, D, room=int(new.max())).to_device()
    T = int(new.sum())
    rows = [_magnitudes(rng, (T, H, D)) for _ in range(2)]
    qs = dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    bl.kv_write(rows[0].cuda(), rows[1].cuda(), c.k, c.v, c.bt, c.sl, qs)
    kv4.write(*c.pools, *(r.double().numpy() for r in rows), c.table, c.lens, new)
    assert all(np.array_equal(a, b) for a, b in zip(c.bytes(), c.pools))
    assert np.array_equal(c.sl.cpu().numpy(), c.lens) and bl.device_errors() == 0
    # read back: the new rows into strided outputs, then whole requests
    wide = torch.zeros((T, H + 2, D), dtype=torch.bfloat16, device="cuda")
    ko, vo = wide[:, 1:1 + H], torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
    bl.kv_read(c.k, c.v, c.bt, c.sl, qs, ko, vo)
    for got, x in ((ko, rows[0]), (vo, rows[1])):
        want = kv4.dequantize(*kv4.quantize(x.double().numpy()))
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    assert not wide[:, 0].any() and not wide[:, -1].any()
    all_ = np.concatenate([[0], np.cumsum(c.lens)]).astype(np.int32)
    ko, vo = (torch.empty((int(all_[-1]), H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bl.kv_read(c.k, c.v, c.bt, c.sl, dev(all_), ko, vo)
    for got, pool, kind in ((ko, c.pools[0], "k"), (vo, c.pools[1], "v")):
        want = np.concatenate([kv4.read_pages(pool, c.table[b, :(L + 15) // 16], kind)[:L] for b, L in enumerate(c.lens)])
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    assert bl.device_errors() == 0


def test_read_of_every_scale_byte_and_code():
    D, H = 128, 1
    k = np.zeros((16, H, 17, D // 2), dtype=np.uint8)
    v = k.copy()
    k[:, 0, :16] = np.resize(np.arange(256, dtype=np.uint8), (16, 16, 64))
    v[:, 0, :16] = np.resize(np.arange(256, dtype=np.uint8)[::-1], (16, 16, 64))
    k[:, 0, 16] = np.resize(np.arange(256, dtype=np.uint8), (16, 64))
    v[:, 0, 16] = np.resize(np.arange(256, dtype=np.uint8)[::-1], (16, 64))
    table = np.arange(16, dtype=np.int32)[None]
    ko, vo = (torch.empty((256, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bl.kv_read(dev(k).view(F4), dev(v).view(F4), dev(table), dev(np.array([256], dtype=np.int32)),
               dev(np.array([0, 256], dtype=np.int32)), ko, vo)
    for got, pool, kind in ((ko, k, "k"), (vo, v, "v")):
        want = torch.from_numpy(kv4.read_pages(pool, table[0], kind)).to(torch.bfloat16).double().numpy()   # (inf past bf16)
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("D", [64, 128])
def test_read_of_other_pools(kv, D):
    rng = np.random.default_rng(D)
    H, B, x = 3, 4, 8 if kv == "bf16" else 16
    lens, n = np.array([33, 0, 16, 70], dtype=np.int32), np.array([33, 0, 7, 20])
    table = rng.permutation(24).astype(np.int32)[:20].reshape(B, 5)
    dt = torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn
    k = torch.randn((24, H, D // x, 16, x)).to(dt)
    v = torch.randn((24, H, D, 16)).to(dt)
    ks, vs = (torch.rand((B, H)) + 0.5 for _ in range(2)) if kv == "fp8" else (None, None)
    qs = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    ko, vo = (torch.empty((int(qs[-1]), H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bl.kv_read(k.cuda(), v.cuda(), dev(table), dev(lens), dev(qs), ko, vo, k_scale=None if ks is None else ks.cuda(),
               v_scale=None if vs is None else vs.cuda())
    for got, pool, sc, perm in ((ko, k, ks, (0, 3, 1, 2, 4)), (vo, v, vs, (0, 3, 1, 2))):
        dense = pool.float().permute(*perm).reshape(24, 16, H, D)
        want = []
        for b in range(B):
            r = dense[table[b].astype(np.int64)].reshape(-1, H, D)[lens[b] - n[b]:lens[b]]
            want.append((r if sc is None else r * sc[b][None, :, None]).to(torch.bfloat16))
        assert torch.equal(got.cpu(), torch.cat(want))
    assert bl.device_errors() == 0


def test_read_of_malformed_requests():
    rng = np.random.default_rng(8)
    c = Cache(rng, [20, 20, 33, 20], 2, 64)
    c.table[2, 1] = -1
    c.lens[3] = 16 * c.table.shape[1] + 1        # past the table
    c.to_device()
    ko, vo = (torch.full((20 + 21 + 33 + 4, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bl.kv_read(c.k, c.v, c.bt, c.sl, dev(np.array([0, 20, 41, 74, 78], dtype=np.int32)), ko, vo)
    assert bl.device_errors() == 2 | 4
    for got in (ko, vo):
        got = got.float().cpu()
        assert not torch.isnan(got[:20]).any() and (got[20:41] == 5).all() and (got[74:] == 5).all()
        assert torch.isnan(got[41 + 16:41 + 32]).all() and not torch.isnan(got[41:57]).any() and not torch.isnan(got[73]).any()
    for bad in ([0, 20, 10, 30, 40], [-1, 0, 0, 0, 0], [0, 0, 0, 0, 79]):
        ko.fill_(5)
        bl.kv_read(c.k, c.v, c.bt, c.sl, dev(np.array(bad, dtype=np.int32)), ko, vo)
        assert bl.device_errors() & 2 and (ko == 5).all()


@pytest.mark.parametrize("H,D", [(8, 128), (17, 64)])
def test_rows_past_the_cache_are_written_as_fewer_are(H, D):
    """More than 128 MB of rows (streamed), and the same in three calls."""
    n = [20000, 1, 14007]
    rng = np.random.default_rng(D)
    need = [(x + 15) // 16 for x in n]
    NP = sum(need)
    bt = np.full((3, max(need)), -1, dtype=np.int32)
    for b, (k, perm) in enumerate(zip(need, np.split(rng.permutation(NP).astype(np.int32), np.cumsum(need)[:2]))):
        bt[b, :k] = perm
    bt = dev(bt)
    g = torch.Generator("cuda").manual_seed(D)
    k, v = (torch.randn((sum(n), H, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    assert k.numel() * 4 > 128 << 20
    at, pools = np.concatenate([[0], np.cumsum(n)]), []
    for parts in (1, 3):
        p = [torch.zeros((NP, H, 17, D // 2), dtype=torch.uint8, device="cuda").view(F4) for _ in range(2)]
        sl = torch.zeros(3, dtype=torch.int32, device="cuda")
        if parts == 1:
            bl.kv_write(k, v, *p, bt, sl, dev(at.astype(np.int32)))
        else:
            for b in range(3):
                s = slice(int(at[b]), int(at[b + 1]))
                bl.kv_write(k[s], v[s], *p, bt[b:b + 1], sl[b:b + 1], dev(np.array([0, n[b]], dtype=np.int32)))
        assert sl.tolist() == n
        pools.append([x.view(torch.uint8) for x in p])
    assert bl.device_errors() == 0
    assert all(torch.equal(a, b) and a.any() for a, b in zip(*pools))


# ----------------------------------------------------------------- decode --

SHAPES = [  # H_q, H_kv, D, lengths
    (8, 2, 64, [1, 17, 200]),
    (4, 4, 128, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65]),
    (7, 1, 64, [0, 64, 128, 129, 0, 300]),
    (32, 8, 128, [0, 0, 1000]),
    (16, 1, 128, [47, 48, 49, 2000, 1]),
    (12, 4, 64, [5, 700, 64]),
    (10, 2, 128, [130] * 70),
]


@pytest.mark.parametrize("H_q,H,D,lens", SHAPES)
def test_decode_shapes_and_splits(H_q, H, D, lens):
    rng = np.random.default_rng(H_q + D)
    c = Cache(rng, lens, H, D).to_device()
    qf, q = bf16(rng.standard_normal((len(lens), H_q, D)) * 2)
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1] * len(lens), D ** -0.5)
    for kw in ({}, dict(max_waves=1), dict(max_waves=2), dict(max_waves=3), dict(max_waves=4), dict(max_waves=37),
               dict(max_waves=40), dict(pages_per_step=4), dict(max_waves=6, xcd_skew=255)):
        out = decode(c, q, D ** -0.5, **kw)
        close(out, ref, mag, dot, DECODE, f"{kw}")
        assert torch.equal(out, decode(c, q, D ** -0.5, **kw)), "not the same twice"
    out = torch.empty_like(out)
    # (16 heads of 128 exceed the fixed array at two workgroups a CU: the documented bound)
    bl.decode_attention_noalloc(q, c.k, c.v, c.bt, c.sl, D ** -0.5, out, max_waves=1900 if H_q // H == 16 else 0)
    assert torch.equal(out, decode(c, q, D ** -0.5))
    assert bl.device_errors() == 0


@pytest.mark.parametrize("seed", range(6))
def test_decode_random_sweep(seed):
    rng = np.random.default_rng(100 + seed)
    G, H, D = int(rng.integers(1, 17)), int(rng.choice([1, 2, 3, 5])), int(rng.choice([64, 128]))
    B = int(rng.integers(1, 40))
    lens = np.where(rng.random(B) < 0.5, rng.integers(0, 8, B) * 64 + rng.integers(-2, 3, B), rng.integers(0, 900, B)).clip(0)
    c = Cache(rng, lens, H, D).to_device()
    qf, q = bf16(rng.standard_normal((B, G * H, D)))
    scale = float(rng.choice([D ** -0.5, 0.0, -0.1, 0.4]))
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1] * B, scale)
    for w in (0, 1, int(rng.integers(2, 200))):
        for pp in (0, 4):
            close(decode(c, q, scale, max_waves=w, pages_per_step=pp), ref, mag, dot, DECODE, f"seed {seed} waves {w} pages {pp}")


def test_decode_strided_queries_outputs_and_wide_table():
    rng = np.random.default_rng(4)
    H_q, H, D, B = 6, 2, 128, 5
    c = Cache(rng, [40, 3, 99, 64, 16], H, D).to_device()
    wide = torch.full((B, 40), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.bt.shape[1]] = c.bt
    c.bt = wide[:, :20]
    qf, q = bf16(rng.standard_normal((B, H_q + 3, D)))
    buf = torch.full((B, H_q + 1, D + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, :H_q, :D]
    bl.decode_attention(q[:, 1:1 + H_q], c.k, c.v, c.bt, c.sl, 0.09, out)
    ref, mag, dot = kv4.attention(qf[:, 1:1 + H_q], *c.pools, c.table, c.lens, [1] * B, 0.09)
    close(out, ref, mag, dot, DECODE)
    assert (buf[:, H_q] == 9).all() and (buf[..., D:] == 9).all()


@pytest.mark.parametrize("D", [64, 128])
def test_nan_blocks(D):
    """A NaN key block takes its (request, head)'s rows, a NaN value block its
    32 dims of them; in a slot past the length neither does anything."""
    rng = np.random.default_rng(D)
    H, G, lens = 2, 3, [70, 70, 70, 33]

    def fill(kind, b, i, shape):
        x = rng.standard_normal(shape)
        if kind == "k" and b == 0 and i == 2:
            x[1, 5, 40] = np.inf
        if kind == "v" and b == 1 and i == 1:
            x[0, 9, 33] = np.nan
        return x
    c = Cache(rng, lens, H, D, fill=fill)
    for pool in c.pools:                         # every dead slot's scale: NaN
        for kind in "kv":
            _, _, sc = kv4.offsets(D, kind)
        for b, L in enumerate(lens):
            t = pool[c.table[b, L // 16]].reshape(H, -1)
            _, _, sc = kv4.offsets(D, "k" if pool is c.pools[0] else "v")
            t[:, sc[L % 16:].ravel()] = 255
            pool[c.table[b, L // 16]] = t.reshape(H, 17, D // 2)
    c.to_device()
    qf, q = bf16(rng.standard_normal((4, G * H, D)))
    with np.errstate(invalid="ignore"):
        ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1] * 4, 0.1)
    # the oracle's own NaNs are those: heads 3..5 of request 0, dims 32..63 of heads 0..2 of request 1
    want = np.zeros(ref.shape, dtype=bool)
    want[0, G:] = True
    want[1, :G, 32:64] = True
    assert np.array_equal(np.isnan(ref), want)
    for kw in ({}, dict(max_waves=1), dict(max_waves=7), dict(pages_per_step=4)):
        close(decode(c, q, 0.1, **kw), ref, mag, dot, DECODE, str(kw))
    # the prompt attention over the same pages: keys that a row sees
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.arange(5, dtype=np.int32)), 0.1, out)
    close(out, ref, mag, dot, PROMPT)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread", [8, 40, 100])
def test_values_of_very_different_sizes(D, spread):
    """Scales from 2^-spread to 2^spread over tokens and blocks; keys too."""
    rng = np.random.default_rng(spread)
    H, G, lens = 2, 4, [300, 64, 17]

    def fill(kind, b, i, shape):
        x = rng.standard_normal(shape)
        if kind == "v":
            x = x * np.repeat(np.exp2(rng.integers(-spread, spread + 1, shape[:2] + (D // 32,))), 32, -1)
        else:
            x = x * np.repeat(np.exp2(rng.integers(-6, 1, shape[:2] + (D // 32,))), 32, -1)
        return x
    c = Cache(rng, lens, H, D, fill=fill).to_device()
    qf, q = bf16(rng.standard_normal((3, G * H, D)) * 3)
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1] * 3, D ** -0.5)
    for kw in ({}, dict(max_waves=1), dict(max_waves=11, pages_per_step=4)):
        close(decode(c, q, D ** -0.5, **kw), ref, mag, dot, DECODE, str(kw))


def test_queries_of_very_different_sizes():
    """Rows from 2^-100 to 2^60 and beyond binary32: each keeps the scores of
    its own size; the largest finite ones pick one token, infinite ones none."""
    rng = np.random.default_rng(2)
    H, G, D = 1, 9, 128
    c = Cache(rng, [100], H, D).to_device()
    qf, q = bf16(rng.standard_normal((1, G, D)) * np.exp2([-100, -20, 0, 2, 4, 5, 6, 60, 126])[None, :, None])
    scale = 0.05
    ref, mag, dot = kv4.attention(qf[:, :8], *c.pools, c.table, c.lens, [1], scale)
    for kw in ({}, dict(max_waves=1), dict(max_waves=3)):
        out = decode(c, q, scale, **kw)
        close(out[:, :7], ref[:, :7], mag[:, :7], dot[:, :7], DECODE)
        close(out[:, 7:8], ref[:, 7:], mag[:, 7:], 0 * dot[:, 7:], DECODE)     # one token's values
        neg = decode(c, -q, -scale, **kw)
        assert torch.equal(out[:, :8], neg[:, :8])
    # the last row's scores overflow binary32 to both infinities
    assert torch.isnan(out[:, 8]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_queries_that_are_not_finite(D):
    rng = np.random.default_rng(D)
    c = Cache(rng, [50, 20], 2, D).to_device()
    qf, q = bf16(rng.standard_normal((2, 8, D)))
    q[0, 1, 7] = float("nan")
    q[0, 6, 0] = float("inf")
    q[1, 3, D - 1] = -float("inf")
    bad = torch.zeros((2, 8), dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[0, 6] = bad[1, 3] = True
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1, 1], 0.1)
    pre = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.arange(3, dtype=np.int32)), 0.1, pre)
    for out, tol in ((decode(c, q, 0.1), DECODE), (pre, PROMPT)):
        assert torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(out).any(-1), bad)
        m = ~bad.cpu().numpy()
        close(out[~bad], ref[m], mag[m], dot[m], tol)


def test_pools_beyond_four_gigabytes():
    """Pages at the far end of pools of 4.5 GiB: every operator's results and
    bytes are those of the same pages in small pools."""
    H, D, NP = 8, 128, 556_000
    rng = np.random.default_rng(77)
    small = Cache(rng, [60, 33], H, D, room=40).to_device()
    n = small.pools[0].shape[0]
    big = [torch.zeros((NP, H, 17, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert big[0].numel() > 1 << 32
    for b, s in zip(big, (small.k, small.v)):
        b[NP - n:] = s.view(torch.uint8)
    bt = torch.where(small.bt >= 0, small.bt + (NP - n), small.bt)
    k, v = torch.randn((42, H, D), device="cuda").to(torch.bfloat16), torch.randn((42, H, D), device="cuda").to(torch.bfloat16)
    q = torch.randn((42, 4 * H, D), device="cuda").to(torch.bfloat16)
    got = []
    for kp, vp, table in ((small.k, small.v, small.bt), (big[0].view(F4), big[1].view(F4), bt)):
        sl, r = dev(small.lens), []
        bl.kv_append(k[:2], v[:2], kp, vp, table, sl)
        out = torch.empty_like(q[:2])
        bl.decode_attention(q[:2], kp, vp, table, sl, 0.09, out)
        qs = torch.tensor([0, 30, 40], dtype=torch.int32, device="cuda")
        bl.kv_write(k[2:], v[2:], kp, vp, table, sl, qs)
        pre, ko, vo = torch.empty_like(q[2:]), torch.empty_like(k[2:]), torch.empty_like(k[2:])
        bl.prefill_attention(q[2:], kp, vp, table, sl, qs, 0.09, pre)
        bl.kv_read(kp, vp, table, sl, qs, ko, vo)
        got.append([out, pre, ko, vo, sl])
    assert bl.device_errors() == 0
    assert all(torch.equal(a, b) for a, b in zip(*got)) and not torch.isnan(got[0][0]).any()
    for b, s in zip(big, (small.k, small.v)):
        assert torch.equal(b[NP - n:], s.view(torch.uint8)) and not b[:NP - n].any()


def test_bad_pages_and_lengths():
    rng = np.random.default_rng(9)
    c = Cache(rng, [100, 100, 33, 40], 2, 128)
    c.table[1, 3] = 10 ** 6
    c.table[2, 0] = -5
    want = c.lens.copy()
    c.lens[3] = 16 * c.table.shape[1] + 9        # clamped to the table, whose last entries are not pages
    c.to_device()
    qf, q = bf16(rng.standard_normal((4, 8, 128)))
    out = decode(c, q, 0.1)
    assert bl.device_errors() == 2 | 4
    ref, mag, dot = kv4.attention(qf[:1], *c.pools, c.table[:1], want[:1], [1], 0.1)
    close(out[:1], ref, mag, dot, DECODE)
    assert torch.isnan(out[1:]).all()


def test_long_requests_and_many_requests():
    rng = np.random.default_rng(12)
    # 30000 tokens on few heads: many waves a request; then 600 short ones
    c = Cache(rng, [30000, 5], 1, 128).to_device()
    qf, q = bf16(rng.standard_normal((2, 8, 128)))
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1, 1], 128 ** -0.5)
    close(decode(c, q, 128 ** -0.5), ref, mag, dot, DECODE)
    lens = rng.integers(0, 50, 600)
    c = Cache(rng, lens, 2, 64).to_device()
    qf, q = bf16(rng.standard_normal((600, 4, 64)))
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1] * 600, 0.125)
    close(decode(c, q, 0.125), ref, mag, dot, DECODE)


# ----------------------------------------------------------------- prompt --

PROMPTS = [  # H_q, H_kv, D, cached, new
    (8, 2, 64, [0, 3, 16, 0], [1, 17, 64, 130]),
    (32, 8, 128, [0, 100], [65, 200]),
    (3, 3, 128, [63, 64, 65, 0, 5], [1, 1, 1, 16, 0]),
    (16, 1, 64, [500], [33]),
    (28, 4, 128, [1000, 40], [20, 7]),
    (4, 2, 128, [3000], [128]),
]


@pytest.mark.parametrize("H_q,H,D,cached,new", PROMPTS)
def test_prompt_shapes(H_q, H, D, cached, new):
    rng = np.random.default_rng(H_q * D)
    c = Cache(rng, np.add(cached, new), H, D).to_device()
    T = int(np.sum(new))
    qf, q = bf16(rng.standard_normal((T, H_q, D)) * 2)
    qs = dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    out = torch.empty_like(q)
    for scale in (D ** -0.5, -0.05):
        ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, new, scale)
        bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, qs, scale, out)
        close(out, ref, mag, dot, PROMPT, f"scale {scale}")
    assert bl.device_errors() == 0


def test_prompt_many_requests():
    rng = np.random.default_rng(31)
    cached, new = rng.integers(0, 90, 80), rng.integers(0, 40, 80)
    c = Cache(rng, cached + new, 2, 64).to_device()
    qf, q = bf16(rng.standard_normal((int(new.sum()), 4, 64)))
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), 0.125, out)
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, new, 0.125)
    close(out, ref, mag, dot, PROMPT)


def test_prompt_page_outside_the_pool():
    rng = np.random.default_rng(32)
    c = Cache(rng, [64, 64], 2, 128)
    c.table[0, 2] = -1                     # keys 32 .. 47 of request 0
    c.to_device()
    qf, q = bf16(rng.standard_normal((128, 4, 128)))
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.array([0, 64, 128], dtype=np.int32)), 0.1, out)
    assert bl.device_errors() == 4
    ref, mag, dot = kv4.attention(qf[64:], *c.pools, c.table[1:], c.lens[1:], [64], 0.1)
    close(out[64:], ref, mag, dot, PROMPT)
    assert torch.isnan(out[32:64]).all() and not torch.isnan(out[:32]).any()


@pytest.mark.parametrize("D", [64, 128])
def test_prompt_nan_blocks_of_later_tokens(D):
    """NaN blocks reach the rows that see their tokens, not earlier rows of the
    same tile, whole calls and keys shared out."""
    rng = np.random.default_rng(D)
    for cached, new in (([0, 30], [150, 100]), ([2500], [90])):
        end = cached[-1] + new[-1]

        def fill(kind, b, i, shape):
            x = rng.standard_normal(shape)
            if b == len(new) - 1:
                for pos, h, d in ((end - 70, 0, 33), (end - 9, 0, 2), (end - 3, 1, 63)):
                    if kind == "v" and i == pos // 16:
                        x[h, pos % 16, d] = np.nan
                if kind == "k" and i == (end - 5) // 16:
                    x[1, (end - 5) % 16, 7] = np.inf
            return x
        c = Cache(rng, np.add(cached, new), 2, D, fill=fill).to_device()
        qf, q = bf16(rng.standard_normal((sum(new), 6, D)))
        qs = dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        out = torch.empty_like(q)
        bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, qs, 0.1, out)
        with np.errstate(invalid="ignore"):
            ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, new, 0.1)
        T = sum(new)
        want = np.zeros(ref.shape, dtype=bool)               # the oracle's own NaNs are those
        want[T - 70:, :3, 32:64] = want[T - 9:, :3, :32] = want[T - 3:, 3:, 32:64] = want[T - 5:, 3:] = True
        assert np.array_equal(np.isnan(ref), want)
        close(out, ref, mag, dot, PROMPT)


@pytest.mark.parametrize("spread", [6, 20])
def test_prompt_values_of_different_sizes(spread):
    rng = np.random.default_rng(spread)

    def fill(kind, b, i, shape):
        x = rng.standard_normal(shape)
        return x * np.exp2(rng.integers(-spread, spread + 1, shape[:2] + (1,))) if kind == "v" else x
    c = Cache(rng, [300], 1, 128, fill=fill).to_device()
    qf, q = bf16(rng.standard_normal((100, 2, 128)))
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.array([0, 100], dtype=np.int32)), 0.1, out)
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [100], 0.1)
    close(out, ref, mag, dot, PROMPT)


# --------------------------------------------------------- used together --

def test_ctypes_path_gives_the_same(monkeypatch):
    rng = np.random.default_rng(40)
    c = Cache(rng, [40, 70], 2, 128, room=1).to_device()
    _, q = bf16(rng.standard_normal((2, 8, 128)))
    _, k = bf16(rng.standard_normal((2, 2, 128)))
    res = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(_binding, "_native", None)
            monkeypatch.setattr(_binding, "_warned", True)
        c.to_device()
        pos, inv = c.sl.clone(), torch.logspace(0, -4, 64, device="cuda")
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        bl.qk_norm_rope(q, k, pos, inv, qo, ko, q_weight=torch.ones(128, device="cuda"))
        bl.kv_append(ko, k, c.k, c.v, c.bt, c.sl)
        out = decode(c, qo, 0.1)
        rk, rv = torch.empty_like(k), torch.empty_like(k)
        qs = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
        bl.kv_read(c.k, c.v, c.bt, c.sl, qs, rk, rv)
        pre = torch.empty_like(q)
        bl.prefill_attention(qo, c.k, c.v, c.bt, c.sl, qs, 0.1, pre)
        res.append([out, rk, rv, pre, qo, ko, *(torch.from_numpy(b) for b in c.bytes())])
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_decode_step_is_the_two_calls():
    rng = np.random.default_rng(41)
    lens = [0, 15, 16, 100, 255, 64]
    a, b = (Cache(np.random.default_rng(7), lens, 2, 128, room=1) for _ in range(2))
    for c in (a, b):
        c.table[3, 6] = -1                   # the page of request 3's slot and of its tokens 96 .. 99
        c.lens[4] = 16 * c.table.shape[1]    # no room
        c.table[4] = c.table[5, 0]
        c.to_device()
    _, q = bf16(rng.standard_normal((6, 8, 128)))
    _, k = bf16(rng.standard_normal((6, 2, 128)))
    _, v = bf16(rng.standard_normal((6, 2, 128)))
    out = torch.empty_like(q)
    bl.decode_step(k, v, q, a.k, a.v, a.bt, a.sl, 0.1, out, max_waves=9)
    f = bl.device_errors()
    bl.kv_append(k, v, b.k, b.v, b.bt, b.sl)
    two = decode(b, q, 0.1, max_waves=9)
    assert f == bl.device_errors() == 1 | 4
    assert torch.equal(out.view(torch.int16), two.view(torch.int16)) and torch.equal(a.sl, b.sl)
    assert torch.isnan(out[3]).all() and not torch.isnan(out[[0, 1, 2, 4, 5]]).any()
    assert all(np.array_equal(x, y) for x, y in zip(a.bytes(), b.bytes()))


def test_step_captured_and_replayed():
    """Norm, rotation, append and attention of a growing batch from a graph."""
    rng = np.random.default_rng(42)
    lens, H, G, D, steps = [30, 1, 500, 64], 2, 4, 128, 5
    c = [Cache(np.random.default_rng(3), lens, H, D, room=steps + 1).to_device() for _ in range(2)]
    inv = torch.logspace(0, -4, D // 2, device="cuda")
    w = torch.rand(D, device="cuda").to(torch.bfloat16)
    x = torch.randn((steps, 4, (G + 2) * H, D), device="cuda").to(torch.bfloat16)
    cur, outs = x[0].clone(), []

    def step(c, rows, out, qo, ko):
        q, k, v = rows[:, :G * H], rows[:, G * H:G * H + H], rows[:, G * H + H:]
        bl.qk_norm_rope(q, k, c.sl, inv, qo, ko, q_weight=w, k_weight=w)
        bl.kv_append(ko, v, c.k, c.v, c.bt, c.sl)
        bl.decode_attention(qo, c.k, c.v, c.bt, c.sl, 0.1, out)
    bufs = [[torch.empty((4, n, D), dtype=torch.bfloat16, device="cuda") for n in (G * H, G * H, H)] for _ in range(2)]
    bl.decode_attention(bufs[0][0].zero_(), c[0].k, c[0].v, c[0].bt, c[0].sl, 0.1, bufs[0][1])   # the workspace grows
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(c[0], cur, *bufs[0])
    for i in range(steps):
        cur.copy_(x[i])
        g.replay()
        torch.cuda.synchronize()
        step(c[1], x[i], *bufs[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*bufs)), i
        assert all(np.array_equal(a, b) for a, b in zip(c[0].bytes(), c[1].bytes())), i
    assert torch.equal(c[0].sl, c[1].sl) and bl.device_errors() == 0


def test_prompt_then_decode_run():
    """Two requests prefilled in chunks and decoded, all operators as a model's
    layer uses them, against the same run in binary64 (rows rounded to bf16
    where the library hands them over)."""
    rng = np.random.default_rng(50)
    H, G, D, F = 2, 4, 128, 64
    inv32 = (10000.0 ** (-np.arange(F) / F)).astype(np.float32)
    wf, w = bf16(1 + 0.1 * rng.standard_normal(D))
    c = Cache(rng, [0, 0], H, D, room=120).to_device()
    inv = dev(inv32)
    for new in ([40, 17], [33, 64], [1, 1], [1, 1]):
        T = sum(new)
        xf, x = bf16(rng.standard_normal((T, (G + 2) * H, D)))
        q, k, v = x[:, :G * H], x[:, G * H:-H], x[:, -H:]
        pos = np.concatenate([c.lens[b] + np.arange(n) for b, n in enumerate(new)]).astype(np.int32)
        qo, ko = torch.empty((T, G * H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
        bl.qk_norm_rope(q, k, dev(pos), inv, qo, ko, q_weight=w, k_weight=w)
        turned = rope.rotate(rope.norm(xf[:, :-H], wf), pos, inv32)
        got = torch.cat([qo, ko], 1).double().cpu().numpy()
        assert (np.abs(got - turned) <= 2.0 ** -8 * np.abs(turned) + 2.0 ** -18 * np.abs(turned).max()).all()
        qs = dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        out = torch.empty_like(qo)
        if new == [1, 1]:
            bl.kv_append(ko, v, c.k, c.v, c.bt, c.sl)
            bl.decode_attention(qo, c.k, c.v, c.bt, c.sl, D ** -0.5, out)
        else:
            bl.kv_write(ko, v, c.k, c.v, c.bt, c.sl, qs)
            bl.prefill_attention(qo, c.k, c.v, c.bt, c.sl, qs, D ** -0.5, out)
        kv4.write(*c.pools, ko.double().cpu().numpy(), xf[:, -H:], c.table, c.lens, new)
        ref, mag, dot = kv4.attention(qo.double().cpu().numpy(), *c.pools, c.table, c.lens, new, D ** -0.5)
        close(out, ref, mag, dot, DECODE if new == [1, 1] else PROMPT)
    assert all(np.array_equal(a, b) for a, b in zip(c.bytes(), c.pools)) and bl.device_errors() == 0


def test_prompt_graphs_share_the_workspace():
    """Write, attention and read back of two batches (planned in the waves, and
    by a launch), a graph each, replayed in turn with eager calls between."""
    rng = np.random.default_rng(70)
    H, G, D, rounds = 2, 2, 64, 3
    kinds = [([40, 3], [37, 70]), (list(rng.integers(0, 60, 70)), list(rng.integers(0, 9, 70)))]
    sets = []
    for cached, new in kinds:
        T = int(sum(new))
        pair = [Cache(np.random.default_rng(5), cached, H, D, room=rounds * max(new)).to_device() for _ in range(2)]
        qs = dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        # five rows that no request owns: left alone
        x = torch.randn((rounds, T + 5, (G + 2) * H, D), device="cuda").to(torch.bfloat16)
        outs = [[torch.full((T + 5, n, D), 3.0, dtype=torch.bfloat16, device="cuda") for n in (G * H, H, H)] for _ in range(2)]
        sets.append((pair, qs, x, outs, x[0].clone(), T))

    def step(c, qs, rows, outs):
        bl.kv_write(rows[:, G * H:-H], rows[:, -H:], c.k, c.v, c.bt, c.sl, qs)
        bl.prefill_attention(rows[:, :G * H], c.k, c.v, c.bt, c.sl, qs, 0.1, outs[0])
        bl.kv_read(c.k, c.v, c.bt, c.sl, qs, outs[1], outs[2])
    graphs = []
    for pair, qs, x, outs, cur, T in sets:           # the workspace grows on caches of no use
        spare = Cache(np.random.default_rng(5), pair[0].lens, H, D, room=99).to_device()
        step(spare, qs, cur, [torch.empty_like(o) for o in outs[0]])
    torch.cuda.synchronize()
    for pair, qs, x, outs, cur, T in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(pair[0], qs, cur, outs[0])
        graphs.append(g)
    bl.device_errors()
    for i in range(rounds):
        for g, (pair, qs, x, outs, cur, T) in zip(graphs, sets):
            cur.copy_(x[i])
            g.replay()
        for pair, qs, x, outs, cur, T in sets:
            step(pair[1], qs, x[i], outs[1])
        torch.cuda.synchronize()
        for pair, qs, x, outs, cur, T in sets:
            assert all(torch.equal(a, b) for a, b in zip(*outs)), i
            assert all((o[T:] == 3).all() for o in outs[0]) and not torch.isnan(outs[0][0]).any()
            assert all(np.array_equal(a, b) for a, b in zip(pair[0].bytes(), pair[1].bytes())), i
    assert bl.device_errors() == 1 | 2                    # the rows of no request
    assert all(torch.equal(p[0].sl, p[1].sl) for p, *_ in sets)


def test_another_stream():
    rng = np.random.default_rng(60)
    c = Cache(rng, [90, 400], 2, 128, room=1).to_device()
    qf, q = bf16(rng.standard_normal((2, 8, 128)))
    kf, k = bf16(rng.standard_normal((2, 2, 128)))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    out = torch.empty_like(q)
    with torch.cuda.stream(st):
        bl.kv_append(k, k, c.k, c.v, c.bt, c.sl)
    bl.decode_attention(q, c.k, c.v, c.bt, c.sl, 0.1, out, stream=st)
    st.synchronize()
    kv4.write(*c.pools, kf, kf, c.table, c.lens, [1, 1])
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1, 1], 0.1)
    close(out, ref, mag, dot, DECODE)


# ------------------------------------------- sizes within one query, one page --

def lost_terms(qf, c, new, scale):
    """[T, H_q, 1]: of each row the largest sum over 32-dim blocks of a query's
    largest magnitude times the key's magnitudes, scaled.  A query dim below
    2^-14 of its block's largest loses bits: it is held within 2^-21 of that."""
    T, H_q, D = qf.shape
    top = np.abs(qf).reshape(T, H_q, D // 32, 32).max(-1)
    out, i = np.zeros((T, H_q, 1)), 0
    for b, n in enumerate(new):
        L = int(c.lens[b])
        k = np.abs(kv4.read_pages(c.pools[0], c.table[b, :(L + 15) // 16], "k")[:L]).reshape(L, c.H, D // 32, 32).sum(-1)
        for h in range(H_q):
            out[i:i + n, h, 0] = (top[i:i + n, h] @ k[:, h // (H_q // c.H)].T).max(-1) * abs(scale)
        i += n
    return out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["blocks", "dims"])
def test_query_dims_of_very_different_sizes(D, where):
    """Dims of 2^-30 to 1 in one query, whose small blocks meet keys as much
    larger, or side by side in a block: every product counts."""
    rng = np.random.default_rng(D)
    H, G, new, scale = 2, 3, [1, 20, 1], D ** -0.5
    lens = [200, 90, 700]
    exps = np.stack([rng.permutation(np.linspace(0, 30, D // 32)).round() for _ in range(H)])       # [H, D / 32]

    def fill(kind, b, i, shape):
        x = rng.standard_normal(shape)
        return x * np.repeat(np.exp2(exps), 32, -1)[:, None] if kind == "k" and where == "blocks" else x
    c = Cache(rng, lens, H, D, fill=fill).to_device()
    T = sum(new)
    size = np.repeat(-exps, 32, -1).repeat(G, 0)[None] if where == "blocks" else rng.integers(-30, 1, (T, G * H, D))
    qf, q = bf16(rng.standard_normal((T, G * H, D)) * np.exp2(size) * 2)
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, new, scale)
    lost = 2.0 ** -8 * lost_terms(qf, c, new, scale)             # 2^-20 of it, in close()'s 2^-12
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), scale, out)
    close(out, ref, mag, dot + lost, PROMPT)
    last = np.cumsum(new) - 1
    for kw in ({}, dict(max_waves=1), dict(max_waves=7)):
        close(decode(c, q[last].contiguous(), scale, **kw), ref[last], mag[last], (dot + lost)[last], DECODE, str(kw))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread", [8, 40, 100])
@pytest.mark.parametrize("cached,new", [([200, 0, 47], [40, 100, 17]), ([2400, 700], [30, 1])], ids=["whole", "keys-shared-out"])
def test_prompt_values_of_very_different_sizes(D, spread, cached, new):
    """Scales from 2^-spread to 2^spread over tokens and blocks.  Beside the
    roundings that close() knows: a value is held within 2^-40 of the largest of
    its 64-token step (the fp16 copy), a weight within 2^-25 of the row's largest
    (fp16), so A grows by 2^-40 / c of the weights times those largest values and
    by 2^-25 / c of the values' sum."""
    rng = np.random.default_rng(spread + D)
    H, G, scale = 2, 3, 0.05

    def fill(kind, b, i, shape):
        x = rng.standard_normal(shape)
        if kind == "v":
            x = x * np.repeat(np.exp2(rng.integers(-spread, spread + 1, shape[:2] + (D // 32,))), 32, -1)
        return x
    c = Cache(rng, np.add(cached, new), H, D, fill=fill).to_device()
    T = sum(new)
    qf, q = bf16(rng.standard_normal((T, G * H, D)))
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), scale, out)
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, new, scale)
    i = 0
    for b, n in enumerate(new):
        L = int(c.lens[b])
        pages = c.table[b, :(L + 15) // 16]
        k, v = kv4.read_pages(c.pools[0], pages, "k")[:L], np.abs(kv4.read_pages(c.pools[1], pages, "v")[:L])
        for h in range(G * H):
            g = h // G
            top = np.array([v[t // 64 * 64:t // 64 * 64 + 64, g].max() for t in range(L)])
            seen = np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]
            w = np.where(seen, np.exp(qf[i:i + n, h] @ k[:, g].T * scale), 0)
            w /= w.sum(-1, keepdims=True)
            mag[i:i + n, h] += (2.0 ** -40 * (w @ top)[:, None] + 2.0 ** -25 * (seen @ v[:, g])) / PROMPT
        i += n
    close(out, ref, mag, dot, PROMPT)
    assert bl.device_errors() == 0


# ------------------------------------------------------- errors as a whole --

def noise(qf, c, new, scale):
    """(out, spread, dot): spread the root of the sum of squares of a row's
    weights times values, what independent relative errors of its weights add up
    to; dot the largest sum of |products| of a score."""
    T, H_q, D = qf.shape
    out, spread, dot, i = np.zeros(qf.shape), np.zeros(qf.shape), np.zeros((T, H_q, 1)), 0
    for b, n in enumerate(new):
        L = int(c.lens[b])
        pages = c.table[b, :(L + 15) // 16]
        k, v = (kv4.read_pages(p, pages, kind)[:L] for p, kind in zip(c.pools, "kv"))
        seen = np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]
        for h in range(H_q):
            g = h // (H_q // c.H)
            s = np.where(seen, qf[i:i + n, h] @ k[:, g].T * scale, -np.inf)
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            out[i:i + n, h] = w @ v[:, g]
            spread[i:i + n, h] = np.sqrt(w ** 2 @ v[:, g] ** 2)
            dot[i:i + n, h, 0] = (np.abs(qf[i:i + n, h]) @ np.abs(k[:, g]).T).max(-1) * abs(scale)
        i += n
    return out, spread, dot


def close_as_a_whole(got, qf, c, new, scale, weight, what=""):
    """The norm of the errors of a call's outputs.  A rounding to bf16 is spread
    over +-2^-8 / (1 .. 2) of the value, rms at most 2^-8 / sqrt(3) of it; a
    weight is off by `weight` and by its score's error, 2^-13 dot at most, from
    key to key independently."""
    ref, spread, dot = noise(qf, c, new, scale)
    got = got.float().cpu().double().numpy()
    bound = 2.0 ** -8 / 3 ** 0.5 * np.linalg.norm(ref) + np.linalg.norm((weight + 2.0 ** -13 * dot) * spread)
    off = np.linalg.norm(got - ref)
    assert off <= bound, f"{what}: {off / np.linalg.norm(ref):.3e} of the outputs, {bound / np.linalg.norm(ref):.3e} allowed"


@pytest.mark.parametrize("D,H,G", [(64, 2, 4), (128, 2, 4), (128, 1, 16), (64, 3, 1)])
@pytest.mark.parametrize("lens", [[50, 200, 7], [9000, 4000]], ids=["short", "long"])
def test_errors_as_a_whole(D, H, G, lens):
    rng = np.random.default_rng(D + H + G)
    scale = D ** -0.5
    c = Cache(rng, lens, H, D).to_device()
    qf, q = bf16(rng.standard_normal((len(lens), G * H, D)))
    for kw in ({}, dict(max_waves=1), dict(max_waves=100)):
        close_as_a_whole(decode(c, q, scale, **kw), qf, c, [1] * len(lens), scale, 2.0 ** -14, f"decode {kw}")
    new = [min(30, n) for n in lens]
    qf, q = bf16(rng.standard_normal((sum(new), G * H, D)))
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), scale, out)
    close_as_a_whole(out, qf, c, new, scale, 2.0 ** -12, "prompt")


@pytest.mark.parametrize("H,waves", [(4, (8, 12, 16)), (2, (6, 8)), (6, (10, 16, 24))])
def test_weighted_shares_of_heads_side_by_side(H, waves):
    """384 pages a wave and more, over workgroups of both weights: the waves that
    take a group's heads side by side share one range of uneven size."""
    rng = np.random.default_rng(H)
    D, scale = 64, 0.125
    lens = [11000, 1, 6500, 0, 8200]
    c = Cache(rng, lens, H, D).to_device()
    qf, q = bf16(rng.standard_normal((5, 2 * H, D)))
    keep = [b for b, n in enumerate(lens) if n]
    pages = H * sum((n + 15) // 16 for n in lens)
    ref, mag, dot = kv4.attention(qf, *c.pools, c.table, c.lens, [1] * 5, scale)
    for w in waves:
        assert pages >= 384 * w and w > 5
        for skew in (255, 0, 100, -1):
            out = decode(c, q, scale, max_waves=w, xcd_skew=skew)
            close(out, ref, mag, dot, DECODE, f"{w} waves, skew {skew}")
            assert not out[3].any() and torch.equal(out, decode(c, q, scale, max_waves=w, xcd_skew=skew))
    sub = Cache.__new__(Cache)
    sub.H, sub.pools, sub.table, sub.lens = c.H, c.pools, c.table[keep], c.lens[keep]
    close_as_a_whole(out[keep], qf[keep], sub, [1] * len(keep), scale, 2.0 ** -14)
    assert bl.device_errors() == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale_byte", [227, 254, 255])
def test_a_page_outside_the_pool_takes_nothing_from_the_first(D, scale_byte):
    """Rows before its tokens are those of the pages they see, whatever the
    pool's first page holds: values of 2^100 and more, infinite ones, NaN."""
    rng = np.random.default_rng(D)
    H, lens = 2, [64, 70]
    c = Cache(rng, lens, H, D, spare=40)
    free = 0                                              # the first page, of no request
    if free in c.table:
        at, other = c.table == free, c.spare[0]
        for pool in c.pools:
            pool[other] = pool[free]
        c.table[at] = other
    for pool in c.pools:
        pool[free, :, 16], pool[free, :, :16] = scale_byte, 0x77
    c.table[0, 1] = c.pools[0].shape[0]
    c.table[1, 4] = -1
    c.to_device()
    qf, q = bf16(rng.standard_normal((sum(lens), 4, D)))
    out = torch.empty_like(q)
    bl.prefill_attention(q, c.k, c.v, c.bt, c.sl, dev(np.array([0, 64, 134], dtype=np.int32)), 0.1, out)
    assert bl.device_errors() == 4
    for b, first, n in ((0, 0, 16), (1, 64, 64)):         # each request's rows before the page
        ref, mag, dot = kv4.attention(qf[first:first + n], *c.pools, c.table[b:b + 1], np.array([n], dtype=np.int32), [n], 0.1)
        close(out[first:first + n], ref, mag, dot, PROMPT, f"request {b}")
    assert torch.isnan(out[16:64]).all() and torch.isnan(out[128:]).all()


def test_one_call_step_captured_and_replayed():
    """bellman_decode_step over 4-bit pools from a graph, a growing batch, with
    eager calls on a second cache between the replays; a refused call leaves
    pools and lengths alone."""
    lens, H, G, D, steps = [30, 1, 500, 64, 0], 2, 4, 64, 4
    a, b = (Cache(np.random.default_rng(3), lens, H, D, room=steps + 1).to_device() for _ in range(2))
    rows = torch.randn((steps, 5, (G + 2) * H, D), device="cuda").to(torch.bfloat16)
    cur, outs = rows[0].clone(), [torch.full((5, G * H, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def step(c, x, out):
        bl.decode_step(x[:, G * H:-H], x[:, -H:], x[:, :G * H], c.k, c.v, c.bt, c.sl, 0.1, out)
    before = a.bytes()
    with pytest.raises(bl.BellmanError):
        step(a, cur, torch.empty((5, G * H + 1, D), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(bl.BellmanError):
        bl.decode_step(cur[:, G * H:-H], cur[:, -H - 1:], cur[:, :G * H], a.k, a.v, a.bt, a.sl, 0.1, outs[0])
    torch.cuda.synchronize()
    assert all(np.array_equal(x, y) for x, y in zip(before, a.bytes())) and a.sl.tolist() == lens
    bl.decode_attention(cur[:, :G * H], a.k, a.v, a.bt, a.sl, 0.1, outs[0])          # the workspace grows
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a, cur, outs[0])
    for i in range(steps):
        cur.copy_(rows[i])
        g.replay()
        step(b, rows[i], outs[1])
        torch.cuda.synchronize()
        assert torch.equal(*outs) and not torch.isnan(outs[0]).any()
        assert all(np.array_equal(x, y) for x, y in zip(a.bytes(), b.bytes()))
    assert torch.equal(a.sl, b.sl) and a.sl.tolist() == [n + steps for n in lens] and bl.device_errors() == 0


@pytest.mark.parametrize("B", [64, 65, 200])      # planned in the waves, and by a launch
def test_read_of_malformed_requests_among_many(B):
    rng = np.random.default_rng(B)
    lens = rng.integers(1, 40, B)
    c = Cache(rng, lens, 1, 64)
    n = np.minimum(lens, rng.integers(0, 40, B))
    n[5] = lens[5] + 1                              # more rows than it has
    c.lens[7] = 16 * c.table.shape[1] + 1           # past the table
    c.lens[9] = -3
    c.to_device()
    at = np.concatenate([[0], np.cumsum(n)])
    ko, vo = (torch.full((int(at[-1]) + 2, 1, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bl.kv_read(c.k, c.v, c.bt, c.sl, dev(at.astype(np.int32)), ko, vo)
    assert bl.device_errors() == 2
    for got, pool, kind in ((ko, c.pools[0], "k"), (vo, c.pools[1], "v")):
        got = got.double().cpu().numpy()
        for b in range(B):
            rows = got[at[b]:at[b + 1]]
            if b in (5, 7, 9):
                assert (rows == 5).all()
            else:
                L = int(lens[b])
                assert np.array_equal(rows, kv4.read_pages(pool, c.table[b, :(L + 15) // 16], kind)[L - n[b]:L])
        assert (got[at[-1]:] == 5).all()
