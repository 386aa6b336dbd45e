// Norm and rotation of queries and keys, before they enter the cache and the
// attention: y = R(p) (x / sqrt(mean(x^2) + eps) * (w + offset)) per head row,
// R(p) turning each pair of the first R dims by position times frequency.
//
// Bound by memory: (H_q + H_kv) D values a token read and written once (36,001
// tokens of 32/8 heads of 128, 737 MB, in 128 us, 5.8 TB/s; 4,613 of 28/4 in
// 15.8 us; 64 tokens 4.1 us, a launch's latency).  Six waves a SIMD (70
// registers; at four, 8,000 tokens of 64 dims took 23 us instead of 17.4, and
// loads a pass ahead cost more registers than they hid).  A row
// is D / 16 lanes, each with two 16-byte units whose values pair up (dims i and
// i + R / 2, or neighbours), so nothing crosses lanes but the sum of squares; a
// wave walks a token's rows, 64 / (D / 16) at a time, queries first.  A lane's
// eight angles are the same for all rows of the token: they are formed once a
// wave, in turns, the product in binary64 (a position of 2^20 times a frequency
// near 1 is within 2^-35 turns there, in binary32 2^-5.7), its fraction, rounded
// to binary32 (2^-26), to the sine and cosine units, which take turns (measured
// within 1.3e-7).
// Everything between the loads and the rounding to bf16 is binary32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"

namespace bellman {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void widen8(const u32x4& u, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ u32x4 round8(const float* y) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 v = {y[2 * i], y[2 * i + 1]};
        u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));   // nearest even
    }
    return u;
}

// Sum over the LPR (4 or 8) neighbouring lanes of a row.
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, true));   // lane ^ 1
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, true));   // lane ^ 2
    if (LPR == 8)
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true));   // half mirror
    return v;
}

constexpr float kTinyMean = 0x1p-100f;   // from it on the squares that count are normal numbers

// STREAM: the stores (1) or loads and stores (2) pass the caches by.
template <int D, bool INTER, int STREAM>
__global__ void __launch_bounds__(256, 6) qk_norm_rope_kernel(RopeArgs a) {
    constexpr int LPR = D / 16, RPW = 64 / LPR;     // lanes a row, rows a pass
    const int lane = threadIdx.x & 63, j = lane % LPR, sub = lane / LPR;
    const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = id / a.chunks;
    if (t >= a.T) return;
    const int c = (int)(id - t * a.chunks);
    const int pq = (a.H_q + RPW - 1) / RPW, passes = pq + (a.H_kv + RPW - 1) / RPW;
    const int p0 = passes * c / a.chunks, p1 = passes * (c + 1) / a.chunks;

    // this lane's units; the first R / 16 lanes of a row rotate theirs
    const bool turns = j < a.R / 16;
    const int ua = !INTER && turns ? 8 * j : 16 * j, ub = !INTER && turns ? 8 * j + a.R / 2 : 16 * j + 8;
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cs[i] = 1.f;
        sn[i] = 0.f;
    }
    if (turns) {
        int pos[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) pos[x] = a.positions[min(x, a.axes - 1) * a.pos_stride + t];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int f = 8 * j + i;
            const int p = f < a.cut[0] ? pos[0] : f < a.cut[1] ? pos[1] : f < a.cut[2] ? pos[2] : pos[3];
            const double r = (double)p * (double)a.inv_freq[f] * 0.15915494309189535;   // 1 / (2 pi)
            const float turn = (float)(r - __builtin_rint(r));
            cs[i] = __builtin_amdgcn_cosf(turn);
            sn[i] = __builtin_amdgcn_sinf(turn);
        }
    }
    float w[16];
    int have = -1;         // whose weights w holds: 0 queries, 1 keys
    for (int p = p0; p < p1; ++p) {
        const bool isk = p >= pq;
        const int H = isk ? a.H_kv : a.H_q;
        const int row = (isk ? p - pq : p) * RPW + sub, h = min(row, H - 1);
        const uint16_t* src = isk ? a.k + t * a.k_st + (int64_t)h * a.k_sh : a.q + t * a.q_st + (int64_t)h * a.q_sh;
        u32x4 xa, xb;
        if (STREAM == 2) {
            xa = __builtin_nontemporal_load((const u32x4*)(src + ua));
            xb = __builtin_nontemporal_load((const u32x4*)(src + ub));
        } else {
            xa = *(const u32x4*)(src + ua);
            xb = *(const u32x4*)(src + ub);
        }
        const void* wp = isk ? a.k_weight : a.q_weight;
        if (wp && have != (int)isk) {
            have = (int)isk;
            if (isk ? a.kw_fp32 : a.qw_fp32) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = ((const float*)wp)[ua + i] + a.offset;
                    w[8 + i] = ((const float*)wp)[ub + i] + a.offset;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = __uint_as_float((uint32_t)((const uint16_t*)wp)[ua + i] << 16) + a.offset;
                    w[8 + i] = __uint_as_float((uint32_t)((const uint16_t*)wp)[ub + i] << 16) + a.offset;
                }
            }
        }
        float x[16];
        widen8(xa, x);
        widen8(xb, x + 8);
        if (wp) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
            float ms = row_sum<LPR>(ss) * (1.f / D) + a.eps;
            if (__any(ms < kTinyMean)) {
                // rows of tiny values under a tiny eps: their squares leave
                // binary32, so they are taken 2^75 times as large
                const float up = ms < kTinyMean ? 0x1p75f : 1.f;
                ss = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[i] *= up;
                    ss = __builtin_fmaf(x[i], x[i], ss);
                }
                ms = row_sum<LPR>(ss) * (1.f / D) + a.eps * up * up;
            }
            const float inv = rsqrtf(ms);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = x[i] * inv * w[i];
        }
        u32x4 ya, yb;
        if (turns) {
            float y[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // the pair of frequency 8 j + i
                const int e = INTER ? 2 * i : i, o = INTER ? 2 * i + 1 : i + 8;
                y[e] = __builtin_fmaf(x[e], cs[i], -(x[o] * sn[i]));
                y[o] = __builtin_fmaf(x[o], cs[i], x[e] * sn[i]);
            }
            ya = round8(y);
            yb = round8(y + 8);
        } else {
            ya = round8(x);
            yb = round8(x + 8);
        }
        if (row < H) {
            uint16_t* dst = isk ? a.k_out + t * a.ko_st + (int64_t)h * a.ko_sh : a.q_out + t * a.qo_st + (int64_t)h * a.qo_sh;
            if (STREAM) {
                __builtin_nontemporal_store(ya, (u32x4*)(dst + ua));
                __builtin_nontemporal_store(yb, (u32x4*)(dst + ub));
            } else {
                *(u32x4*)(dst + ua) = ya;
                *(u32x4*)(dst + ub) = yb;
            }
        }
    }
}

}  // namespace

void launch_qk_norm_rope(const RopeArgs& args, hipStream_t s) {
    RopeArgs a = args;
    const int rpw = 64 / (a.D / 16);
    const int passes = (a.H_q + rpw - 1) / rpw + (a.H_kv + rpw - 1) / rpw;
    // A token's passes go over as many waves as it takes to have 2048 (two a SIMD);
    // from 2048 tokens on one wave takes a token and forms its angles once (for
    // 1024, 2048, 4096 waves, us: 1,024 tokens of 32/8 heads of 128 7.0, 6.5, 7.1,
    // 2,048 8.4, 8.3, 8.9, 256 5.3, 5.1, 5.1).
    a.chunks = (int)std::min<int64_t>(passes, (2048 + a.T - 1) / a.T);
    const dim3 grid((unsigned)(((int64_t)a.T * a.chunks + 3) / 4));
    // Streamed (stores; loads and stores / neither, us; rows of 32/8 heads): stores
    // of pairs (i, i + F) at head_dim 128, where an instruction writes whole lines:
    // 2,048 tokens 8.4 / 10.8, 8,000 29.9 / 30.1, 20,000 65 / 82.  The others once
    // input and output pass the 256 MB memory-side cache: head_dim 64 20,000 37.7 /
    // 34.1, 72,000 137 / 144, neighbouring pairs 9,000 of 28/4 31 / 28, 20,000 77 /
    // 87.  The loads too, of whole lines, once the input alone is well past it:
    // 30,000 107 / 105 with stores alone, 33,000 118 / 122, 60,000 210 / 225.
    const int64_t in = (int64_t)a.T * (a.H_q + a.H_kv) * a.D * 2;
    const bool lines = a.D == 128 && !a.interleaved;
    const int stream = lines ? 1 + (a.R == a.D && in > (320 << 20)) : 2 * in > (256 << 20);
    const auto kernel =
        a.D == 128 ? (a.interleaved ? (stream ? qk_norm_rope_kernel<128, true, 1> : qk_norm_rope_kernel<128, true, 0>)
                                    : (stream == 2 ? qk_norm_rope_kernel<128, false, 2> : qk_norm_rope_kernel<128, false, 1>))
                   : (a.interleaved ? (stream ? qk_norm_rope_kernel<64, true, 1> : qk_norm_rope_kernel<64, true, 0>)
                                    : (stream ? qk_norm_rope_kernel<64, false, 1> : qk_norm_rope_kernel<64, false, 0>));
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
}

}  // namespace bellman
