// Rotary positions, and the step between W_kv_a and the attention (LayerNorm of the latent and rotation of the
// shared key in one pass), forward and backward.  The paper takes q_rope and k_pe as already rotated; these
// kernels are what rotates them.
//
//   angle(m, j) = position_m * freq_j,   j = 0 .. d_rot/2 - 1
//   (a, b) -> mscale * (a cos - b sin, b cos + a sin)        inverse: sin -> -sin, which is the transpose, i.e.
//                                                            the gradient (mscale included)
// for the pairs (2j, 2j+1) of the rotated channels (interleaved) or (j, j + d_rot/2) (half).
//
// The angle needs more than fp32: at position 4e6 an fp32 product is off by a quarter of a radian.  It is formed in fixed point: freq /
// (2 pi), reduced to its fraction in fp64, becomes a 64-bit fraction of a turn, and position times that, modulo 2^64, is the
// fraction of a turn -- two integer multiplications, where fp64 arithmetic cost three times the instructions.  Errors: fp64's rounding of
// freq / (2 pi), position * freq * 2^-52 radians (2^-30 at position 4e6 and freq 1, 2^-21 at 2^31); the 32 bits kept, 2^-32 of a turn; their
// conversion to fp32 radians, 3 pi 2^-24.  Sine and cosine of the reduced angle in [-pi, pi] come from the special-function unit,
// whose absolute error is below 2^-21.  Together 2^-19 at any 32-bit position and freq up to 1: far under the half step (2^-8) of the
// bf16 result.
//
// Everything here reads and writes every element once; the kernels come close enough to HBM speed that instructions count
// (a warp moves 512 bytes per load, and an SM gets 4 instructions per clock for about 23 bytes per clock).
#pragma once
#include "layernorm_sm100.cuh"
#include "sm100_ptx.cuh"

namespace laga {

constexpr int kRopeMaxD = 1024;        // channels of a head
constexpr int kRopeMaxRot = 256;       // rotated channels
constexpr int kRopeRowsPerThread = 4;

struct Rotary {
    const int* positions;              // [M]
    const double* freqs;               // [d_rot / 2], radians per position
    float mscale;
    int interleaved, inverse;
};

// freq (radians per position) as a 64-bit fraction of a turn per position
__device__ __forceinline__ unsigned long long rotary_step(double freq) {
    const double turns = freq * 0.15915494309189533577;
    return static_cast<unsigned long long>((turns - floor(turns)) * 18446744073709551616.0);
}
// (cos, sin) * mscale of a pair at one position; `inverse` turns the other way.
__device__ __forceinline__ float2 rotary_turn(const Rotary& r, int position, unsigned long long step) {
    const unsigned long long turn = static_cast<unsigned long long>(static_cast<long long>(position)) * step;
    const float phi = static_cast<float>(static_cast<int>(turn >> 32)) * 1.4629180792671596e-9f;      // 2 pi / 2^32
    float s, c;
    __sincosf(phi, &s, &c);
    if (r.inverse) s = -s;
    return make_float2(c * r.mscale, s * r.mscale);
}
__device__ __forceinline__ float2 rotary_apply(float2 turn, float a, float b) {
    return make_float2(fmaf(a, turn.x, -b * turn.y), fmaf(b, turn.x, a * turn.y));
}

// y[m, i, :] = x[m, i, :] with channels [rot_begin, rot_begin + d_rot) rotated.  Rows of h heads of d channels, row
// pitches in elements.  A block takes rows_per_block = blockDim.y * 4 rows (m, i) of the flattened [M, h]: the loads
// go out first, then the block's threads fill the table of (cos, sin) of the tokens those rows touch (once per token,
// not once per head: with 16 heads that is 1/16 of the integer and special-function work), then each thread rotates or
// copies its 16 bytes.  threadIdx.x is the unit within the head, so no index needs a division but the token's.
// A unit is eight channels: a 16-byte chunk, or in half layout, among the rotated channels, four of the first half and
// their four partners, so that in both layouts a unit is whole pairs and x and y may be the same buffer.
// in_place: only the rotated units run.
// Bound by HBM: 16384 tokens of 16 heads of 192 channels 32.0 us, 6.3 TB/s; 8192 tokens of 128 heads, half layout, 122 us, 6.6 TB/s (a plain
// copy here: 6.45).  Eight tokens of 16 heads: 2.4 us, the launch and two round trips.
struct RopeArgs {
    const __nv_bfloat16* x;
    __nv_bfloat16* y;
    unsigned x_pitch, y_pitch;             // bytes
    int M, h, d, rot_begin, d_rot, in_place;
    unsigned h_magic;                      // ceil(2^32 / h) for h <= kRopeMagicHeads
    Rotary rot;
};
constexpr int kRopeMagicHeads = 1024;

template <bool kInterleaved>
__global__ void __launch_bounds__(256, 5)
rope_kernel(const RopeArgs a) {
    extern __shared__ float2 turns[];                       // [tokens of this block][d_rot / 2]
    const int n_pairs = a.d_rot >> 1;
    const int before = a.in_place ? 0 : a.rot_begin >> 3;   // units copied in front of the rotated ones
    const int u = static_cast<int>(threadIdx.x) - before;   // rotated unit, if it is one
    const bool rotates = u >= 0 && u < (a.d_rot >> 3);
    const bool split = !kInterleaved && rotates;            // two runs of four channels, n_pairs apart
    const int c0 = split ? a.rot_begin + u * 4 : rotates ? a.rot_begin + u * 8 : static_cast<int>(threadIdx.x) * 8;
    const long long row0 = static_cast<long long>(blockIdx.x) * (blockDim.y * kRopeRowsPerThread);
    const int n_rows = static_cast<int>(min(static_cast<long long>(blockDim.y * kRopeRowsPerThread), static_cast<long long>(a.M) * a.h - row0));
    const int first_token = static_cast<int>(row0 / a.h), first_head = static_cast<int>(row0 - static_cast<long long>(first_token) * a.h);
    // (token, head) of the block's row i: i + first_head is below h + 1024
    auto token_of = [&](int i) -> int {
        const unsigned r = static_cast<unsigned>(i + first_head);
        return a.h <= kRopeMagicHeads ? static_cast<int>(__umulhi(r, a.h_magic)) : static_cast<int>(r >= static_cast<unsigned>(a.h));
    };
    const uint8_t* x0 = reinterpret_cast<const uint8_t*>(a.x) + static_cast<long long>(first_token) * a.x_pitch + c0 * 2;
    uint8_t* y0 = reinterpret_cast<uint8_t*>(a.y) + static_cast<long long>(first_token) * a.y_pitch + c0 * 2;
    const int gap = split ? n_pairs * 2 : 8;                // bytes between the unit's halves

    uint4 v[kRopeRowsPerThread];
    int token[kRopeRowsPerThread], head_at[kRopeRowsPerThread];
#pragma unroll
    for (int k = 0; k < kRopeRowsPerThread; ++k) {
        const int i = threadIdx.y + k * blockDim.y;
        token[k] = a.h == 1 ? i : token_of(i);
        head_at[k] = (i + first_head - token[k] * a.h) * a.d * 2;
        if (i < n_rows) {
            const uint8_t* src = x0 + static_cast<unsigned long long>(static_cast<unsigned>(token[k])) * a.x_pitch + head_at[k];
            if (split) {
                const uint2 lo = *reinterpret_cast<const uint2*>(src), hi = *reinterpret_cast<const uint2*>(src + gap);
                v[k] = make_uint4(lo.x, lo.y, hi.x, hi.y);
            } else {
                v[k] = *reinterpret_cast<const uint4*>(src);
            }
        }
    }
    const int n_tokens = (a.h == 1 ? n_rows - 1 : token_of(n_rows - 1)) + 1;
    for (int t = threadIdx.y * blockDim.x + threadIdx.x; t < n_tokens * n_pairs; t += blockDim.x * blockDim.y) {
        const int tok = t / n_pairs;
        turns[t] = rotary_turn(a.rot, __ldg(a.rot.positions + first_token + tok), rotary_step(__ldg(a.rot.freqs + t - tok * n_pairs)));
    }
    __syncthreads();
    if (rotates) {
#pragma unroll
        for (int k = 0; k < kRopeRowsPerThread; ++k) {
            if (static_cast<int>(threadIdx.y + k * blockDim.y) >= n_rows) break;
            const float4* turn = reinterpret_cast<const float4*>(turns + token[k] * n_pairs + u * 4);
            const float4 t01 = turn[0], t23 = turn[1];
            const float2 t[4] = {make_float2(t01.x, t01.y), make_float2(t01.z, t01.w), make_float2(t23.x, t23.y), make_float2(t23.z, t23.w)};
            float f[8];
            ln_unpack(v[k], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float& p = kInterleaved ? f[2 * e] : f[e];
                float& q = kInterleaved ? f[2 * e + 1] : f[4 + e];
                const float2 r = rotary_apply(t[e], p, q);
                p = r.x;
                q = r.y;
            }
            v[k] = ln_pack(f);
        }
    }
#pragma unroll
    for (int k = 0; k < kRopeRowsPerThread; ++k) {
        if (static_cast<int>(threadIdx.y + k * blockDim.y) >= n_rows) break;
        uint8_t* dst = y0 + static_cast<unsigned long long>(static_cast<unsigned>(token[k])) * a.y_pitch + head_at[k];
        if (split) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(v[k].x, v[k].y);
            *reinterpret_cast<uint2*>(dst + gap) = make_uint2(v[k].z, v[k].w);
        } else {
            *reinterpret_cast<uint4*>(dst) = v[k];
        }
    }
}

// ---- latent norm + key rotation ----------------------------------------------------------------------------
// kv_a rows are D latent channels followed by R key channels (what W_kv_a delivers).  The latent is normalised exactly as
// layernorm_fwd_kernel does it (mean first, then the squares of the differences), and a lane rotates its pairs of the key with a
// sine and cosine of its own: no table, no exchange.  Destinations, each optional: dense latent [M, D] and k_pe [M, R],
// and the row slots[m] of a cache whose rows are the D + R channels side by side (a slot outside [0, n_slots) writes
// nothing: padding).
struct LatentNormRopeArgs {
    const __nv_bfloat16* kv_a;
    long long kv_a_pitch;
    const __nv_bfloat16 *gamma, *beta;     // beta may be null
    int M, D, R;
    float eps;
    Rotary rot;
    __nv_bfloat16 *latent, *k_pe;          // both or neither
    float *mean, *rstd;                    // each may be null
    __nv_bfloat16* cache;                  // null: no cache
    const int* slots;
    int n_slots;
};

__device__ __forceinline__ void rotary_store_pair(__nv_bfloat16* dst, int j, int n_pairs, bool interleaved, float2 v) {
    if (interleaved) {
        *reinterpret_cast<__nv_bfloat162*>(dst + 2 * j) = __floats2bfloat162_rn(v.x, v.y);
    } else {
        dst[j] = __float2bfloat16_rn(v.x);
        dst[j + n_pairs] = __float2bfloat16_rn(v.y);
    }
}

// The two channels of pair j among the rotated ones.
__device__ __forceinline__ float2 rotary_load_pair(const __nv_bfloat16* src, int j, int n_pairs, bool interleaved) {
    if (interleaved) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(src + 2 * j));
    return make_float2(__bfloat162float(src[j]), __bfloat162float(src[j + n_pairs]));
}

// Rows on their way to shared memory: a warp's row is a chain (load, sums, store) whose latency it cannot hide by itself, so
// each warp keeps a ring of rows in flight (asynchronous 16-byte copies, one group per row) and no register waits.
__device__ __forceinline__ void row_copy16(void* smem_dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem_dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void row_copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void row_copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }
// Two fp32 values in one register pair: one instruction for two additions, products or fused multiply-adds.
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 f2_parts(F2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ void f2_unpack(const uint4& v, F2* f) {     // eight bf16
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = f2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
}
__device__ __forceinline__ uint4 f2_pack(const F2* f) {
    uint4 v;
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 t = f2_parts(f[k]);
        w[k] = pack_bf16x2(t.x, t.y);
    }
    return v;
}

// Half a warp per row: what a row costs beside its elements (addresses, position, slot, reductions, loop) is issued once for two rows;
// with a warp per row those instructions were more than half of the kernel (330 a row, now 247).  Measured at 65536 rows of 512 + 64
// channels into the cache: 28.2 us, 5.4 TB/s (a warp per row, ring of four: 30.7; one row ahead in registers: 36.4).
// kLatentDepth rows per half warp are in shared memory or on their way; gamma and beta stay in registers as bf16, and the
// arithmetic runs two values at a time.  kChunks = ceil(D / 128) chunks of eight channels a lane; kFull: D is kChunks * 128.
constexpr int kLatentDepth = 2;
constexpr int kLatentMaxRows = 1 << 30;      // row numbers one or two strides ahead stay within 31 bits
__host__ __device__ constexpr int latent_fwd_smem(int D, int R) { return kLnWarps * 2 * kLatentDepth * (D + R) * 2; }
__device__ __forceinline__ float half_warp_sum(float v) {
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
template <int kChunks, bool kFull>
__global__ void __launch_bounds__(kLnWarps * 32, kChunks <= 4 ? 2 : 1)
latent_norm_rope_fwd_kernel(const LatentNormRopeArgs a) {
    extern __shared__ __align__(16) uint8_t ring[];          // [warps][2][kLatentDepth][D + R] bf16
    const int lane = threadIdx.x & 31, q = lane & 15;
    const int stride = gridDim.x * kLnWarps * 2;
    const float inv_d = 1.0f / static_cast<float>(a.D);
    const int n_pairs = a.R >> 1, row_bytes = (a.D + a.R) * 2;
    uint8_t* rows = ring + (threadIdx.x >> 4) * kLatentDepth * row_bytes;
    int m = (blockIdx.x * kLnWarps + (threadIdx.x >> 5)) * 2;              // the warp's first row; this half's is m + (lane >> 4)
    const int sub = lane >> 4;
    auto fetch = [&](int r, int stage) {
        if (r < a.M) {
            const __nv_bfloat16* src = a.kv_a + r * a.kv_a_pitch;
            uint8_t* dst = rows + stage * row_bytes;
            for (int c = q * 8; c < a.D + a.R; c += 128) row_copy16(dst + c * 2, src + c);
        }
        row_copy_commit();                                   // (an empty group keeps the count)
    };
#pragma unroll
    for (int k = 0; k < kLatentDepth - 1; ++k) fetch(m + sub + k * stride, k);
    int position = 0, slot = -1;
    if (m + sub < a.M) {
        position = __ldg(a.rot.positions + m + sub);
        if (a.cache != nullptr) slot = __ldg(a.slots + m + sub);
    }
    uint4 gamma[kChunks], beta[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = i * 128 + q * 8;
        const bool in = kFull || c < a.D;
        gamma[i] = in ? __ldg(reinterpret_cast<const uint4*>(a.gamma + c)) : make_uint4(0u, 0u, 0u, 0u);
        beta[i] = in && a.beta != nullptr ? __ldg(reinterpret_cast<const uint4*>(a.beta + c)) : make_uint4(0u, 0u, 0u, 0u);
    }
    const unsigned long long step0 = q < n_pairs ? rotary_step(__ldg(a.rot.freqs + q)) : 0ull,
                             step1 = q + 16 < n_pairs ? rotary_step(__ldg(a.rot.freqs + q + 16)) : 0ull;
    int stage = 0;
    for (; m < a.M; m += stride) {
        const int mine = m + sub;
        __syncwarp();                                        // the row this fetch replaces has been read by every lane
        fetch(mine + (kLatentDepth - 1) * stride, stage == 0 ? kLatentDepth - 1 : stage - 1);
        const int here = position, to = slot;
        if (mine + stride < a.M) {
            position = __ldg(a.rot.positions + mine + stride);
            if (a.cache != nullptr) slot = __ldg(a.slots + mine + stride);
        }
        row_copy_wait<kLatentDepth - 1>();
        __syncwarp();
        const uint8_t* row = rows + stage * row_bytes;
        if (++stage == kLatentDepth) stage = 0;
        const bool live = mine < a.M;                        // (the second half of the last warp may have no row)
        const bool dense = live && a.latent != nullptr, cached = live && to >= 0 && to < a.n_slots;
        __nv_bfloat16* cache_row = a.cache + static_cast<size_t>(cached ? to : 0) * (a.D + a.R);
        F2 v[kChunks][4], sum = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int c = i * 128 + q * 8;
            f2_unpack(kFull || c < a.D ? *reinterpret_cast<const uint4*>(row + c * 2) : make_uint4(0u, 0u, 0u, 0u), v[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = f2_add(sum, v[i][k]);
        }
        const float2 sums = f2_parts(sum);
        const float mean = half_warp_sum(sums.x + sums.y) * inv_d;
        const F2 minus = f2(-mean, -mean);
        F2 sq = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
            if (kFull || i * 128 + q * 8 < a.D)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[i][k] = f2_add(v[i][k], minus);
                    sq = f2_fma(v[i][k], v[i][k], sq);
                }
        // the key, under the second sum
        const __nv_bfloat16* key = reinterpret_cast<const __nv_bfloat16*>(row) + a.D;
        auto turn_pair = [&](int j, unsigned long long step) {
            const float2 in = rotary_load_pair(key, j, n_pairs, a.rot.interleaved);
            const float2 out = rotary_apply(rotary_turn(a.rot, here, step), in.x, in.y);
            if (dense) rotary_store_pair(a.k_pe + static_cast<size_t>(mine) * a.R, j, n_pairs, a.rot.interleaved, out);
            if (cached) rotary_store_pair(cache_row + a.D, j, n_pairs, a.rot.interleaved, out);
        };
        if (q < n_pairs) turn_pair(q, step0);
        if (q + 16 < n_pairs) turn_pair(q + 16, step1);
        for (int j = q + 32; j < n_pairs; j += 16) turn_pair(j, rotary_step(__ldg(a.rot.freqs + j)));
        const float2 sqs = f2_parts(sq);
        const float rstd = rsqrtf(half_warp_sum(sqs.x + sqs.y) * inv_d + a.eps);
        const F2 scale = f2(rstd, rstd);
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int c = i * 128 + q * 8;
            if (kFull || c < a.D) {
                F2 gm[4], bt[4];
                f2_unpack(gamma[i], gm);
                f2_unpack(beta[i], bt);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i][k] = f2_fma(f2_mul(v[i][k], scale), gm[k], bt[k]);
                const uint4 packed = f2_pack(v[i]);
                if (dense) *reinterpret_cast<uint4*>(a.latent + static_cast<size_t>(mine) * a.D + c) = packed;
                if (cached) *reinterpret_cast<uint4*>(cache_row + c) = packed;
            }
        }
        if (q == 0 && live) {
            if (a.mean != nullptr) a.mean[mine] = mean;
            if (a.rstd != nullptr) a.rstd[mine] = rstd;
        }
    }
}

// Backward: dkv_a[m] = [ LayerNorm^T dlatent[m] , rotation^T dk_pe[m] ], with per-block sums of dgamma and dbeta over the
// block's rows in `partial` [blocks][2][D].  latent_norm_sums_kernel adds those in block order: the result does not depend
// on the order in which blocks run (the fp32 atomics of layernorm_bwd_kernel do).
// A warp per row, the next row in registers.  Measured with D = 512, R = 64: 16384 rows 13.3 us (inputs partly in L2; 14.1 not), 65536
// rows 39 us without the second kernel, 5.8 TB/s.  Instructions bound the rows (340 each), the second kernel adds 2 to 3 us; fetching rows further ahead, in
// shared memory or into L2, only adds instructions (16.2 and 15.4 us).
struct LatentNormRopeBwdArgs {
    const __nv_bfloat16 *dlatent, *dk_pe, *kv_a;
    long long kv_a_pitch;
    const __nv_bfloat16* gamma;
    const float *mean, *rstd;
    int M, D, R;
    Rotary rot;                            // inverse already set
    __nv_bfloat16* dkv_a;                  // [M, D + R]
    float* partial;
};

// A pair as it lies in memory, for rows fetched ahead in registers (the backward keeps one row ahead there: its sums leave few
// registers, and a ring in shared memory as the forward's measured 16.2 us against 13.4 at M = 16384, the extra trip
// through shared memory costing instructions that this kernel does not have).
__device__ __forceinline__ uint32_t rotary_fetch_pair(const __nv_bfloat16* src, int j, int n_pairs, bool interleaved) {
    if (interleaved) return *reinterpret_cast<const uint32_t*>(src + 2 * j);
    const unsigned short* u = reinterpret_cast<const unsigned short*>(src);
    return u[j] | (static_cast<uint32_t>(u[j + n_pairs]) << 16);
}
__device__ __forceinline__ float2 rotary_pair_of(uint32_t raw) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw)); }

template <int kLnChunks>
struct LatentBwdRow {
    uint4 x[kLnChunks], dy[kLnChunks];
    uint32_t pair;
    int position;
    float mean, rstd;
};
template <int kLnChunks, bool kFull>
__device__ __forceinline__ void latent_bwd_fetch(const LatentNormRopeBwdArgs& a, int m, int lane, LatentBwdRow<kLnChunks>& r) {
    const __nv_bfloat16* x = a.kv_a + m * a.kv_a_pitch;
    const __nv_bfloat16* dy = a.dlatent + static_cast<size_t>(m) * a.D;
#pragma unroll
    for (int i = 0; i < kLnChunks; ++i) {
        const int c = i * 256 + lane * 8;
        r.x[i] = kFull || c < a.D ? *reinterpret_cast<const uint4*>(x + c) : make_uint4(0u, 0u, 0u, 0u);
        r.dy[i] = kFull || c < a.D ? *reinterpret_cast<const uint4*>(dy + c) : make_uint4(0u, 0u, 0u, 0u);
    }
    r.pair = lane < (a.R >> 1) ? rotary_fetch_pair(a.dk_pe + static_cast<size_t>(m) * a.R, lane, a.R >> 1, a.rot.interleaved) : 0u;
    r.position = __ldg(a.rot.positions + m);
    r.mean = __ldg(a.mean + m);
    r.rstd = __ldg(a.rstd + m);
}

template <int kLnChunks, bool kFull>
__global__ void __launch_bounds__(kLnWarps * 32, kLnChunks <= 2 ? 2 : 1)
latent_norm_rope_bwd_kernel(const LatentNormRopeBwdArgs a) {
    __shared__ float part[kLnWarps][kLnChunks * 256];
    grid_launch_dependents();                                // the sums' blocks may take their places as these leave theirs
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_warps = gridDim.x * kLnWarps;
    const float inv_d = 1.0f / static_cast<float>(a.D);
    const int n_pairs = a.R >> 1;
    F2 acc_g[kLnChunks][4], acc_b[kLnChunks][4];
    uint4 gamma[kLnChunks];
#pragma unroll
    for (int i = 0; i < kLnChunks; ++i) {
        const int c = i * 256 + lane * 8;
        gamma[i] = kFull || c < a.D ? __ldg(reinterpret_cast<const uint4*>(a.gamma + c)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc_g[i][k] = acc_b[i][k] = f2(0.f, 0.f);
    }
    const unsigned long long step = lane < n_pairs ? rotary_step(__ldg(a.rot.freqs + lane)) : 0ull;
    int m = blockIdx.x * kLnWarps + warp;
    LatentBwdRow<kLnChunks> next;
    if (m < a.M) latent_bwd_fetch<kLnChunks, kFull>(a, m, lane, next);
    for (; m < a.M; m += n_warps) {
        const LatentBwdRow<kLnChunks> row = next;
        if (m + n_warps < a.M) latent_bwd_fetch<kLnChunks, kFull>(a, m + n_warps, lane, next);
        __nv_bfloat16* out = a.dkv_a + static_cast<size_t>(m) * (a.D + a.R);
        const F2 rstd = f2(row.rstd, row.rstd), shift = f2(-row.mean * row.rstd, -row.mean * row.rstd);
        F2 xh[kLnChunks][4], g[kLnChunks][4], t1 = f2(0.f, 0.f), t2 = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i) {
            F2 dv[4];
            f2_unpack(row.x[i], xh[i]);
            f2_unpack(row.dy[i], dv);
            f2_unpack(gamma[i], g[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                xh[i][k] = f2_fma(xh[i][k], rstd, shift);
                g[i][k] = f2_mul(dv[k], g[i][k]);                       // (zeros beyond D: dy is)
                t1 = f2_add(t1, g[i][k]);
                t2 = f2_fma(g[i][k], xh[i][k], t2);
                acc_g[i][k] = f2_fma(dv[k], xh[i][k], acc_g[i][k]);
                acc_b[i][k] = f2_add(acc_b[i][k], dv[k]);
            }
        }
        if (lane < n_pairs) {
            const float2 in = rotary_pair_of(row.pair);
            rotary_store_pair(out + a.D, lane, n_pairs, a.rot.interleaved, rotary_apply(rotary_turn(a.rot, row.position, step), in.x, in.y));
        }
        for (int j = lane + 32; j < n_pairs; j += 32) {                 // keys wider than 64 channels
            const float2 in = rotary_pair_of(rotary_fetch_pair(a.dk_pe + static_cast<size_t>(m) * a.R, j, n_pairs, a.rot.interleaved));
            rotary_store_pair(out + a.D, j, n_pairs, a.rot.interleaved,
                              rotary_apply(rotary_turn(a.rot, row.position, rotary_step(__ldg(a.rot.freqs + j))), in.x, in.y));
        }
        const float2 u1 = f2_parts(t1), u2 = f2_parts(t2);
        float s1 = u1.x + u1.y, s2 = u2.x + u2.y;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            s1 += __shfl_xor_sync(0xffffffffu, s1, d);
            s2 += __shfl_xor_sync(0xffffffffu, s2, d);
        }
        // rstd * (g - s1 - xhat * s2)
        s1 *= -inv_d * row.rstd;
        s2 *= -inv_d * row.rstd;
        const F2 p1 = f2(s1, s1), p2 = f2(s2, s2);
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i) {
            const int c = i * 256 + lane * 8;
            if (kFull || c < a.D) {
#pragma unroll
                for (int k = 0; k < 4; ++k) g[i][k] = f2_fma(xh[i][k], p2, f2_fma(g[i][k], rstd, p1));
                *reinterpret_cast<uint4*>(out + c) = f2_pack(g[i]);
            }
        }
    }
    float* dst = a.partial + static_cast<size_t>(blockIdx.x) * 2 * a.D;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i) {
            const int c = i * 256 + lane * 8;
            if (c < a.D)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *reinterpret_cast<float2*>(&part[warp][c + 2 * k]) = f2_parts(pass == 0 ? acc_g[i][k] : acc_b[i][k]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += kLnWarps * 32) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kLnWarps; ++w) s += part[w][c];
            dst[pass * a.D + c] = s;
        }
    }
}

// dgamma and dbeta from the per-block sums: 32 columns a block, 32 warps on interleaved blocks' rows (ten loads each, all in
// flight at once: the kernel is one round trip to L2), added in a fixed order.  Columns [0, D) are dgamma, [D, 2D) dbeta
// (dropped when dbeta is null).
__global__ void __launch_bounds__(1024)
latent_norm_sums_kernel(const float* partial, int n_blocks, int D, float* dgamma, float* dbeta) {
    __shared__ float part[32][33];
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < 2 * D) {
#pragma unroll 10
        for (int b = warp; b < n_blocks; b += 32) s += partial[static_cast<size_t>(b) * 2 * D + c];
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < 2 * D) {
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 32; ++w) s += part[w][lane];
        if (c < D) dgamma[c] = s;
        else if (dbeta != nullptr) dbeta[c - D] = s;
    }
}

}  // namespace laga
