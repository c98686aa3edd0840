// Rotary positions, and the step between W_kv_a and the attention (LayerNorm of the latent and rotation of the
// shared key in one pass), forward and backward.  The paper takes q_rope and k_pe as already rotated; these
// kernels are what rotates them.
//
//   angle(m, j) = position_m * freq_j,   j = 0 .. d_rot/2 - 1
//   (a, b) -> mscale * (a cos - b sin, b cos + a sin)        inverse: sin -> -sin, which is the transpose, i.e.
//                                                            the gradient (mscale included)
// for the pairs (2j, 2j+1) of the rotated channels (interleaved) or (j, j + d_rot/2) (half).
//
// The angle is formed in fp64: at position 4e6 an fp32 product is off by a quarter of a radian.  It is reduced to a
// fraction of a turn there (one multiplication, one rounding, one subtraction; B200 has fp64 at half the fp32 rate),
// and sine and cosine of the reduced angle in [-pi, pi] come from the special-function unit, whose absolute error
// below 2^-21 is far under the half step (2^-9) of the bf16 result.
//
// Everything here is bound by HBM: one read and one write of every element.
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

// (cos, sin) * mscale of one pair at one position; `inverse` turns the other way.
__device__ __forceinline__ float2 rotary_turn(const Rotary& r, int position, int pair) {
    constexpr double kInvTwoPi = 0.15915494309189533577;
    const double turns = static_cast<double>(position) * (__ldg(r.freqs + pair) * kInvTwoPi);
    const float phi = static_cast<float>(turns - rint(turns)) * 6.2831853071795865f;
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
// not once per head: with 16 heads that is 1/16 of the fp64 and special-function work), then each thread rotates or
// copies its 16-byte chunks.  threadIdx.x is the chunk within the head, so no index needs a division but the token's.
// Half layout: the thread of a chunk in the first half of the rotated channels also owns the partner chunk, and the
// partner's own thread does not exist (units_per_head counts it out), so x and y may be the same buffer.
// in_place: only the rotated units run.
template <bool kInterleaved>
__global__ void __launch_bounds__(256)
rope_kernel(const __nv_bfloat16* x, long long x_pitch, __nv_bfloat16* y, long long y_pitch, int M, int h, int d,
            int rot_begin, int d_rot, int in_place, Rotary rot) {
    extern __shared__ float2 turns[];                       // [tokens of this block][d_rot / 2]
    const int n_pairs = d_rot >> 1;
    const int rot_units = kInterleaved ? d_rot >> 3 : d_rot >> 4;
    const int before = in_place ? 0 : rot_begin >> 3;       // units copied in front of the rotated ones
    const int u = threadIdx.x;
    const bool rotates = u >= before && u < before + rot_units;
    // first channel of this thread's unit
    const int c0 = u < before ? u * 8 : rotates ? rot_begin + (u - before) * 8 : rot_begin + d_rot + (u - before - rot_units) * 8;
    const long long rows = static_cast<long long>(M) * h;
    const long long row0 = static_cast<long long>(blockIdx.x) * (blockDim.y * kRopeRowsPerThread);
    const long long row_end = min(rows, row0 + blockDim.y * kRopeRowsPerThread);
    const int first_token = static_cast<int>(row0 / h);
    const int n_tokens = static_cast<int>((row_end - 1) / h) - first_token + 1;

    uint4 v[kRopeRowsPerThread], w[kRopeRowsPerThread];
    int token[kRopeRowsPerThread], head[kRopeRowsPerThread];
#pragma unroll
    for (int k = 0; k < kRopeRowsPerThread; ++k) {
        const long long row = row0 + threadIdx.y + k * blockDim.y;
        token[k] = -1;
        if (row < row_end) {
            // row - first_token * h is below 2^31 and small: 32-bit division
            const unsigned r = static_cast<unsigned>(row - static_cast<long long>(first_token) * h);
            token[k] = static_cast<int>(r / static_cast<unsigned>(h));
            head[k] = static_cast<int>(r) - token[k] * h;
            const __nv_bfloat16* src = x + (first_token + token[k]) * x_pitch + head[k] * d + c0;
            v[k] = *reinterpret_cast<const uint4*>(src);
            if (!kInterleaved && rotates) w[k] = *reinterpret_cast<const uint4*>(src + n_pairs);
        }
    }
    for (int t = threadIdx.y * blockDim.x + threadIdx.x; t < n_tokens * n_pairs; t += blockDim.x * blockDim.y) {
        const int tok = t / n_pairs;
        turns[t] = rotary_turn(rot, __ldg(rot.positions + first_token + tok), t - tok * n_pairs);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRopeRowsPerThread; ++k) {
        if (token[k] < 0) continue;
        __nv_bfloat16* dst = y + (first_token + token[k]) * y_pitch + head[k] * d + c0;
        if (rotates) {
            const float2* turn = turns + token[k] * n_pairs;
            float a[8], b[8];
            ln_unpack(v[k], a);
            if (kInterleaved) {
                turn += (u - before) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 r = rotary_apply(turn[e], a[2 * e], a[2 * e + 1]);
                    a[2 * e] = r.x;
                    a[2 * e + 1] = r.y;
                }
            } else {
                turn += (u - before) * 8;
                ln_unpack(w[k], b);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 r = rotary_apply(turn[e], a[e], b[e]);
                    a[e] = r.x;
                    b[e] = r.y;
                }
                *reinterpret_cast<uint4*>(dst + n_pairs) = ln_pack(b);
            }
            v[k] = ln_pack(a);
        }
        *reinterpret_cast<uint4*>(dst) = v[k];
    }
}

// ---- latent norm + key rotation ----------------------------------------------------------------------------
// kv_a rows are D latent channels followed by R key channels (what W_kv_a delivers).  One warp per row: the latent is
// normalised exactly as layernorm_fwd_kernel does it, and the key is rotated with one pair per lane (a row's 32 pairs are
// 32 lanes' sine and cosine: no table, no exchange).  Destinations, each optional: dense latent [M, D] and k_pe [M, R],
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

// The two channels of pair j among the rotated ones.
__device__ __forceinline__ float2 rotary_load_pair(const __nv_bfloat16* src, int j, int n_pairs, bool interleaved) {
    if (interleaved) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(src + 2 * j));
    return make_float2(__bfloat162float(src[j]), __bfloat162float(src[j + n_pairs]));
}
__device__ __forceinline__ void rotary_store_pair(__nv_bfloat16* dst, int j, int n_pairs, bool interleaved, float2 v) {
    if (interleaved) {
        *reinterpret_cast<__nv_bfloat162*>(dst + 2 * j) = __floats2bfloat162_rn(v.x, v.y);
    } else {
        dst[j] = __float2bfloat16_rn(v.x);
        dst[j + n_pairs] = __float2bfloat16_rn(v.y);
    }
}

template <int kLnChunks>
__global__ void __launch_bounds__(kLnWarps * 32)
latent_norm_rope_fwd_kernel(const LatentNormRopeArgs a) {
    const int lane = threadIdx.x & 31;
    const int n_warps = gridDim.x * kLnWarps;
    const float inv_d = 1.0f / static_cast<float>(a.D);
    const int n_pairs = a.R >> 1;
    for (int m = blockIdx.x * kLnWarps + (threadIdx.x >> 5); m < a.M; m += n_warps) {
        const __nv_bfloat16* row = a.kv_a + m * a.kv_a_pitch;
        __nv_bfloat16* cache_row = nullptr;
        if (a.cache != nullptr) {
            const int slot = __ldg(a.slots + m);
            if (slot >= 0 && slot < a.n_slots) cache_row = a.cache + static_cast<size_t>(slot) * (a.D + a.R);
            else if (a.latent == nullptr) continue;                     // nothing of this row goes anywhere
        }
        const int position = __ldg(a.rot.positions + m);
        float v[kLnChunks][8];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i) {
            const int c = i * 256 + lane * 8;
            if (c < a.D) {
                ln_unpack(*reinterpret_cast<const uint4*>(row + c), v[i]);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum += v[i][k];
            }
        }
        // the key, under the latent's loads
        for (int j = lane; j < n_pairs; j += 32) {
            const float2 in = rotary_load_pair(row + a.D, j, n_pairs, a.rot.interleaved);
            const float2 out = rotary_apply(rotary_turn(a.rot, position, j), in.x, in.y);
            if (a.k_pe != nullptr) rotary_store_pair(a.k_pe + static_cast<size_t>(m) * a.R, j, n_pairs, a.rot.interleaved, out);
            if (cache_row != nullptr) rotary_store_pair(cache_row + a.D, j, n_pairs, a.rot.interleaved, out);
        }
        const float mean = ln_warp_sum(sum) * inv_d;
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i)
            if (i * 256 + lane * 8 < a.D)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float t = v[i][k] - mean;
                    sq = fmaf(t, t, sq);
                }
        const float rstd = rsqrtf(ln_warp_sum(sq) * inv_d + a.eps);
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i) {
            const int c = i * 256 + lane * 8;
            if (c < a.D) {
                float gm[8], bt[8], o[8];
                ln_unpack(__ldg(reinterpret_cast<const uint4*>(a.gamma + c)), gm);
                if (a.beta != nullptr) ln_unpack(__ldg(reinterpret_cast<const uint4*>(a.beta + c)), bt);
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = fmaf((v[i][k] - mean) * rstd, gm[k], a.beta != nullptr ? bt[k] : 0.f);
                const uint4 packed = ln_pack(o);
                if (a.latent != nullptr) *reinterpret_cast<uint4*>(a.latent + static_cast<size_t>(m) * a.D + c) = packed;
                if (cache_row != nullptr) *reinterpret_cast<uint4*>(cache_row + c) = packed;
            }
        }
        if (lane == 0) {
            if (a.mean != nullptr) a.mean[m] = mean;
            if (a.rstd != nullptr) a.rstd[m] = rstd;
        }
    }
}

// Backward: dkv_a[m] = [ LayerNorm^T dlatent[m] , rotation^T dk_pe[m] ], with per-block sums of dgamma and dbeta over the
// block's rows in `partial` [blocks][2][D].  latent_norm_sums_kernel adds those in block order: the result does not depend
// on the order in which blocks run (the fp32 atomics of layernorm_bwd_kernel do).
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

template <int kLnChunks>
__global__ void __launch_bounds__(kLnWarps * 32)
latent_norm_rope_bwd_kernel(const LatentNormRopeBwdArgs a) {
    __shared__ float part[kLnWarps][kLnChunks * 256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_warps = gridDim.x * kLnWarps;
    const float inv_d = 1.0f / static_cast<float>(a.D);
    const int n_pairs = a.R >> 1;
    float acc_g[kLnChunks][8], acc_b[kLnChunks][8];
#pragma unroll
    for (int i = 0; i < kLnChunks; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc_g[i][k] = acc_b[i][k] = 0.f;
    for (int m = blockIdx.x * kLnWarps + warp; m < a.M; m += n_warps) {
        const float mean = __ldg(a.mean + m), rstd = __ldg(a.rstd + m);
        const int position = __ldg(a.rot.positions + m);
        const __nv_bfloat16* xr = a.kv_a + m * a.kv_a_pitch;
        const __nv_bfloat16* gr = a.dlatent + static_cast<size_t>(m) * a.D;
        __nv_bfloat16* out = a.dkv_a + static_cast<size_t>(m) * (a.D + a.R);
        float xh[kLnChunks][8], g[kLnChunks][8];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i) {
            const int c = i * 256 + lane * 8;
            if (c < a.D) {
                float xv[8], dv[8], gm[8];
                ln_unpack(*reinterpret_cast<const uint4*>(xr + c), xv);
                ln_unpack(*reinterpret_cast<const uint4*>(gr + c), dv);
                ln_unpack(__ldg(reinterpret_cast<const uint4*>(a.gamma + c)), gm);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    xh[i][k] = (xv[k] - mean) * rstd;
                    g[i][k] = dv[k] * gm[k];
                    s1 += g[i][k];
                    s2 = fmaf(g[i][k], xh[i][k], s2);
                    acc_g[i][k] = fmaf(dv[k], xh[i][k], acc_g[i][k]);
                    acc_b[i][k] += dv[k];
                }
            }
        }
        for (int j = lane; j < n_pairs; j += 32) {
            const float2 in = rotary_load_pair(a.dk_pe + static_cast<size_t>(m) * a.R, j, n_pairs, a.rot.interleaved);
            rotary_store_pair(out + a.D, j, n_pairs, a.rot.interleaved, rotary_apply(rotary_turn(a.rot, position, j), in.x, in.y));
        }
        s1 = ln_warp_sum(s1) * inv_d;
        s2 = ln_warp_sum(s2) * inv_d;
#pragma unroll
        for (int i = 0; i < kLnChunks; ++i) {
            const int c = i * 256 + lane * 8;
            if (c < a.D) {
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = rstd * (g[i][k] - s1 - xh[i][k] * s2);
                *reinterpret_cast<uint4*>(out + c) = ln_pack(o);
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
                for (int k = 0; k < 8; ++k) part[warp][c + k] = pass == 0 ? acc_g[i][k] : acc_b[i][k];
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

// dgamma and dbeta from the per-block sums: 32 columns a block, eight warps on interleaved blocks' rows, added in a
// fixed order.  Columns [0, D) are dgamma, [D, 2D) dbeta (dropped when dbeta is null).
__global__ void __launch_bounds__(256)
latent_norm_sums_kernel(const float* __restrict__ partial, int n_blocks, int D, float* dgamma, float* dbeta) {
    __shared__ float part[8][33];
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < 2 * D)
        for (int b = warp; b < n_blocks; b += 8) s += partial[static_cast<size_t>(b) * 2 * D + c];
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < 2 * D) {
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += part[w][lane];
        if (c < D) dgamma[c] = s;
        else if (dbeta != nullptr) dbeta[c - D] = s;
    }
}

}  // namespace laga
