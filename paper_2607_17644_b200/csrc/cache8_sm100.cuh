// The paged latent cache in 8 bits: how a token is held, and the kernels that write and read tokens.
//
// A token is the 512 channels x of its normalised latent and the 64 channels k of the rotated shared key.  With
//     s = the smallest power of two, 2^-32 at least, such that no channel exceeds 448 s     (448: the largest e4m3 number)
// it is held as codes, latent e4m3(x / s), key e4m3(k / s), and what the key's rounding left, e4m3(k / s - first code): read back as
// x = s code, k = s (code + second code).  e4m3 has four binary digits: a latent channel is off by at most 2^-4 of itself, a key
// channel by at most 2^-8, half a step of bf16: scores lie on the key's positions, and 64 of 576 channels cost little.  Where that is less than 2^-10 s -- a
// latent channel below 2^-6 s, a key channel below 2^-2 s -- they are held to 2^-10 s.  s is a power of two because nothing is gained by another (the codes are floating) and everything that
// multiplies by it stays exact; one s for latent and key, so that a score is one product of codes.  One s a token, because a token
// that joins a page must not change those that are there.  A token with a channel that is not finite has s = NaN: all of it reads as NaN.
//
// A page of n tokens is n rows of 640 codes (latent, key, rest of the key), then the rows' n scales in fp32: 644 bytes a token against 1152
// in bf16; every row starts on a 128-byte boundary of its page, so that 128 channels of a tile of rows are one operand slab.
#pragma once
#include "rope_sm100.cuh"
#include "sm100_ptx.cuh"

namespace laga {

constexpr int kC8Lat = 512, kC8Key = 64;
constexpr int kC8Row = kC8Lat + 2 * kC8Key;          // codes of a token
constexpr int kC8Token = kC8Row + 4;                 // ... and its scale

struct Cache8 {
    uint8_t* base;
    int page_shift, n_slots;                         // n_slots: pages * page size
    __host__ __device__ size_t page_bytes() const { return static_cast<size_t>(kC8Token) << page_shift; }
    __device__ __forceinline__ uint8_t* row(int slot) const {
        return base + (slot >> page_shift) * page_bytes() + static_cast<size_t>(slot & ((1 << page_shift) - 1)) * kC8Row;
    }
    __device__ __forceinline__ float* scale(int slot) const {
        return reinterpret_cast<float*>(base + (slot >> page_shift) * page_bytes() + (static_cast<size_t>(kC8Row) << page_shift)) +
               (slot & ((1 << page_shift) - 1));
    }
};

// log2 of the smallest power of two that brings a magnitude (given as the bits of its absolute value) within 448 = 1.75 * 2^8.  128 or more,
// the exponent of what is not finite, for infinity and NaN.
__device__ __forceinline__ int scale_exponent(uint32_t abs_bits) {
    const int e = static_cast<int>(abs_bits >> 23);
    return e == 255 ? 128 : e - 127 - 8 + ((abs_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
}
// 2^e for e in [-126, 127], NaN for 128
__device__ __forceinline__ float exact_exp2(int e) { return e == 128 ? __uint_as_float(0x7fc00000u) : __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

struct Cache8AppendArgs {
    const __nv_bfloat16* kv_a;
    long long kv_a_pitch;
    const __nv_bfloat16 *gamma, *beta;               // beta may be null
    int M;
    float eps;
    Rotary rot;
    Cache8 cache;
    const int* slots;
};

// Half a warp per row and a ring of rows in shared memory, as latent_norm_rope_fwd_kernel has it (the arithmetic up to the rounding is the
// same); what it adds is the largest magnitude of the row, the codes and half the bytes to write.  Instructions bound it: 65535 rows 22.9 us
// without beta, 5.2 TB/s (magnitudes as masked integers and beta's zeros added: 26.1; rings of three and four rows: 23.4 and 24.6).
// The largest magnitude of three, NaN if one is.
__device__ __forceinline__ float largest3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
template <bool kInterleaved, bool kBeta>
__global__ void __launch_bounds__(kLnWarps * 32, 2)
cache8_append_kernel(const Cache8AppendArgs a) {
    constexpr int kRowBytes = (kC8Lat + kC8Key) * 2, kPairs = kC8Key / 2;
    __shared__ __align__(16) uint8_t ring[kLnWarps * 2 * kLatentDepth * kRowBytes];
    const int lane = threadIdx.x & 31, q = lane & 15, sub = lane >> 4;
    const int stride = gridDim.x * kLnWarps * 2;
    uint8_t* rows = ring + (threadIdx.x >> 4) * kLatentDepth * kRowBytes;
    int m = (blockIdx.x * kLnWarps + (threadIdx.x >> 5)) * 2;              // the warp's first row; this half's is m + sub
    auto fetch = [&](int r, int stage) {
        if (r < a.M) {
            const __nv_bfloat16* src = a.kv_a + r * a.kv_a_pitch;
            uint8_t* dst = rows + stage * kRowBytes;
#pragma unroll
            for (int c = q * 8; c < kC8Lat + kC8Key; c += 128) row_copy16(dst + c * 2, src + c);
        }
        row_copy_commit();                                   // (an empty group keeps the count)
    };
#pragma unroll
    for (int k = 0; k < kLatentDepth - 1; ++k) fetch(m + sub + k * stride, k);
    int position = 0, slot = -1;
    if (m + sub < a.M) {
        position = __ldg(a.rot.positions + m + sub);
        slot = __ldg(a.slots + m + sub);
    }
    uint4 gamma[4], beta[kBeta ? 4 : 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        gamma[i] = __ldg(reinterpret_cast<const uint4*>(a.gamma + i * 128 + q * 8));
        if constexpr (kBeta) beta[i] = __ldg(reinterpret_cast<const uint4*>(a.beta + i * 128 + q * 8));
    }
    const unsigned long long step[2] = {rotary_step(__ldg(a.rot.freqs + q)), rotary_step(__ldg(a.rot.freqs + q + 16))};
    int stage = 0;
    for (; m < a.M; m += stride) {
        const int mine = m + sub;
        __syncwarp();                                        // the row this fetch replaces has been read by every lane
        fetch(mine + (kLatentDepth - 1) * stride, stage == 0 ? kLatentDepth - 1 : stage - 1);
        const int here = position, to = slot;
        if (mine + stride < a.M) {
            position = __ldg(a.rot.positions + mine + stride);
            slot = __ldg(a.slots + mine + stride);
        }
        row_copy_wait<kLatentDepth - 1>();
        __syncwarp();
        const uint8_t* row = rows + stage * kRowBytes;
        if (++stage == kLatentDepth) stage = 0;
        const bool cached = mine < a.M && to >= 0 && to < a.cache.n_slots;
        F2 v[4][4], sum = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f2_unpack(*reinterpret_cast<const uint4*>(row + (i * 128 + q * 8) * 2), v[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = f2_add(sum, v[i][k]);
        }
        const float2 sums = f2_parts(sum);
        const float mean = half_warp_sum(sums.x + sums.y) * (1.0f / kC8Lat);
        const F2 minus = f2(-mean, -mean);
        F2 sq = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[i][k] = f2_add(v[i][k], minus);
                sq = f2_fma(v[i][k], v[i][k], sq);
            }
        // the key, under the second sum: pairs q and q + 16
        const __nv_bfloat16* key = reinterpret_cast<const __nv_bfloat16*>(row) + kC8Lat;
        float2 k2[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float2 in = rotary_load_pair(key, q + 16 * t, kPairs, kInterleaved);
            k2[t] = rotary_apply(rotary_turn(a.rot, here, step[t]), in.x, in.y);
        }
        float most = largest3(largest3(k2[0].x, k2[0].y, k2[1].x), k2[1].y, 0.f);
        const float2 sqs = f2_parts(sq);
        // (rsqrtf and the products after it: of 33.5 million codes 37 to 43 are the neighbours of those that exact arithmetic gives; with a root and a division
        // in fp32, 36 to 45)
        const float rstd = rsqrtf(half_warp_sum(sqs.x + sqs.y) * (1.0f / kC8Lat) + a.eps);
        const F2 scale = f2(rstd, rstd);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            F2 gm[4], bt[4];
            f2_unpack(gamma[i], gm);
            if constexpr (kBeta) f2_unpack(beta[i], bt);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[i][k] = f2_mul(v[i][k], scale);
                if constexpr (kBeta) v[i][k] = f2_fma(v[i][k], gm[k], bt[k]);
                else v[i][k] = f2_mul(v[i][k], gm[k]);
                const float2 x = f2_parts(v[i][k]);
                most = largest3(most, x.x, x.y);
            }
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) most = largest3(most, __shfl_xor_sync(0xffffffffu, most, d), 0.f);
        const int e = max(scale_exponent(__float_as_uint(most) & 0x7fffffffu), -32);
        const float inv = e == 128 ? 0.f : exact_exp2(-e);
        const F2 inv2 = f2(inv, inv);
        uint8_t* codes = a.cache.row(cached ? to : 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t c[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 x = f2_parts(f2_mul(v[i][k], inv2));
                c[k] = e4m3x2(x.x, x.y);
            }
            if (cached) *reinterpret_cast<uint2*>(codes + i * 128 + q * 8) = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float x = k2[t].x * inv, y = k2[t].y * inv;
            const uint32_t first = e4m3x2(x, y);
            const float2 held = float2_of_half2(half2_of_e4m3x2(first));
            const uint32_t rest = e4m3x2(x - held.x, y - held.y);
            const int j = q + 16 * t;
            if (cached) {
                uint8_t* dst = codes + kC8Lat;
                if constexpr (kInterleaved) {
                    *reinterpret_cast<uint16_t*>(dst + 2 * j) = static_cast<uint16_t>(first);
                    *reinterpret_cast<uint16_t*>(dst + kC8Key + 2 * j) = static_cast<uint16_t>(rest);
                } else {
                    dst[j] = static_cast<uint8_t>(first);
                    dst[j + kPairs] = static_cast<uint8_t>(first >> 8);
                    dst[kC8Key + j] = static_cast<uint8_t>(rest);
                    dst[kC8Key + j + kPairs] = static_cast<uint8_t>(rest >> 8);
                }
            }
        }
        if (q == 0 && cached) *a.cache.scale(to) = exact_exp2(e);
    }
}

// Rows slots[m] of the cache as the dense bf16 rows that the attention over a whole prompt takes: latent[m] and k_pe[m]; zeros where the slot
// is outside the cache.  The latent is exact (four digits times a power of two), the key is rounded once to bf16.
// A thread turns 16 codes (of a key: 16 and their rests) into 32 bytes: 36 threads a row, kC8ReadRows rows a thread, whose loads go out together.
// HBM bounds it: 131072 rows 38.5 us, 6.1 TB/s (with four rows a thread, of which fewer are resident, 42.0; with two 16-byte stores for one of 32, 43.8).
constexpr int kC8ReadUnits = kC8Row / 16 - kC8Key / 16, kC8ReadY = 7, kC8ReadRows = 2;
struct Cache8ReadArgs {
    Cache8 cache;
    const int* slots;
    int M;
    __nv_bfloat16 *latent, *k_pe;
};
template <bool kWide>                                        // the results begin on 32-byte boundaries
__global__ void __launch_bounds__(kC8ReadUnits * kC8ReadY)
cache8_read_kernel(const Cache8ReadArgs a) {
    const int u = threadIdx.x;
    const bool is_key = u >= kC8Lat / 16;
    const int m0 = blockIdx.x * (kC8ReadY * kC8ReadRows) + threadIdx.y;
    uint4 first[kC8ReadRows], rest[kC8ReadRows];
    float s[kC8ReadRows];
#pragma unroll
    for (int k = 0; k < kC8ReadRows; ++k) {
        const int m = m0 + k * kC8ReadY, slot = m < a.M ? __ldg(a.slots + m) : -1;
        first[k] = rest[k] = make_uint4(0u, 0u, 0u, 0u);
        s[k] = 0.f;
        if (slot >= 0 && slot < a.cache.n_slots) {
            const uint8_t* row = a.cache.row(slot) + u * 16;
            first[k] = __ldcs(reinterpret_cast<const uint4*>(row));
            if (is_key) rest[k] = __ldcs(reinterpret_cast<const uint4*>(row + kC8Key));
            s[k] = __ldg(a.cache.scale(slot));
        }
    }
#pragma unroll
    for (int k = 0; k < kC8ReadRows; ++k) {
        const int m = m0 + k * kC8ReadY;
        if (m >= a.M) break;
        const uint32_t w[4] = {first[k].x, first[k].y, first[k].z, first[k].w}, r[4] = {rest[k].x, rest[k].y, rest[k].z, rest[k].w};
        uint32_t o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float2 x = float2_of_half2(half2_of_e4m3x2(w[j >> 1] >> (16 * (j & 1))));
            if (is_key) {
                const float2 y = float2_of_half2(half2_of_e4m3x2(r[j >> 1] >> (16 * (j & 1))));
                x = make_float2(x.x + y.x, x.y + y.y);
            }
            o[j] = pack_bf16x2(x.x * s[k], x.y * s[k]);
        }
        __nv_bfloat16* dst = is_key ? a.k_pe + static_cast<size_t>(m) * kC8Key + (u - kC8Lat / 16) * 16 : a.latent + static_cast<size_t>(m) * kC8Lat + u * 16;
        if (kWide) {
            st_global_v8(dst, o);
        } else {
            *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4*>(dst + 8) = make_uint4(o[4], o[5], o[6], o[7]);
        }
    }
}

}  // namespace laga
