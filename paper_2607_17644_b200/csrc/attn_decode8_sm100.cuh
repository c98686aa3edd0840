// Attention of one new token per request over the paged latent cache in 8 bits (cache8_sm100.cuh has the format): the operator of
// attn_decode_sm100.cuh over rows of 640 codes and a scale s_t, 644 bytes a token where bf16 takes 1152.
//
// The codes are never widened: they go from the cache to shared memory by TMA and from there to the tensor cores (kind::f8f6f4) as
// they are.  What multiplies them is brought to 8 bits instead, in two parts each, which together hold as much as a bf16 number:
//   queries        q_lat / r = hi + lo, both e4m3, with a power of two r per (request, head): off by at most 2^-4 * 2^-4 = 2^-8 of a
//                  channel, half a step of bf16, or 2^-10 r (the largest channel is 224 r or more).  The key's 64 channels multiply both the key's codes and their rests.
//   probabilities  p / 2^m = hi + lo likewise.  Up to 32 heads a CTA the parts are columns of one MMA (hi e4m3, lo 32 times the rest
//                  in e4m3); with 64 heads TMEM has no room for those columns, so that lo is a second MMA into the same accumulator,
//                  cannot be scaled, and hi is e5m2, whose range is wide enough for the weights of which lo keeps nothing (2^-7).
// The token's scale belongs to both products: scores are s_t r f (hi + lo) . row_t, and as 2^m p_t c_t = s_t p_t code_t the scale goes
// into the probability, whose exponent it adds to (it is a power of two):
//     y_t = score_t log2(e) + log2 s_t,   P_t = 2^(y_t - m),   O = sum P_t code_t,   l = sum P_t / s_t,   out = O / l
// What e4m3 can hold of P is 2^17, so the reference m is kept near the tile's maximum of y, both ways: where a tile's lies outside [m, m + 11]
// it becomes that maximum less 7 (never more than 2^40 below its highest: what came before is then all that counts, and the
// accumulator must not overflow), and O and l are rescaled.  Up to 32 heads a CTA weights are held to 2^-12 of a tile's largest, and typically to
// 2^-19; with 64, to 2^-10 and 2^-17 (and, as e5m2 reaches further, to 2^-3 of themselves down to 2^-14 and 2^-21).  A few that stand far above all others
// are no part of P (kD8Places).
//
// Scores are computed the other way round from the bf16 kernel, S^T[128 keys x (hi, lo columns of the heads)] = K (A) . Q^T (B): the long
// operand is read from shared memory once for both parts, a thread has all 16 heads' scores of one key, so no reduction is on
// the way of a tile: instead of the maximum the threads vote whether m still holds (one word a warp).
//   output   O^T[512 latents x heads] (+)= V^T (A, MN-major: the same slabs) . P (B, MN-major: a key's probabilities are 16 bytes of a row)
//
// Work split: the line of 64-key units of all requests in equal stretches, as there, with a gap before each request (decode8_gap); a tile is two
// units, or one where a piece ends in an odd one.  A tile is five slabs of 128 keys x 128 codes around a ring with a barrier per slab: the
// key's first (only scores read it).
//   warps 0 .. 4g-1  softmax: group w / 4 has 8 heads (16 where the CTA has 64), its thread l of warp w % 4 key 32 (w % 4) + l; and the drain
//   then four warps: TMA producer of the latent's last two slabs; value MMAs; score MMAs (and the first queries); TMA producer of the rest
//
// What bounds it.  Bytes are 644 a token, once for all heads; the MMAs, M = 128 from shared memory, take 41, 49 and 66 clocks for 32, 64 and 128 columns
// whatever the type's width, 36 of them for a tile up to 32 heads a CTA and 52 with 64.  Measured, the whole call replayed (and this kernel under a profiler), scores of
// deviation about 1: 64 requests of up to 8192 tokens, 16 heads, pages of 64, 42.5 us (35; a tile in 3.5 K clocks, HBM's rate); 200 of about 2000, 32 heads, pages
// of 128, 76 us (64; HBM's rate too, and 5 K clocks for each switch of request); 8 of up to 65536, 128 heads, pages of 64, 131 us, in long runs, at the
// card's power limit, 153 (128; 4.2 K clocks a tile against 2.9 K of MMAs: two tiles are in flight, and a slab's life -- load 1.8 K, scores, softmax 2.4 K,
// values 1.6 K -- is more than twice that); 250 of up to 600, 64 heads, 60 us with pages of 64 and 67 with pages of 16 (48 with pages of 16; one or two switches a CTA,
// 10 K clocks each: 128 KB of accumulator to L2 and a tile without references; the three kernels' starts overlap).  Pages of 16 tokens are 40 copies a tile for two
// lanes where pages of 64 are 10: 64 x 8192 64 us, 200 x 2000 106.
// Scores of deviation 2 and 3, the same four (250 x 600 with pages of 64): 46, 90, 176, 65 and 51, 98, 191, 74: of a softmax group's ten tiles 4 and 7 to
// 9 find a reference that does not hold, against one (and a piece's first, which has none): two meetings more, the weights a second time, the values of the tile before waited for.
#pragma once
#include "armed_ring.cuh"
#include "attn_decode_sm100.cuh"
#include "cache8_sm100.cuh"

namespace laga {

constexpr int kD8Keys = 128;                 // keys of a tile
constexpr int kD8Unit = kDecKeys;            // keys of a unit of the line: a tile is one or two
constexpr float kD8Lift = 7.0f;              // where a tile's maximum is put ...
constexpr float kD8High = 11.0f;             // ... and the most it may become; the least is 0
constexpr float kD8Fall = 40.0f;
// Weights that stand apart.  What P can hold is relative to its tile's largest weight, so that a token with a large key (and with it a large scale), a high score and
// a small value, as they are found where a context begins, would drown its neighbours: with 13 nats between them and 2^7 between the scales, all 127 of them.
// So a key that is more than 2^kApart above the rest of its tile is no part of P: the reference is put where the rest needs it, the key's d are kept in the
// piece's place of the workspace, which is written only when the piece ends, and before the accumulator is drained the token's codes are fetched from the cache
// once more and multiplied in fp32.  The reference goes down no further than 2^kD8Fall below what is left out.
// Which: in a piece's first tile, keys of some warps (32 neighbours each) where as many others have nothing near (of a tile with three warps' keys, or two,
// one other; with one's, every fourth key counts as another's); in a later one, keys that far above the window.  Of each warp kD8Places in a piece at
// most; where there are more, the tile's largest weight sets the reference as it does otherwise.
// A tile with some costs 2 to 4 us, meetings and latencies (with one in each request: 511 tokens 16.5 -> 17.3 us, 64 of up to 8192, 16 heads 42.2 -> 44.8, 200 of about
// 2000, 32 heads 75.8 -> 82.5, 250 of up to 600, 64 heads 60 -> 71.5); that they may come costs 0.6 us a call and 2 % where scores are flat, and some 5 to 15 % of scores of
// deviation 2 and more, whose references move often.  (Kept per head instead of for the group's heads together, at the end by a walk over their places: 3 to 5 us a
// tile.  As called functions: 5 % lost where nothing stands apart.)
constexpr int kD8Places = 4;
constexpr int kD8Looks = 2;                  // tiles of a piece from which keys may be left out
constexpr int kD8Place = 36;                 // words of a kept key: d of up to 16 heads, its place in the request, 1 / its scale, and m of then
constexpr float kD8LoScale = 32.0f;

// Two pairs of fp16 numbers as four codes and the codes of what is left: e4m3, and 32 times the rest; or e5m2, and the rest in e4m3.  (One block of
// instructions: halves of registers that the compiler sees one by one are moved about.)
__device__ __forceinline__ void parts_e4m3_scaled(uint32_t x, uint32_t y, uint32_t& hi, uint32_t& lo) {
    asm("{\n\t.reg .b16 a, b;\n\t.reg .b32 u, v, s;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 a, %2;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, %3;\n\t"
        "mov.b32 %0, {a, b};\n\tcvt.rn.f16x2.e4m3x2 u, a;\n\tcvt.rn.f16x2.e4m3x2 v, b;\n\t"
        "mov.b32 s, 0x50005000;\n\t"                        // 32 twice
        "sub.rn.f16x2 u, %2, u;\n\tsub.rn.f16x2 v, %3, v;\n\tmul.rn.f16x2 u, u, s;\n\tmul.rn.f16x2 v, v, s;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 a, u;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, v;\n\tmov.b32 %1, {a, b};\n\t}"
        : "=&r"(hi), "=&r"(lo)
        : "r"(x), "r"(y));
}
__device__ __forceinline__ void parts_e5m2_e4m3(uint32_t x, uint32_t y, uint32_t& hi, uint32_t& lo) {
    asm("{\n\t.reg .b16 a, b;\n\t.reg .b32 u, v;\n\t"
        "cvt.rn.satfinite.e5m2x2.f16x2 a, %2;\n\tcvt.rn.satfinite.e5m2x2.f16x2 b, %3;\n\t"
        "mov.b32 %0, {a, b};\n\tcvt.rn.f16x2.e5m2x2 u, a;\n\tcvt.rn.f16x2.e5m2x2 v, b;\n\t"
        "sub.rn.f16x2 u, %2, u;\n\tsub.rn.f16x2 v, %3, v;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 a, u;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, v;\n\tmov.b32 %1, {a, b};\n\t}"
        : "=&r"(hi), "=&r"(lo)
        : "r"(x), "r"(y));
}

template <int kHeads>
struct AttnDecode8Smem {
    static constexpr int kPer = kHeads == 64 ? 16 : 8;         // heads of a softmax group
    static constexpr int kGroups = kHeads / kPer;
    static constexpr int kSoftWarps = 4 * kGroups;
    static constexpr int kThreads = 32 * (kSoftWarps + 4);
    static constexpr bool kSplit = kHeads <= 32;               // both parts of P as columns
    // One copy of the instructions that make P of scores, not two: fewer registers, of which 20 warps have 96 each (saves 1.4 us for 200 requests
    // of about 2000 tokens, 32 heads, costs 4 for 1024 of up to 300; would cost 0.4 at 64 x 8192 with 16 heads and 1 to 2 at 8 x 65536 with 128)
    static constexpr bool kOneCopy = kHeads == 32;
    static constexpr float kApart = kSplit ? 11.0f : 10.0f;    // how far above the rest of its tile a weight stands that is left out of P
    static constexpr float kDrop = kSplit ? 3.0f : 0.0f;       // P = 2^(d - kDrop): at most 2^8 in e4m3 (hi and 32 times the rest), 2^11 in e5m2 and its rest
    static constexpr int kCols = kSplit ? 2 * kHeads : kHeads; // TMEM columns of 128 latents of O^T
    static constexpr int kPRow = kSplit ? 2 * kHeads : kHeads; // bytes of a key's row of P
    static constexpr int kPTile = kD8Keys * kPRow;
    static constexpr int kSlabs = kHeads == 16 ? 12 : kHeads == 32 ? 10 : 8;
    // With 64 heads' queries there are slabs for two tiles but not for their keys' too: the key's slab comes first, into the place of the latent's
    // first, and is scored while that is still on its way.  (A ring of five slabs a tile let a tile's last slab in only after the values of the
    // tile before: 8 x 65536, 128 heads 153 us against 133.5.  A place of 8 KB for the key's codes and then their rests, beside eight for the latent, which one
    // copy of the queries' rotated part would leave room for: 138.)
    static constexpr bool kKeyFirst = kHeads == 64;
    static constexpr int kScales = kHeads == 64 ? 2 : 4;       // tiles whose scales are held
    static constexpr int kQSlab = 2 * kHeads * 128;            // 32 rows for every 16 heads, hi then lo, x 128 channels
    static constexpr int kSlab = kD8Keys * 128;
    static constexpr int kQ = 0;
    static constexpr int kP = kQ + 5 * kQSlab;                 // two buffers, or the two parts
    static constexpr int kSlab0 = kP + 2 * kPTile;
    static constexpr int kScale = kSlab0 + kSlabs * kSlab;
    static constexpr int kRef = kScale + kScales * kD8Keys * 4;    // per head: m; query factor, step of m and its power, tile maximum (these four: a piece's sums, a row a warp); maximum of the rest
    static constexpr int kVote = kRef + 6 * kHeads * 4;            // [2][groups][4 warps]
    static constexpr int kBar = kVote + 2 * kGroups * 16;
    static constexpr int kBars = 2 * kSlabs + 12 + kScales + kGroups;
    static constexpr int kMisc = kBar + kBars * 8;             // TMEM slot, abort flag, start, scan
    static constexpr int kTotalBytes = kMisc + 16 + 4 * (kThreads / 32);
    static_assert(4 * kD8Places * kD8Place <= 2 * 512, "what is left out does not fit two heads of a piece");
    static_assert(kTotalBytes <= 232448 && kSlab0 % 1024 == 0 && kP % 1024 == 0 && kVote % 16 == 0 && kBar % 8 == 0, "decode kernel's shared memory");
};

struct AttnDecode8Args {
    AttnDecodeArgs d;
    Cache8 cache;
    const float* q_scale;              // [B][h_pad]; written by the kernel before, which may still run when this one starts: no load of constants (here and in the joins)
};

// Where the line's units lie.  A request with tokens begins with a gap as long as what its switch costs -- queries, a tile without references, the accumulator
// to drain -- and is then its units: stretches of the line are equal work, not equal units, and one that would begin within a gap begins with the request.
// (Saves 13.6 us for 250 requests of up to 600 tokens, 64 heads, 11 for 1024 of up to 300, 32 heads, 7.7 for 130 of up to 900, 128 heads, 1.7 each for 200 of about 2000, 32
// heads, and 64 of up to 8192, 16 heads, with pages of 64, and costs 0.8 for one of 511.  Gaps of 8, 6 and 5 units, or of 3, 3 and 2, were 0.1 to 2.4 us worse in one or other of these.)
constexpr int decode8_gap(int heads) { return heads == 64 ? 5 : heads == 32 ? 4 : 3; }

// Walks the tiles of one CTA's stretch of the line.
struct Decode8Cursor {
    int left, b, t, n, len, gap;       // of the stretch left; request; unit within it; its units; its length
    __device__ __forceinline__ void open(const AttnDecodeArgs& a) {
        for (; b < a.B; ++b) {
            len = decode_len(a, b);
            n = (len + kD8Unit - 1) / kD8Unit;
            if (t < n) return;
            t = 0;
        }
        left = 0;                      // the lengths changed under the kernel: stop
    }
    __device__ __forceinline__ Decode8Cursor(const AttnDecodeArgs& a, int gap_, int left_, int b_, int t_) : left(left_), b(b_), t(t_), n(0), len(0), gap(gap_) {
        if (left > 0) open(a);
    }
    __device__ __forceinline__ bool done() const { return left <= 0; }
    __device__ __forceinline__ int units() const { return min(min(2, n - t), left); }
    __device__ __forceinline__ bool ends_piece() const { return t + 2 >= n || left <= 2; }
    __device__ __forceinline__ int valid() const { return min(units() * kD8Unit, len - t * kD8Unit); }
    __device__ __forceinline__ void next(const AttnDecodeArgs& a) { advance(a, units()); }
    // The same by pieces: the keys of this one from here on, tiles of kD8Keys and what is left; and the next one.
    __device__ __forceinline__ int piece_keys() const { return min(min(n - t, left) * kD8Unit, len - t * kD8Unit); }
    __device__ __forceinline__ void next_piece(const AttnDecodeArgs& a) { advance(a, min(n - t, left)); }
    __device__ __forceinline__ void advance(const AttnDecodeArgs& a, int u) {
        left -= u;
        t += u;
        if (t >= n && left > 0) { t = 0; ++b; open(a); left -= gap; }
    }
};

// kN values a lane, each reduced over the warp: the halves of the values change sides until a lane has one, value lane / (32 / kN).  (kN plus a
// few shuffles; the warp-wide reduction instruction is one for each value, but takes some 18 clocks of a unit that the SM's warps share.)
template <int kN, class Op>
__device__ __forceinline__ float warp_reduce_each(float (&v)[kN], int lane, Op op) {
    int dist = 16;
#pragma unroll
    for (int n = kN / 2; n > 0; n >>= 1, dist >>= 1) {
        const bool upper = (lane & dist) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float out = upper ? v[i] : v[i + n], keep = upper ? v[i + n] : v[i];
            v[i] = op(keep, __shfl_xor_sync(0xffffffffu, out, dist));
        }
    }
#pragma unroll
    for (int e = 16 / kN; e > 0; e >>= 1) v[0] = op(v[0], __shfl_xor_sync(0xffffffffu, v[0], e));
    return v[0];
}
// Floats as integers of the same order, and back.
__device__ __forceinline__ int ordered(float x) {
    const int i = __float_as_int(x);
    return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }
constexpr int kOrderedLowest = static_cast<int>(0x80000000u);
template <int kHeads>
__global__ void __launch_bounds__(AttnDecode8Smem<kHeads>::kThreads, 1)
attn_decode8_sm100_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_codes, const AttnDecode8Args all) {
    using L = AttnDecode8Smem<kHeads>;
    const AttnDecodeArgs& args = all.d;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBar);
    uint64_t* full = bars;                            // [kSlabs] slab has landed (the key's: and the tile's scales)
    uint64_t* empty = full + L::kSlabs;               // ... has been scored and multiplied
    uint64_t* q_full = empty + L::kSlabs;             // the piece's queries
    uint64_t* q_empty = q_full + 1;
    uint64_t* s_full = q_empty + 1;                   // [2] scores of tile T are in TMEM buffer T & 1
    uint64_t* p_full = s_full + 2;                    // [2] P of tile T is in shared memory, O^T is rescaled
    uint64_t* pv_done = p_full + 2;                   // [2] O^T += V^T P of tile T has completed
    uint64_t* o_full = pv_done + 2;                   // a piece's accumulator is complete
    uint64_t* o_free = o_full + 1;                    // ... and has been drained
    uint64_t* quiesce_bar = o_free + 1;               // [2] abort path only: the issuers' last commits
    // [kScales] scales of tile T are in buffer T % kScales.  (Not the key slab's barrier: that slab is free again once scored, so its barrier may
    // be a phase further when the softmax looks.)
    uint64_t* c_full = quiesce_bar + 2;
    uint64_t* group_bar = c_full + L::kScales;        // [kGroups] a softmax group's warps meet: a wait with a limit, as every wait here
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    int* start_b = reinterpret_cast<int*>(tmem_slot + 2);
    int* start_t = start_b + 1;
    int* scan = start_b + 2;                          // per-warp sums of the unit counts
    float* ref_s = reinterpret_cast<float*>(smem + L::kRef);
    float *factor_s = ref_s + kHeads, *step_s = factor_s + kHeads, *alpha_s = step_s + kHeads;
    int *top_s = reinterpret_cast<int*>(alpha_s + kHeads), *rest_s = top_s + kHeads;
    float* most_s = step_s;                           // [4 warps][kHeads], in a piece's first tile before the four have their values
    // once the stretch is found: keys that each softmax warp has left out of P in this piece; for each group, how many of its tiles something stands apart in
    // (upper half), and for which heads of this one
    int *took_s = scan, *apart_s = scan + L::kSoftWarps;

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int group = static_cast<int>(blockIdx.x) % args.n_groups;
    const int cta = static_cast<int>(blockIdx.x) / args.n_groups;
    const int head0 = group * kHeads;
    constexpr int kProducerWarp2 = L::kSoftWarps, kValueWarp = kProducerWarp2 + 1, kScoreWarp = kProducerWarp2 + 2, kProducerWarp = kProducerWarp2 + 3;

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kSlabs; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        mbar_init(q_full, 1); mbar_init(q_empty, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_full[i], L::kSoftWarps); mbar_init(&pv_done[i], 1); mbar_init(&quiesce_bar[i], 1); }
        mbar_init(o_full, 1); mbar_init(o_free, L::kSoftWarps);
        for (int i = 0; i < L::kScales; ++i) mbar_init(&c_full[i], 1);
        for (int i = 0; i < L::kGroups; ++i) mbar_init(&group_bar[i], 4);
        abort_flag->value = (smem_u32(smem) & 1023u) != 0u ? 1u : 0u;
        *start_b = 0; *start_t = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tmap_q); tma_prefetch_desc(&tmap_codes);
    }
    if (warp == kScoreWarp) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_launch_dependents();
    // Launched to overlap decode_absorb8_kernel, the call's first: only the queries (and the status word, which it clears) are its work, so
    // only who touches those waits for it.  All 512 columns are this CTA's, so they start at column 0 (checked, not trusted).
    constexpr uint32_t tmem_base = 0, tmem_s = 256;
    if (threadIdx.x == 0 && (abort_flag->value != 0u || *tmem_slot != tmem_base)) {
        abort_flag->value = 1u;
        atomicCAS(args.status, kStatusOk, kStatusCheck | 0xD5u);
    }

    constexpr int kGap = decode8_gap(kHeads);
    // ---- the line of units, and where this CTA's stretch begins ---------------------------------------------
    int my_units = 0;
    {
        const int run = (args.B + L::kThreads - 1) / L::kThreads;
        const int b0 = min(args.B, static_cast<int>(threadIdx.x) * run), b1 = min(args.B, b0 + run);
        auto line_of = [&](int b) {
            const int n = (decode_len(args, b) + kD8Unit - 1) / kD8Unit;
            return n > 0 ? n + kGap : 0;
        };
        int sum = 0;
        for (int b = b0; b < b1; ++b) sum += line_of(b);
        int incl = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += v;
        }
        if (lane == 31) scan[warp] = incl;
        __syncthreads();
        int before = incl - sum, total = 0;
#pragma unroll
        for (int w = 0; w < L::kThreads / 32; ++w) {
            if (w < warp) before += scan[w];
            total += scan[w];
        }
        const int per = (total + args.ctas_per_group - 1) / args.ctas_per_group;
        const int g0 = cta * per;
        my_units = min(per, total - g0);               // may be negative: nothing to do
        for (int b = b0; b < b1; ++b) {
            const int n = line_of(b);
            if (g0 >= before && g0 < before + n) { *start_b = b; *start_t = g0 - before - kGap; }
            before += n;
        }
        __syncthreads();
    }
    const int first_b = *start_b, first_t = max(0, *start_t);
    my_units += min(0, *start_t);                      // what is left of a gap; nothing to do where the stretch ends in it

    auto fetch_queries = [&](int b) {
        grid_dependency_wait();                              // (returns at once after the first time)
        mbar_arrive_expect_tx(q_full, 5 * L::kQSlab);
        for (int k = 0; k < 5; ++k)
            tma_load_2d_chk(args.status, smem + L::kQ + k * L::kQSlab, &tmap_q, q_full, k * 128, 2 * (b * args.h_pad + head0));
    };

    // ---- producers: boxes of min(page, 64) keys, kSubs of them a slab ----------------------------------------
    // Two lanes share a tile's slabs.  What limits them is their instruction count -- a lane beside busy softmax warps runs at four to six
    // clocks an instruction, a copy's operands go through uniform registers -- so addresses are plain words, and what is in flight is worked
    // out only where a wait has given up.  kFirst: the lane with the key's slab, the latent's first two, the scales and the queries.
    auto produce = [&](auto subs, auto first_half) {
        constexpr int kSubs = decltype(subs)::value, kBox = kD8Keys / kSubs;
        constexpr bool kFirst = decltype(first_half)::value;
        constexpr uint32_t kBegin = kFirst ? 0 : 3, kCount = kFirst ? 3 : 2;
        const uint64_t once = args.n_groups == 1 ? l2_evict_first() : l2_evict_normal();      // (head groups read a tile one after another)
        const int shift = args.page_shift, in_page = (1 << shift) - 1, n_pages = args.n_pages;
        const uint32_t full_a = smem_u32(full), empty_a = smem_u32(empty), slab_a = smem_u32(smem + L::kSlab0);
        int pages[kSubs], pages_next[kSubs];                 // of the tile's boxes; a tile ahead
        auto fetch_pages = [&](const Decode8Cursor& c, int* p) {
            if (c.done()) return;
            const int* row = args.block_table + static_cast<size_t>(c.b) * args.columns;
            const int k0 = c.t * kD8Unit;
#pragma unroll
            for (int i = 0; i < kSubs; ++i) p[i] = k0 + i * kBox < c.len ? __ldg(row + ((k0 + i * kBox) >> shift)) : 0;
        };
        Decode8Cursor cur(args, kGap, my_units, first_b, first_t);
        fetch_pages(cur, pages);
        uint32_t slot = kBegin, par = 0, pieces = 0, T = 0;
        ArmedRing<L::kScales> armed_scales;                  // (tile T's, in the lane that has them)
        bool new_piece = true, ok = true;
        // a piece's queries behind its first loads: they wait for the last scores of the piece before (the first are the score warp's)
        auto piece_queries = [&](int b) -> bool {
            if (!new_piece) return true;
            if (pieces > 0) {
                if (!mbar_wait(q_empty, (pieces & 1u) ^ 1u, abort_flag, args.status, 0x81)) return false;
                fetch_queries(b);
            }
            ++pieces;
            return true;
        };
        while (!cur.done()) {
            Decode8Cursor next = cur;
            next.next(args);
            fetch_pages(next, pages_next);
            const int boxes = (cur.valid() + kBox - 1) / kBox, row0 = (cur.t * kD8Unit) & in_page;       // boxes of this tile that hold a key
            float* scales = reinterpret_cast<float*>(smem + L::kScale) + armed_scales.at() * kD8Keys;
            bool all_there = true;
#pragma unroll
            for (int i = 0; i < kSubs; ++i) all_there = all_there && static_cast<uint32_t>(pages[i]) < static_cast<uint32_t>(n_pages);
            uint32_t there = static_cast<uint32_t>(boxes);   // boxes whose page is one
            if (!all_there) {
#pragma unroll
                for (int i = 0; i < kSubs; ++i) {
                    if (i >= boxes || static_cast<uint32_t>(pages[i]) < static_cast<uint32_t>(n_pages)) continue;
                    pages[i] = n_pages;                      // out of the map's range: TMA fills zeros
                    --there;
                    atomicCAS(args.status, kStatusOk, kStatusCheck | 0xF2u);
                }
            }
#pragma unroll
            for (uint32_t s = 0; s < kCount; ++s) {          // the key's slab, then the latent's four (kKeyFirst: the first of them last)
                int channel = kBegin + s == 0 ? kC8Lat : static_cast<int>(kBegin + s - 1) * 128;
                if constexpr (L::kKeyFirst) {
                    // The tile's four places; the latent's quarter too but for the key's slab.  The first is filled twice a tile, both times by this
                    // lane, which sees every phase of its barrier one after another (one that did not could take a phase for the one before the last).
                    const uint32_t which = kFirst ? s & 1u : s + 2u;
                    slot = (T & 1u) * 4 + which;
                    par = which > 0 ? (T >> 1) & 1u : s >> 1;
                    channel = kFirst && s == 0 ? kC8Lat : static_cast<int>(which) * 128;
                    if (kFirst && s == 2) {                  // (waits for the key's scores, which need the queries)
                        ok = piece_queries(cur.b);
                        if (!ok) break;
                    }
                }
                const uint32_t bar = full_a + slot * 8;
                if (!mbar_test_wait_u32(empty_a + slot * 8, par ^ 1u)) ok = mbar_wait(&empty[slot], par ^ 1u, abort_flag, args.status, 0x80);
                if (!ok) break;
                mbar_arrive_expect_tx_u32(bar, boxes * (kBox * 128));
                const uint32_t dst = slab_a + slot * L::kSlab;
#pragma unroll
                for (int i = 0; i < kSubs; ++i)
                    if (i < boxes) tma_load_codes_chk(args.status, dst + i * (kBox * 128), &tmap_codes, bar, channel, (row0 + i * kBox) & in_page, pages[i], once);
                if (kFirst && s == 0) {                      // (the scales that were in this buffer have been read: their tile's values are multiplied)
                    if (there != static_cast<uint32_t>(boxes)) {
                        for (int k = 0; k < boxes * kBox; ++k) scales[k] = 1.0f;
                        fence_async_shared();
                    }
                    uint64_t* c_bar = &c_full[armed_scales.at()];
                    mbar_arrive_expect_tx(c_bar, there * (kBox * 4));
                    armed_scales.arm();
#pragma unroll
                    for (int i = 0; i < kSubs; ++i)
                        if (i < boxes && pages[i] < n_pages)
                            bulk_load(scales + i * kBox, all.cache.base + pages[i] * all.cache.page_bytes() + (static_cast<size_t>(kC8Row) << shift) +
                                      ((row0 + i * kBox) & in_page) * 4, kBox * 4, c_bar);
                }
                if constexpr (!L::kKeyFirst) {
                    slot += s + 1 < kCount ? 1u : 6u - kCount;
                    if (slot >= L::kSlabs) { slot -= L::kSlabs; par ^= 1u; }
                }
            }
            if (!ok) break;
            if constexpr (kFirst && !L::kKeyFirst) {
                ok = piece_queries(cur.b);
                if (!ok) break;
            }
            new_piece = cur.ends_piece();
            cur = next;
#pragma unroll
            for (int i = 0; i < kSubs; ++i) pages[i] = pages_next[i];
            ++T;
        }
        // What a lane has armed is complete when every barrier has left the phase that it was armed for last: slots behind `slot` are a round
        // behind.  (A barrier that was never armed, or is the other lane's, costs the limit at most.)
        if (abort_flag->value != 0u) {
            for (uint32_t i = 0; i < L::kSlabs; ++i) {
                if constexpr (L::kKeyFirst) {                // (armed for either)
                    mbar_wait_quiesce(&full[i], 0);
                    mbar_wait_quiesce(&full[i], 1);
                } else {
                    mbar_wait_quiesce(&full[i], i < slot ? par : par ^ 1u);
                }
            }
            if (kFirst) {
                armed_scales.last_phases([&](uint32_t i, uint32_t parity) { mbar_wait_quiesce(&c_full[i], parity); });
                if (pieces > 0) mbar_wait_quiesce(q_full, (pieces - 1) & 1u);
            }
        }
    };
    auto produce_half = [&](auto first_half) {
        if (args.page_shift >= 6) produce(std::integral_constant<int, 2>{}, first_half);
        else if (args.page_shift == 5) produce(std::integral_constant<int, 4>{}, first_half);
        else produce(std::integral_constant<int, 8>{}, first_half);
    };

    if (abort_flag->value != 0u || my_units <= 0) {
        // nothing to do (or nothing may be done): fall through to the common exit
    } else if (warp == kProducerWarp) {
        if (elect_one()) produce_half(std::true_type{});
    } else if (warp == kProducerWarp2) {
        if (elect_one()) produce_half(std::false_type{});
    } else if (warp == kScoreWarp) {
        // ---- issuer of the score MMAs ------------------------------------------------------------------------
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_f8(kE4m3, kE4m3, 128, 2 * kHeads, 0, 0);
            const uint32_t k_lo = desc_lo(desc_k_major(smem_u32(smem + L::kSlab0))), q_lo = desc_lo(desc_k_major(smem_u32(smem + L::kQ))),
                           hi = desc_hi(desc_k_major(0));
            uint32_t slot = 0, par = 0, pieces = 0;
            bool ok = true, new_piece = true;
            fetch_queries(first_b);                          // (a unit of first_b is here, so it is the first request with tokens)
            Decode8Cursor cur(args, kGap, my_units, first_b, first_t);
            for (uint32_t T = 0; !cur.done(); ++T) {
                const uint32_t buf = T & 1u, d = tmem_s + buf * (2 * kHeads);
                if (T >= 2) ok = mbar_wait(&p_full[buf], ((T >> 1) & 1u) ^ 1u, abort_flag, args.status, 0x82);     // the scores of tile T - 2 have been read
                if (ok && new_piece) ok = mbar_wait(q_full, pieces & 1u, abort_flag, args.status, 0x83);
                if (!ok) break;
                new_piece = cur.ends_piece();
                cur.next(args);
                // A barrier probe queues behind the lane's MMAs until the tensor pipe has taken them, so the next slab's is made before this one's.
                // kKeyFirst: the key's slab, the latent's second to fourth, its first.
                if constexpr (L::kKeyFirst) { slot = buf * 4; par = 0; }
                bool here = mbar_test_wait(&full[slot], par);
#pragma unroll 1
                for (int s = 0; s < 5; ++s) {
                    if (!here) ok = mbar_wait(&full[slot], par, abort_flag, args.status, 0x84);
                    if (!ok) break;
                    const uint32_t at = slot;
                    if constexpr (L::kKeyFirst) {
                        slot = buf * 4 + ((s + 1) & 3);
                        par = s == 3 ? 1u : (T >> 1) & 1u;
                    } else if (++slot == L::kSlabs) {
                        slot = 0;
                        par ^= 1u;
                    }
                    if (s < 4) here = mbar_test_wait(&full[slot], par);
                    tc_fence_after_sync();
                    const int quarter = s == 0 ? 4 : L::kKeyFirst ? s & 3 : s - 1;       // of the queries' channels
                    mma8_ss_chain4<2, 2>(d, k_lo + at * (L::kSlab / 16), hi, q_lo + quarter * (L::kQSlab / 16), hi, idesc, s > 0 ? 1u : 0u);
                    if (s == 0) mma_commit(&empty[at]);
                }
                if (!ok) break;
                mma_commit(&s_full[buf]);
                if (new_piece) { mma_commit(q_empty); ++pieces; }
            }
            if (abort_flag->value != 0u) { mma_commit(quiesce_bar); mbar_wait_quiesce(quiesce_bar, 0); }
        }
    } else if (warp == kValueWarp) {
        // ---- issuer of the value MMAs ------------------------------------------------------------------------
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_f8(kE4m3, L::kSplit ? kE4m3 : kE5m2, 128, L::kCols, 1, 1), idesc_lo = make_idesc_f8(kE4m3, kE4m3, 128, L::kCols, 1, 1);
            constexpr int kAStep = 32 * 128 / 16, kBStep = 32 * L::kPRow / 16;
            const uint32_t v_lo = desc_lo(desc_mn_major(smem_u32(smem + L::kSlab0), L::kSlab)), v_hi = desc_hi(desc_mn_major(0, L::kSlab)),
                           p_lo = desc_lo(desc_mn_major_narrow<L::kPRow>(smem_u32(smem + L::kP))), p_hi = desc_hi(desc_mn_major_narrow<L::kPRow>(0));
            uint32_t slot = 0, pieces = 0;
            bool ok = true, new_piece = true;
            Decode8Cursor cur(args, kGap, my_units, first_b, first_t);
            for (uint32_t T = 0; !cur.done(); ++T) {
                const uint32_t buf = T & 1u;
                const int k_steps = (cur.valid() + 31) >> 5;
                ok = mbar_wait(&p_full[buf], (T >> 1) & 1u, abort_flag, args.status, 0x85);
                // the first tile of a piece overwrites O^T: the piece before it must have been drained
                if (ok && new_piece && pieces > 0) ok = mbar_wait(o_free, (pieces - 1) & 1u, abort_flag, args.status, 0x86);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t b_lo = p_lo + (L::kSplit ? buf * (L::kPTile / 16) : 0u);
                if constexpr (L::kKeyFirst) slot = buf * 4;
                else if (++slot == L::kSlabs) slot = 0;      // the key's slab
#pragma unroll 1
                for (uint32_t s = 0; s < 4; ++s) {
                    const uint32_t a_lo = v_lo + slot * (L::kSlab / 16), d = tmem_base + s * L::kCols;
                    if (k_steps == 4) {
                        mma8_ss_chain4<kAStep, kBStep>(d, a_lo, v_hi, b_lo, p_hi, idesc, new_piece ? 0u : 1u);
                        if constexpr (!L::kSplit) mma8_ss_chain4<kAStep, kBStep>(d, a_lo, v_hi, b_lo + L::kPTile / 16, p_hi, idesc_lo, 1u);
                    } else {
#pragma unroll 1
                        for (int k = 0; k < k_steps; ++k) {
                            mma8_ss(d, desc_of(a_lo + k * kAStep, v_hi), desc_of(b_lo + k * kBStep, p_hi), idesc, (!new_piece || k > 0) ? 1u : 0u);
                            if constexpr (!L::kSplit)
                                mma8_ss(d, desc_of(a_lo + k * kAStep, v_hi), desc_of(b_lo + L::kPTile / 16 + k * kBStep, p_hi), idesc_lo, 1u);
                        }
                    }
                    mma_commit(&empty[slot]);
                    if (++slot == L::kSlabs) slot = 0;
                }
                mma_commit(&pv_done[buf]);
                new_piece = cur.ends_piece();
                if (new_piece) { mma_commit(o_full); ++pieces; }
                cur.next(args);
            }
            if (abort_flag->value != 0u) { mma_commit(quiesce_bar + 1); mbar_wait_quiesce(quiesce_bar + 1, 0); }
        }
    } else if (warp < L::kSoftWarps) {
        // ---- softmax, rescaling, drain -----------------------------------------------------------------------
        constexpr int kPer = L::kPer, kPairs = kPer / 2, kShare = 32 / kPer;
        const int g = warp >> 2, quarter = warp & 3, key = quarter * 32 + lane, tid = key;      // (thread of the group)
        const int h0 = g * kPer;                               // the group's heads within the CTA's
        const int n_live = max(0, min(kPer, args.h - head0 - h0));
        const uint32_t live = ((1u << n_live) - 1u) << (kPer - n_live);      // bit kPer - 1 - i: the group's head i is one
        const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
        // sixteen heads' scores are 32 columns, first the products with hi, then those with lo; so are their columns of O^T where P has two parts
        const uint32_t sixteen = static_cast<uint32_t>(h0 >> 4), within = static_cast<uint32_t>(h0 & 15);
        const uint32_t col_s = tmem_s + lane_addr + sixteen * 32 + within, col_o = tmem_base + lane_addr + (L::kSplit ? sixteen * 32 + within : h0);
        int* vote_s = reinterpret_cast<int*>(smem + L::kVote) + g * 4;
        float* lsum_s = factor_s;                              // [4 warps][kHeads], where a piece's per-head words are no longer needed
        F2 l2[kPairs];                                         // this key's part of the sums
        uint32_t T = 0, pieces = 0, pos = 0, meetings = 0;     // pos: the tile's first slab
        bool ok = true, first = true, seen = false;            // seen, peak: of the group's head `tid`, whether some key had a weight, and its highest m
        float peak = kDecLowest;
        auto arrive = [&]() {                                  // the group's four warps meet: what they wrote to shared memory is there
            __syncwarp();
            if (lane == 0) mbar_arrive(&group_bar[g]);
        };
        auto wait_for_group = [&]() -> bool { return mbar_wait_warp(&group_bar[g], meetings++ & 1u, abort_flag, args.status, 0x87); };
        auto place_of = [&](int held, uint32_t few) -> int {   // of the warp's places that are not held, this lane's
            uint32_t left = ~static_cast<uint32_t>(held);
            for (uint32_t before = few & ((1u << lane) - 1u); before != 0u; before &= before - 1u) left &= left - 1u;
            return __ffs(static_cast<int>(left)) - 1;
        };
        Decode8Cursor cur(args, kGap, my_units, first_b, first_t);
        auto query_scale = [&](const Decode8Cursor& c) -> float {
            return tid < n_live && !c.done() ? all.q_scale[static_cast<size_t>(c.b) * args.h_pad + head0 + h0 + tid] * args.scale_log2 : 0.f;
        };
        grid_dependency_wait();
        float factor = query_scale(cur);
        int keys_left = cur.piece_keys();
        while (!cur.done()) {
            const uint32_t buf = T & 1u, par = (T >> 1) & 1u;
            const int valid = min(kD8Keys, keys_left);
            if (first) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) l2[i] = f2(0.f, 0.f);
                if (tid < kPer) {
                    factor_s[h0 + tid] = factor;
                    ref_s[h0 + tid] = tid < n_live ? 0.f : 1e30f;        // (a head that is none: every weight zero, and no rescaling for it)
                    rest_s[h0 + tid] = kOrderedLowest;
                }
                if (lane == 0) took_s[warp] = 0;
                if (tid == 0) apart_s[g] = 0;
                seen = false;
                peak = kDecLowest;
                arrive();
                if (!wait_for_group()) break;
            }
            {
                // (asked together: an answer takes some 90 clocks even where it is yes)
                const bool scales = mbar_test_wait(&c_full[T % L::kScales], (T / L::kScales) & 1u), scores = mbar_test_wait(&s_full[buf], par);
                if (!__all_sync(0xffffffffu, scales && scores)) {
                    ok = mbar_wait_warp(&c_full[T % L::kScales], (T / L::kScales) & 1u, abort_flag, args.status, 0x88);
                    if (ok) ok = mbar_wait_warp(&s_full[buf], par, abort_flag, args.status, 0x89);
                    if (!ok) break;
                }
            }
            tc_fence_after_sync();
            // d = y - m
            F2 d[kPairs];
            float s = reinterpret_cast<const float*>(smem + L::kScale)[(T % L::kScales) * kD8Keys + key];
            {
                uint32_t raw[2 * kPer];                        // the products with hi, then those with lo
                if constexpr (kPer == 16) {
                    tmem_ld_x32(col_s + buf * (2 * kHeads), raw);
                } else {
                    tmem_ld_x8(col_s + buf * (2 * kHeads), raw);
                    tmem_ld_x8(col_s + buf * (2 * kHeads) + 16, raw + kPer);
                }
                if (key >= valid || s == 0.f) s = 1.0f;        // (a page as it was made, of zeros: a row of zeros)
                const float ef = static_cast<float>(static_cast<int>(__float_as_uint(s) >> 23 & 0xffu) - 127);
                const F2 s2 = f2(s, s), e2 = f2(ef, ef), minus1 = f2(-1.0f, -1.0f);
                const ulonglong2 *f = reinterpret_cast<const ulonglong2*>(factor_s + h0), *m = reinterpret_cast<const ulonglong2*>(ref_s + h0);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < kPairs; i += 2) {
                    const ulonglong2 f4 = f[i >> 1], m4 = m[i >> 1];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int c = 2 * (i + j);
                        const F2 both = f2_add(f2(__uint_as_float(raw[c]), __uint_as_float(raw[c + 1])), f2(__uint_as_float(raw[kPer + c]), __uint_as_float(raw[kPer + c + 1])));
                        // (y rounded before m is taken off: the largest score of a tile is then at its place whatever its size)
                        const F2 y = f2_fma(both, f2_mul(F2{j == 0 ? f4.x : f4.y}, s2), e2);
                        d[i + j] = f2_fma(F2{j == 0 ? m4.x : m4.y}, minus1, y);
                    }
                }
            }
            if (key >= valid) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) d[i] = f2(-INFINITY, -INFINITY);
            }
            // Does the reference hold?  For every head some key must have d >= 0, and none more than kD8High: the signs of d, a bit a head (the first
            // head's the highest of them), across the keys, and a bit that is set where nothing is above.  (A piece's first tile has no reference yet.)
            if (!first) {
                uint32_t below = 0u;
                float most = -INFINITY;
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float2 v = f2_parts(d[i]);
                    below = __funnelshift_l(__float_as_uint(v.x), below, 1);
                    below = __funnelshift_l(__float_as_uint(v.y), below, 1);
                    most = fmax3(most, v.x, v.y);
                }
                below = __reduce_and_sync(0xffffffffu, below | (most > kD8High ? 0u : 0x80000000u));
                if (lane == 0) vote_s[buf * (4 * L::kGroups) + quarter] = static_cast<int>(below);
                arrive();
            }
            // Probabilities and their parts, while the group's other warps vote.
            F2 p[kPairs];
            uint32_t hi[kPer / 4], lo[kPer / 4];
            auto weigh = [&]() {
#pragma unroll
                for (int i = 0; i < kPer / 4; ++i) {
                    uint32_t p16[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float2 v = f2_parts(L::kSplit ? f2_add(d[2 * i + j], f2(-L::kDrop, -L::kDrop)) : d[2 * i + j]);
                        const float2 w = make_float2(fast_exp2(v.x), fast_exp2(v.y));
                        p[2 * i + j] = f2(w.x, w.y);
                        const __half2 ph = __floats2half2_rn(w.x, w.y);
                        p16[j] = *reinterpret_cast<const uint32_t*>(&ph);
                    }
                    if constexpr (L::kSplit) parts_e4m3_scaled(p16[0], p16[1], hi[i], lo[i]);
                    else parts_e5m2_e4m3(p16[0], p16[1], hi[i], lo[i]);
                }
            };
            // Where the references do not hold, once more with those that do (a piece's first tile has none, and does not weigh before).  kOneCopy: in a
            // second turn of the loop.
            const uint32_t prev = T - (L::kSplit ? 2 : 1);
            bool p_free = true, settled = false;
#pragma unroll 1
            for (;;) {
                if (settled || !first) weigh();
                if (settled) break;
                settled = true;
                // (asked now: P's buffer, whose last use must have been multiplied)
                p_free = T < (L::kSplit ? 2 : 1) || mbar_test_wait(&pv_done[prev & 1u], (prev >> 1) & 1u);
                if (!first) {
                    ok = wait_for_group();
                    if (!ok) break;
                    const int4 votes = *reinterpret_cast<const int4*>(vote_s + buf * (4 * L::kGroups));
                    const uint32_t below = static_cast<uint32_t>(votes.x & votes.y & votes.z & votes.w);
                    if ((below & (0x80000000u | live)) == 0x80000000u) {
                        seen = true;
                        break;
                    }
                }
                // The heads' maxima over the tile, then the references they ask for.
                float tops[kPer];
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float2 v = f2_parts(d[i]);
                    tops[2 * i] = v.x;
                    tops[2 * i + 1] = v.y;
                }
                const float most = warp_reduce_each(tops, lane, [](float x, float y) { return fmaxf(x, y); });
                if (!first) {
                    if ((lane & (kShare - 1)) == 0) atomicMax(&top_s[h0 + lane / kShare], ordered(most));
                } else if (valid > 32 || valid == 1) {
                    if ((lane & (kShare - 1)) == 0) most_s[quarter * kHeads + h0 + lane / kShare] = most;
                } else if (quarter == 0) {                     // all keys are one warp's: as if every fourth were another's
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) {
                            const float2 v = f2_parts(d[i]);
                            tops[2 * i] = (lane & 3) == c ? v.x : -INFINITY;
                            tops[2 * i + 1] = (lane & 3) == c ? v.y : -INFINITY;
                        }
                        const float most_c = warp_reduce_each(tops, lane, [](float x, float y) { return fmaxf(x, y); });
                        if ((lane & (kShare - 1)) == 0) most_s[c * kHeads + h0 + lane / kShare] = most_c;
                    }
                }
                arrive();
                ok = wait_for_group();
                if (!ok) break;
                bool apart = false;
                if (tid < kPer) {
                    const float m = ref_s[h0 + tid];
                    float top;
                    // Does something stand apart?  Then it is far above what the reference was for; in the first tile, one warp has it, and no other anything near it.
                    if (first) {
                        const float* of = most_s + h0 + tid;
                        const float a = fmaxf(of[0], of[kHeads]), b = fmaxf(of[2 * kHeads], of[3 * kHeads]), u = fminf(a, b),
                                    v = fmaxf(fminf(of[0], of[kHeads]), fminf(of[2 * kHeads], of[3 * kHeads]));
                        top = fmaxf(a, b);                     // of the warps' maxima; behind it the larger of u and v, then the smaller
                        rest_s[h0 + tid] = kOrderedLowest;
                        apart = valid > 1 && top - (valid > 64 || (valid >= 4 && valid <= 32) ? fminf(u, v) : fmaxf(u, v)) > L::kApart;
                    } else {
                        top = unordered(top_s[h0 + tid]);
                        apart = top > kD8High + L::kApart && apart_s[g] < kD8Looks << 16;
                    }
                    top_s[h0 + tid] = kOrderedLowest;
                    if (seen) peak = fmaxf(peak, m);
                    const bool given = tid < n_live && top > -INFINITY;
                    apart = apart && given;
                    float to = m;
                    if (given && !apart && (first || !(top >= 0.f && top <= kD8High))) to = fmaxf(m + (top - kD8Lift), peak - kD8Fall);
                    ref_s[h0 + tid] = to;
                    step_s[h0 + tid] = to - m;                 // (the step that was taken, with the sum's rounding)
                    alpha_s[h0 + tid] = apart ? top : fast_exp2(m - to);
                    seen = seen || top > -INFINITY;
                }
                if (quarter == 0) {
                    const uint32_t heads = __ballot_sync(0xffffffffu, apart);
                    if (heads != 0u && lane == 0) apart_s[g] += 0x10000 + static_cast<int>(heads);
                }
                arrive();
                ok = wait_for_group();
                if (!ok) break;
                const uint32_t apart_heads = static_cast<uint32_t>(apart_s[g]) & 0xffffu;        // (the same for the whole group)
                bool may_leave = false;                        // this key is one of few that are far above all others of their warp
                if (__builtin_expect(apart_heads != 0u, 0)) {
                    // The largest of the rest, and the references that it asks for.
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        const float2 v = f2_parts(d[i >> 1]);
                        tops[i] = (i & 1) ? v.y : v.x;
                        const float limit = __shfl_sync(0xffffffffu, most, i * kShare) - L::kApart;
                        may_leave = may_leave || ((apart_heads >> i & 1u) != 0u && tops[i] > limit);
                    }
                    const int held = took_s[warp];             // a bit a place
                    const uint32_t few = __ballot_sync(0xffffffffu, may_leave);
                    may_leave = may_leave && __popc(few) <= kD8Places - __popc(held);
                    if (may_leave) {                           // kept for the end of the piece, if it is left out: d and m of all the group's heads, its place in the request, 1 / s
                        const uint32_t slot = static_cast<uint32_t>(cta + cur.b);
                        float* place = args.part_o + static_cast<size_t>(slot * args.h_pad + head0 + h0 + kPer - 2) * kDecLat + (quarter * kD8Places + place_of(held, few)) * kD8Place;
                        if (device_check(slot < static_cast<uint32_t>(args.ctas_per_group + args.B), args.status, 0xEB0000u | cta)) {
#pragma unroll
                            for (int i = 0; i < kPairs; i += 2) reinterpret_cast<ulonglong2*>(place)[i >> 1] = make_ulonglong2(d[i].v, d[i + 1].v);
                            place[16] = __int_as_float(cur.t * kD8Unit + cur.piece_keys() - keys_left + key);
                            place[17] = __uint_as_float((254u - min(254u, __float_as_uint(s) >> 23 & 0xffu)) << 23);
#pragma unroll 1
                            for (int i = 0; i < kPer; ++i) place[20 + i] = ref_s[h0 + i] - step_s[h0 + i];      // (heads that do not look have taken theirs)
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kPer; ++i) tops[i] = may_leave ? -INFINITY : tops[i];
                    const float rest = warp_reduce_each(tops, lane, [](float x, float y) { return fmaxf(x, y); });
                    if ((lane & (kShare - 1)) == 0) atomicMax(&rest_s[h0 + lane / kShare], ordered(rest));
                    arrive();
                    ok = wait_for_group();
                    if (!ok) break;
                    if (apart) {
                        const float top = alpha_s[h0 + tid], others = unordered(rest_s[h0 + tid]), m = ref_s[h0 + tid];
                        const float aim = others > -INFINITY && top - others > L::kApart ? others : top;
                        float to = aim >= 0.f && aim <= kD8High ? m : fmaxf(m + (aim - kD8Lift), peak - kD8Fall);
                        to = fmaxf(to, m + (top - kD8Lift) - kD8Fall);
                        if (top - (to - m) > kD8High) peak = fmaxf(peak, m + (top - kD8Lift));
                        ref_s[h0 + tid] = to;
                        step_s[h0 + tid] = to - m;
                        alpha_s[h0 + tid] = fast_exp2(m - to);
                    }
                    if (tid < kPer) rest_s[h0 + tid] = kOrderedLowest;
                    if (tid == 0) apart_s[g] &= ~0xffff;
                    arrive();
                    ok = wait_for_group();
                    if (!ok) break;
                }
                const ulonglong2 *step = reinterpret_cast<const ulonglong2*>(step_s + h0), *alpha = reinterpret_cast<const ulonglong2*>(alpha_s + h0);
                const F2 minus1 = f2(-1.0f, -1.0f);
#pragma unroll
                for (int i = 0; i < kPairs; i += 2) {
                    const ulonglong2 t4 = step[i >> 1], a4 = alpha[i >> 1];
                    d[i] = f2_fma(F2{t4.x}, minus1, d[i]);
                    d[i + 1] = f2_fma(F2{t4.y}, minus1, d[i + 1]);
                    if (!first) {
                        l2[i] = f2_mul(l2[i], F2{a4.x});
                        l2[i + 1] = f2_mul(l2[i + 1], F2{a4.y});
                    }
                }
                if (const uint32_t few = __ballot_sync(0xffffffffu, may_leave); __builtin_expect(few != 0u, 0)) {
                    // A key that is above the window now is left out, for all of the group's heads.
                    float largest = -INFINITY;
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        const float2 v = f2_parts(d[i]);
                        largest = fmax3(largest, v.x, v.y);
                    }
                    const bool out = may_leave && largest > kD8High;
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) d[i] = out ? f2(-INFINITY, -INFINITY) : d[i];
                    const int held = took_s[warp];
                    const uint32_t more = __reduce_or_sync(0xffffffffu, out ? 1u << place_of(held, few) : 0u);
                    if (lane == 0) took_s[warp] = held | static_cast<int>(more);
                }
                if constexpr (!L::kOneCopy) weigh();
                if (!first) {
                    // O^T is at rest once the values of the tile before have been multiplied; this tile's wait for p_full below
                    ok = mbar_wait_warp(&pv_done[(T - 1) & 1u], ((T - 1) >> 1) & 1u, abort_flag, args.status, 0x8A);
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int h = 0; h < kPer; ++h) {           // (mostly one head's reference has moved: its columns alone)
                        if (step_s[h0 + h] == 0.f) continue;   // (the same for the whole group)
                        const float by = alpha_s[h0 + h];
                        uint32_t o[4], rest[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            tmem_ld_x1(col_o + c * L::kCols + h, &o[c]);
                            if constexpr (L::kSplit) tmem_ld_x1(col_o + c * L::kCols + 16 + h, &rest[c]);
                        }
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            tmem_st_x1(col_o + c * L::kCols + h, __float_as_uint(__uint_as_float(o[c]) * by));
                            if constexpr (L::kSplit) tmem_st_x1(col_o + c * L::kCols + 16 + h, __float_as_uint(__uint_as_float(rest[c]) * by));
                        }
                    }
                    tmem_st_wait();
                }
                if constexpr (!L::kOneCopy) break;
            }
            if (!ok) break;
            {
                const float inv = __uint_as_float((254u - min(254u, __float_as_uint(s) >> 23 & 0xffu)) << 23);      // 1 / s
                const F2 inv2 = f2(inv, inv);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) l2[i] = f2_fma(p[i], inv2, l2[i]);
            }
            if (!__all_sync(0xffffffffu, p_free)) {
                ok = mbar_wait_warp(&pv_done[prev & 1u], (prev >> 1) & 1u, abort_flag, args.status, 0x8B);
                if (!ok) break;
            }
            {
                uint8_t* row = smem + L::kP + (L::kSplit ? buf * L::kPTile : 0) + key * L::kPRow;
                const int turn = L::kPRow == 32 ? (key >> 2) & 1 : (key >> 1) & 3;
                if constexpr (L::kSplit) {                     // sixteen heads: a chunk of hi, a chunk of lo; this group's are half of each
                    *reinterpret_cast<uint2*>(row + (((2 * sixteen) ^ turn) << 4) + within) = make_uint2(hi[0], hi[1]);
                    *reinterpret_cast<uint2*>(row + (((2 * sixteen + 1) ^ turn) << 4) + within) = make_uint2(lo[0], lo[1]);
                } else {
                    *reinterpret_cast<uint4*>(row + ((g ^ turn) << 4)) = make_uint4(hi[0], hi[1], hi[kPer / 4 - 2], hi[kPer / 4 - 1]);
                    *reinterpret_cast<uint4*>(row + L::kPTile + ((g ^ turn) << 4)) = make_uint4(lo[0], lo[1], lo[kPer / 4 - 2], lo[kPer / 4 - 1]);
                }
            }
            if (g == 0 && (valid & 31)) {     // rows of the last 32-key step that no token owns: zero, whatever the page holds (0 * NaN is NaN)
                const int n_zero = 32 - (valid & 31);
                for (int i = tid; i < 4 * 8 * n_zero; i += 128) {                    // 4 slabs x rows x eight 16-byte chunks
                    const int slab = i / (8 * n_zero), r = valid + (i >> 3) % n_zero;
                    uint32_t slot = pos + (L::kKeyFirst ? 0 : 1) + slab;
                    if (slot >= L::kSlabs) slot -= L::kSlabs;
                    *reinterpret_cast<uint4*>(smem + L::kSlab0 + slot * L::kSlab + r * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
            fence_async_shared();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[buf]);
            first = false;
            keys_left -= kD8Keys;
            if (keys_left <= 0) {
                const int b = cur.b;
                cur.next_piece(args);
                keys_left = cur.piece_keys();
                factor = query_scale(cur);                     // the next piece's, on its way meanwhile
                // the sums over the 128 keys, within the warp
                float sums[kPer];
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float2 v = f2_parts(l2[i]);
                    sums[2 * i] = v.x;
                    sums[2 * i + 1] = v.y;
                }
                const float sum = warp_reduce_each(sums, lane, [](float x, float y) { return x + y; });
                ok = mbar_wait_warp(o_full, pieces & 1u, abort_flag, args.status, 0x8C);
                if (!ok) break;
                tc_fence_after_sync();
                // (O is complete: every warp of the group has handed over its P, so the per-head words but m have been read)
                if ((lane & (kShare - 1)) == 0) lsum_s[quarter * kHeads + h0 + lane / kShare] = sum;
                arrive();
                const size_t slot = static_cast<size_t>(cta) + b;
                // (a slot past the workspace would mean that the roles disagree about the pieces)
                const bool store = device_check(slot < static_cast<size_t>(args.ctas_per_group) + args.B, args.status, 0xEB0000u | cta);
                const bool any_taken = store && apart_s[g] != 0;       // (or looked at, at least)
                const float* places = args.part_o + (slot * args.h_pad + head0 + h0 + kPer - 2) * kDecLat;
                if (__builtin_expect(any_taken, 0)) {
                    ok = wait_for_group();
                    if (!ok) break;
                    // What was left out, in a fixed order: the token's codes from the cache once more, into the accumulator of each head.
#pragma unroll 1
                    for (int k = 0; k < 4 * kD8Places; ++k) {
                        if ((took_s[g * 4 + k / kD8Places] >> k % kD8Places & 1) == 0) continue;
                        const float* place = places + k * kD8Place;
                        auto weight = [&](int i) { return fast_exp2(place[i] + place[20 + i] - (ref_s[h0 + i] + L::kDrop)); };
                        if (tid < n_live) lsum_s[h0 + tid] += weight(tid) * place[17];
                        __syncwarp();
                        const int at = __float_as_int(place[16]);
                        if (static_cast<uint32_t>(at) >= static_cast<uint32_t>(args.columns) << args.page_shift) continue;       // (checked, not trusted)
                        const int page = __ldg(args.block_table + static_cast<size_t>(b) * args.columns + (at >> args.page_shift));
                        if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(args.n_pages)) continue;        // (zeros)
                        const int token = (page << args.page_shift) | (at & ((1 << args.page_shift) - 1));
                        const uint8_t* row = all.cache.row(token) + key;
                        float codes[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) codes[c] = float2_of_half2(half2_of_e4m3x2(row[c * 128])).x;
#pragma unroll 1
                        for (int i = 0; i < kPer; ++i) {
                            const float w = weight(i);
                            uint32_t o[4];
#pragma unroll
                            for (int c = 0; c < 4; ++c) tmem_ld_x1(col_o + c * L::kCols + i, &o[c]);
                            tmem_ld_wait();
#pragma unroll
                            for (int c = 0; c < 4; ++c) tmem_st_x1(col_o + c * L::kCols + i, __float_as_uint(fmaf(w, codes[c], __uint_as_float(o[c]))));
                        }
                        tmem_st_wait();                        // (the next key reads them)
                    }
                    arrive();                                  // (the places are read by all before they are written over)
                    ok = wait_for_group();
                    if (!ok) break;
                }
                // A head's 512 latents in the order that a thread has them in, latent 128 c + l at 4 l + c: 16 bytes a store, 512 of a warp side by side.
                float4* dst = reinterpret_cast<float4*>(args.part_o + (slot * args.h_pad + head0 + h0) * kDecLat) + key;
#pragma unroll 1
                for (int v0 = 0; v0 < kPer; v0 += 8) {
                    float x[8][4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t o[8], rest[8];
                        tmem_ld_x8(col_o + c * L::kCols + v0, o);
                        if constexpr (L::kSplit) tmem_ld_x8(col_o + c * L::kCols + 16, rest);
                        tmem_ld_wait();
#pragma unroll
                        for (int v = 0; v < 8; ++v) {
                            x[v][c] = __uint_as_float(o[v]);
                            if constexpr (L::kSplit) x[v][c] = fmaf(__uint_as_float(rest[v]), 1.0f / kD8LoScale, x[v][c]);
                        }
                    }
                    if (v0 + 8 == kPer) {                      // the next piece's values may be multiplied while these are stored
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(o_free);
                    }
#pragma unroll
                    for (int v = 0; v < 8; ++v)
                        if (store && v0 + v < n_live) dst[(v0 + v) * (kDecLat / 4)] = make_float4(x[v][0], x[v][1], x[v][2], x[v][3]);
                }
                if (!any_taken && !wait_for_group()) break;
                if (store && tid < n_live) {
                    const float l = ((lsum_s[h0 + tid] + lsum_s[kHeads + h0 + tid]) + lsum_s[2 * kHeads + h0 + tid]) + lsum_s[3 * kHeads + h0 + tid];
                    // (no weight at all: nothing that another piece's reference should be compared with)
                    args.part_ml[slot * args.h_pad + head0 + h0 + tid] = make_float2(l == 0.f ? kDecLowest : ref_s[h0 + tid] + L::kDrop, l);
                }
                ++pieces;
                first = true;
            }
            ++T;
            pos += L::kKeyFirst ? 4 : 5;
            if (pos >= L::kSlabs) pos -= L::kSlabs;
        }
    }
    grid_dependency_wait();          // a CTA without work too: this kernel's completion stands for the one before it
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kScoreWarp) { tc_fence_after_sync(); tmem_dealloc(*tmem_slot, 512); }
}

// The queries as the kernel above takes them: decode_absorb_kernel's product, q_abs[b, i, :] = W_uk[i] q_nope[b, i, :], and the rotated part
// beside it, over the smallest power of two that brings the 576 channels within 448, in two e4m3 parts:
//     rows ((b * h_pad / 16 + i / 16) * 2 + part) * 16 + i % 16 of 640 codes: 512 absorbed, the rotated part twice (for the key's codes and
//     for their rests);   q_scale[b][i] the power of two
//
// Few requests, decode_absorb8_kernel: a CTA has all 512 latents of a head, 128 KB of W_uk, for 16 requests; four groups of four warps have
// 128 latents each, D[128 latents x 16 requests] = W_uk (A) . q^T (B).  A lane has a latent, nothing is padded but columns.
// Many, decode_absorb8_rows_kernel: a CTA has 128 latents of a head for 128 requests, D[128 requests x 128 latents] = q (A) . W_uk^T (B).  A thread
// has a request's row, whose magnitude needs no other lane; the four CTAs of a head are a cluster and tell one another theirs.
// The loops over a row are rolled: a CTA goes through them once, and instructions that are taken in for one use are slow ones.
constexpr int kAbsorb8Threads = 512;
struct DecodeAbsorb8Smem {
    static constexpr int kTile = 16;                             // requests
    static constexpr int kW = 0;                                 // four blocks of 128 latents, two slabs of 64 channels each; later the parts' boxes
    static constexpr int kWBlock = 2 * 128 * 128;
    static constexpr int kQ = kW + 4 * kWBlock;                  // two slabs of kTile rows
    static constexpr int kMax = kQ + 2 * kTile * 128;            // [17][16]: largest magnitudes of 16 warps and of the rotated part; then 1 / scale
    static constexpr int kBar = kMax + 18 * 16 * 4;
    static constexpr int kTotalBytes = kBar + 8 * 8 + 16;
};
static_assert(DecodeAbsorb8Smem::kTotalBytes <= 232448, "shared memory of the absorption");

// A pair of values as codes and the codes of what is left (taken of the value rounded to fp16: 2^-12 of it, where the parts together hold 2^-8).
__device__ __forceinline__ void absorb8_parts(F2 x, float inv, uint32_t& hi, uint32_t& lo) {
    const float2 w = f2_parts(f2_mul(x, f2(inv, inv)));
    const __half2 w16 = __floats2half2_rn(w.x, w.y);
    hi = e4m3x2_of_half2(*reinterpret_cast<const uint32_t*>(&w16));
    const uint32_t held = half2_of_e4m3x2(hi);
    const __half2 rest = __hsub2(w16, *reinterpret_cast<const __half2*>(&held));
    lo = e4m3x2_of_half2(*reinterpret_cast<const uint32_t*>(&rest));
}
__device__ __forceinline__ int absorb8_exponent(float most) { return max(scale_exponent(__float_as_uint(most)), -100); }
// Eight rotated channels c .. of a request (row: its head's first part of the queries' rows), twice: for the key's codes and for their rests.
__device__ __forceinline__ void absorb8_store_rotated(uint4 v, uint8_t* row, int c, float inv) {
    float t[8];
    ln_unpack(v, t);
    uint32_t a[4], b[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) absorb8_parts(f2(t[2 * m], t[2 * m + 1]), inv, a[m], b[m]);
    const uint2 hi = make_uint2(__byte_perm(a[0], a[1], 0x5410), __byte_perm(a[2], a[3], 0x5410)),
                lo = make_uint2(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410));
    uint8_t* dst = row + kC8Lat + c;
    *reinterpret_cast<uint2*>(dst) = hi;
    *reinterpret_cast<uint2*>(dst + kC8Key) = hi;
    *reinterpret_cast<uint2*>(dst + 16 * kC8Row) = lo;
    *reinterpret_cast<uint2*>(dst + 16 * kC8Row + kC8Key) = lo;
}
__device__ __forceinline__ float absorb8_magnitude(uint4 v) {
    float t[8], most = 0.f;
    ln_unpack(v, t);
#pragma unroll
    for (int i = 0; i < 8; i += 2) most = fmax3(most, fabsf(t[i]), fabsf(t[i + 1]));      // (a NaN loses: its code says so by itself)
    return most;
}

__global__ void __launch_bounds__(kAbsorb8Threads, 1)
decode_absorb8_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_out,
                      const __nv_bfloat16* __restrict__ q, int B, int h, int h_pad, uint8_t* __restrict__ rows, float* __restrict__ q_scale,
                      unsigned* status, int status_words) {
    using L = DecodeAbsorb8Smem;
    constexpr int kTile = L::kTile;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);      // [4] a block's weights (the first: and the queries)
    uint64_t* done = full + 4;                                         // [4] its product
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(full + 8);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    float *warp_max = reinterpret_cast<float*>(smem + L::kMax), *inv_s = warp_max + 17 * 16;
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int block = warp >> 2, head = blockIdx.x, b0 = blockIdx.y * kTile;
    // the status slot, before any kernel of the call can write to it (as in decode_absorb_kernel)
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < status_words) {
        status[threadIdx.x] = 0u;
        __threadfence();
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < 8; ++i) mbar_init(&full[i], 1);
        abort_flag->value = 0;
        mbar_fence_init();
        for (int j = 0; j < 4; ++j) {
            mbar_arrive_expect_tx(&full[j], L::kWBlock + (j == 0 ? 2 * kTile * 128 : 0));
            for (int k = 0; k < 2; ++k) {
                if (j == 0) tma_load_2d_chk(status, smem + L::kQ + k * kTile * 128, &tmap_q, full, head * 192 + k * 64, b0);
                tma_load_2d_chk(status, smem + L::kW + j * L::kWBlock + k * 128 * 128, &tmap_w, &full[j], head * 256 + k * 64, j * 128);
            }
        }
    }
    if (warp == 1) { tmem_alloc(tmem_slot, 64); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    if (warp == 0) {
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_bf16(128, kTile, 0, 0);
            const uint64_t dq = desc_k_major(smem_u32(smem + L::kQ));
            bool ok = true;
            for (int j = 0; j < 4 && ok; ++j) {
                ok = mbar_wait(&full[j], 0, abort_flag, status, 0x90);
                if (!ok) break;
                tc_fence_after_sync();
                const uint64_t dw = desc_k_major(smem_u32(smem + L::kW + j * L::kWBlock));
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    mma_ss(tmem + j * kTile, dw + (kk >> 2) * (128 * 128 / 16) + (kk & 3) * 2, dq + (kk >> 2) * (kTile * 128 / 16) + (kk & 3) * 2, idesc,
                           kk > 0 ? 1u : 0u);
                mma_commit(&done[j]);
            }
            if (!ok)
                for (int j = 0; j < 4; ++j) mbar_wait_quiesce(&full[j], 0);
        }
        __syncwarp();
    }
    const size_t row0 = (head >> 4) * 32 + (head & 15);          // of the request's 2 h_pad rows: the head's first part; the second 16 on
    // the rotated part: eight threads a request, eight channels a thread
    const int r8 = threadIdx.x >> 3, c8 = (threadIdx.x & 7) * 8;
    uint4 turned = make_uint4(0u, 0u, 0u, 0u);
    if (warp < 4) {
        if (r8 < B - b0) turned = *reinterpret_cast<const uint4*>(q + (static_cast<size_t>(b0 + r8) * h + head) * 192 + 128 + c8);
        float most = absorb8_magnitude(turned);
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        if ((threadIdx.x & 7) == 0) warp_max[16 * 16 + r8] = most;
    }
    const bool ok = mbar_wait_warp(&done[block], 0, abort_flag, status, 0x91);
    tc_fence_after_sync();
    uint32_t v[16];
    tmem_ld_x16(tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + block * kTile, v);
    tmem_ld_wait();
    float mags[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) mags[r] = fabsf(__uint_as_float(v[r]));
    const float mine = warp_reduce_each(mags, lane, [](float x, float y) { return fmaxf(x, y); });
    if ((lane & 1) == 0) warp_max[warp * 16 + (lane >> 1)] = mine;
    __syncthreads();
    if (threadIdx.x < 16) {
        const int r = threadIdx.x;
        float most = 0.f;
#pragma unroll
        for (int w = 0; w < 17; ++w) most = fmaxf(most, warp_max[w * 16 + r]);
        const int e = absorb8_exponent(most);
        inv_s[r] = e == 128 ? 0.f : exact_exp2(-e);
        if (b0 + r < B) q_scale[static_cast<size_t>(b0 + r) * h_pad + head] = exact_exp2(e);
    }
    __syncthreads();
    // D is latents x requests, a part's box requests x 128 latents: transposed on the way through shared memory (over the weights, which the
    // MMAs have read); requests past B are clipped by the map.
    uint8_t* box = smem + L::kW + block * 2 * (16 * 128) + (warp & 3) * 32 + lane;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
        const float2 x = make_float2(__uint_as_float(v[r]) * inv_s[r], __uint_as_float(v[r + 1]) * inv_s[r + 1]);
        uint32_t hi, lo;
        absorb8_parts(f2(x.x, x.y), 1.0f, hi, lo);
        uint8_t* at = box + r * 128;
        at[0] = static_cast<uint8_t>(hi);
        at[128] = static_cast<uint8_t>(hi >> 8);
        at[16 * 128] = static_cast<uint8_t>(lo);
        at[16 * 128 + 128] = static_cast<uint8_t>(lo >> 8);
    }
    fence_async_shared();
    if (warp < 4 && r8 < B - b0) absorb8_store_rotated(turned, rows + (static_cast<size_t>(b0 + r8) * 2 * h_pad + row0) * kC8Row, c8, inv_s[r8]);
    if (__syncthreads_and(ok) && threadIdx.x == 0) {
        for (int j = 0; j < 4; ++j)
            for (int part = 0; part < 2; ++part)
                tma_store_2d(&tmap_out, smem + L::kW + (2 * j + part) * (16 * 128), (static_cast<int>(row0) + part * 16) * kC8Row + j * 128, b0);
        tma_store_commit();
        tma_store_wait_all();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) { tc_fence_after_sync(); tmem_dealloc(tmem, 64); }
}

constexpr int kAbsorbRows = 128, kAbsorbRowsThreads = 256;
// kSlabs of the queries in shared memory: both halves of q_nope's channels, three CTAs an SM; or one after the other in one place, four an SM, for
// more CTAs than that.  (250 requests, 64 heads, 512 CTAs: 16.6 us with two, 13.8 with one; 200 requests, 32 heads, 256 CTAs: 8.0, 8.7.)
template <int kSlabs>
struct DecodeAbsorb8RowsSmem {
    static constexpr int kW = 0;                                 // two slabs of 128 rows x 64 channels; later the parts' boxes
    static constexpr int kQ = kW + 2 * 128 * 128;
    static constexpr int kMax = kQ + kSlabs * 128 * 128;         // [2 groups][128], [4 CTAs][128], [128] of the rotated part
    static constexpr int kBar = kMax + 7 * 128 * 4;
    static constexpr int kTotalBytes = kBar + 40;
};
template <int kSlabs>
__global__ void __cluster_dims__(4, 1, 1) __launch_bounds__(kAbsorbRowsThreads)
decode_absorb8_rows_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_out,
                           const __nv_bfloat16* __restrict__ q, int B, int h, int h_pad, uint8_t* __restrict__ rows, float* __restrict__ q_scale,
                           unsigned* status, int status_words) {
    using L = DecodeAbsorb8RowsSmem<kSlabs>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);      // [2] 64 channels of weights and queries
    uint64_t* done = full + 2;                                   // [2] their product
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(full + 4);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    float *group_max = reinterpret_cast<float*>(smem + L::kMax), *cta_max = group_max + 2 * kAbsorbRows, *turned_max = cta_max + 4 * kAbsorbRows;
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_cta_rank()), head = blockIdx.y, b0 = blockIdx.z * kAbsorbRows, c0 = rank * 128;
    const int half = warp >> 2, r = (warp & 3) * 32 + lane;      // this thread's request; its half of the latents
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < status_words) {       // (as in decode_absorb_kernel)
        status[threadIdx.x] = 0u;
        __threadfence();
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4; ++i) mbar_init(&full[i], 1);
        abort_flag->value = 0;
        mbar_fence_init();
        for (int k = 0; k < 2; ++k) {
            mbar_arrive_expect_tx(&full[k], 2 * 128 * 128);
            tma_load_2d_chk(status, smem + L::kW + k * 128 * 128, &tmap_w, &full[k], head * 256 + k * 64, c0);
            if (k < kSlabs) tma_load_2d_chk(status, smem + L::kQ + k * 128 * 128, &tmap_q, &full[k], head * 192 + k * 64, b0);
        }
    }
    if (warp == 1) { tmem_alloc(tmem_slot, 128); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (the peers run: waited for before the first word to them)
    grid_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    if (warp == 0) {
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_bf16(128, 128, 0, 0);
            const uint64_t da = desc_k_major(smem_u32(smem + L::kQ)), db = desc_k_major(smem_u32(smem + L::kW));
            bool ok = true;
#pragma unroll 1
            for (int k = 0; k < 2 && ok; ++k) {
                if (k >= kSlabs) {
                    ok = mbar_wait(done, 0, abort_flag, status, 0x97);
                    if (!ok) break;
                    tma_load_2d_chk(status, smem + L::kQ, &tmap_q, full + 1, head * 192 + 64, b0);
                }
                ok = mbar_wait(&full[k], 0, abort_flag, status, 0x92);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) mma_ss(tmem, da + (k < kSlabs ? k : 0) * (128 * 128 / 16) + kk * 2, db + k * (128 * 128 / 16) + kk * 2, idesc, (k > 0 || kk > 0) ? 1u : 0u);
                mma_commit(&done[k]);
            }
            if (!ok) {
                mbar_wait_quiesce(full, 0);
                mbar_wait_quiesce(full + 1, 0);                  // (without its queries it costs the limit, which is longer than any load)
            }
        }
        __syncwarp();
    }
    // The rotated part of a quarter of the requests, eight threads a request: this CTA's.
    const int r8 = rank * 32 + static_cast<int>(threadIdx.x >> 3), c8 = (threadIdx.x & 7) * 8;
    const bool live8 = b0 + r8 < B;
    uint4 turned = make_uint4(0u, 0u, 0u, 0u);
    if (live8) turned = *reinterpret_cast<const uint4*>(q + (static_cast<size_t>(b0 + r8) * h + head) * 192 + 128 + c8);
    {
        float most = absorb8_magnitude(turned);
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        if ((threadIdx.x & 7) == 0) turned_max[r8] = most;
    }
    const bool ok = mbar_wait_warp(done + 1, 0, abort_flag, status, 0x93);
    tc_fence_after_sync();
    const uint32_t column = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + half * 64;
    float most = 0.f;
    uint32_t v[32];
#pragma unroll 1
    for (int c = 0; c < 64; c += 32) {
        tmem_ld_x32(column + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; i += 2) most = fmax3(most, fabsf(__uint_as_float(v[i])), fabsf(__uint_as_float(v[i + 1])));
    }
    group_max[half * kAbsorbRows + r] = most;
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (half == 0) {
        most = fmaxf(most, group_max[kAbsorbRows + r]);
        if (r >> 5 == rank) most = fmaxf(most, turned_max[r]);
#pragma unroll
        for (uint32_t peer = 0; peer < 4; ++peer)
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_map(cta_max + rank * kAbsorbRows + r, peer)), "f"(most) : "memory");
    }
    cluster_sync();
    auto exponent = [&](int i) {
        return absorb8_exponent(fmaxf(fmaxf(cta_max[i], cta_max[kAbsorbRows + i]), fmaxf(cta_max[2 * kAbsorbRows + i], cta_max[3 * kAbsorbRows + i])));
    };
    const int e = exponent(r);
    const float inv = e == 128 ? 0.f : exact_exp2(-e);
    if (rank == 0 && half == 0 && b0 + r < B) q_scale[static_cast<size_t>(b0 + r) * h_pad + head] = exact_exp2(e);
    // The two parts' boxes of 128 requests x 128 codes over the weights, which the MMAs have read (each thread has seen that above), and from there
    // whole rows by TMA: a lane that stored its own row would touch 32 lines an instruction.  Requests past B are clipped by the map.
    uint8_t* line = smem + L::kW + r * 128;                      // + part * 16 KB; 16-byte chunk c at c ^ (r & 7)
#pragma unroll 1
    for (int k = 0; k < 4; ++k) {
        tmem_ld_x16(column + 16 * k, v);
        tmem_ld_wait();
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[2], b[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) absorb8_parts(f2(__uint_as_float(v[4 * i + 2 * m]), __uint_as_float(v[4 * i + 2 * m + 1])), inv, a[m], b[m]);
            hi[i] = __byte_perm(a[0], a[1], 0x5410);
            lo[i] = __byte_perm(b[0], b[1], 0x5410);
        }
        const int chunk = ((half * 4 + k) ^ (r & 7)) << 4;
        *reinterpret_cast<uint4*>(line + chunk) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(line + 128 * 128 + chunk) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    fence_async_shared();
    const size_t row0 = (head >> 4) * 32 + (head & 15);          // of the request's 2 h_pad rows: the head's first part; the second 16 on
    if (live8) {
        const int e8 = exponent(r8);
        absorb8_store_rotated(turned, rows + (static_cast<size_t>(b0 + r8) * 2 * h_pad + row0) * kC8Row, c8, e8 == 128 ? 0.f : exact_exp2(-e8));
    }
    if (__syncthreads_and(ok) && threadIdx.x == 0) {
        for (int part = 0; part < 2; ++part)
            tma_store_2d(&tmap_out, smem + L::kW + part * (128 * 128), (static_cast<int>(row0) + part * 16) * kC8Row + c0, b0);
        tma_store_commit();
        tma_store_wait_all();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) { tc_fence_after_sync(); tmem_dealloc(tmem, 128); }
}

// Joining the pieces and the value dimension for many requests.  (decode_project_kernel keeps a head's weights and goes through its requests sixteen at a
// time, a chain of loads, sums, stores and MMAs each; two kernels, for the sums and for the product, pass 2 KB a request and head through L2.  250
// requests of 1 to 600 tokens, 64 heads, pages of 64, the call replayed: 68.6 us with the first, 55.5 so; the two were 3.3 better than the first.  Itself, alone, 15.4 us, of which L2
// needs some 8 for 52 MB of pieces; the rest are the weights of the sum, eight steps' latencies, and a launch and W_uv's load, which the call hides.)
// A CTA has a head and up to 128 requests:
//     w_p = 2^(m_p - M) / sum_p 2^(m_p - M) l_p,   o[c] = sum_p w_p o_p[c] as bf16(o) and bf16(o - bf16(o)),   out[v] = sum_c W_uv[c, v] (both parts)[c]
// D[128 requests x 128 values] = the parts (A, K-major) . W_uv (B, MN-major, rows in the pieces' order), 64 latents at a time: sixteen warps sum
// those of all requests, half a warp a request, the next 64 on their way from L2 meanwhile, while the seventeenth multiplies the last.  A
// request of more than kJoinAlone pieces, of which half a warp would make a long chain, is summed by all of them first, into its first piece's place.
constexpr int kJoinWarps = 16, kJoinThreads = 32 * (kJoinWarps + 1), kJoinRows = 128, kJoinSteps = kDecLat / 64, kJoinAlone = 8;
struct Decode8JoinSmem {
    static constexpr int kSlab = 128 * 128;                      // 128 requests x 64 latents; or 2 x (64 latents x 64 values)
    static constexpr int kW = 0;                                 // all of a head's, a slab a step
    static constexpr int kA = kW + kJoinSteps * kSlab;           // two buffers of both parts; later the results' boxes
    static constexpr int kMaxPieces = kDecMaxCtas + kJoinRows;
    static constexpr int kPieces = kA + 4 * kSlab;               // a request's first stretch, how many pieces, where their weights begin
    static constexpr int kWeights = kPieces + kJoinRows * 16;
    static constexpr int kScan = kWeights + kMaxPieces * 4;
    static constexpr int kLong = kScan + 40 * 4;                 // requests of more than kJoinAlone pieces: how many, then which
    static constexpr int kBar = kLong + (1 + kMaxPieces / (kJoinAlone + 1) + 1) * 4;
    static constexpr int kTotalBytes = kBar + (kJoinSteps + 5) * 8 + 16;
    static_assert(kTotalBytes <= 232448 && kBar % 8 == 0 && kPieces % 16 == 0, "shared memory of the join");
};
__global__ void __launch_bounds__(kJoinThreads, 1)
decode8_join_kernel(const __grid_constant__ CUtensorMap tmap_wv, const __grid_constant__ CUtensorMap tmap_out, float* part_o,
                    const float2* part_ml, const int* __restrict__ seq_lens, int columns, int page_shift, int B, int h, int h_pad,
                    int ctas_per_group, int gap, int n_rows, float* __restrict__ lse, unsigned* status) {
    using L = Decode8JoinSmem;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* w_full = reinterpret_cast<uint64_t*>(smem + L::kBar);      // [kJoinSteps]
    uint64_t* a_full = w_full + kJoinSteps;                              // [2] both parts of 64 latents are in buffer i
    uint64_t* a_empty = a_full + 2;                                      // [2] ... have been multiplied
    uint64_t* done = a_empty + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    int4* pieces = reinterpret_cast<int4*>(smem + L::kPieces);
    float* weights = reinterpret_cast<float*>(smem + L::kWeights);
    int *scan = reinterpret_cast<int*>(smem + L::kScan), *long_ones = reinterpret_cast<int*>(smem + L::kLong);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int head = blockIdx.x, b0 = blockIdx.y * n_rows;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kJoinSteps; ++i) mbar_init(&w_full[i], 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&a_full[i], kJoinWarps); mbar_init(&a_empty[i], 1); }
        mbar_init(done, 1);
        abort_flag->value = 0;
        mbar_fence_init();
        for (int k = 0; k < kJoinSteps; ++k) {                   // (weights are an input: nothing to wait for)
            mbar_arrive_expect_tx(&w_full[k], L::kSlab);
            for (int i = 0; i < 2; ++i)
                tma_load_turned_chk(status, smem + L::kW + k * L::kSlab + i * (L::kSlab / 2), &tmap_wv, &w_full[k], head * 256 + i * 64, k * 16);
        }
    }
    if (warp == kJoinWarps) { tmem_alloc(tmem_slot, 128); tmem_relinquish(); }
    // Where the requests lie on the line, from the lengths (an input too).
    auto units_of = [&](int b) { return (decode_clamp(__ldg(seq_lens + b), columns, page_shift) + kD8Unit - 1) / kD8Unit; };
    {
        int sum = 0, before = 0;
        for (int b = threadIdx.x; b < B; b += kJoinThreads) {
            const int n = units_of(b), line = n > 0 ? n + gap : 0;
            sum += line;
            before += b < b0 ? line : 0;
        }
        sum = __reduce_add_sync(0xffffffffu, sum);
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) { scan[warp] = sum; scan[20 + warp] = before; }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    if (warp == 0) {                                             // four requests a lane, then over the lanes
        int sum = lane <= kJoinWarps ? scan[lane] : 0, position = lane <= kJoinWarps ? scan[20 + lane] : 0;
        sum = __reduce_add_sync(0xffffffffu, sum);
        position = __reduce_add_sync(0xffffffffu, position);
        const int per = max(1, (sum + ctas_per_group - 1) / ctas_per_group);
        int n[4], line = 0, count[4], total = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = lane * 4 + i;
            n[i] = r < n_rows && b0 + r < B ? units_of(b0 + r) : 0;
            line += n[i] > 0 ? n[i] + gap : 0;
        }
        auto before_lane = [&](int v) {
            int incl = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += o;
            }
            return incl - v;
        };
        position += before_lane(line);
        int first[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n[i] > 0) position += gap;
            // (the bounds hold anyway, unless the lengths change under the kernel)
            first[i] = min(position / per, ctas_per_group - 1);
            count[i] = n[i] > 0 ? min((position + n[i] - 1) / per, ctas_per_group - 1) - first[i] + 1 : 0;
            position += n[i];
            total += count[i];
        }
        int base = before_lane(total), n_long = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            count[i] = max(0, min(count[i], L::kMaxPieces - base));
            pieces[lane * 4 + i] = make_int4(first[i], count[i], base, 0);
            base += count[i];
            const uint32_t many = __ballot_sync(0xffffffffu, count[i] > kJoinAlone);
            if (count[i] > kJoinAlone) long_ones[1 + n_long + __popc(many & ((1u << lane) - 1u))] = lane * 4 + i;
            n_long += __popc(many);
        }
        if (lane == 0) long_ones[0] = n_long;
    }
    __syncthreads();
    grid_dependency_wait();
    bool ok = true;
    if (warp == kJoinWarps) {
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_bf16(128, 128, 0, 1);
            for (int k = 0; k < kJoinSteps; ++k) {
                const int buf = k & 1;
                ok = mbar_wait(&w_full[k], 0, abort_flag, status, 0x94);
                if (ok) ok = mbar_wait(&a_full[buf], (k >> 1) & 1, abort_flag, status, 0x95);
                if (!ok) break;
                tc_fence_after_sync();
                const uint64_t db = desc_mn_major(smem_u32(smem + L::kW + k * L::kSlab), L::kSlab / 2);
                for (int part = 0; part < 2; ++part) {
                    const uint64_t da = desc_k_major(smem_u32(smem + L::kA + (2 * buf + part) * L::kSlab));
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) mma_ss(tmem, da + kk * 2, db + kk * 128, idesc, (k > 0 || part > 0 || kk > 0) ? 1u : 0u);
                }
                mma_commit(&a_empty[buf]);
            }
            mma_commit(done);
            if (!ok) {
                for (int k = 0; k < kJoinSteps; ++k) mbar_wait_quiesce(&w_full[k], 0);
                mbar_wait_quiesce(done, 0);
            }
        }
        __syncwarp();
    } else {
        // ---- weights: four lanes a request, of the eight that this warp sums below ------------------------------
        {
            const int r = (lane >> 3) * (2 * kJoinWarps) + warp * 2 + ((lane >> 2) & 1), q = lane & 3;
            const bool mine = r < n_rows && b0 + r < B;
            const int4 p = mine ? pieces[r] : make_int4(0, 0, 0, 0);
            const float2* ml = part_ml + static_cast<size_t>(p.x + b0 + r) * h_pad + head;
            float M = -INFINITY, l = 0.f;
#pragma unroll 4
            for (int c = q; c < p.y; c += 4) M = fmaxf(M, ml[static_cast<size_t>(c) * h_pad].x);
            M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 1));
            M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 2));
#pragma unroll 4
            for (int c = q; c < p.y; c += 4) {
                const float2 x = ml[static_cast<size_t>(c) * h_pad];
                const float w = fast_exp2(x.x - M);
                weights[p.z + c] = w;
                l = fmaf(w, x.y, l);
            }
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            const float inv = l == 0.f ? 0.f : 1.0f / l;         // (nothing left: every score was -inf; a NaN stays one)
            for (int c = q; c < p.y; c += 4) weights[p.z + c] *= inv;
            if (mine && q == 0 && lse != nullptr)
                lse[static_cast<size_t>(b0 + r) * h + head] = p.y > 0 ? (M + log2f(l)) * 0.6931471805599453f : -INFINITY;
        }
        __syncwarp();
        const size_t step = static_cast<size_t>(h_pad) * (kDecLat / 4);
        auto add = [](float4 x, float w, float4 a) { return make_float4(fmaf(x.x, w, a.x), fmaf(x.y, w, a.y), fmaf(x.z, w, a.z), fmaf(x.w, w, a.w)); };
        const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
        // ---- requests of many pieces: a quarter of the warps every fourth piece, then the four quarters -----------------
        if (const int n_long = long_ones[0]; n_long > 0) {
            auto joiners_meet = []() { asm volatile("bar.sync 1, %0;" ::"n"(kJoinWarps * 32) : "memory"); };
            float4* quarters = reinterpret_cast<float4*>(smem + L::kA);
            const int col = threadIdx.x & 127, part = threadIdx.x >> 7;
            joiners_meet();                                      // (all weights are there)
            for (int i = 0; i < n_long; ++i) {
                const int r = long_ones[1 + i];
                const int4 p = pieces[r];
                float4* o = reinterpret_cast<float4*>(part_o + (static_cast<size_t>(p.x + b0 + r) * h_pad + head) * kDecLat) + col;
                float4 sum = none;
#pragma unroll 8
                for (int c = part; c < p.y; c += 4) sum = add(__ldcs(o + c * step), weights[p.z + c], sum);
                quarters[part * 128 + col] = sum;
                joiners_meet();
                if (part == 0) {
                    *o = add(quarters[384 + col], 1.f, add(quarters[256 + col], 1.f, add(quarters[128 + col], 1.f, sum)));
                    if (col == 0) {
                        pieces[r].y = 1;
                        weights[p.z] = 1.f;
                    }
                }
                joiners_meet();
            }
        }
        // ---- sums: half a warp a request, four latents a lane; the first two pieces' a step ahead ---------------
        constexpr int kMost = kJoinRows / (2 * kJoinWarps);
        const int quad = lane & 15;
        const float4* src[kMost];
        int count[kMost], base[kMost];
        float w0[kMost], w1[kMost];
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const int r = i * (2 * kJoinWarps) + warp * 2 + (lane >> 4);
            const int4 p = r < n_rows && b0 + r < B ? pieces[r] : make_int4(0, 0, 0, 0);
            src[i] = reinterpret_cast<const float4*>(part_o + (static_cast<size_t>(p.x + b0 + r) * h_pad + head) * kDecLat) + quad;
            count[i] = p.y;
            base[i] = p.z;
            w0[i] = p.y > 0 ? weights[p.z] : 0.f;
            w1[i] = p.y > 1 ? weights[p.z + 1] : 0.f;
        }
        float4 x0[kMost], x1[kMost];
        auto fetch = [&](int k) {
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                x0[i] = count[i] > 0 ? __ldcs(src[i] + k * 16) : none;
                x1[i] = count[i] > 1 ? __ldcs(src[i] + step + k * 16) : none;
            }
        };
        fetch(0);
#pragma unroll 1
        for (int k = 0; k < kJoinSteps; ++k) {
            const int buf = k & 1;
            float4 acc[kMost];
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                acc[i] = add(x1[i], w1[i], add(x0[i], w0[i], none));
                for (int c = 2; c < count[i]; ++c) acc[i] = add(__ldcs(src[i] + c * step + k * 16), weights[base[i] + c], acc[i]);
            }
            if (k + 1 < kJoinSteps) fetch(k + 1);
            ok = mbar_wait_warp(&a_empty[buf], ((k >> 1) & 1) ^ 1, abort_flag, status, 0x96);
            if (!ok) break;
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const int r = i * (2 * kJoinWarps) + warp * 2 + (lane >> 4);
                if (r >= n_rows) break;                          // (rows that are nobody's: their results are not stored)
                const uint32_t h0 = pack_bf16x2(acc[i].x, acc[i].y), h1 = pack_bf16x2(acc[i].z, acc[i].w);
                auto rest = [](float a, float b, uint32_t both) { return pack_bf16x2(a - __uint_as_float(both << 16), b - __uint_as_float(both & 0xffff0000u)); };
                uint8_t* at = smem + L::kA + 2 * buf * L::kSlab + r * 128 + (((quad >> 1) ^ (r & 7)) << 4) + (quad & 1) * 8;
                *reinterpret_cast<uint2*>(at) = make_uint2(h0, h1);
                *reinterpret_cast<uint2*>(at + L::kSlab) = make_uint2(rest(acc[i].x, acc[i].y, h0), rest(acc[i].z, acc[i].w, h1));
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(&a_full[buf]);
        }
        if (ok) ok = mbar_wait_warp(done, 0, abort_flag, status, 0x98);
        ok = __all_sync(0xffffffffu, ok && abort_flag->value == 0u);
        tc_fence_after_sync();
        // two boxes of requests x 64 values, over the parts, which have been multiplied
        const int r = (warp & 3) * 32 + lane, c0 = (warp >> 2) * 32;
        uint32_t v[32];
        tmem_ld_x32(tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + c0, v);
        tmem_ld_wait();
        uint8_t* line = smem + L::kA + (c0 >> 6) * L::kSlab + r * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(__uint_as_float(v[8 * i + 2 * j]), __uint_as_float(v[8 * i + 2 * j + 1]));
            *reinterpret_cast<uint4*>(line + (((((c0 & 63) >> 3) + i) ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        fence_async_shared();
    }
    if (__syncthreads_and(ok) && threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) tma_store_2d(&tmap_out, smem + L::kA + i * L::kSlab, head * 128 + i * 64, b0);
        tma_store_commit();
        tma_store_wait_all();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kJoinWarps) { tc_fence_after_sync(); tmem_dealloc(tmem, 128); }
}

}  // namespace laga
