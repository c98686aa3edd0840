// Attention of one new token per request over the paged latent cache in 8 bits (cache8_sm100.cuh has the format): the operator of
// attn_decode_sm100.cuh over rows of 640 codes and a scale s_t, 644 bytes a token where bf16 takes 1152.
//
// The codes are never widened: they go from the cache to shared memory by TMA and from there to the tensor cores (kind::f8f6f4) as
// they are.  What multiplies them is brought to 8 bits instead, in two parts each, which together hold as much as a bf16 number:
//   queries        q_lat / r = hi + lo, both e4m3, with a power of two r per (request, head): off by at most 2^-4 * 2^-4 = 2^-8 of a
//                  channel, half a step of bf16.  The key's 64 channels multiply both the key's codes and their rests.
//   probabilities  p / 2^m = hi + lo likewise.  Up to 32 heads a CTA the parts are columns of one MMA (hi e4m3, lo 32 times the rest
//                  in e4m3); with 64 heads TMEM has no room for those columns, so that lo is a second MMA into the same accumulator,
//                  cannot be scaled, and hi is e5m2, whose range is wide enough for the weights of which lo keeps nothing (2^-7).
// The token's scale belongs to both products: scores are s_t r f (hi + lo) . row_t, and as 2^m p_t c_t = s_t p_t code_t the scale goes
// into the probability, whose exponent it adds to (it is a power of two):
//     y_t = score_t log2(e) + log2 s_t,   P_t = 2^(y_t - m),   O = sum P_t code_t,   l = sum P_t / s_t,   out = O / l
// What e4m3 can hold of P is 2^17, so the reference m is kept near the tile's maximum of y, both ways: where a tile's lies outside (m + 1, m + 8]
// it becomes that maximum less 5 (never more than 2^40 below its highest: what came before is then all that counts, and the
// accumulator must not overflow), and O and l are rescaled.  Weights of 2^-16 of a tile's largest are kept with 32 heads.
//
// Scores are computed the other way round from the bf16 kernel, S^T[128 keys x (hi, lo columns of the heads)] = K (A) . Q^T (B): the long
// operand is read from shared memory once for both parts, a thread has all 16 heads' scores of one key, so no reduction is on
// the way of a tile: instead of the maximum the threads vote whether m still holds (one word a warp).
//   output   O^T[512 latents x heads] (+)= V^T (A, MN-major: the same slabs) . P (B, MN-major: a key's probabilities are 16 bytes of a row)
//
// Work split: the line of 64-key units of all requests in equal stretches, as there; a tile is two units, or one where a piece ends in an
// odd one.  A tile is five slabs of 128 keys x 128 codes around a ring with a barrier per slab: the key's first (only scores read it).
//   warps 0 .. 4g-1  softmax: group w / 4 has heads 16 (w / 4) .., its thread l of warp w % 4 key 32 (w % 4) + l; and the drain
//   then four warps: first queries; value MMAs; score MMAs; TMA producer
#pragma once
#include "attn_decode_sm100.cuh"
#include "cache8_sm100.cuh"

namespace laga {

constexpr int kD8Keys = 128;                 // keys of a tile
constexpr int kD8Unit = kDecKeys;            // keys of a unit of the line
constexpr float kD8Lift = 5.0f;              // a tile's maximum starts at 2^5
constexpr float kD8Low = 1.0f, kD8High = 8.0f;
constexpr float kD8Fall = 40.0f;
constexpr float kD8LoScale = 32.0f;

template <int kHeads>
struct AttnDecode8Smem {
    static constexpr int kGroups = kHeads / 16;
    static constexpr int kSoftWarps = 4 * kGroups;
    static constexpr int kThreads = 32 * (kSoftWarps + 4);
    static constexpr bool kSplit = kHeads <= 32;               // both parts of P as columns
    static constexpr int kCols = kSplit ? 2 * kHeads : kHeads; // TMEM columns of 128 latents of O^T
    static constexpr int kPRow = kSplit ? 2 * kHeads : kHeads; // bytes of a key's row of P
    static constexpr int kPTile = kD8Keys * kPRow;
    static constexpr int kSlabs = kHeads == 16 ? 12 : kHeads == 32 ? 10 : 8;
    static constexpr int kScales = kHeads == 64 ? 2 : 4;       // tiles whose scales are held
    static constexpr int kQSlab = 2 * kHeads * 128;            // 32 rows for every 16 heads, hi then lo, x 128 channels
    static constexpr int kSlab = kD8Keys * 128;
    static constexpr int kQ = 0;
    static constexpr int kP = kQ + 5 * kQSlab;                 // two buffers, or the two parts
    static constexpr int kSlab0 = kP + 2 * kPTile;
    static constexpr int kScale = kSlab0 + kSlabs * kSlab;
    static constexpr int kRef = kScale + kScales * kD8Keys * 4;    // per head: m, query factor, rescaling factor, highest m, tile maximum
    static constexpr int kVote = kRef + 5 * kHeads * 4;            // [2][groups][4 warps]
    static constexpr int kBar = kVote + 2 * kGroups * 16;
    static constexpr int kBars = 2 * kSlabs + 12 + kScales + kGroups;
    static constexpr int kMisc = kBar + kBars * 8;             // TMEM slot, abort flag, start, scan
    static constexpr int kTotalBytes = kMisc + 16 + 4 * (kThreads / 32);
    static_assert(kTotalBytes <= 232448 && kSlab0 % 1024 == 0 && kP % 1024 == 0 && kVote % 16 == 0 && kBar % 8 == 0, "decode kernel's shared memory");
};

struct AttnDecode8Args {
    AttnDecodeArgs d;
    Cache8 cache;
    const float* q_scale;              // [B][h_pad]
};

// Walks the tiles of one CTA's stretch of the line.
struct Decode8Cursor {
    int left, b, t, n, len;            // units left; request; unit within it; its units; its length
    __device__ __forceinline__ void open(const AttnDecodeArgs& a) {
        for (; b < a.B; ++b) {
            len = decode_len(a, b);
            n = (len + kD8Unit - 1) / kD8Unit;
            if (t < n) return;
            t = 0;
        }
        left = 0;                      // the lengths changed under the kernel: stop
    }
    __device__ __forceinline__ Decode8Cursor(const AttnDecodeArgs& a, int left_, int b_, int t_) : left(left_), b(b_), t(t_), n(0), len(0) {
        if (left > 0) open(a);
    }
    __device__ __forceinline__ bool done() const { return left <= 0; }
    __device__ __forceinline__ int units() const { return min(min(2, n - t), left); }
    __device__ __forceinline__ bool ends_piece() const { return t + 2 >= n || left <= 2; }
    __device__ __forceinline__ int valid() const { return min(units() * kD8Unit, len - t * kD8Unit); }
    __device__ __forceinline__ void next(const AttnDecodeArgs& a) {
        const int u = units();
        left -= u;
        t += u;
        if (t >= n && left > 0) { t = 0; ++b; open(a); }
    }
};

// Floats as integers of the same order (NaN above or below everything), and back.
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
    float *factor_s = ref_s + kHeads, *alpha_s = factor_s + kHeads, *peak_s = alpha_s + kHeads;
    int* top_s = reinterpret_cast<int*>(peak_s + kHeads);

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int group = static_cast<int>(blockIdx.x) % args.n_groups;
    const int cta = static_cast<int>(blockIdx.x) / args.n_groups;
    const int head0 = group * kHeads;
    constexpr int kQueryWarp = L::kSoftWarps, kValueWarp = kQueryWarp + 1, kScoreWarp = kQueryWarp + 2, kProducerWarp = kQueryWarp + 3;

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
    if (threadIdx.x < kHeads) top_s[threadIdx.x] = kOrderedLowest;
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

    // ---- the line of units, and where this CTA's stretch begins ---------------------------------------------
    int my_units = 0;
    {
        const int run = (args.B + L::kThreads - 1) / L::kThreads;
        const int b0 = min(args.B, static_cast<int>(threadIdx.x) * run), b1 = min(args.B, b0 + run);
        int sum = 0;
        for (int b = b0; b < b1; ++b) sum += (decode_len(args, b) + kD8Unit - 1) / kD8Unit;
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
            const int n = (decode_len(args, b) + kD8Unit - 1) / kD8Unit;
            if (g0 >= before && g0 < before + n) { *start_b = b; *start_t = g0 - before; }
            before += n;
        }
        __syncthreads();
    }
    const int first_b = *start_b, first_t = *start_t;

    auto fetch_queries = [&](int b) {
        grid_dependency_wait();                              // (returns at once after the first time)
        mbar_arrive_expect_tx(q_full, 5 * L::kQSlab);
        for (int k = 0; k < 5; ++k)
            tma_load_2d_chk(args.status, smem + L::kQ + k * L::kQSlab, &tmap_q, q_full, k * 128, 2 * (b * args.h_pad + head0));
    };

    if (abort_flag->value != 0u || my_units <= 0) {
        // nothing to do (or nothing may be done): fall through to the common exit
    } else if (warp == kProducerWarp) {
        // ---- producer: a lane per box of min(page, 64) keys -------------------------------------------------
        // Lane l also keeps the page of box l of the next 32.
        const uint64_t once = l2_evict_first();
        const int shift = args.page_shift, box_shift = min(shift, 6), box = 1 << box_shift, n_sub = kD8Keys >> box_shift;
        auto page_of = [&](const Decode8Cursor& c, int i) -> int {
            const long long key = static_cast<long long>(i) << box_shift;
            if (key >= c.len) return args.n_pages;                             // beyond the request: never issued
            const int page = __ldg(args.block_table + static_cast<size_t>(c.b) * args.columns + (key >> shift));
            if (page >= 0 && page < args.n_pages) return page;
            atomicCAS(args.status, kStatusOk, kStatusCheck | 0xF2u);           // a bad entry: zeros, and a status
            return args.n_pages;                                               // out of the map's range: TMA fills zeros
        };
        ArmedBarriers armed(bars);
        Decode8Cursor cur(args, my_units, first_b, first_t);
        uint32_t slot = 0, par = 0, pieces = 0, T = 0;
        bool new_piece = true, ok = true;
        int batch = 0, page_cur = 0, page_next = 0;          // first box of the batch; pages of box batch + lane and batch + 32 + lane
        while (!cur.done()) {
            const int first = cur.t << (6 - box_shift);
            if (new_piece) {
                batch = first;
                page_cur = page_of(cur, batch + lane);
                page_next = page_of(cur, batch + 32 + lane);
            }
            if (first - batch >= 32) {
                batch += 32;
                page_cur = page_next;
                page_next = page_of(cur, batch + 32 + lane);
            }
            const int boxes = (cur.valid() + box - 1) >> box_shift;                 // boxes of this tile that hold a key
            const int page = __shfl_sync(0xffffffffu, page_cur, first - batch + (lane & (n_sub - 1)));
            const int row = ((first + lane) << box_shift) & ((1 << shift) - 1);
            const bool there = page < args.n_pages;
            const uint32_t bytes = static_cast<uint32_t>(boxes) << (box_shift + 7);
            const uint32_t scale_bytes = __popc(__ballot_sync(0xffffffffu, lane < boxes && there)) << (box_shift + 2);
            uint64_t* c_bar = &c_full[T % L::kScales];
            float* scales = reinterpret_cast<float*>(smem + L::kScale) + (T % L::kScales) * kD8Keys + (lane << box_shift);
#pragma unroll 1
            for (int s = 0; s < 5; ++s) {                    // the key's slab, then the latent's four
                ok = mbar_wait_warp(&empty[slot], par ^ 1u, abort_flag, args.status, 0x80);
                if (!ok) break;
                if (s == 0 && lane < boxes && !there) {
                    for (int i = 0; i < box; ++i) scales[i] = 1.0f;
                    fence_async_shared();
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_expect_tx(&full[slot], bytes);
                    armed.arm(&full[slot], par);
                    if (s == 0) {
                        mbar_arrive_expect_tx(c_bar, scale_bytes);
                        armed.arm(c_bar, T / L::kScales);
                    }
                }
                __syncwarp();
                if (lane < boxes) {
                    tma_load_codes_chk(args.status, smem + L::kSlab0 + slot * L::kSlab + (lane << (box_shift + 7)), &tmap_codes, &full[slot],
                                       s == 0 ? kC8Lat : (s - 1) * 128, row, page, once);
                    if (s == 0 && there)
                        bulk_load(scales, all.cache.base + page * all.cache.page_bytes() + (static_cast<size_t>(kC8Row) << shift) + row * 4, box * 4, c_bar);
                }
                if (++slot == L::kSlabs) { slot = 0; par ^= 1u; }
            }
            // a piece's queries after its first tile: they wait for the last scores of the piece before (the first are the query warp's)
            if (ok && new_piece) {
                if (lane == 0 && pieces > 0) {
                    ok = mbar_wait(q_empty, (pieces & 1u) ^ 1u, abort_flag, args.status, 0x81);
                    if (ok) fetch_queries(cur.b);
                }
                if (lane == 0 && ok) armed.arm(q_full, pieces);
                ++pieces;
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            new_piece = cur.ends_piece();
            cur.next(args);
            ++T;
        }
        __syncwarp();
        if (lane == 0 && abort_flag->value != 0u) armed.quiesce();
    } else if (warp == kQueryWarp) {
        if (elect_one()) fetch_queries(first_b);             // (a unit of first_b is here, so it is the first request with tokens)
    } else if (warp == kScoreWarp) {
        // ---- issuer of the score MMAs ------------------------------------------------------------------------
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_f8(kE4m3, kE4m3, 128, 2 * kHeads, 0, 0);
            const uint32_t k_lo = desc_lo(desc_k_major(smem_u32(smem + L::kSlab0))), q_lo = desc_lo(desc_k_major(smem_u32(smem + L::kQ))),
                           hi = desc_hi(desc_k_major(0));
            uint32_t slot = 0, par = 0, pieces = 0;
            bool ok = true, new_piece = true;
            Decode8Cursor cur(args, my_units, first_b, first_t);
            for (uint32_t T = 0; !cur.done(); ++T) {
                const uint32_t buf = T & 1u, d = tmem_s + buf * (2 * kHeads);
                if (T >= 2) ok = mbar_wait(&p_full[buf], ((T >> 1) & 1u) ^ 1u, abort_flag, args.status, 0x82);     // the scores of tile T - 2 have been read
                if (ok && new_piece) ok = mbar_wait(q_full, pieces & 1u, abort_flag, args.status, 0x83);
                if (!ok) break;
                new_piece = cur.ends_piece();
                cur.next(args);
#pragma unroll 1
                for (int s = 0; s < 5; ++s) {
                    ok = mbar_wait(&full[slot], par, abort_flag, args.status, 0x84);
                    if (!ok) break;
                    tc_fence_after_sync();
                    mma8_ss_chain4<2, 2>(d, k_lo + slot * (L::kSlab / 16), hi, q_lo + (s == 0 ? 4 : s - 1) * (L::kQSlab / 16), hi, idesc, s > 0 ? 1u : 0u);
                    if (s == 0) mma_commit(&empty[slot]);
                    if (++slot == L::kSlabs) { slot = 0; par ^= 1u; }
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
            Decode8Cursor cur(args, my_units, first_b, first_t);
            for (uint32_t T = 0; !cur.done(); ++T) {
                const uint32_t buf = T & 1u;
                const int k_steps = (cur.valid() + 31) >> 5;
                ok = mbar_wait(&p_full[buf], (T >> 1) & 1u, abort_flag, args.status, 0x85);
                // the first tile of a piece overwrites O^T: the piece before it must have been drained
                if (ok && new_piece && pieces > 0) ok = mbar_wait(o_free, (pieces - 1) & 1u, abort_flag, args.status, 0x86);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t b_lo = p_lo + (L::kSplit ? buf * (L::kPTile / 16) : 0u);
                if (++slot == L::kSlabs) slot = 0;           // the key's slab
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
        const int g = warp >> 2, quarter = warp & 3, key = quarter * 32 + lane, tid = key;      // (thread of the group)
        const int h0 = g * 16;                                 // the group's heads within the CTA's
        const int n_live = max(0, min(16, args.h - head0 - h0));
        const uint32_t live = (1u << n_live) - 1u;
        const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t col_o = tmem_base + lane_addr + (L::kSplit ? g * 32 : g * 16);
        int* vote_s = reinterpret_cast<int*>(smem + L::kVote) + g * 4;
        F2 l2[8];                                              // this key's part of the sums
        uint32_t T = 0, pieces = 0, pos = 0, meetings = 0;     // pos: the tile's first slab
        bool ok = true, first = true;
        auto meet = [&]() -> bool {                            // the group's four warps, and what they wrote to shared memory
            __syncwarp();
            if (lane == 0) mbar_arrive(&group_bar[g]);
            return mbar_wait_warp(&group_bar[g], meetings++ & 1u, abort_flag, args.status, 0x87);
        };
        Decode8Cursor cur(args, my_units, first_b, first_t);
        grid_dependency_wait();
        while (!cur.done()) {
            const uint32_t buf = T & 1u, par = (T >> 1) & 1u;
            const int valid = cur.valid();
            if (first) {
#pragma unroll
                for (int i = 0; i < 8; ++i) l2[i] = f2(0.f, 0.f);
                if (tid < 16) {
                    ref_s[h0 + tid] = peak_s[h0 + tid] = kDecLowest;
                    factor_s[h0 + tid] = __ldg(all.q_scale + static_cast<size_t>(cur.b) * args.h_pad + head0 + h0 + tid) * args.scale_log2;
                }
                if (!meet()) break;
            }
            ok = mbar_wait_warp(&c_full[T % L::kScales], (T / L::kScales) & 1u, abort_flag, args.status, 0x88);
            if (ok) ok = mbar_wait_warp(&s_full[buf], par, abort_flag, args.status, 0x89);
            if (!ok) break;
            tc_fence_after_sync();
            F2 y[8];
            float s = reinterpret_cast<const float*>(smem + L::kScale)[(T % L::kScales) * kD8Keys + key];
            {
                uint32_t raw[32];
                tmem_ld_x32(tmem_s + buf * (2 * kHeads) + g * 32 + lane_addr, raw);
                if (key >= valid) s = 1.0f;
                const uint32_t e = __float_as_uint(s) >> 23 & 0xffu;
                const float ef = static_cast<float>(static_cast<int>(e) - 127);
                tmem_ld_wait();
                const F2 s2 = f2(s, s), e2 = f2(ef, ef);
                const ulonglong2* f = reinterpret_cast<const ulonglong2*>(factor_s + h0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const ulonglong2 f4 = f[i];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int c = 4 * i + 2 * j;
                        const F2 both = f2_add(f2(__uint_as_float(raw[c]), __uint_as_float(raw[c + 1])), f2(__uint_as_float(raw[16 + c]), __uint_as_float(raw[17 + c])));
                        y[2 * i + j] = f2_fma(f2_mul(both, s2), F2{j == 0 ? f4.x : f4.y}, e2);
                    }
                }
            }
            if (key >= valid) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = f2(-INFINITY, -INFINITY);
            }
            // Does the reference hold?  For every head some key must lie above m + 1, and none above m + 8.
            {
                const ulonglong2* m = reinterpret_cast<const ulonglong2*>(ref_s + h0);
                uint32_t above = 0u;
                float most = -INFINITY;
                const F2 minus1 = f2(-1.0f, -1.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const ulonglong2 m4 = m[i];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float2 d = f2_parts(f2_fma(F2{j == 0 ? m4.x : m4.y}, minus1, y[2 * i + j]));
                        above |= (d.x > kD8Low ? 1u : 0u) << (4 * i + 2 * j);
                        above |= (d.y > kD8Low ? 1u : 0u) << (4 * i + 2 * j + 1);
                        if (4 * i + 2 * j < n_live) most = fmaxf(most, d.x);
                        if (4 * i + 2 * j + 1 < n_live) most = fmaxf(most, d.y);
                    }
                }
                above |= (most > kD8High ? 1u : 0u) << 16;
                above = __reduce_or_sync(0xffffffffu, above);
                if (lane == 0) vote_s[buf * (4 * L::kGroups) + quarter] = static_cast<int>(above);
            }
            if (!meet()) break;
            const int4 votes = *reinterpret_cast<const int4*>(vote_s + buf * (4 * L::kGroups));
            const uint32_t vote = static_cast<uint32_t>(votes.x | votes.y | votes.z | votes.w);
            if ((vote & 0x10000u) != 0u || (vote & live) != live) {
                // The heads' maxima over the tile, then the references they ask for.
                int mine = kOrderedLowest;
#pragma unroll
                for (int h = 0; h < 16; ++h) {
                    const float2 v = f2_parts(y[h >> 1]);
                    const int most = __reduce_max_sync(0xffffffffu, ordered((h & 1) ? v.y : v.x));
                    if (lane == h) mine = most;
                }
                if (lane < 16) atomicMax(&top_s[h0 + lane], mine);
                if (!meet()) break;
                if (tid < 16) {
                    const float top = unordered(top_s[h0 + tid]), m = ref_s[h0 + tid], peak = peak_s[h0 + tid];
                    top_s[h0 + tid] = kOrderedLowest;
                    float to = m;
                    if (top > -INFINITY && !(top - m > kD8Low && top - m <= kD8High)) to = fmaxf(top - kD8Lift, peak - kD8Fall);
                    alpha_s[h0 + tid] = to == m ? 1.0f : fast_exp2(m - to);
                    ref_s[h0 + tid] = to;
                    peak_s[h0 + tid] = fmaxf(peak, to);
                }
                if (!meet()) break;
                const float* alpha = alpha_s + h0;
#pragma unroll
                for (int i = 0; i < 8; ++i) l2[i] = f2_mul(l2[i], f2(alpha[2 * i], alpha[2 * i + 1]));
                if (!first) {
                    // O^T is at rest once the values of the tile before have been multiplied; this tile's wait for p_full below
                    ok = mbar_wait_warp(&pv_done[(T - 1) & 1u], ((T - 1) >> 1) & 1u, abort_flag, args.status, 0x8A);
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int c = 0; c < 4 * L::kCols; c += L::kCols) {
#pragma unroll 1
                        for (int part = 0; part < (L::kSplit ? 2 : 1); ++part) {
                            uint32_t o[16];
                            tmem_ld_x16(col_o + c + part * 16, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int v = 0; v < 16; ++v) o[v] = __float_as_uint(__uint_as_float(o[v]) * alpha[v]);
                            tmem_st_x16(col_o + c + part * 16, o);
                        }
                    }
                    tmem_st_wait();
                }
            }
            // Probabilities and their parts
            uint32_t hi[4], lo[4];
            {
                const float inv = __uint_as_float((254u - min(254u, __float_as_uint(s) >> 23 & 0xffu)) << 23);      // 1 / s
                const F2 inv2 = f2(inv, inv), minus1 = f2(-1.0f, -1.0f);
                const ulonglong2* m = reinterpret_cast<const ulonglong2*>(ref_s + h0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const ulonglong2 m4 = m[i];
                    uint32_t a[2], b[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float2 d = f2_parts(f2_fma(F2{j == 0 ? m4.x : m4.y}, minus1, y[2 * i + j]));
                        const float2 p = make_float2(fast_exp2(d.x), fast_exp2(d.y));
                        l2[2 * i + j] = f2_fma(f2(p.x, p.y), inv2, l2[2 * i + j]);
                        const __half2 ph = __floats2half2_rn(p.x, p.y);
                        const uint32_t p16 = *reinterpret_cast<const uint32_t*>(&ph);
                        if constexpr (L::kSplit) {
                            a[j] = e4m3x2_of_half2(p16);
                            const uint32_t h16 = half2_of_e4m3x2(a[j]);
                            const __half2 rest = __hmul2(__hsub2(ph, *reinterpret_cast<const __half2*>(&h16)), __float2half2_rn(kD8LoScale));
                            b[j] = e4m3x2_of_half2(*reinterpret_cast<const uint32_t*>(&rest));
                        } else {
                            a[j] = e5m2x2_of_half2(p16);
                            const uint32_t h16 = half2_of_e5m2x2(a[j]);
                            const __half2 rest = __hsub2(ph, *reinterpret_cast<const __half2*>(&h16));
                            b[j] = e4m3x2_of_half2(*reinterpret_cast<const uint32_t*>(&rest));
                        }
                    }
                    hi[i] = a[0] | (a[1] << 16);
                    lo[i] = b[0] | (b[1] << 16);
                }
            }
            // the buffer's last use has been multiplied
            if (L::kSplit ? T >= 2 : T >= 1) {
                const uint32_t prev = T - (L::kSplit ? 2 : 1);
                ok = mbar_wait_warp(&pv_done[prev & 1u], (prev >> 1) & 1u, abort_flag, args.status, 0x8B);
                if (!ok) break;
            }
            {
                uint8_t* row = smem + L::kP + (L::kSplit ? buf * L::kPTile : 0) + key * L::kPRow;
                const int turn = L::kPRow == 32 ? (key >> 2) & 1 : (key >> 1) & 3;
                const int c_hi = L::kSplit ? 2 * g : g, c_lo = L::kSplit ? 2 * g + 1 : g;
                *reinterpret_cast<uint4*>(row + ((c_hi ^ turn) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4*>(row + (L::kSplit ? 0 : L::kPTile) + ((c_lo ^ turn) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
            if (g == 0 && (valid & 31)) {     // rows of the last 32-key step that no token owns: zero, whatever the page holds (0 * NaN is NaN)
                const int n_zero = 32 - (valid & 31);
                for (int i = tid; i < 4 * 8 * n_zero; i += 128) {                    // 4 slabs x rows x eight 16-byte chunks
                    const int slab = i / (8 * n_zero), r = valid + (i >> 3) % n_zero;
                    uint32_t slot = pos + 1 + slab;
                    if (slot >= L::kSlabs) slot -= L::kSlabs;
                    *reinterpret_cast<uint4*>(smem + L::kSlab0 + slot * L::kSlab + r * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
            fence_async_shared();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[buf]);
            first = false;
            if (cur.ends_piece()) {
                ok = mbar_wait_warp(o_full, pieces & 1u, abort_flag, args.status, 0x8C);
                if (!ok) break;
                tc_fence_after_sync();
                const size_t slot = static_cast<size_t>(cta) + cur.b;
                // (a slot past the workspace would mean that the roles disagree about the pieces)
                const bool store = device_check(slot < static_cast<size_t>(args.ctas_per_group) + args.B, args.status, 0xEB0000u | cta);
                float* dst = args.part_o + (slot * args.h_pad + head0 + h0) * kDecLat + key;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[L::kSplit ? 32 : 16];
                    if constexpr (L::kSplit) tmem_ld_x32(col_o + c * L::kCols, o);
                    else tmem_ld_x16(col_o + c * L::kCols, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        float x = __uint_as_float(o[v]);
                        if constexpr (L::kSplit) x = fmaf(__uint_as_float(o[(16 + v) % (L::kSplit ? 32 : 16)]), 1.0f / kD8LoScale, x);
                        if (store && v < n_live) dst[v * kDecLat + c * 128] = x;
                    }
                }
                // the sums over the 128 keys: within the warp, then the warps one after another (a fixed order)
                float sums = 0.f;
#pragma unroll
                for (int h = 0; h < 16; ++h) {
                    const float2 v = f2_parts(l2[h >> 1]);
                    float x = (h & 1) ? v.y : v.x;
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
                    if (lane == h) sums = x;
                }
#pragma unroll 1
                for (int w = 0; w < 4; ++w) {
                    if (quarter == w && lane < 16) alpha_s[h0 + lane] = (w == 0 ? 0.f : alpha_s[h0 + lane]) + sums;
                    if (ok) ok = meet();
                }
                if (!ok) break;
                if (store && tid < n_live) args.part_ml[slot * args.h_pad + head0 + h0 + tid] = make_float2(ref_s[h0 + tid], alpha_s[h0 + tid]);
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_free);
                ++pieces;
                first = true;
                if (!meet()) break;          // the references have been read
            }
            cur.next(args);
            ++T;
            pos += 5;
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
// A CTA has 128 latents of a head; the four of a head are a cluster and tell one another their largest magnitudes.
template <int kRequests>
struct DecodeAbsorb8Smem {
    static constexpr int kW = 0;                                 // two slabs of 128 rows x 64 channels; later the two parts' boxes
    static constexpr int kQ = kW + 2 * 128 * 128;                // two slabs of kRequests rows
    static constexpr int kMax = kQ + 2 * kRequests * 128;        // [4 warps][kRequests], [kRequests] of the rotated part, [4 CTAs][kRequests]
    static constexpr int kInv = kMax + 9 * kRequests * 4;        // [kRequests] 1 / scale
    static constexpr int kBar = kInv + kRequests * 4;
    static constexpr int kTotalBytes = kBar + 32;
};
template <int kRequests>
__global__ void __cluster_dims__(4, 1, 1) __launch_bounds__(kAbsorbThreads)
decode_absorb8_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_out,
                      const __nv_bfloat16* __restrict__ q, int B, int h, int h_pad, uint8_t* __restrict__ rows, float* __restrict__ q_scale,
                      unsigned* status, int status_words) {
    using L = DecodeAbsorb8Smem<kRequests>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);
    uint64_t* done = full + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(full + 2);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    uint32_t *warp_max = reinterpret_cast<uint32_t*>(smem + L::kMax), *rope_max = warp_max + 4 * kRequests, *cta_max = rope_max + kRequests;
    float* inv_s = reinterpret_cast<float*>(smem + L::kInv);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_cta_rank()), head = blockIdx.y, b0 = blockIdx.z * kRequests, c0 = rank * 128;
    constexpr uint32_t kCols = kRequests < 32 ? 32 : kRequests;
    // the status slot, before any kernel of the call can write to it (as in decode_absorb_kernel)
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < status_words) {
        status[threadIdx.x] = 0u;
        __threadfence();
    }
    if (threadIdx.x == 0) {
        mbar_init(full, 1); mbar_init(done, 1);
        abort_flag->value = 0;
        mbar_fence_init();
    }
    if (warp == 0) { tmem_alloc(tmem_slot, kCols); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (the peers run: waited for before the first word to them)
    grid_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    if (warp == 0) {
        if (elect_one()) {
            mbar_arrive_expect_tx(full, 2 * 128 * 128 + 2 * kRequests * 128);
            for (int k = 0; k < 2; ++k) {
                tma_load_2d_chk(status, smem + L::kW + k * 128 * 128, &tmap_w, full, head * 256 + k * 64, c0);
                tma_load_2d_chk(status, smem + L::kQ + k * kRequests * 128, &tmap_q, full, head * 192 + k * 64, b0);
            }
            if (mbar_wait(full, 0, abort_flag, status, 0x90)) {
                tc_fence_after_sync();
                constexpr uint32_t idesc = make_idesc_bf16(128, kRequests, 0, 0);
                const uint64_t da = desc_k_major(smem_u32(smem + L::kW)), db = desc_k_major(smem_u32(smem + L::kQ));
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    mma_ss(tmem, da + (kk >> 2) * (128 * 128 / 16) + (kk & 3) * 2, db + (kk >> 2) * (kRequests * 128 / 16) + (kk & 3) * 2, idesc,
                           kk > 0 ? 1u : 0u);
                mma_commit(done);
            } else {
                mbar_wait_quiesce(full, 0);
            }
        }
        __syncwarp();
    }
    // The rotated part, eight threads a request, eight channels a thread: sixteen requests at a time.
    const int j = threadIdx.x & 7;
    auto rotated = [&](int r) {
        return r < B - b0 ? *reinterpret_cast<const uint4*>(q + (static_cast<size_t>(b0 + r) * h + head) * 192 + 128 + j * 8) : make_uint4(0u, 0u, 0u, 0u);
    };
#pragma unroll
    for (int r0 = 0; r0 < kRequests; r0 += 16) {
        const int r = r0 + static_cast<int>(threadIdx.x >> 3);
        const uint4 v = rotated(r);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t most = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) most = max(most, max((w[k] << 16) & 0x7fffffffu, w[k] & 0x7fff0000u));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
        if (j == 0) rope_max[r] = most;
    }
    const bool ok = mbar_wait_warp(done, 0, abort_flag, status, 0x91);
    tc_fence_after_sync();
    const uint32_t column = tmem + (static_cast<uint32_t>(warp * 32) << 16);
#pragma unroll 1
    for (int r0 = 0; r0 < kRequests; r0 += 16) {
        uint32_t v[16], mine = 0u;
        tmem_ld_x16(column + r0, v);
        tmem_ld_wait();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const uint32_t most = __reduce_max_sync(0xffffffffu, v[r] & 0x7fffffffu);
            if (lane == r) mine = most;
        }
        if (lane < 16) warp_max[warp * kRequests + r0 + lane] = mine;
    }
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x < kRequests) {
        const int r = threadIdx.x;
        uint32_t most = rope_max[r];
#pragma unroll
        for (int w = 0; w < 4; ++w) most = max(most, warp_max[w * kRequests + r]);
#pragma unroll
        for (uint32_t peer = 0; peer < 4; ++peer)
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(cluster_map(cta_max + rank * kRequests + r, peer)), "r"(most) : "memory");
    }
    cluster_sync();
    if (threadIdx.x < kRequests) {
        const int r = threadIdx.x;
        const uint32_t most = max(max(cta_max[r], cta_max[kRequests + r]), max(cta_max[2 * kRequests + r], cta_max[3 * kRequests + r]));
        const int e = max(scale_exponent(most), -100);
        inv_s[r] = e == 128 ? 0.f : exact_exp2(-e);
        if (rank == 0 && b0 + r < B) q_scale[static_cast<size_t>(b0 + r) * h_pad + head] = exact_exp2(e);
    }
    __syncthreads();
    // D is latents x requests, a part's box requests x 128 latents: transposed on the way through shared memory (over the weights, which the
    // MMAs have read); requests past B are clipped by the map.
    uint8_t* box = smem + L::kW + warp * 32 + lane;
#pragma unroll 1
    for (int r0 = 0; r0 < kRequests; r0 += 16) {
        uint32_t v[16];
        tmem_ld_x16(column + r0, v);
        tmem_ld_wait();
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            const float x = __uint_as_float(v[r]) * inv_s[r0 + r], y = __uint_as_float(v[r + 1]) * inv_s[r0 + r + 1];
            const uint32_t hi = e4m3x2(x, y);
            const float2 held = float2_of_half2(half2_of_e4m3x2(hi));
            const uint32_t lo = e4m3x2(x - held.x, y - held.y);
            uint8_t* at = box + (r0 + r) * 128;
            at[0] = static_cast<uint8_t>(hi);
            at[128] = static_cast<uint8_t>(hi >> 8);
            at[kRequests * 128] = static_cast<uint8_t>(lo);
            at[kRequests * 128 + 128] = static_cast<uint8_t>(lo >> 8);
        }
    }
    fence_async_shared();
    const int row0 = (head >> 4) * 32 + (head & 15);             // of the request's 2 h_pad rows: the head's first part; the second 16 on
    // the rotated part: each CTA of the cluster takes its share of the requests
#pragma unroll
    for (int r0 = 0; r0 < kRequests; r0 += 16) {
        const int r = r0 + static_cast<int>(threadIdx.x >> 3);
        if ((r0 >> 4) % 4 != rank || r >= B - b0) continue;
        const uint4 v = rotated(r);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        const float inv = inv_s[r];
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float x = __uint_as_float(w[k] << 16) * inv, y = __uint_as_float(w[k] & 0xffff0000u) * inv;
            hi[k] = e4m3x2(x, y);
            const float2 held = float2_of_half2(half2_of_e4m3x2(hi[k]));
            lo[k] = e4m3x2(x - held.x, y - held.y);
        }
        uint8_t* dst = rows + (static_cast<size_t>(b0 + r) * 2 * h_pad + row0) * kC8Row + kC8Lat + j * 8;
        const uint2 h2 = make_uint2(hi[0] | (hi[1] << 16), hi[2] | (hi[3] << 16)), l2 = make_uint2(lo[0] | (lo[1] << 16), lo[2] | (lo[3] << 16));
        *reinterpret_cast<uint2*>(dst) = h2;
        *reinterpret_cast<uint2*>(dst + kC8Key) = h2;
        *reinterpret_cast<uint2*>(dst + 16 * kC8Row) = l2;
        *reinterpret_cast<uint2*>(dst + 16 * kC8Row + kC8Key) = l2;
    }
    if (__syncthreads_and(ok) && threadIdx.x == 0) {
        for (int part = 0; part < 2; ++part)
            tma_store_2d(&tmap_out, smem + L::kW + part * kRequests * 128, (row0 + part * 16) * kC8Row + c0, b0);
        tma_store_commit();
        tma_store_wait_all();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) { tc_fence_after_sync(); tmem_dealloc(tmem, kCols); }
}

}  // namespace laga
