// Attention of one new token per request over a paged latent cache, in the absorbed form (Section 3.2): a cached token
// is its latent and the shared rotated key side by side, 576 channels that serve every head, so with
//     q_lat[b,i,:] = ( W_uk[i] q_nope[b,i,:] , q_rope[b,i,:] )
// the scores of request b are s[i,t] = scale * q_lat[b,i,:] . row_t, the latent-space output is
// o_lat[b,i,:] = sum_t softmax_t(s[i,:]) c_t, and W_uv[i] carries it to the value dimension afterwards.  Per cached token
// 1152 bytes are read and 2176 FLOP per head done: with 16 heads 30 FLOP per byte, far on the memory side (the ridge is
// at 260); with 128 heads it is at the ridge.
//
// Work split.  The 64-key tiles of all requests form one line; CTA c of a head group takes the c-th stretch of
// ceil(total / CTAs) tiles, whatever requests it crosses, so ragged batches and one long request alike fill the GPU
// (one CTA per SM, no counter).  Each (CTA, request) piece leaves its unnormalised accumulator, running maximum and sum
// in the workspace at slot c + b -- both only grow along the line and one of them does at every step, so no two pieces share a
// slot -- and decode_project_kernel joins a request's pieces.
//
// Tiles.  kHeads (16, 32 or 64) heads per CTA; more heads are more CTAs over the same keys (L2 serves the second read).
//   scores   S[heads x 64 keys] = Q (A, rows = heads; of the 64 MMA rows only the first kHeads mean anything, the others read
//            whatever shared memory follows and are ignored) . K^T (B, K-major key tile).  Rows 16w .. 16w+15 of an M = 64
//            product lie in lanes 32w .. 32w+15 of TMEM: sixteen heads per softmax warp, read so that all 32 threads
//            have 32 scores each (tmem_ld_16x64)
//   output   O^T[512 latents x heads] (+)= V^T (A, MN-major: the very same key tile) . P^T (B: the softmax's bf16 P in shared memory):
//            the long side is the MMA's M, so few heads waste nothing and O takes 4 * kHeads TMEM columns.  Up to 32 heads a CTA P
//            comes in two parts, bf16(p) and bf16(p - bf16(p)), as further columns that the drain adds up: an MMA of 128 x 32 costs
//            its issue, as one of 128 x 16 does, and of the path's three roundings to bf16 (q W_uk, P, the result) one goes (error against
//            float64 with 16 heads 2.5e-3 -> 2.2e-3; the result's rounding alone is 1.7e-3).  With 64 heads the columns would
//            neither be free (the MMAs bound that case) nor fit TMEM beside the scores.
// The tile is loaded once, in nine 64-channel slabs: the rope slab, which only the scores read, and two halves of four slabs (256
// latents), which go around a ring with a barrier per entry, so that the next tiles' loads are in flight while this
// tile is scored, exponentiated and multiplied.
//
//   warps 0..3  softmax (16 heads per warp), rescaling of O^T when a running maximum moved by more than 2^8, drain
//   warp 7      TMA producer (page table entries are fetched ahead of their use)
//   warp 4      fetches the first queries, beside the producer's way to the first tile (lengths, page table; one request of 511 tokens:
//               the call 14.6 -> 13.7 us); then it is done, and keeps the others off the scheduler of softmax warp 0
//   warps 6, 5  issuers of the score and of the value MMAs: apart, because a lane that has issued MMAs sees no barrier until the tensor
//               pipe has taken them, and neither product's start should wait for the other's
//
// Measured, the whole call (absorption, this kernel, projection): 64 requests of up to 8192 tokens, 16 heads, 302 MB of cache: 60 us, of
// which this kernel's main loop 51 (6.0 TB/s: HBM bounds it), absorption and set-up 4, the last CTA's lag and the projection 5.
// 8 requests of up to 65536 tokens, 128 heads, 440 MB, 0.106 TFLOP: 145 us; in long runs, at the card's power limit, 160 to 170.
// There shared memory bounds it: 74 KB of queries leave two tiles, and a half tile's life (load 1500 clocks, scores 2000, softmax 940,
// values 750) sets 2600 clocks a tile against 1920 of MMAs.  One request of 511 tokens: 13.4 us, three kernels' latencies.
//
// Rows behind a request's last token may hold anything, NaN included: their scores are replaced by -inf, and their
// rows of the tile are zeroed in shared memory before P.V (0 * NaN is NaN).
#pragma once
#include <type_traits>

#include "attn_fwd_sm100.cuh"
#include "sm100_ptx.cuh"

namespace laga {

constexpr int kDecThreads = 256;
constexpr int kDecProducerWarp = 7, kDecScoreWarp = 6, kDecValueWarp = 5, kDecQueryWarp = 4;
constexpr int kDecKeys = 64;
constexpr int kDecMaxCtas = 148;             // CTAs over all head groups (the workspace is sized by it)
constexpr int kDecRow = 576;                 // channels of a cached token
constexpr int kDecLat = 512;
constexpr float kDecLowest = -3.402823466e38f;      // the lowest fp32 number

// Shared memory for kHeads heads per CTA: what the queries and P leave holds the tiles, 3, 2.5 or 2 of them.
template <int kHeads>
struct AttnDecodeSmem {
    static constexpr int kHalves = kHeads == 16 ? 6 : kHeads == 32 ? 5 : 4;      // half tiles in the ring
    static constexpr int kQSlab = kHeads * 128;               // kHeads rows x 64 channels
    static constexpr int kParts = kHeads <= 32 ? 2 : 1;       // P as bf16(p) and bf16(p - bf16(p)), or as bf16(p) alone
    static constexpr int kCols = kParts * kHeads;             // rows of the P tile, and TMEM columns of 128 latents of O^T
    static constexpr int kPTile = kCols * 128;                // kCols rows x 64 keys
    static constexpr int kSlab = kDecKeys * 128;              // 64 keys x 64 channels
    static constexpr int kHalf = 4 * kSlab;                   // 64 keys x 256 latents
    static constexpr int kQ = 0;
    static constexpr int kP = kQ + 9 * kQSlab;                // two buffers
    static constexpr int kRope = kP + 2 * kPTile;             // one slab: it is free again as soon as it has been scored
    static constexpr int kHalf0 = kRope + kSlab;
    static constexpr int kAlpha = kHalf0 + kHalves * kHalf;   // two buffers of kHeads factors, then of a word per warp
    static constexpr int kBar = kAlpha + 2 * kHeads * 4 + 32;
    static constexpr int kTotalBytes = kBar + 48 * 8;
    // the MMA's rows kHeads..63 of the last query slab read up to here
    static_assert(kQ + 8 * kQSlab + 64 * 128 <= kAlpha, "score MMAs read past the operand area");
};
static_assert(AttnDecodeSmem<16>::kTotalBytes <= 232448 && AttnDecodeSmem<32>::kTotalBytes <= 232448 &&
              AttnDecodeSmem<64>::kTotalBytes <= 232448, "decode kernel exceeds the 227 KB of shared memory per CTA");

struct AttnDecodeArgs {
    int B, h, n_groups, ctas_per_group;
    float scale_log2;                  // softmax_scale * log2(e)
    const int* seq_lens;               // [B]
    const int* block_table;            // [B, columns]
    int columns, page_shift, n_pages;
    float* part_o;                     // [slots][h_pad][512], unnormalised
    float2* part_ml;                   // [slots][h_pad]: running maximum (log2 domain), sum
    int h_pad;
    unsigned* status;
};

// Length of a request, held within the table's row whatever the caller's array says (2^30 tokens at most).
__device__ __forceinline__ int decode_clamp(int len, int columns, int page_shift) { return max(0, min(len, columns << page_shift)); }
__device__ __forceinline__ int decode_len(const AttnDecodeArgs& a, int b) {
    const int given = __ldg(a.seq_lens + b), len = decode_clamp(given, a.columns, a.page_shift);
    if (len != given) atomicCAS(a.status, kStatusOk, kStatusCheck | 0xF0u);
    return len;
}

// Walks the pieces (request, tiles) of one CTA's stretch of the line.
struct DecodeCursor {
    int left;          // tiles of the stretch not yet handed out, this one included
    int b;             // request
    int t, n;          // tile within the request; tiles the request has
    int len;
    __device__ __forceinline__ void open(const AttnDecodeArgs& a) {      // the next request with something in it
        for (; b < a.B; ++b) {
            len = decode_len(a, b);
            n = (len + kDecKeys - 1) / kDecKeys;
            if (n > 0) return;
        }
        left = 0;                                                        // the lengths changed under the kernel: stop
    }
    __device__ __forceinline__ DecodeCursor(const AttnDecodeArgs& a, int left_, int b_, int t_) : left(left_), b(b_), t(t_), n(0), len(0) {
        if (left > 0) open(a);
    }
    __device__ __forceinline__ bool done() const { return left <= 0; }
    __device__ __forceinline__ bool ends_piece() const { return t + 1 == n || left == 1; }
    __device__ __forceinline__ int valid() const { return min(kDecKeys, len - t * kDecKeys); }
    __device__ __forceinline__ void next(const AttnDecodeArgs& a) {
        --left;
        if (++t == n && left > 0) { t = 0; ++b; open(a); }
    }
};

template <int kHeads>
__global__ void __launch_bounds__(kDecThreads, 1)
attn_decode_sm100_kernel(const __grid_constant__ CUtensorMap tmap_qabs, const __grid_constant__ CUtensorMap tmap_q,
                         const __grid_constant__ CUtensorMap tmap_rope, const __grid_constant__ CUtensorMap tmap_lat,
                         const AttnDecodeArgs args) {
    using L = AttnDecodeSmem<kHeads>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBar);
    uint64_t* h_full = bars;                          // [kHalves] half tile has landed
    uint64_t* h_empty = h_full + L::kHalves;          // ... has been scored and multiplied
    uint64_t* r_full = h_empty + L::kHalves;          // rope slab
    uint64_t* r_empty = r_full + 1;
    uint64_t* q_full = r_empty + 1;                   // the piece's queries
    uint64_t* q_empty = q_full + 1;
    uint64_t* s_full = q_empty + 1;                    // [2] scores of tile T are in TMEM buffer T & 1
    uint64_t* p_full = s_full + 2;                    // [2] P of tile T is in shared memory, O^T is rescaled
    uint64_t* pv_done = p_full + 2;                   // [2] O^T += V^T P^T of tile T has completed
    uint64_t* a_full = pv_done + 2;                   // [2] rescaling factors of tile T are in shared memory
    uint64_t* o_full = a_full + 2;                    // a piece's accumulator is complete
    uint64_t* o_free = o_full + 1;                    // ... and has been drained
    uint64_t* quiesce_bar = o_free + 1;               // [2] abort path only: the issuers' last commits
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 36);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    int* start_b = reinterpret_cast<int*>(tmem_slot + 2);
    int* start_t = start_b + 1;
    int* scan = start_b + 2;                          // [8] per-warp sums of the tile counts
    static_assert(2 * L::kHalves + 4 + 12 <= 36, "barriers overlap the scalars");
    float* alpha_s = reinterpret_cast<float*>(smem + L::kAlpha);
    int* moved_s = reinterpret_cast<int*>(alpha_s + 2 * kHeads);     // [2 buffers][4 warps]: the tile (+ 1) that wrote it last

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;   // (warp-uniform for the compiler)
    const int group = static_cast<int>(blockIdx.x) % args.n_groups;
    const int cta = static_cast<int>(blockIdx.x) / args.n_groups;
    const int head0 = group * kHeads;

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kHalves; ++i) { mbar_init(&h_full[i], 1); mbar_init(&h_empty[i], 1); }
        mbar_init(r_full, 1); mbar_init(r_empty, 1); mbar_init(q_full, 1); mbar_init(q_empty, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_full[i], 4); mbar_init(&pv_done[i], 1); mbar_init(&a_full[i], kHeads / 16); }
        mbar_init(o_full, 1); mbar_init(o_free, 4); mbar_init(quiesce_bar, 1); mbar_init(quiesce_bar + 1, 1);
        abort_flag->value = (smem_u32(smem) & 1023u) != 0u ? 1u : 0u;
        *start_b = 0; *start_t = 0;
        for (int i = 0; i < 8; ++i) moved_s[i] = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tmap_qabs); tma_prefetch_desc(&tmap_q); tma_prefetch_desc(&tmap_rope); tma_prefetch_desc(&tmap_lat);
    }
    if (warp == kDecScoreWarp) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_launch_dependents();
    // Launched to overlap decode_absorb_kernel, the only kernel of the call before this one, which itself starts after everything
    // earlier on the stream.  Only the absorbed queries (and the status word, which it clears) are its work: lengths, page
    // table and cache are read at once, and only who fetches queries waits for it first.
    // All 512 columns are this CTA's, so they start at column 0: an immediate in every MMA (checked, not trusted).
    constexpr uint32_t tmem_base = 0, tmem_s = 256;
    if (threadIdx.x == 0 && (abort_flag->value != 0u || *tmem_slot != tmem_base)) {
        abort_flag->value = 1u;
        atomicCAS(args.status, kStatusOk, kStatusCheck | 0xD4u);
    }

    // ---- the line of tiles, and where this CTA's stretch begins --------------------------------------------
    int my_tiles = 0;
    {
        const int run = (args.B + kDecThreads - 1) / kDecThreads;
        const int b0 = min(args.B, static_cast<int>(threadIdx.x) * run), b1 = min(args.B, b0 + run);
        int sum = 0;
        for (int b = b0; b < b1; ++b) sum += (decode_len(args, b) + kDecKeys - 1) / kDecKeys;
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
        for (int w = 0; w < kDecThreads / 32; ++w) {
            if (w < warp) before += scan[w];
            total += scan[w];
        }
        const int per = (total + args.ctas_per_group - 1) / args.ctas_per_group;
        const int g0 = cta * per;
        my_tiles = min(per, total - g0);               // may be negative: nothing to do
        for (int b = b0; b < b1; ++b) {
            const int n = (decode_len(args, b) + kDecKeys - 1) / kDecKeys;
            if (g0 >= before && g0 < before + n) { *start_b = b; *start_t = g0 - before; }
            before += n;
        }
        __syncthreads();
    }
    const int first_b = *start_b, first_t = *start_t;

    auto fetch_queries = [&](int b) {
        grid_dependency_wait();                              // (returns at once after the first time)
        mbar_arrive_expect_tx(q_full, 9 * L::kQSlab);
        uint8_t* dst = smem + L::kQ;
        tma_load_2d_chk(args.status, dst, &tmap_q, q_full, 128, b * args.h + head0);          // rope band first
        for (int k = 0; k < 8; ++k)
            tma_load_2d_chk(args.status, dst + (1 + k) * L::kQSlab, &tmap_qabs, q_full, k * 64, b * args.h + head0);
    };

    if (abort_flag->value != 0u || my_tiles <= 0) {
        // nothing to do (or nothing may be done): fall through to the common exit
    } else if (warp == kDecProducerWarp) {
        // ---- producer ------------------------------------------------------------------------------------
        const int n_rows = args.n_pages << args.page_shift;
        const uint64_t once = l2_evict_first();              // (the head groups that share a tile read it at nearly the same time)
        // first cache row of the keys from `key` on, within one page
        auto row_of = [&](const DecodeCursor& c, int key) -> int {
            if (key >= c.len) return n_rows;                                   // beyond the request: never issued
            const int page = __ldg(args.block_table + static_cast<size_t>(c.b) * args.columns + (key >> args.page_shift));
            if (page < 0 || page >= args.n_pages) {                            // a bad entry: zeros, and a status
                atomicCAS(args.status, kStatusOk, kStatusCheck | 0xF1u);
                return n_rows;                                                 // out of the map's range: TMA fills zeros
            }
            return (page << args.page_shift) + (key & ((1 << args.page_shift) - 1));
        };
        auto load_queries = [&](const DecodeCursor& c, uint32_t piece, ArmedBarriers& armed) -> bool {
            if (piece > 0 && !mbar_wait(q_empty, (piece & 1u) ^ 1u, abort_flag, args.status, 0xB0)) return false;
            armed.arm(q_full, piece);
            if (piece > 0) fetch_queries(c.b);               // (the first are the query warp's)
            return true;
        };
        uint32_t slot = 0, par = 0, r_par = 0, pieces = 0;
        bool new_piece = true, ok = true;
        if (args.page_shift >= 6) {
            // A tile lies in one page: three copies, by one lane.  A 3-d view of the cache (64 channels, rows, nine channel groups)
            // lets one copy fill four slabs; what limits this warp is its instruction count, as it does the MMA lanes'.
            if (elect_one()) {
                ArmedBarriers armed(bars);
                DecodeCursor cur(args, my_tiles, first_b, first_t);
                int row = row_of(cur, cur.t * kDecKeys);
                while (!cur.done()) {
                    DecodeCursor next = cur;
                    next.next(args);
                    const int next_row = next.done() ? 0 : row_of(next, next.t * kDecKeys);         // a tile ahead
                    if (!mbar_wait(r_empty, r_par ^ 1u, abort_flag, args.status, 0xB1)) break;
                    mbar_arrive_expect_tx(r_full, L::kSlab);
                    armed.arm(r_full, r_par);
                    tma_load_3d_chk(args.status, smem + L::kRope, &tmap_rope, r_full, 0, row, 8, once);
                    r_par ^= 1u;
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        ok = mbar_wait(&h_empty[slot], par ^ 1u, abort_flag, args.status, 0xB8);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&h_full[slot], L::kHalf);
                        armed.arm(&h_full[slot], par);
                        tma_load_3d_chk(args.status, smem + L::kHalf0 + slot * L::kHalf, &tmap_lat, &h_full[slot], 0, row, half * 4, once);
                        if (++slot == L::kHalves) { slot = 0; par ^= 1u; }
                    }
                    // a piece's queries after its first tile: they wait for the last scores of the piece before
                    if (ok && new_piece) ok = load_queries(cur, pieces++, armed);
                    if (!ok) break;
                    new_piece = cur.ends_piece();
                    cur = next;
                    row = next_row;
                }
                if (abort_flag->value != 0u) armed.quiesce();
            }
        } else {
            // Pages of 16 or 32 rows: four or two boxes a slab, a box per lane.  Lane l also keeps the page of box l of the next 32.
            ArmedBarriers armed(bars);
            const int n_sub = kDecKeys >> args.page_shift, page = 1 << args.page_shift;
            DecodeCursor cur(args, my_tiles, first_b, first_t);
            int batch = 0, row_cur = 0, row_next = 0;       // first box of the batch; rows of box batch + lane and batch + 32 + lane
            while (!cur.done()) {
                if (new_piece) {
                    batch = cur.t * n_sub;
                    row_cur = row_of(cur, (batch + lane) << args.page_shift);
                    row_next = row_of(cur, (batch + 32 + lane) << args.page_shift);
                }
                if (cur.t * n_sub - batch >= 32) {
                    batch += 32;
                    row_cur = row_next;
                    row_next = row_of(cur, (batch + 32 + lane) << args.page_shift);
                }
                const int boxes = (cur.valid() + page - 1) >> args.page_shift;              // boxes of this tile that hold a key
                const int sub = lane & (n_sub - 1);
                const int row = __shfl_sync(0xffffffffu, row_cur, cur.t * n_sub - batch + sub);
                const uint32_t bytes = static_cast<uint32_t>(boxes) * page * 128;
                if (lane == 0) {
                    ok = mbar_wait(r_empty, r_par ^ 1u, abort_flag, args.status, 0xB1);
                    if (ok) {
                        mbar_arrive_expect_tx(r_full, bytes);
                        armed.arm(r_full, r_par);
                    }
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane < boxes) tma_load_3d_chk(args.status, smem + L::kRope + lane * page * 128, &tmap_rope, r_full, 0, row, 8, once);
                r_par ^= 1u;
                for (int half = 0; half < 2; ++half) {
                    if (lane == 0) {
                        ok = mbar_wait(&h_empty[slot], par ^ 1u, abort_flag, args.status, 0xB8);
                        if (ok) {
                            mbar_arrive_expect_tx(&h_full[slot], 4 * bytes);
                            armed.arm(&h_full[slot], par);
                        }
                    }
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    const int slab = lane / n_sub;                                          // lanes 0 .. 4 n_sub - 1: box `sub` of slab `slab`
                    if (slab < 4 && sub < boxes)
                        tma_load_3d_chk(args.status, smem + L::kHalf0 + slot * L::kHalf + slab * L::kSlab + sub * page * 128, &tmap_rope, &h_full[slot], 0, row,
                                    half * 4 + slab, once);
                    if (++slot == L::kHalves) { slot = 0; par ^= 1u; }
                }
                if (ok && new_piece && lane == 0) ok = load_queries(cur, pieces++, armed);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                new_piece = cur.ends_piece();
                cur.next(args);
            }
            __syncwarp();
            if (lane == 0 && abort_flag->value != 0u) armed.quiesce();
        }
    } else if (warp == kDecQueryWarp) {
        if (elect_one()) fetch_queries(first_b);             // (the first request with tokens at or behind first_b is first_b: a tile of it is here)
    } else if (warp == kDecScoreWarp) {
        // ---- issuer of the score MMAs ----------------------------------------------------------------------
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_bf16(64, kDecKeys, 0, 0);
            const uint32_t q_lo = desc_lo(desc_k_major(smem_u32(smem + L::kQ))), r_lo = desc_lo(desc_k_major(smem_u32(smem + L::kRope))),
                           k_lo = desc_lo(desc_k_major(smem_u32(smem + L::kHalf0))), hi = desc_hi(desc_k_major(0));
            uint32_t slot = 0, h_par = 0, pieces = 0;
            bool ok = true, new_piece = true, early = false;
            DecodeCursor cur(args, my_tiles, first_b, first_t);
            for (uint32_t T = 0; !cur.done(); ++T) {
                const uint32_t buf = T & 1u, par = (T >> 1) & 1u, d = tmem_s + buf * kDecKeys;
                // A barrier probe queues behind the lane's MMAs until the tensor pipe has taken them, so each is made before the
                // MMAs that precede its use: `early` holds this tile's, made before the last MMAs of the tile before.
                if (!early) {
                    if (T >= 2) ok = mbar_wait(&p_full[buf], par ^ 1u, abort_flag, args.status, 0xB2);     // the scores of tile T - 2 have been read
                    if (ok) ok = mbar_wait(r_full, T & 1u, abort_flag, args.status, 0xB4);
                }
                if (ok && new_piece) ok = mbar_wait(q_full, pieces & 1u, abort_flag, args.status, 0xB3);
                if (!ok) break;
                bool here = mbar_test_wait(&h_full[slot], h_par);
                tc_fence_after_sync();
                uint32_t a_lo = q_lo;
                mma_ss_chain4_first(d, a_lo, hi, r_lo, hi, idesc);
                mma_commit(r_empty);
                a_lo += L::kQSlab / 16;
                new_piece = cur.ends_piece();
                cur.next(args);
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    if (!here) ok = mbar_wait(&h_full[slot], h_par, abort_flag, args.status, 0xB5);
                    if (!ok) break;
                    const uint32_t b_lo = k_lo + slot * (L::kHalf / 16);
                    if (++slot == L::kHalves) { slot = 0; h_par ^= 1u; }
                    if (half == 0) here = mbar_test_wait(&h_full[slot], h_par);
                    tc_fence_after_sync();
                    mma_ss_chain8_two_slabs<L::kQSlab / 16, L::kSlab / 16>(d, a_lo, hi, b_lo, hi, idesc);
                    if (half == 1) {
                        const bool taken = T < 1 || mbar_test_wait(&p_full[buf ^ 1u], ((T + 1) >> 1 & 1u) ^ 1u), landed = mbar_test_wait(r_full, (T + 1) & 1u);
                        early = taken && landed;
                    }
                    mma_ss_chain8_two_slabs<L::kQSlab / 16, L::kSlab / 16>(d, a_lo + 2 * L::kQSlab / 16, hi, b_lo + 2 * L::kSlab / 16, hi, idesc);
                    a_lo += 4 * L::kQSlab / 16;
                }
                if (!ok) break;
                mma_commit(&s_full[buf]);
                if (new_piece) { mma_commit(q_empty); ++pieces; }
            }
            if (abort_flag->value != 0u) { mma_commit(quiesce_bar); mbar_wait_quiesce(quiesce_bar, 0); }
        }
    } else if (warp == kDecValueWarp) {
        // ---- issuer of the value MMAs ----------------------------------------------------------------------
        if (elect_one()) {
            constexpr uint32_t idesc = make_idesc_bf16(128, L::kCols, 1, 0);
            const uint32_t v_lo = desc_lo(desc_mn_major(smem_u32(smem + L::kHalf0), L::kSlab)), v_hi = desc_hi(desc_mn_major(0, L::kSlab)),
                           p_lo = desc_lo(desc_k_major(smem_u32(smem + L::kP))), p_hi = desc_hi(desc_k_major(0));
            uint32_t slot = 0, pieces = 0;
            bool ok = true, new_piece = true;
            DecodeCursor cur(args, my_tiles, first_b, first_t);
            for (uint32_t T = 0; !cur.done(); ++T) {
                const uint32_t buf = T & 1u;
                const int k_steps = (cur.valid() + 15) >> 4;
                ok = mbar_wait(&p_full[buf], (T >> 1) & 1u, abort_flag, args.status, 0xB6);
                // the first tile of a piece overwrites O^T: the piece before it must have been drained
                if (ok && new_piece && pieces > 0) ok = mbar_wait(o_free, (pieces - 1) & 1u, abort_flag, args.status, 0xB7);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t b_lo = p_lo + buf * (L::kPTile / 16);
#pragma unroll 1
                for (uint32_t half = 0; half < 2; ++half) {
                    const uint32_t a_lo = v_lo + slot * (L::kHalf / 16), d = tmem_base + half * (2 * L::kCols);
                    if (k_steps == 4) {
                        mma_ss_chain4_mn_k(d, a_lo, v_hi, b_lo, p_hi, idesc, new_piece ? 0u : 1u);
                        mma_ss_chain4_mn_k(d + L::kCols, a_lo + 2 * L::kSlab / 16, v_hi, b_lo, p_hi, idesc, new_piece ? 0u : 1u);
                    } else {
#pragma unroll 1
                        for (int kk = 0; kk < 2 * k_steps; ++kk) {
                            const int u = kk >= k_steps, k = kk - u * k_steps;
                            mma_ss(d + u * L::kCols, desc_of(a_lo + u * (2 * L::kSlab / 16) + k * 128, v_hi), desc_of(b_lo + k * 2, p_hi), idesc,
                                   (!new_piece || k > 0) ? 1u : 0u);
                        }
                    }
                    mma_commit(&h_empty[slot]);
                    if (++slot == L::kHalves) slot = 0;
                }
                mma_commit(&pv_done[buf]);
                new_piece = cur.ends_piece();
                if (new_piece) { mma_commit(o_full); ++pieces; }
                cur.next(args);
            }
            if (abort_flag->value != 0u) { mma_commit(quiesce_bar + 1); mbar_wait_quiesce(quiesce_bar + 1, 0); }
        }
    } else if (warp < 4) {
        // ---- softmax, rescaling, drain -------------------------------------------------------------------
        // Warp w owns heads 16w .. 16w+15 of the group (its sixteen lanes of the M = 64 score tile); thread l holds sixteen
        // scores of head 16w + l/4 and sixteen of head 16w + l/4 + 8, so that a head's row is four neighbouring threads'.
        const bool softmax_warp = warp * 16 < kHeads;
        const int r0 = warp * 16 + (lane >> 2), r1 = r0 + 8;   // heads within the group
        const bool live0 = head0 + r0 < args.h, live1 = head0 + r1 < args.h;
        const uint32_t lane_addr = static_cast<uint32_t>(warp * 32) << 16;
        // running maxima (log2 domain) and this thread's part of the sums; a maximum starts at the lowest number, not at -inf, so
        // that keys whose score is -inf weigh exp2(-inf) = 0 even where there is nothing else yet (-inf - -inf is NaN)
        float m0 = kDecLowest, m1 = kDecLowest, l0 = 0.f, l1 = 0.f;
        uint32_t T = 0, pieces = 0;
        bool ok = true, first = true;
        DecodeCursor cur(args, my_tiles, first_b, first_t);
        while (!cur.done()) {
            const uint32_t buf = T & 1u, par = (T >> 1) & 1u;
            const int valid = cur.valid();
            const int tag = static_cast<int>(T) + 1;
            int4 flags;                                       // per softmax warp: tag if one of its maxima moved in this tile
            if (softmax_warp) {
                ok = mbar_wait_warp(&s_full[buf], par, abort_flag, args.status, 0xC0);
                if (!ok) break;
                tc_fence_after_sync();
                uint32_t sv[32];
                tmem_ld_16x64(tmem_s + buf * kDecKeys + lane_addr, sv);
                tmem_ld_wait();
                if (valid < kDecKeys) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if ((i >> 2) * 8 + (lane & 3) * 2 + (i & 1) >= valid) sv[i] = __float_as_uint(-INFINITY);
                }
                float x0[4], x1[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x0[e] = fmaxf(__uint_as_float(sv[8 * e]), __uint_as_float(sv[8 * e + 1]));
                    x1[e] = fmaxf(__uint_as_float(sv[8 * e + 2]), __uint_as_float(sv[8 * e + 3]));
                    x0[e] = fmax3(x0[e], __uint_as_float(sv[8 * e + 4]), __uint_as_float(sv[8 * e + 5]));
                    x1[e] = fmax3(x1[e], __uint_as_float(sv[8 * e + 6]), __uint_as_float(sv[8 * e + 7]));
                }
                float mx0 = fmaxf(fmax3(x0[0], x0[1], x0[2]), x0[3]), mx1 = fmaxf(fmax3(x1[0], x1[1], x1[2]), x1[3]);
#pragma unroll
                for (int d = 1; d < 4; d <<= 1) {
                    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, d));
                    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, d));
                }
                const float c0 = fmaxf(m0, mx0 * args.scale_log2), c1 = fmaxf(m1, mx1 * args.scale_log2);
                const bool move0 = live0 && (c0 - m0) > 8.0f, move1 = live1 && (c1 - m1) > 8.0f;   // lazy: only when it fell behind by 2^8
                const float n0 = (move0 || first) ? c0 : m0, n1 = (move1 || first) ? c1 : m1;
                if (__any_sync(0xffffffffu, (move0 || move1) && !first)) {
                    const float f0 = move0 ? fast_exp2(m0 - n0) : 1.0f, f1 = move1 ? fast_exp2(m1 - n1) : 1.0f;
                    l0 *= f0; l1 *= f1;
                    if ((lane & 3) == 0) { alpha_s[buf * kHeads + r0] = f0; alpha_s[buf * kHeads + r1] = f1; }
                    if (lane == 0) moved_s[buf * 4 + warp] = tag;
                    __syncwarp();
                }
                m0 = n0; m1 = n1;
                if (lane == 0) mbar_arrive(&a_full[buf]);
                float s0[2] = {0.f, 0.f}, s1[2] = {0.f, 0.f};
                // pk[2j], pk[2j+1]: columns 8j + 2(l%4), +1 of heads r0 and r1; pr: what their rounding left
                uint32_t pk[16], pr[L::kParts == 2 ? 16 : 1];
                auto rest = [](float a, float b, uint32_t both) {
                    return pack_bf16x2(a - __uint_as_float(both << 16), b - __uint_as_float(both & 0xffff0000u));
                };
                // The product is rounded as the maximum's was, not fused with the subtraction: the largest score's exponent is then 0 whatever its
                // size (fused, it is the maximum's rounding: 1e30 where every score is near the lowest number).
                auto exps = [&](int j) {
                    const float a0 = fast_exp2(__fmul_rn(__uint_as_float(sv[4 * j]), args.scale_log2) - n0);
                    const float a1 = fast_exp2(__fmul_rn(__uint_as_float(sv[4 * j + 1]), args.scale_log2) - n0);
                    const float b0 = fast_exp2(__fmul_rn(__uint_as_float(sv[4 * j + 2]), args.scale_log2) - n1);
                    const float b1 = fast_exp2(__fmul_rn(__uint_as_float(sv[4 * j + 3]), args.scale_log2) - n1);
                    s0[j & 1] += a0 + a1;
                    s1[j & 1] += b0 + b1;
                    pk[2 * j] = pack_bf16x2(a0, a1);
                    pk[2 * j + 1] = pack_bf16x2(b0, b1);
                    if constexpr (L::kParts == 2) {
                        pr[2 * j] = rest(a0, a1, pk[2 * j]);
                        pr[2 * j + 1] = rest(b0, b1, pk[2 * j + 1]);
                    }
                };
#pragma unroll
                for (int j = 0; j < 5; ++j) exps(j);
                // the two barriers this tile still needs, asked while there are exponentials to do: P of the tile that used the buffer
                // before has been multiplied; every softmax warp has said whether its maxima moved
                const bool p_free = T < 2 || mbar_test_wait(&pv_done[buf], par ^ 1u), told = mbar_test_wait(&a_full[buf], par);
#pragma unroll
                for (int j = 5; j < 8; ++j) exps(j);
                l0 += s0[0] + s0[1];
                l1 += s1[0] + s1[1];
                if (!__all_sync(0xffffffffu, p_free)) {
                    ok = mbar_wait_warp(&pv_done[buf], par ^ 1u, abort_flag, args.status, 0xC1);
                    if (!ok) break;
                }
                // rows of 128 bytes (64 keys of a head), 16-byte chunks swizzled like every operand tile; blocks: heads 0..7 and 8..15 of the
                // warp, key groups 2j and 2j + 1
                const int prow = warp * 16 + ((lane >> 3) & 1) * 8 + (lane & 7);
                const uint32_t pbase = smem_u32(smem + L::kP + buf * L::kPTile) + prow * 128;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    stmatrix_x4(pbase + (((2 * j + (lane >> 4)) ^ (lane & 7)) << 4), pk[4 * j], pk[4 * j + 1], pk[4 * j + 2], pk[4 * j + 3]);
                if constexpr (L::kParts == 2) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        stmatrix_x4(pbase + kHeads * 128 + (((2 * j + (lane >> 4)) ^ (lane & 7)) << 4), pr[4 * j], pr[4 * j + 1], pr[4 * j + 2],
                                    pr[4 * j + 3]);
                }
                if (!__all_sync(0xffffffffu, told)) {
                    ok = mbar_wait_warp(&a_full[buf], par, abort_flag, args.status, 0xC4);
                    if (!ok) break;
                }
            } else {
                ok = mbar_wait_warp(&a_full[buf], par, abort_flag, args.status, 0xC4);
                if (!ok) break;
                tc_fence_after_sync();
            }
            flags = reinterpret_cast<const int4*>(moved_s)[buf];
            if (flags.x == tag || flags.y == tag || flags.z == tag || flags.w == tag) {
                // O^T is at rest once P.V of the previous tile has completed; this tile's waits for p_full below
                const uint32_t prev = T - 1;
                ok = mbar_wait_warp(&pv_done[prev & 1u], (prev >> 1) & 1u, abort_flag, args.status, 0xC2);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < 4 * L::kCols; c += 16) {
                    const int w = (c % kHeads) >> 4;          // sixteen columns: the heads of softmax warp w
                    if ((w == 0 ? flags.x : w == 1 ? flags.y : w == 2 ? flags.z : flags.w) != tag) continue;
                    uint32_t o[16];
                    tmem_ld_x16(tmem_base + lane_addr + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[v] = __float_as_uint(__uint_as_float(o[v]) * alpha_s[buf * kHeads + c % kHeads + v]);
                    tmem_st_x16(tmem_base + lane_addr + c, o);
                }
                tmem_st_wait();
            }
            if (valid & 15) {             // rows of the last 16-key step that no token owns: zero, whatever the page holds
                const int n_zero = 16 - (valid & 15);
                for (int i = threadIdx.x; i < 8 * 8 * n_zero; i += 128) {       // 8 slabs x rows x eight 16-byte chunks
                    const int slab = i / (8 * n_zero), r = valid + (i >> 3) % n_zero;
                    const uint32_t slot = (2 * T + (slab >> 2)) % L::kHalves;
                    *reinterpret_cast<uint4*>(smem + L::kHalf0 + slot * L::kHalf + (slab & 3) * L::kSlab + r * 128 + (i & 7) * 16) =
                        make_uint4(0u, 0u, 0u, 0u);
                }
            }
            fence_async_shared();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[buf]);
            first = false;
            const bool ends = cur.ends_piece();
            if (ends) {
                ok = mbar_wait_warp(o_full, pieces & 1u, abort_flag, args.status, 0xC3);
                if (!ok) break;
                tc_fence_after_sync();
                const size_t slot = static_cast<size_t>(cta) + cur.b;
                float* dst = args.part_o + (slot * args.h_pad + head0) * kDecLat + warp * 32 + lane;
                // (a slot past the workspace would mean that the roles disagree about the pieces)
                const int n_heads = device_check(slot < static_cast<size_t>(args.ctas_per_group) + args.B, args.status, 0xEA0000u | cta) ? min(kHeads, args.h - head0) : 0;
                // Columns c .. c+31 of TMEM are latents (c / kCols) * 128 + lane of heads c % kHeads ..: a store of a warp is 128 bytes of one
                // head's row.  The accumulator is up to 256 columns and nothing else of the CTA moves meanwhile, so the loop is
                // unrolled (constant offsets) and the next columns are on their way while these are stored.  A step holds all parts
                // of its values: 32 columns, or with 32 heads twice that.
                constexpr int kStep = kHeads == 32 ? 64 : 32;
                uint32_t o[2][kStep];
                auto load = [&](int c, uint32_t* r) {
#pragma unroll
                    for (int k = 0; k < kStep; k += 32) tmem_ld_x32(tmem_base + lane_addr + c + k, r + k);
                };
                load(0, o[0]);
#pragma unroll
                for (int c = 0; c < 4 * L::kCols; c += kStep) {
                    tmem_ld_wait();
                    if (c + kStep < 4 * L::kCols) load(c + kStep, o[(c / kStep + 1) & 1]);
                    const uint32_t* r = o[(c / kStep) & 1];
#pragma unroll
                    for (int v = 0; v < kStep / L::kParts; ++v) {
                        const int head = (c + v) % kHeads, latent = (c + v) / L::kCols * 128;
                        float x = __uint_as_float(r[v]);
                        if constexpr (L::kParts == 2) x += __uint_as_float(r[v + kHeads]);
                        if (head < n_heads) dst[head * kDecLat + latent] = x;
                    }
                }
                if (softmax_warp && n_heads > 0) {
#pragma unroll
                    for (int d = 1; d < 4; d <<= 1) {
                        l0 += __shfl_xor_sync(0xffffffffu, l0, d);
                        l1 += __shfl_xor_sync(0xffffffffu, l1, d);
                    }
                    float2* ml = args.part_ml + slot * args.h_pad + head0;
                    if ((lane & 3) == 0 && live0) ml[r0] = make_float2(m0, l0);
                    if ((lane & 3) == 0 && live1) ml[r1] = make_float2(m1, l1);
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_free);
                ++pieces;
                m0 = m1 = kDecLowest; l0 = l1 = 0.f;
                first = true;
            }
            cur.next(args);
            ++T;
        }
    }
    grid_dependency_wait();          // a CTA without work too: this kernel's completion stands for the one before it
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kDecScoreWarp) { tc_fence_after_sync(); tmem_dealloc(*tmem_slot, 512); }
}

// q_abs[b, i, :] = W_uk[i] q_nope[b, i, :] for a tile of kRequests requests: D[128 latents x requests] = W_uk (A: rows = latents,
// K-major as it lies) . q^T (B: rows = requests), eight MMAs.  The weights are the M side, so a small batch pads
// nothing but the result's columns, and 4 * h CTAs share the read of W_uk.  First kernel of the call: clears the status slot.
// Latency bounds it (one tile load, eight MMAs, one store per CTA): about 3 us of a call with warm weights.  The result leaves through
// shared memory and TMA, whole rows instead of two bytes a thread (64 requests of 8192: the call 61.8 -> 59.9 us).
constexpr int kAbsorbThreads = 128;
template <int kRequests>
struct DecodeAbsorbSmem {
    static constexpr int kW = 0;                                 // two slabs of 128 rows x 64 channels
    static constexpr int kQ = kW + 2 * 128 * 128;                // two slabs of kRequests rows
    static constexpr int kBar = kQ + 2 * kRequests * 128;
    static constexpr int kTotalBytes = kBar + 32;
};
template <int kRequests>
__global__ void __launch_bounds__(kAbsorbThreads)
decode_absorb_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_q,
                     const __grid_constant__ CUtensorMap tmap_out, unsigned* status, int status_words) {
    using L = DecodeAbsorbSmem<kRequests>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);
    uint64_t* done = full + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(full + 2);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int c0 = blockIdx.x * 128, head = blockIdx.y, b0 = blockIdx.z * kRequests;
    constexpr uint32_t kCols = kRequests < 32 ? 32 : kRequests;
    // the status slot, before any kernel of the call can write to it: the attention kernel starts once every CTA has come by the
    // launch signal below, and no wait of this kernel gives up within two seconds
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
    grid_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    if (warp == 0) {
        if (elect_one()) {
            mbar_arrive_expect_tx(full, 2 * 128 * 128 + 2 * kRequests * 128);
            for (int k = 0; k < 2; ++k) {
                tma_load_2d_chk(status, smem + L::kW + k * 128 * 128, &tmap_w, full, head * 256 + k * 64, c0);
                tma_load_2d_chk(status, smem + L::kQ + k * kRequests * 128, &tmap_q, full, head * 192 + k * 64, b0);
            }
            if (mbar_wait(full, 0, abort_flag, status, 0xB9)) {
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
    const bool ok = mbar_wait_warp(done, 0, abort_flag, status, 0xBA);
    if (ok) {
        // D is latents x requests, the output requests x latents: transposed on its way through shared memory (over the weights, which
        // the MMAs have read), in the boxes of 64 latents that TMA stores; requests past B are clipped by the map.
        tc_fence_after_sync();
        const int c = warp * 32 + lane;
        uint8_t* box = smem + L::kW + (c >> 6) * (kRequests * 128) + (c & 7) * 2;
        const int chunk = (c & 63) >> 3;
#pragma unroll
        for (int r0 = 0; r0 < kRequests; r0 += 16) {
            uint32_t v[16];
            tmem_ld_x16(tmem + (static_cast<uint32_t>(warp * 32) << 16) + r0, v);
            tmem_ld_wait();
#pragma unroll
            for (int r = 0; r < 16; ++r)
                *reinterpret_cast<__nv_bfloat16*>(box + (r0 + r) * 128 + ((chunk ^ (r & 7)) << 4)) = __float2bfloat16_rn(__uint_as_float(v[r]));
        }
        fence_async_shared();
    }
    if (__syncthreads_and(ok) && threadIdx.x == 0) {
        for (int k = 0; k < 2; ++k) tma_store_2d(&tmap_out, smem + L::kW + k * kRequests * 128, head * kDecLat + c0 + k * 64, b0);
        tma_store_commit();
        tma_store_wait_all();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) { tc_fence_after_sync(); tmem_dealloc(tmem, kCols); }
}

// Joins the pieces of each (request, head) and carries the result to the value dimension:
//     o[c] = sum_p 2^(m_p - M) o_p[c] / sum_p 2^(m_p - M) l_p,      out[v] = sum_c W_uv[c, v] o[c]
// A CTA keeps one head's W_uv (128 KB) in shared memory and takes tiles of up to 16 requests: D[128 values x 32] = W_uv^T (A, MN-major, 512
// rows of the weights as they lie) . o^T (B).  o is fp32; rounded to bf16 it would cost as much accuracy as the result's own
// rounding, so B holds it in two parts, hi = bf16(o) in rows 0..15 and lo = bf16(o - hi) in rows 16..31 -- columns that the MMA
// computes in the time of sixteen -- and the two halves of D are added.
// The weights' tile is requested before this kernel waits for the attention kernel (nothing in the call writes them).  Half
// a warp per request turns the maxima and sums into weights, so that the loads of the pieces themselves (2 KB each) depend on nothing.
// With few requests a CTA has one tile, all of this is latency, and all warps sum pieces.  With many it is a pipeline: warps 0..15 sum
// this tile's pieces (four requests a thread at once) while warps 16..23 make the next tile's weights, 24..27 write the tile before and
// warp 31 issues MMAs; one barrier per tile.
// A request without tokens has no piece, and one whose every score is -inf has sums of 0: zeros, LSE -inf.
// Few requests: about 4 us, latency; the first pieces are read while their weights are made (one request of 511 tokens: the call 13.7 ->
// 13.4 us).  Many: the sums bound it (2 KB a piece from L2, four loads in flight a thread).  The call, before the
// pipeline -> now: 130 requests of up to 900 tokens, 128 heads, 121 -> 82 us; 250 of up to 60, 64 heads, 80 -> 45; 2048 of 128, 16 heads,
// 202 -> 130.
constexpr int kProjectThreads = 1024;
struct DecodeProjectSmem {
    static constexpr int kW = 0;                                 // two slabs of 512 rows x 64 values
    static constexpr int kWSlab = 512 * 128;
    static constexpr int kO = kW + 2 * kWSlab;                   // two buffers of eight slabs of 32 rows x 64 latents
    static constexpr int kOSlab = 32 * 128;
    static constexpr int kRed = kO + 2 * 8 * kOSlab;             // [8 groups][512] floats
    static constexpr int kWeights = kRed + 8 * 512 * 4;     // two buffers: (weight, sum) per piece, at most one piece per CTA and one more per request
    static constexpr int kMaxPieces = kDecMaxCtas + 20;
    static constexpr int kTable = kWeights + 2 * kMaxPieces * 8;  // three tiles' pieces: 16 int4 each
    static constexpr int kBar = kTable + 3 * 16 * 16;
    static constexpr int kTotalBytes = kBar + 48;
};
static_assert(DecodeProjectSmem::kTotalBytes <= 232448 && DecodeProjectSmem::kBar % 8 == 0, "projection kernel's shared memory");
__global__ void __launch_bounds__(kProjectThreads, 1)
decode_project_kernel(const __grid_constant__ CUtensorMap tmap_wv, const float* __restrict__ part_o, const float2* __restrict__ part_ml,
                      const int* __restrict__ seq_lens, int columns, int page_shift, int B, int h, int h_pad, int ctas_per_group,
                      int tile_requests, __nv_bfloat16* __restrict__ out, float* __restrict__ lse, unsigned* status) {
    using L = DecodeProjectSmem;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);
    uint64_t* done = full + 1;                                   // [2] the MMAs of the tile in buffer i have completed
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(full + 3);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    float* red = reinterpret_cast<float*>(smem + L::kRed);
    int* sums = reinterpret_cast<int*>(red);                     // 64 words, before `red` is needed
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int head = blockIdx.x;
    const int n_tiles = (B + tile_requests - 1) / tile_requests, tiles_each = (n_tiles + gridDim.y - 1) / gridDim.y;
    const int tile0 = blockIdx.y * tiles_each, my_tiles = min(tiles_each, n_tiles - tile0);      // (may be none)
    if (threadIdx.x == 0) {
        mbar_init(full, 1); mbar_init(done, 1); mbar_init(done + 1, 1);
        abort_flag->value = 0;
        mbar_fence_init();
        if (my_tiles > 0) {
            mbar_arrive_expect_tx(full, 2 * L::kWSlab);
            for (int k = 0; k < 4; ++k)                          // slab k / 2, rows 256 (k % 2) ..
                tma_load_2d_chk(status, smem + L::kW + k * (L::kWSlab / 2), &tmap_wv, full, head * 256 + (k >> 1) * 64, (k & 1) * 256);
        }
    }
    if (warp == 0) { __syncwarp(); tmem_alloc(tmem_slot, 64); tmem_relinquish(); }
    // rows of B that no request fills: zero (their columns of D are never read, but nothing uninitialised should be multiplied)
    for (int i = threadIdx.x; i < 2 * 8 * 32 * 8; i += kProjectThreads)
        *reinterpret_cast<uint4*>(smem + L::kO + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    grid_launch_dependents();

    // Where the requests' tiles lie on the line, from the lengths again (an input of the call: nothing to wait for).
    auto tiles_of = [&](int b) { return (decode_clamp(__ldg(seq_lens + b), columns, page_shift) + kDecKeys - 1) / kDecKeys; };
    int per, position;                                           // tiles of a stretch; position on the line of the next tile's first request
    {
        const int b_first = tile0 * tile_requests;
        const int run = (B + kProjectThreads - 1) / kProjectThreads;
        const int s0 = min(B, static_cast<int>(threadIdx.x) * run), s1 = min(B, s0 + run);
        int sum = 0, before = 0;                                 // tiles of this thread's requests, and of those of them before b_first
        for (int b = s0; b < s1; ++b) {
            const int n = tiles_of(b);
            sum += n;
            before += b < b_first ? n : 0;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, d);
            before += __shfl_xor_sync(0xffffffffu, before, d);
        }
        if (lane == 0) { sums[warp] = sum; sums[32 + warp] = before; }
        __syncthreads();
        sum = sums[lane];
        before = sums[32 + lane];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, d);
            before += __shfl_xor_sync(0xffffffffu, before, d);
        }
        per = max(1, (sum + ctas_per_group - 1) / ctas_per_group);
        position = before;
    }
    // The pieces of the tile's request l -- first stretch, how many, where their weights begin -- go to the table of the tile (three, by
    // tile number), one warp's work: warp 28's, two tiles ahead, in the order of the tiles.
    int4* table = reinterpret_cast<int4*>(smem + L::kTable);
    auto locate = [&](int i) {
        const int b = (tile0 + i) * tile_requests + lane;
        const int mine = lane < tile_requests && b < B && i < my_tiles ? tiles_of(b) : 0;
        int incl = mine;
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += v;
        }
        const int begin = position + incl - mine, first = begin / per;
        const int count = mine > 0 ? (begin + mine - 1) / per - first + 1 : 0;
        position += __shfl_sync(0xffffffffu, incl, 15);
        int base = count;
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, base, d);
            if (lane >= d) base += v;
        }
        if (lane < 16) table[i % 3 * 16 + lane] = make_int4(first, count, base - count, 0);
    };
    struct Tile { int b0, n_req; const int4* pieces; };
    auto tile_at = [&](int i) {
        const int b = (tile0 + i) * tile_requests;
        return Tile{b, min(tile_requests, B - b), table + i % 3 * 16};
    };
    // Weights: half a warp per request, warps 16..23.
    auto make_weights = [&](const Tile& t, int buf) {
        if (warp < 16 || warp >= 24) return;
        const int r = (warp - 16) * 2 + (lane >> 4), q = lane & 15;
        const int4 p = t.pieces[r];                              // (first, count, base)
        const int n = r < t.n_req ? p.y : 0;
        float2* weights = reinterpret_cast<float2*>(smem + L::kWeights) + buf * L::kMaxPieces + p.z;
        const float2* src = part_ml + static_cast<size_t>(p.x + t.b0 + r) * h_pad + head;
        float M = -INFINITY, l = 0.f;
#pragma unroll 4
        for (int c = q; c < n; c += 16) {
            const float2 ml = src[static_cast<size_t>(c) * h_pad];
            weights[c] = ml;
            M = fmaxf(M, ml.x);
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
        for (int c = q; c < n; c += 16) {                        // (a lane reads what it wrote)
            const float2 ml = weights[c];
            const float w = fast_exp2(ml.x - M);
            l = fmaf(w, ml.y, l);
            weights[c].x = w;
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        const float inv = l == 0.f ? 0.f : 1.0f / l;             // (nothing left: every score was -inf; a NaN stays one)
        for (int c = q; c < n; c += 16) weights[c].x *= inv;
        if (lse != nullptr && q == 0 && r < t.n_req)
            lse[static_cast<size_t>(t.b0 + r) * h + head] = n > 0 ? (M + log2f(l)) * 0.6931471805599453f : -INFINITY;
    };
    // Sums: groups of 128 threads, four channels a thread, kEach requests a group at once; with fewer requests than groups, the groups
    // that share one take every second, fourth or eighth piece.
    const int group = warp >> 2, cg = threadIdx.x & 127;
    auto store_row = [&](int buf, int r, float4 o) {             // both parts of request r's row, swizzled
        const float x[4] = {o.x, o.y, o.z, o.w};
        float rest[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) rest[e] = x[e] - __bfloat162float(__float2bfloat16_rn(x[e]));
        uint8_t* slab = smem + L::kO + (buf * 8 + (cg >> 4)) * L::kOSlab;      // 16 threads of four channels per slab
        const int chunk = (cg & 15) >> 1, in_chunk = (cg & 1) * 8;
        *reinterpret_cast<uint2*>(slab + r * 128 + ((chunk ^ (r & 7)) << 4) + in_chunk) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
        *reinterpret_cast<uint2*>(slab + (16 + r) * 128 + ((chunk ^ (r & 7)) << 4) + in_chunk) =
            make_uint2(pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3]));
    };
    const size_t step = static_cast<size_t>(h_pad) * (kDecLat / 4);
    auto sum_pieces = [&](auto each, const Tile& t, int buf) {
        constexpr int kEach = decltype(each)::value, kGroups = 16 / kEach, kLogGroups = kEach == 4 ? 2 : 3;
        constexpr bool kFew = kEach == 2;                    // a CTA's only tile: the weights are made here, under the first pieces' loads
        const float2* weights = reinterpret_cast<const float2*>(smem + L::kWeights) + buf * L::kMaxPieces;
        const int log_split = t.n_req == 1 ? kLogGroups : t.n_req == 2 ? kLogGroups - 1 : t.n_req <= kGroups / 2 ? kLogGroups - 2 : 0;
        const int split = 1 << log_split, share = group & (split - 1);
        const float4* o[kEach];
        const float2* w[kEach];
        int n[kEach], most = 0;
        float4 acc[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int r = (group >> log_split) + k * kGroups, at = r & 15;     // (k > 0 only where split is 1)
            const bool in = r < t.n_req && (k == 0 || split == 1);
            const int4 p = t.pieces[at];
            o[k] = reinterpret_cast<const float4*>(part_o + (static_cast<size_t>(p.x + t.b0 + at) * h_pad + head) * kDecLat) + cg;
            w[k] = weights + p.z;
            n[k] = in ? p.y : 0;
            most = max(most, n[k]);
            acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        // two pieces: the first of each request where split is 1, this group's first two of its request otherwise
        float4 ahead[kFew ? kEach : 1];
        if constexpr (kFew) {
            const bool whole = split == 1;
            const int at0 = whole ? 0 : share, at1 = whole ? 0 : share + split;
            const bool has0 = at0 < n[0], has1 = at1 < (whole ? n[1] : n[0]);
            if (has0) ahead[0] = o[0][at0 * step];
            if (has1) ahead[1] = (whole ? o[1] : o[0])[at1 * step];
            make_weights(t, buf);
            __syncthreads();
            const float w0 = has0 ? w[0][at0].x : 0.f, w1 = has1 ? (whole ? w[1] : w[0])[at1].x : 0.f;
            if (has0) acc[0] = make_float4(ahead[0].x * w0, ahead[0].y * w0, ahead[0].z * w0, ahead[0].w * w0);
            if (has1) {
                const float4 x = make_float4(ahead[1].x * w1, ahead[1].y * w1, ahead[1].z * w1, ahead[1].w * w1);
                if (whole) acc[1] = x;
                else acc[0] = make_float4(acc[0].x + x.x, acc[0].y + x.y, acc[0].z + x.z, acc[0].w + x.w);
            }
        }
        if (split == 1) {
#pragma unroll 2
            for (int c = kFew ? 1 : 0; c < most; ++c)
#pragma unroll
                for (int k = 0; k < kEach; ++k)
                    if (c < n[k]) {
                        const float4 x = o[k][c * step];
                        const float wc = w[k][c].x;
                        acc[k].x = fmaf(x.x, wc, acc[k].x); acc[k].y = fmaf(x.y, wc, acc[k].y);
                        acc[k].z = fmaf(x.z, wc, acc[k].z); acc[k].w = fmaf(x.w, wc, acc[k].w);
                    }
        } else {
#pragma unroll 8
            for (int c = share + (kFew ? kEach * split : 0); c < n[0]; c += split) {
                const float4 x = o[0][c * step];
                const float wc = w[0][c].x;
                acc[0].x = fmaf(x.x, wc, acc[0].x); acc[0].y = fmaf(x.y, wc, acc[0].y);
                acc[0].z = fmaf(x.z, wc, acc[0].z); acc[0].w = fmaf(x.w, wc, acc[0].w);
            }
            reinterpret_cast<float4*>(red)[group * 128 + cg] = acc[0];
            asm volatile("bar.sync 1, %0;" ::"n"(kGroups * 128) : "memory");   // the summing warps; none of them ever leaves early
            acc[0] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < split; ++k) {
                const float4 x = reinterpret_cast<const float4*>(red)[(group - share + k) * 128 + cg];
                acc[0].x += x.x; acc[0].y += x.y; acc[0].z += x.z; acc[0].w += x.w;
            }
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int r = (group >> log_split) + k * kGroups;
            if (r < t.n_req && share == 0 && (k == 0 || split == 1)) store_row(buf, r, acc[k]);
        }
    };
    auto write_out = [&](int b0, int n_req, int buf) {           // warps 24..27: D of a tile whose MMAs have completed
        tc_fence_after_sync();
        uint32_t v[32];
        tmem_ld_x32(tmem + buf * 32 + (static_cast<uint32_t>((warp & 3) * 32) << 16), v);
        tmem_ld_wait();
        __nv_bfloat16* dst = out + (static_cast<size_t>(b0) * h + head) * 128 + (warp & 3) * 32 + lane;
        const size_t pitch = static_cast<size_t>(h) * 128;
#pragma unroll
        for (int r = 0; r < 16; ++r, dst += pitch)
            if (r < n_req) *dst = __float2bfloat16_rn(__uint_as_float(v[r]) + __uint_as_float(v[16 + r]));
        tc_fence_before_sync();
    };

    // (No role leaves this loop early: a wait that gave up skips its work and the rest of the launch runs through.)
    const bool pipelined = my_tiles > 1, writer = warp >= 24 && warp < 28;
    if (warp == 28) {
        locate(0);
        locate(1);
    }
    __syncthreads();
    grid_dependency_wait();
    if (my_tiles > 0) {
        if (pipelined) {
            make_weights(tile_at(0), 0);
            __syncthreads();
        }
        for (int i = 0; i < my_tiles; ++i) {
            const int buf = i & 1;
            const Tile t = tile_at(i);
            if (!pipelined) {
                sum_pieces(std::integral_constant<int, 2>{}, t, buf);
            } else {
                if (warp < 16) {
                    // the MMAs that read this buffer two tiles ago have completed
                    const bool free = i < 2 || mbar_wait_warp(&done[buf], ((i >> 1) & 1u) ^ 1u, abort_flag, status, 0xBB);
                    if (free || t.n_req <= 4) sum_pieces(std::integral_constant<int, 4>{}, t, buf);    // (few requests: its barrier wants every summing warp)
                } else {
                    if (i > 0 && writer && mbar_wait_warp(&done[buf ^ 1], ((i - 1) >> 1) & 1u, abort_flag, status, 0xBD))
                        write_out(t.b0 - tile_requests, tile_requests, buf ^ 1);
                    if (i + 1 < my_tiles) make_weights(tile_at(i + 1), buf ^ 1);
                    if (warp == 28) locate(i + 2);
                }
            }
            fence_async_shared();
            tc_fence_before_sync();
            __syncthreads();
            if (warp == 31) {
                if (elect_one()) {
                    if (i > 0 || mbar_wait(full, 0, abort_flag, status, 0xBC)) {
                        tc_fence_after_sync();
                        constexpr uint32_t idesc = make_idesc_bf16(128, 32, 1, 0);
                        const uint32_t a_lo = desc_lo(desc_mn_major(smem_u32(smem + L::kW), L::kWSlab)), a_hi = desc_hi(desc_mn_major(0, L::kWSlab)),
                                       b_lo = desc_lo(desc_k_major(smem_u32(smem + L::kO + buf * 8 * L::kOSlab))), b_hi = desc_hi(desc_k_major(0));
#pragma unroll 1
                        for (uint32_t s = 0; s < 8; ++s)         // 64 latents: four steps of 16 rows of W_uv
                            mma_ss_chain4_mn_k(tmem + buf * 32, a_lo + s * (64 * 128 / 16), a_hi, b_lo + s * (L::kOSlab / 16), b_hi, idesc, s > 0 ? 1u : 0u);
                        mma_commit(&done[buf]);
                    } else {
                        mbar_wait_quiesce(full, 0);
                    }
                }
                __syncwarp();
            }
            if (i + 1 == my_tiles && writer && mbar_wait_warp(&done[buf], (i >> 1) & 1u, abort_flag, status, 0xBE)) write_out(t.b0, t.n_req, buf);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) { tc_fence_after_sync(); tmem_dealloc(tmem, 64); }
}

}  // namespace laga
