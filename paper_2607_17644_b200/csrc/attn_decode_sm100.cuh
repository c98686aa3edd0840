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
// slot -- and decode_combine_kernel joins a request's pieces.
//
// Tiles.  kHeads (16, 32 or 64) heads per CTA; more heads are more CTAs over the same keys (L2 serves the second read).
//   scores   S[heads x 64 keys] = Q (A, rows = heads, of 128 MMA rows only the first kHeads mean anything; the others read
//            whatever shared memory follows and are ignored) . K^T (B, K-major key tile): a head's row sits in one TMEM lane, so
//            the softmax needs no exchange between threads
//   output   O^T[512 latents x heads] (+)= V^T (A, MN-major: the very same key tile) . P^T (B: the softmax's bf16 P in shared memory):
//            the long side is the MMA's M, so few heads waste nothing and O takes 4 * kHeads TMEM columns
// The tile is loaded once, in nine 64-channel slabs: the rope slab (only the scores read it) and four units of two slabs (128
// latents).  Rope slabs and units go around two rings with a barrier per entry, so the next tiles' loads are always in
// flight while this tile is scored, exponentiated and multiplied.
//
//   warps 0..3  softmax (thread = head row), rescaling of O^T when a running maximum moved by more than 2^8, drain
//   warp 4      TMA producer (page table entries are fetched 32 at a time, one batch ahead)
//   warp 5      MMA issuer: takes whatever is ready, P.V first (it frees units), else the next unit's score MMAs
//
// Rows behind a request's last token may hold anything, NaN included: their scores are replaced by -inf, and their
// rows of the tile are zeroed in shared memory before P.V (0 * NaN is NaN).
#pragma once
#include "attn_fwd_sm100.cuh"
#include "sm100_ptx.cuh"

namespace laga {

constexpr int kDecThreads = 192;
constexpr int kDecKeys = 64;
constexpr int kDecMaxCtas = 148;             // CTAs over all head groups (the workspace is sized by it)
constexpr int kDecRow = 576;                 // channels of a cached token
constexpr int kDecLat = 512;

// Shared memory for kHeads heads per CTA.  Shared memory is what limits the loads in flight: 64 heads' queries take 72 KB
// of it, so that variant keeps one P buffer.
template <int kHeads>
struct AttnDecodeSmem {
    static constexpr int kQBufs = kHeads == 16 ? 2 : 1;
    static constexpr int kPBufs = kHeads == 64 ? 1 : 2;
    static constexpr int kRopes = kHeads == 64 ? 2 : kHeads == 32 ? 3 : 4;
    static constexpr int kUnits = kHeads == 64 ? 8 : 9;
    static constexpr int kQSlab = kHeads * 128;               // kHeads rows x 64 channels
    static constexpr int kPTile = kHeads * 128;               // kHeads rows x 64 keys
    static constexpr int kSlab = kDecKeys * 128;              // 64 keys x 64 channels
    static constexpr int kUnit = 2 * kSlab;
    static constexpr int kQ = 0;
    static constexpr int kP = kQ + kQBufs * 9 * kQSlab;
    static constexpr int kRope = kP + kPBufs * kPTile;
    static constexpr int kUnit0 = kRope + kRopes * kSlab;
    static constexpr int kAlpha = kUnit0 + kUnits * kUnit;    // two buffers of kHeads factors, then of a word per warp
    static constexpr int kBar = kAlpha + 2 * kHeads * 4 + 32;
    static constexpr int kTotalBytes = kBar + 64 * 8;
    // the MMA's rows kHeads..127 of the last query slab read up to here
    static_assert(kQ + (kQBufs * 9 - 1) * kQSlab + 128 * 128 <= kAlpha, "score MMAs read past the operand area");
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
    int* tile_start;                   // [B + 1] first tile of each request on the line; written by CTA 0 for the combine
    unsigned* status;
};

__device__ __forceinline__ int decode_len(const AttnDecodeArgs& a, int b) {
    const int len = __ldg(a.seq_lens + b);
    const long long most = static_cast<long long>(a.columns) << a.page_shift;
    if (len < 0 || len > most) {       // never read past the table's row
        atomicCAS(a.status, kStatusOk, kStatusCheck | 0xF0u);
        return len < 0 ? 0 : static_cast<int>(most);
    }
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
                         const __grid_constant__ CUtensorMap tmap_cache, const AttnDecodeArgs args) {
    using L = AttnDecodeSmem<kHeads>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kBar);
    uint64_t* u_full = bars;                          // [kUnits]
    uint64_t* u_empty = u_full + L::kUnits;
    uint64_t* r_full = u_empty + L::kUnits;           // [kRopes]
    uint64_t* r_empty = r_full + L::kRopes;
    uint64_t* q_full = r_empty + L::kRopes;           // [kQBufs]
    uint64_t* q_empty = q_full + L::kQBufs;
    uint64_t* s_full = q_empty + L::kQBufs;           // [2] scores of tile T are in TMEM buffer T & 1
    uint64_t* p_full = s_full + 2;                    // [2] P of tile T is in shared memory, O^T is rescaled
    uint64_t* pv_done = p_full + 2;                   // [2] O^T += V^T P^T of tile T has completed
    uint64_t* a_full = pv_done + 2;                   // [2] rescaling factors of tile T are in shared memory
    uint64_t* o_full = a_full + 2;                    // a piece's accumulator is complete
    uint64_t* o_free = o_full + 1;                    // ... and has been drained
    uint64_t* quiesce_bar = o_free + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 48);
    AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(tmem_slot + 1);
    int* start_b = reinterpret_cast<int*>(tmem_slot + 2);
    int* start_t = start_b + 1;
    int* scan = start_b + 2;                          // [6] per-warp sums of the tile counts
    static_assert(2 * L::kUnits + 2 * L::kRopes + 2 * L::kQBufs + 11 <= 48, "barriers overlap the scalars");
    float* alpha_s = reinterpret_cast<float*>(smem + L::kAlpha);
    volatile int* moved_s = reinterpret_cast<volatile int*>(alpha_s + 2 * kHeads);     // [2 buffers][4 warps]

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = static_cast<int>(blockIdx.x) % args.n_groups;
    const int cta = static_cast<int>(blockIdx.x) / args.n_groups;
    const int head0 = group * kHeads;

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kUnits; ++i) { mbar_init(&u_full[i], 1); mbar_init(&u_empty[i], 1); }
        for (int i = 0; i < L::kRopes; ++i) { mbar_init(&r_full[i], 1); mbar_init(&r_empty[i], 1); }
        for (int i = 0; i < L::kQBufs; ++i) { mbar_init(&q_full[i], 1); mbar_init(&q_empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_full[i], 128); mbar_init(&pv_done[i], 1); mbar_init(&a_full[i], kHeads < 32 ? 32 : kHeads); }
        mbar_init(o_full, 1); mbar_init(o_free, 128); mbar_init(quiesce_bar, 1);
        abort_flag->value = (smem_u32(smem) & 1023u) != 0u ? 1u : 0u;
        *start_b = 0; *start_t = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tmap_qabs); tma_prefetch_desc(&tmap_q); tma_prefetch_desc(&tmap_cache);
    }
    if (warp == 5) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_launch_dependents();
    grid_dependency_wait();          // global memory from here on
    const uint32_t tmem_base = *tmem_slot;
    const uint32_t tmem_s = tmem_base + 256;
    if (threadIdx.x == 0 && abort_flag->value != 0u) atomicCAS(args.status, kStatusOk, kStatusCheck | 0xD4u);

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
        const bool publish = blockIdx.x == 0;
        for (int b = b0; b < b1; ++b) {
            const int n = (decode_len(args, b) + kDecKeys - 1) / kDecKeys;
            if (publish) args.tile_start[b] = before;
            if (g0 >= before && g0 < before + n) { *start_b = b; *start_t = g0 - before; }
            before += n;
        }
        if (publish && threadIdx.x == 0) args.tile_start[args.B] = total;
        __syncthreads();
    }
    const int first_b = *start_b, first_t = *start_t;

    if (abort_flag->value != 0u || my_tiles <= 0) {
        // nothing to do (or nothing may be done): fall through to the common exit
    } else if (warp == 4) {
        // ---- producer ------------------------------------------------------------------------------------
        ArmedBarriers armed(bars);
        uint32_t nu = 0, nr = 0, nq = 0;
        const int sub_shift = args.page_shift < 6 ? args.page_shift : 6;       // a box is one page or a whole tile, if smaller
        const int n_sub = kDecKeys >> sub_shift, sub_rows = 1 << sub_shift;
        const int n_rows = args.n_pages << args.page_shift;
        bool ok = true;
        DecodeCursor cur(args, my_tiles, first_b, first_t);
        bool new_piece = true;
        int batch0 = 0, row_cur = 0, row_next = 0;       // first row of sub-box (batch0 + lane), and of the batch after it
        // first cache row of sub-box s of the request (s counts boxes of sub_rows keys)
        auto sub_row = [&](int b, int len, int s) -> int {
            const int key = s << sub_shift;
            if (key >= len || key < 0) return n_rows;                          // beyond the request: never issued
            const int page = __ldg(args.block_table + static_cast<size_t>(b) * args.columns + (key >> args.page_shift));
            if (page < 0 || page >= args.n_pages) {                            // a bad entry: zeros, and a status
                atomicCAS(args.status, kStatusOk, kStatusCheck | 0xF1u);
                return n_rows;                                                 // out of the map's range: TMA fills zeros
            }
            return (page << args.page_shift) + (key & ((1 << args.page_shift) - 1));
        };
        while (!cur.done()) {
            if (new_piece) {
                const uint32_t qb = nq % L::kQBufs;
                ok = mbar_wait(&q_empty[qb], ((nq / L::kQBufs) & 1u) ^ 1u, abort_flag, args.status, 0xB0);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(&q_full[qb], 9 * L::kQSlab);
                    armed.arm(&q_full[qb], nq / L::kQBufs);
                    uint8_t* dst = smem + L::kQ + qb * 9 * L::kQSlab;
                    tma_load_2d_chk(args.status, dst, &tmap_q, &q_full[qb], 128, cur.b * args.h + head0);          // rope band first
                    for (int c = 0; c < 8; ++c)
                        tma_load_2d_chk(args.status, dst + (1 + c) * L::kQSlab, &tmap_qabs, &q_full[qb], c * 64, cur.b * args.h + head0);
                }
                ++nq;
                batch0 = cur.t * n_sub;
                row_cur = sub_row(cur.b, cur.len, batch0 + lane);
                row_next = sub_row(cur.b, cur.len, batch0 + 32 + lane);
                new_piece = false;
            }
            const int s0 = cur.t * n_sub;
            if (s0 - batch0 >= 32) {
                batch0 += 32;
                row_cur = row_next;
                row_next = sub_row(cur.b, cur.len, batch0 + 32 + lane);
            }
            const int valid = cur.valid();
            const int boxes = (valid + sub_rows - 1) >> sub_shift;              // sub-boxes of this tile that hold a key
            const int row = __shfl_sync(0xffffffffu, row_cur, (s0 - batch0 + lane) & 31);   // lane s: sub-box s of this tile
            const uint32_t box_bytes = static_cast<uint32_t>(boxes) * sub_rows * 128;
#pragma unroll 1
            for (int e = 0; e < 5; ++e) {                                       // the rope slab, then the four units
                uint64_t *full, *empty;
                uint8_t* dst;
                uint32_t phase, slot;
                if (e == 0) {
                    slot = nr % L::kRopes; phase = nr / L::kRopes; ++nr;
                    full = &r_full[slot]; empty = &r_empty[slot]; dst = smem + L::kRope + slot * L::kSlab;
                } else {
                    slot = nu % L::kUnits; phase = nu / L::kUnits; ++nu;
                    full = &u_full[slot]; empty = &u_empty[slot]; dst = smem + L::kUnit0 + slot * L::kUnit;
                }
                ok = mbar_wait(empty, (phase & 1u) ^ 1u, abort_flag, args.status, 0xB1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(full, e == 0 ? box_bytes : 2 * box_bytes);
                    armed.arm(full, phase);
                }
                __syncwarp();
                if (lane < boxes) {
                    uint8_t* at = dst + lane * sub_rows * 128;
                    if (e == 0) {
                        tma_load_2d(at, &tmap_cache, full, kDecLat, row);
                    } else {
                        tma_load_2d(at, &tmap_cache, full, (e - 1) * 128, row);
                        tma_load_2d(at + L::kSlab, &tmap_cache, full, (e - 1) * 128 + 64, row);
                    }
                }
            }
            if (!ok) break;
            new_piece = cur.ends_piece();
            cur.next(args);
        }
        __syncwarp();
        if (lane == 0 && abort_flag->value != 0u) armed.quiesce();
    } else if (warp == 5) {
        // ---- MMA issuer ----------------------------------------------------------------------------------
        if (elect_one()) {
            constexpr uint32_t idesc_qk = make_idesc_bf16(128, kDecKeys, 0, 0);
            constexpr uint32_t idesc_pv = make_idesc_bf16(128, kHeads, 1, 0);
            DecodeCursor qk(args, my_tiles, first_b, first_t), pv = qk;
            uint32_t Tq = 0, Tp = 0;                 // tiles scored / multiplied so far
            uint32_t nu = 0, nr = 0, nq = 0;         // ring entries the score MMAs have taken
            uint32_t pv_unit = 0, pieces = 0;
            int part = 0;                            // of the tile being scored: 0 = rope slab next, 1..4 = unit next
            bool qk_new = true, pv_new = true, ok = true;
            unsigned long long t0 = global_timer_ns();
            uint32_t polls = 0;
            while (!pv.done()) {
                bool progress = false;
                if (Tp < Tq && mbar_try_wait(&p_full[Tp & 1u], (Tp >> 1) & 1u)) {
                    // the first tile of a piece overwrites O^T: the piece before it must have been drained
                    if (pv_new && pieces > 0) {
                        ok = mbar_wait(o_free, (pieces - 1) & 1u, abort_flag, args.status, 0xB3);
                        if (!ok) break;
                    }
                    tc_fence_after_sync();
                    const int k_steps = (pv.valid() + 15) >> 4;
                    const uint32_t sp = smem_u32(smem + L::kP + (Tp % L::kPBufs) * L::kPTile);
                    for (int u = 0; u < 4; ++u) {
                        const uint32_t slot = pv_unit % L::kUnits;
                        ++pv_unit;
                        const uint32_t sv = smem_u32(smem + L::kUnit0 + slot * L::kUnit);
                        for (int kk = 0; kk < k_steps; ++kk)
                            mma_ss(tmem_base + u * kHeads, desc_mn_major(sv + kk * 2048, L::kSlab), desc_k_major(sp + kk * 32), idesc_pv,
                                   (!pv_new || kk > 0) ? 1u : 0u);
                        mma_commit(&u_empty[slot]);
                    }
                    mma_commit(&pv_done[Tp & 1u]);
                    pv_new = pv.ends_piece();
                    if (pv_new) { mma_commit(o_full); ++pieces; }
                    pv.next(args);
                    ++Tp;
                    progress = true;
                } else if (!qk.done() && Tq <= Tp + 1) {     // at most two score tiles: the older one's P has been taken
                    const uint32_t qb = nq % L::kQBufs;
                    if (part == 0) {
                        const uint32_t slot = nr % L::kRopes;
                        if (mbar_try_wait(&r_full[slot], (nr / L::kRopes) & 1u) &&
                            (!qk_new || mbar_try_wait(&q_full[qb], (nq / L::kQBufs) & 1u))) {
                            qk_new = false;
                            tc_fence_after_sync();
                            const uint32_t sq = smem_u32(smem + L::kQ + qb * 9 * L::kQSlab);
                            const uint32_t sk = smem_u32(smem + L::kRope + slot * L::kSlab);
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                mma_ss(tmem_s + (Tq & 1u) * kDecKeys, desc_k_major(sq + kk * 32), desc_k_major(sk + kk * 32), idesc_qk, kk > 0 ? 1u : 0u);
                            mma_commit(&r_empty[slot]);
                            ++nr;
                            part = 1;
                            progress = true;
                        }
                    } else {
                        const uint32_t slot = nu % L::kUnits;
                        if (mbar_try_wait(&u_full[slot], (nu / L::kUnits) & 1u)) {
                            tc_fence_after_sync();
                            const uint32_t sq = smem_u32(smem + L::kQ + qb * 9 * L::kQSlab) + (2 * part - 1) * L::kQSlab;
                            const uint32_t sk = smem_u32(smem + L::kUnit0 + slot * L::kUnit);
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)
                                mma_ss(tmem_s + (Tq & 1u) * kDecKeys, desc_k_major(sq + (kk >> 2) * L::kQSlab + (kk & 3) * 32),
                                       desc_k_major(sk + (kk >> 2) * L::kSlab + (kk & 3) * 32), idesc_qk, 1u);
                            ++nu;
                            progress = true;
                            if (++part == 5) {
                                part = 0;
                                mma_commit(&s_full[Tq & 1u]);
                                qk_new = qk.ends_piece();
                                if (qk_new) { mma_commit(&q_empty[qb]); ++nq; }
                                qk.next(args);
                                ++Tq;
                            }
                        }
                    }
                }
                if (progress) {
                    polls = 0;
                } else if ((++polls & 0xffu) == 0u) {        // bounded, like every wait
                    if (polls == 256u) t0 = global_timer_ns();
                    if (abort_flag->value != 0u) break;
                    if (global_timer_ns() - t0 > kWaitBudgetNs) {
                        abort_flag->value = 1u;
                        atomicCAS(args.status, kStatusOk, kStatusTimeout | 0xB4u);
                        break;
                    }
                }
            }
            if (abort_flag->value != 0u) { mma_commit(quiesce_bar); mbar_wait_quiesce(quiesce_bar, 0); }
        }
    } else {
        // ---- softmax, rescaling, drain -------------------------------------------------------------------
        const int row = warp * 32 + lane;                     // head within the group == TMEM lane
        const bool softmax_warp = warp * 32 < kHeads;
        const bool live = row < kHeads && head0 + row < args.h;
        const uint32_t lane_addr = static_cast<uint32_t>(warp * 32) << 16;
        float m_run = -INFINITY, l_run = 0.f;
        uint32_t T = 0, pieces = 0;
        bool ok = true, first = true;
        DecodeCursor cur(args, my_tiles, first_b, first_t);
        while (!cur.done()) {
            const uint32_t buf = T & 1u, par = (T >> 1) & 1u;
            ok = mbar_wait_warp(&s_full[buf], par, abort_flag, args.status, 0xC0);
            if (!ok) break;
            tc_fence_after_sync();
            const int valid = cur.valid();
            if (softmax_warp) {
                uint32_t sv[kDecKeys];
                tmem_ld_x32(tmem_s + buf * kDecKeys + lane_addr, sv);
                tmem_ld_x32(tmem_s + buf * kDecKeys + lane_addr + 32, sv + 32);
                tmem_ld_wait();
                if (valid < kDecKeys) {
#pragma unroll
                    for (int c = 0; c < kDecKeys; ++c)
                        if (c >= valid) sv[c] = __float_as_uint(-INFINITY);
                }
                float mx = __uint_as_float(sv[0]);
#pragma unroll
                for (int c = 1; c < kDecKeys - 1; c += 2) mx = fmax3(mx, __uint_as_float(sv[c]), __uint_as_float(sv[c + 1]));
                mx = fmaxf(mx, __uint_as_float(sv[kDecKeys - 1]));
                const float m_cand = fmaxf(m_run, mx * args.scale_log2);
                const bool move = live && (m_cand - m_run) > 8.0f;        // lazy rescale: only when it fell behind by 2^8
                const float m_new = (move || first) ? m_cand : m_run;
                const float alpha = move && !first ? fast_exp2(m_run - m_new) : 1.0f;
                m_run = m_new;
                float sums[4] = {0.f, 0.f, 0.f, 0.f};
                uint32_t pk[kDecKeys / 2];
#pragma unroll
                for (int c = 0; c < kDecKeys / 2; ++c) {
                    const float p0 = fast_exp2(fmaf(__uint_as_float(sv[2 * c]), args.scale_log2, -m_new));
                    const float p1 = fast_exp2(fmaf(__uint_as_float(sv[2 * c + 1]), args.scale_log2, -m_new));
                    sums[c & 3] += p0 + p1;
                    pk[c] = pack_bf16x2(p0, p1);
                }
                l_run = l_run * alpha + ((sums[0] + sums[1]) + (sums[2] + sums[3]));
                if (row < kHeads) alpha_s[buf * kHeads + row] = alpha;
                const bool any = __any_sync(0xffffffffu, move && !first);
                if (lane == 0) moved_s[buf * 4 + warp] = any ? 1 : 0;
                __syncwarp();
                mbar_arrive(&a_full[buf]);
                // P of the tile that used this buffer before has been multiplied
                if (T >= L::kPBufs) {
                    const uint32_t prev = T - L::kPBufs;
                    ok = mbar_wait_warp(&pv_done[prev & 1u], (prev >> 1) & 1u, abort_flag, args.status, 0xC1);
                    if (!ok) break;
                }
                if (row < kHeads) {       // row of 128 bytes, 16-byte chunks swizzled like every operand tile
                    uint8_t* dst = smem + L::kP + (T % L::kPBufs) * L::kPTile + row * 128;
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        *reinterpret_cast<uint4*>(dst + ((c ^ (row & 7)) << 4)) = make_uint4(pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]);
                }
            }
            ok = mbar_wait_warp(&a_full[buf], par, abort_flag, args.status, 0xC4);    // factors and flags are written
            if (!ok) break;
            bool moved = false;
#pragma unroll
            for (int w = 0; w * 32 < kHeads; ++w) moved |= moved_s[buf * 4 + w] != 0;
            if (moved) {
                // O^T is at rest once P.V of the previous tile has completed; this tile's waits for p_full below
                const uint32_t prev = T - 1;
                ok = mbar_wait_warp(&pv_done[prev & 1u], (prev >> 1) & 1u, abort_flag, args.status, 0xC2);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < 4 * kHeads; c += 16) {
                    uint32_t o[16];
                    tmem_ld_x16(tmem_base + lane_addr + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[v] = __float_as_uint(__uint_as_float(o[v]) * alpha_s[buf * kHeads + (c + v) % kHeads]);
                    tmem_st_x16(tmem_base + lane_addr + c, o);
                }
                tmem_st_wait();
            }
            if (valid & 15) {             // rows of the last 16-key step that no token owns: zero, whatever the page holds
                const int n_zero = 16 - (valid & 15);
                for (int i = threadIdx.x; i < 8 * 8 * n_zero; i += 128) {       // 8 slabs x rows x eight 16-byte chunks
                    const int slab = i / (8 * n_zero), r = valid + (i >> 3) % n_zero;
                    const uint32_t slot = (4 * T + (slab >> 1)) % L::kUnits;
                    *reinterpret_cast<uint4*>(smem + L::kUnit0 + slot * L::kUnit + (slab & 1) * L::kSlab + r * 128 + (i & 7) * 16) =
                        make_uint4(0u, 0u, 0u, 0u);
                }
            }
            fence_async_shared();
            tc_fence_before_sync();
            mbar_arrive(&p_full[buf]);
            first = false;
            const bool ends = cur.ends_piece();
            if (ends) {
                ok = mbar_wait_warp(o_full, pieces & 1u, abort_flag, args.status, 0xC3);
                if (!ok) break;
                tc_fence_after_sync();
                const size_t slot = static_cast<size_t>(cta) + cur.b;
                float* dst = args.part_o + (slot * args.h_pad + head0) * kDecLat + row;
                const int n_heads = min(kHeads, args.h - head0);
#pragma unroll 1
                for (int c = 0; c < 4 * kHeads; c += 16) {    // latents (c / kHeads) * 128 + row of heads c % kHeads ..
                    uint32_t o[16];
                    tmem_ld_x16(tmem_base + lane_addr + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if ((c % kHeads) + v < n_heads) dst[static_cast<size_t>((c % kHeads) + v) * kDecLat + (c / kHeads) * 128] = __uint_as_float(o[v]);
                }
                if (live) args.part_ml[slot * args.h_pad + head0 + row] = make_float2(m_run, l_run);
                tc_fence_before_sync();
                mbar_arrive(o_free);
                ++pieces;
                m_run = -INFINITY; l_run = 0.f;
                first = true;
            }
            cur.next(args);
            ++T;
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 5) { tc_fence_after_sync(); tmem_dealloc(tmem_base, 512); }
}

// Joins the pieces of one (request, head): o_lat = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c, rounded once to bf16
// for the value projection's tensor-core product.  A request without tokens has no piece: zeros, LSE -inf.
__global__ void __launch_bounds__(128)
decode_combine_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, const int* __restrict__ tile_start,
                      int B, int h, int h_pad, int ctas_per_group, __nv_bfloat16* __restrict__ o_lat, float* __restrict__ lse) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int b = blockIdx.x / h, head = blockIdx.x - b * h;
    const int total = tile_start[B], begin = tile_start[b], end = tile_start[b + 1];
    const int per = max(1, (total + ctas_per_group - 1) / ctas_per_group);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float M = -INFINITY, l = 0.f;
    if (end > begin) {
        const int c0 = begin / per, c1 = (end - 1) / per;
        for (int c = c0; c <= c1; ++c) {
            const float m = part_ml[static_cast<size_t>(c + b) * h_pad + head].x;
            M = c == c0 ? m : fmaxf(M, m);
        }
        for (int c = c0; c <= c1; ++c) {
            const size_t at = static_cast<size_t>(c + b) * h_pad + head;
            const float2 ml = part_ml[at];
            const float w = fast_exp2(ml.x - M);
            const float4 o = reinterpret_cast<const float4*>(part_o + at * kDecLat)[threadIdx.x];
            l = fmaf(ml.y, w, l);
            acc.x = fmaf(o.x, w, acc.x); acc.y = fmaf(o.y, w, acc.y);
            acc.z = fmaf(o.z, w, acc.z); acc.w = fmaf(o.w, w, acc.w);
        }
        const float inv = 1.0f / l;
        acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    }
    reinterpret_cast<uint2*>(o_lat + static_cast<size_t>(blockIdx.x) * kDecLat)[threadIdx.x] =
        make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
    if (lse != nullptr && threadIdx.x == 0) lse[blockIdx.x] = end > begin ? (M + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace laga
