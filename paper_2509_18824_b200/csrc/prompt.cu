// Causal GQA attention of packed new tokens over the paged cache.
//
// out = softmax(scale q . K^T) V over the keys t <= len + i, a pass over the keys with a row's weights relative to one of its first scores
// (see kSumLimit: the reference moves only where a block's weights add up to more than 2^40, so that no maximum is looked for and nothing
// is rescaled in the usual block).
//
// A CTA per SM works through its entries of the plan (prompt_plan.cuh): two row tiles A and B of 128 rows - the query heads of a KV head
// for 128 / G tokens each - against the same key tiles of 128 keys.  Tensor memory holds S and O of both (4 x 128 columns); P, in bf16,
// lies over the scores that it comes from.  Per key tile the tensor pipe computes P.V of A, the next S of A, then the same of B, while the
// four warps of A (of B) turn scores into weights: what one tile's soft-max takes hides behind the other's products.  K and V pass through
// one ring of five 32 KiB slots.  Warps: 0-3 soft-max A, 4-7 soft-max B, 8-11 results (normalise and store while the next entry
// begins), 12 issues the products, 13 the copies.
#include "attention_shared.cuh"
#include "prompt_plan.cuh"

namespace sdv {

namespace {
constexpr int kPThreads = 448;
constexpr int kPMmaWarp = 12, kPTmaWarp = 13;
constexpr int kPStages = 5;
constexpr int kPHalf = kPromptTile * 128;      // bytes of one D-half of a key tile: [128 keys][64] bf16, swizzled (16 KiB)
constexpr int kPStage = 2 * kPHalf;
constexpr int kPQBytes = 2 * kRowTile * 128;   // of one row tile
constexpr int kPBars = 256;
constexpr int kPSmem = 2 * kPQBytes + kPStages * kPStage + kPBars + 2 * kRowTile * 8;
constexpr int kMergeThreads = 256;

struct PromptShared {
    uint8_t *q_smem, *ring;
    uint64_t* kv_full;      // [5] TMA -> MMA (and whoever clears V rows)
    uint64_t* kv_empty;     // [5] MMA -> TMA
    uint64_t* q_full;       // [2] TMA -> MMA, per row tile from here on
    uint64_t* q_empty;      // MMA -> TMA: the entry's last scores are there
    uint64_t* s_full;       // MMA -> soft-max: scores of a key tile
    uint64_t* p_full;       // [2][2] soft-max -> MMA: weights of a block of 64 keys, the tile's first and second (a warp may be a block ahead)
    uint64_t* o_done;       // MMA -> soft-max: O updated by a block
    uint64_t* o_full;       // MMA -> results: O updated by the entry's last block
    uint64_t* o_empty;      // results -> MMA, soft-max: O, reference and sum have been read
    uint64_t* sum_full;     // soft-max -> results: reference and sum
    uint64_t* unwound;      // MMA: every product that was issued has completed
    uint32_t* tmem_slot;
    int* abort_flag;
    float2* sums;           // [2][128] reference and sum of a row

    __device__ __forceinline__ explicit PromptShared(uint8_t* smem) {
        q_smem = smem;
        ring = smem + 2 * kPQBytes;
        uint64_t* bars = reinterpret_cast<uint64_t*>(ring + kPStages * kPStage);
        kv_full = bars; kv_empty = bars + 5;
        q_full = bars + 10; q_empty = bars + 12; s_full = bars + 14; p_full = bars + 16; o_done = bars + 20; o_full = bars + 22;
        o_empty = bars + 24; sum_full = bars + 26; unwound = bars + 28;
        tmem_slot = reinterpret_cast<uint32_t*>(bars + 29);
        abort_flag = reinterpret_cast<int*>(bars + 30);
        sums = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(bars) + kPBars);
    }
    // (one thread)
    __device__ __forceinline__ void init_barriers() const {
        *abort_flag = 0;
        for (int i = 0; i < kPStages; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); }
        for (int w = 0; w < 2; ++w) {
            mbar_init(&q_full[w], 1); mbar_init(&q_empty[w], 1); mbar_init(&s_full[w], 1); mbar_init(&p_full[2 * w], 4); mbar_init(&p_full[2 * w + 1], 4);
            mbar_init(&o_done[w], 1); mbar_init(&o_full[w], 1); mbar_init(&o_empty[w], 4); mbar_init(&sum_full[w], 4);
        }
        mbar_init(unwound, 1);
    }
};

// position in a ring of n barriers: slot, and parity of the phase
template <int N>
struct RingAt {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() { if (++slot == N) { slot = 0; phase ^= 1u; } }
};

// An entry as a CTA sees it: which blocks of its keys the rows of either tile see.
struct PromptWork {
    PromptEntry e;
    int h;                  // KV head
    int nb[2];              // key blocks of row tiles A and B, from kb0 on
    __device__ __forceinline__ int blocks() const { return max(nb[0], nb[1]); }
};

struct PromptArgs {
    sd_prompts p;
    PromptGeom g;
    __nv_bfloat16* out;
    long long ldo;
    float* lse;
    float* partial;
    int num_blocks;
    float scale_log2;
    long long wait_cycles;
    int withhold;
};

// the CTA's k-th piece of work; false: there is none
__device__ __forceinline__ bool prompt_work(const PromptArgs& a, int k, int entries, PromptWork& w) {
    const int ctas = gridDim.x, c = blockIdx.x;
    const long long i = (long long)k * ctas + ((k & 1) ? ctas - 1 - c : c);
    if (i >= (long long)entries * a.p.Hkv) return false;
    const int4* src = reinterpret_cast<const int4*>(plan_entries(a.p.plan) + i / a.p.Hkv);
    const int4 x = __ldcg(src), y = __ldcg(src + 1);
    w.e = PromptEntry{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    w.h = (int)(i % a.p.Hkv);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int last = min((t + 1) * a.g.tokens, w.e.tokens);      // the tile's last token sees the most
        w.nb[t] = last > t * a.g.tokens ? max(min((w.e.pos0 + last + kBlock - 1) / kBlock, w.e.kb1) - w.e.kb0, 0) : 0;
    }
    return true;
}
}  // namespace

__global__ void __launch_bounds__(kPThreads, 1)
prompt_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
              const __grid_constant__ PromptArgs a, int32_t* status) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const PromptShared sh(smem);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const long long limit = a.wait_cycles;
    int* const abort_flag = sh.abort_flag;

    griddep_launch_dependents();
    const bool aligned = (smem_u32(smem) & 1023u) == 0;    // swizzled tiles need 1 KiB alignment
    if (!aligned) {
        if (threadIdx.x == 0) set_status(status, SD_ERR_UNSUPPORTED);
        griddep_wait();
        return;
    }
    if (warp == kPTmaWarp) {
        if (lane == 0) {
            sh.init_barriers();
            fence_barrier_init();
            fence_proxy_async_smem();
            prefetch_tensormap(&q_map); prefetch_tensormap(&k_map); prefetch_tensormap(&v_map);
        }
        __syncwarp();
        tmem_alloc(sh.tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();                                       // barriers and tensor memory are set up
    tc_fence_after_sync();
    const uint32_t tmem = *sh.tmem_slot;                   // S of A and B, O of A and B: 128 columns each
    griddep_wait();                                        // global memory from here on
    const int entries = __ldcg(&plan_header(a.p.plan)->entries);
    PromptWork w;

    if (warp == kPTmaWarp) {
        // ------------------------------------------------------------ copies (a whole warp in uniform control flow)
        const uint64_t keep = policy_evict_last(), once = policy_evict_first();
        RingAt<kPStages> at;
        uint32_t q_phase[2] = {1u, 1u};                    // (empty at first)
        bool ok = true;
        for (int k = 0; ok && prompt_work(a, k, entries, w); ++k) {
            const int nb = w.blocks();
            const int32_t* table = a.p.block_table + (size_t)w.e.b * a.p.max_blocks_per_seq + w.e.kb0;
            int held = 0;                                  // 32 entries of the table
            const auto block_of = [&](int i) {
                int blk = __shfl_sync(0xffffffffu, held, i & 31);
                if (blk < 0 || blk >= a.num_blocks) { if (lane == 0) set_status(status, SD_ERR_BOUNDS); blk = 0; }
                return blk;
            };
            const auto load = [&](const CUtensorMap* m, int j) -> bool {
                if (!mbar_wait_warp(&sh.kv_empty[at.slot], at.phase ^ 1u, abort_flag, limit)) return false;
                const bool two = 2 * j + 1 < nb;
                const int y0 = (block_of(2 * j) * a.p.Hkv + w.h) * kBlock, y1 = two ? (block_of(2 * j + 1) * a.p.Hkv + w.h) * kBlock : 0;
                uint8_t* dst = sh.ring + at.slot * kPStage;
                uint64_t* full = &sh.kv_full[at.slot];
                if (elect_one()) {
                    mbar_arrive_expect_tx(full, two ? kPStage : kPStage / 2);
                    tma_load_2d(dst, m, 0, y0, full, keep);
                    tma_load_2d(dst + kPHalf, m, 64, y0, full, keep);
                    if (two) {
                        tma_load_2d(dst + kPHalf / 2, m, 0, y1, full, keep);
                        tma_load_2d(dst + kPHalf + kPHalf / 2, m, 64, y1, full, keep);
                    }
                }
                __syncwarp();
                at.next();
                return true;
            };
            for (int j = 0; ok && 2 * j < nb; ++j) {
                if ((j & 15) == 0) held = 2 * j + lane < nb ? __ldcg(table + 2 * j + lane) : 0;
                ok = load(&k_map, j);
                if (j == 0)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (!ok || w.nb[t] == 0) continue;
                        ok = mbar_wait_warp(&sh.q_empty[t], q_phase[t], abort_flag, limit);
                        if (!ok) continue;
                        q_phase[t] ^= 1u;
                        if (elect_one()) {
                            uint8_t* dst = sh.q_smem + t * kPQBytes;
                            const int row = w.e.row0 + t * a.g.tokens;
                            mbar_arrive_expect_tx(&sh.q_full[t], (uint32_t)(a.g.tokens * a.g.G) * kD * 2);
                            tma_load_3d(dst, &q_map, 0, w.h * a.g.G, row, &sh.q_full[t], once);
                            tma_load_3d(dst + kRowTile * 128, &q_map, 64, w.h * a.g.G, row, &sh.q_full[t], once);
                        }
                        __syncwarp();
                    }
                if (ok) ok = load(&v_map, j);
            }
        }
        if (!ok) {
            if (lane == 0) set_status(status, SD_ERR_TIMEOUT);
            unwind_pause();
        }
    } else if (warp == kPMmaWarp) {
        // ------------------------------------------------------------ products (a whole warp in uniform control flow)
        const uint32_t idesc_s = make_idesc_bf16(kRowTile, kPromptTile, false, false), idesc_s_half = make_idesc_bf16(kRowTile, kBlock, false, false);
        const uint32_t idesc_o = make_idesc_bf16(kRowTile, kD, false, true);
        const uint64_t q_desc = make_smem_desc(smem_u32(sh.q_smem), 16, 1024, 128);
        const uint64_t k_desc = make_smem_desc(smem_u32(sh.ring), 16, 1024, 128);
        const uint64_t v_desc = make_smem_desc(smem_u32(sh.ring), kPHalf, 1024, 128);   // [key][d]: N (= d) contiguous
        RingAt<kPStages> at;                               // the next K or V
        uint32_t q_phase[2] = {0u, 0u}, p_phase[4] = {0u, 0u, 0u, 0u}, o_phase[2] = {1u, 1u};
        const auto scores = [&](int t, int j, int slot) {
            const uint64_t kd = k_desc + (uint64_t)(slot * (kPStage >> 4)), qd = q_desc + (uint64_t)(t * (kPQBytes >> 4));
            const uint32_t d = tmem + t * kPromptTile;
            const uint32_t idesc = 2 * j + 1 < w.nb[t] ? idesc_s : idesc_s_half;
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < kD / 16; ++k)
                    mma_ss(d, qd + (uint64_t)((k >> 2) * ((kRowTile * 128) >> 4) + (k & 3) * 2),
                           kd + (uint64_t)((k >> 2) * (kPHalf >> 4) + (k & 3) * 2), idesc, k != 0 ? 1u : 0u);
                mma_commit(&sh.s_full[t]);
                if (2 * (j + 1) >= w.nb[t]) mma_commit(&sh.q_empty[t]);
            }
            __syncwarp();
        };
        bool ok = true;
        for (int k = 0; ok && prompt_work(a, k, entries, w); ++k) {
            const int nb = w.blocks(), nt = (nb + 1) / 2;
            if (nt == 0) continue;
            if (!(ok = mbar_wait_warp(&sh.kv_full[at.slot], at.phase, abort_flag, limit))) break;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (!ok || w.nb[t] == 0) continue;
                ok = mbar_wait_warp(&sh.q_full[t], q_phase[t], abort_flag, limit);
                if (!ok) continue;
                q_phase[t] ^= 1u;
                tc_fence_after_sync();
                scores(t, 0, at.slot);
            }
            if (!ok) break;
            if (elect_one()) mma_commit(&sh.kv_empty[at.slot]);
            __syncwarp();
            at.next();
            for (int j = 0; ok && j < nt; ++j) {
                const RingAt<kPStages> v_at = at;
                RingAt<kPStages> k_at = at;
                k_at.next();
                bool have_v = false, have_k = false;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (!ok || 2 * j >= w.nb[t]) continue;
                    if (j == 0) {                          // the entry before has left O
                        ok = mbar_wait_warp(&sh.o_empty[t], o_phase[t], abort_flag, limit);
                        o_phase[t] ^= 1u;
                    }
                    if (ok && !have_v) { ok = mbar_wait_warp(&sh.kv_full[v_at.slot], v_at.phase, abort_flag, limit); have_v = true; }
                    const uint64_t vd = v_desc + (uint64_t)(v_at.slot * (kPStage >> 4));
                    const uint32_t o = tmem + 2 * kPromptTile + t * kD, pa = tmem + t * kPromptTile;
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb) {       // blocks of 64 keys: P of 16 keys = 8 columns
                        if (!ok || 2 * j + hb >= w.nb[t]) continue;
                        ok = mbar_wait_warp(&sh.p_full[2 * t + hb], p_phase[2 * t + hb], abort_flag, limit);
                        if (!ok) continue;
                        p_phase[2 * t + hb] ^= 1u;
                        tc_fence_after_sync();
                        if (elect_one()) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                mma_ts(o, pa + (hb * 4 + i) * 8, vd + (uint64_t)((hb * 4 + i) * (2048 >> 4)), idesc_o,
                                       (j | hb | i) != 0 ? 1u : 0u);
                            mma_commit(&sh.o_done[t]);
                            if (2 * j + hb + 1 == w.nb[t]) mma_commit(&sh.o_full[t]);
                        }
                        __syncwarp();
                    }
                    if (ok && 2 * (j + 1) < w.nb[t]) {
                        if (!have_k) { ok = mbar_wait_warp(&sh.kv_full[k_at.slot], k_at.phase, abort_flag, limit); have_k = true; }
                        tc_fence_after_sync();
                        if (ok) scores(t, j + 1, k_at.slot);
                    }
                }
                if (!ok) break;
                if (elect_one()) {
                    mma_commit(&sh.kv_empty[v_at.slot]);
                    if (j + 1 < nt) mma_commit(&sh.kv_empty[k_at.slot]);
                }
                __syncwarp();
                at.next();
                if (j + 1 < nt) at.next();
            }
        }
        if (elect_one()) mma_commit(sh.unwound);
        __syncwarp();
        if (!ok && lane == 0) set_status(status, SD_ERR_TIMEOUT);
        mbar_wait_plain(sh.unwound, 0, limit);             // (nothing gives tensor memory back while a product runs)
        if (!ok) unwind_pause();
    } else if (warp < 8) {
        // ------------------------------------------------------------ soft-max: one thread per row
        const int t = warp >> 2, quad = warp & 3;          // row tile, TMEM quadrant
        const int r = quad * 32 + lane;                    // TMEM lane
        const int token = t * a.g.tokens + a.g.token_of(r);
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t ts = tmem + lanes + t * kPromptTile, to = tmem + lanes + 2 * kPromptTile + t * kD;
        const uint64_t scale2 = pack_f32x2(a.scale_log2, a.scale_log2);
        RingAt<kPStages> at;                               // the entry's first K
        uint32_t s_phase = 0u, done_phase = 1u, read_phase = 1u;
        bool ok = true;
        for (int k = 0; ok && prompt_work(a, k, entries, w); ++k) {
            const int nb = w.nb[t];
            const int fills = 2 * ((w.blocks() + 1) / 2);  // K and V tiles of the entry in the ring
            const bool row_ok = token < w.e.tokens && a.g.token_of(r) < a.g.tokens;
            const int seen = w.e.pos0 + token + 1 - w.e.kb0 * kBlock;          // keys from kb0 on that this row sees
            const int all_see = w.e.pos0 + t * a.g.tokens + 1 - w.e.kb0 * kBlock;   // ... that every row of the tile sees
            const int filled = w.e.end - w.e.kb0 * kBlock;  // ... that have been written
            float m_used = 0.f, l = 0.f;
            uint64_t neg_m2 = 0ull;
            uint32_t ra[32], rb[32];
            RingAt<kPStages> v_at = at;
            v_at.next();
            for (int i = 0; i < nb; ++i) {                 // blocks of 64 keys, two to a tile of scores
                const uint32_t tb = ts + (i & 1) * kBlock;
                if ((i & 1) == 0) {
                    if (!(ok = mbar_wait_warp(&sh.s_full[t], s_phase, abort_flag, limit))) break;
                    s_phase ^= 1u;
                    tc_fence_after_sync();
                    tmem_ld32(tb, ra);
                }
                const int vis = max(min(seen - i * kBlock, kBlock), 0);
                const bool masked = all_see < (i + 1) * kBlock;
                uint32_t mask_lo = ~0u, mask_hi = ~0u;
                if (masked && row_ok) {
                    mask_lo = vis >= 32 ? ~0u : (1u << vis) - 1u;
                    mask_hi = vis >= 64 ? ~0u : (vis > 32 ? (1u << (vis - 32)) - 1u : 0u);
                }
                // V rows behind the request's last token carry weight 0, but 0 x NaN would still reach O: cleared before P.V reads them
                // (by the tile whose P.V comes first)
                if (filled < (i + 1) * kBlock && (t == 0 || i >= w.nb[0])) {
                    if (!(ok = mbar_wait_warp(&sh.kv_full[v_at.slot], v_at.phase, abort_flag, limit))) break;
                    if ((r & 63) >= filled - i * kBlock) {
                        uint4* z = reinterpret_cast<uint4*>(sh.ring + v_at.slot * kPStage + (r >> 6) * kPHalf + ((i & 1) * kBlock + (r & 63)) * 128);
#pragma unroll
                        for (int c = 0; c < 8; ++c) z[c] = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                    }
                }
                tmem_ld_wait();
                tmem_ld32(tb + 32, rb);
                if (masked) mask_scores(ra, mask_lo);
                if (i == 0) {                              // the reference: the largest of the first 32 scores
                    float mt = fmaxf(__uint_as_float(ra[0]), __uint_as_float(ra[1]));
#pragma unroll
                    for (int c = 2; c < 32; c += 2) mt = max3(mt, __uint_as_float(ra[c]), __uint_as_float(ra[c + 1]));
                    m_used = row_ok && mt > -INFINITY ? mt * a.scale_log2 : 0.f;
                    neg_m2 = pack_f32x2(-m_used, -m_used);
                }
                uint32_t pk[32];
                uint64_t ps[2] = {0ull, 0ull};
                exp_pack(ra, scale2, neg_m2, pk, ps);
                tmem_ld_wait();
                if ((i & 1) == 0 && i + 1 < nb) tmem_ld32(tb + kBlock, ra);    // the next block's first half
                if (masked) mask_scores(rb, mask_hi);
                exp_pack(rb, scale2, neg_m2, pk + 16, ps);
                float psum = sum_f32x2(add_f32x2(ps[0], ps[1]));
                // too large for the reference (or not a number), or, where no score has counted so far, too small
                const bool off = row_ok && vis > 0 && (!(psum <= kSumLimit) || l + psum == 0.f);
                if (__any_sync(0xffffffffu, off)) {
                    float mt = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        uint32_t s[16];
                        tmem_ld16(tb + c * 16, s);
                        tmem_ld_wait();
                        if (masked) mask_scores(s, (c < 2 ? mask_lo : mask_hi) >> ((c & 1) * 16));
#pragma unroll
                        for (int x = 0; x < 16; x += 2) mt = max3(mt, __uint_as_float(s[x]), __uint_as_float(s[x + 1]));
                    }
                    mt *= a.scale_log2;
                    const bool raise = off && mt > -INFINITY && (l == 0.f || mt > m_used + kRaiseAbove);
                    const float alpha = raise && l != 0.f ? exp2f(m_used - mt) : 1.f;
                    if (__any_sync(0xffffffffu, alpha != 1.f)) {               // (then a block has been added to O)
                        if (!(ok = mbar_wait_warp(&sh.o_done[t], done_phase, abort_flag, limit))) break;
                        tc_fence_after_sync();
#pragma unroll 1
                        for (int c = 0; c < 8; ++c) {
                            uint32_t o[16];
                            tmem_ld16(to + c * 16, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                            tmem_st16(to + c * 16, o);
                        }
                        tmem_st_wait();
                        l *= alpha;
                    }
                    if (raise) m_used = mt;
                    neg_m2 = pack_f32x2(-m_used, -m_used);
                    uint64_t again[2] = {0ull, 0ull};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t s[16];
                        tmem_ld16(tb + c * 16, s);
                        tmem_ld_wait();
                        if (masked) mask_scores(s, (c < 2 ? mask_lo : mask_hi) >> ((c & 1) * 16));
                        exp_pack(s, scale2, neg_m2, pk + c * 8, again);
                    }
                    psum = sum_f32x2(add_f32x2(again[0], again[1]));
                }
                l += psum;
                done_phase ^= 1u;
                tmem_st32(ts + (i & 1) * 32, pk);          // over scores that have been read
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0 && !a.withhold) mbar_arrive(&sh.p_full[2 * t + (i & 1)]);
                if (i & 1) { v_at.next(); v_at.next(); }
            }
            if (!ok) break;
            for (int i = 0; i < fills; ++i) at.next();
            if (nb == 0) continue;
            if (!(ok = mbar_wait_warp(&sh.o_empty[t], read_phase, abort_flag, limit))) break;
            read_phase ^= 1u;
            sh.sums[t * kRowTile + r] = make_float2(m_used, l);
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.sum_full[t]);
        }
        if (!ok) {
            if (lane == 0) set_status(status, SD_ERR_TIMEOUT);
            unwind_pause();
        }
    } else {
        // ------------------------------------------------------------ results: one thread per row
        const int quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const int row_token = a.g.token_of(r), head = r - row_token * a.g.G;
        uint32_t phase[2] = {0u, 0u};
        bool ok = true;
        for (int k = 0; ok && prompt_work(a, k, entries, w); ++k) {
#pragma unroll 1
            for (int t = 0; t < 2 && ok; ++t) {
                const int token = t * a.g.tokens + row_token;
                const bool row_ok = row_token < a.g.tokens && token < w.e.tokens;
                float* const part = w.e.slot < 0 ? nullptr : a.partial + (size_t)(w.e.slot + w.h) * a.g.slot_floats() + (size_t)t * a.g.rows * kD;
                float2* const part_sum = w.e.slot < 0 ? nullptr
                    : reinterpret_cast<float2*>(a.partial + (size_t)(w.e.slot + w.h) * a.g.slot_floats() + (size_t)a.g.tiles * a.g.rows * kD) + t * a.g.rows;
                if (w.nb[t] == 0) {                        // none of its rows sees a key of this chunk
                    if (row_ok && part) part_sum[r] = make_float2(0.f, 0.f);
                    continue;
                }
                if (!(ok = mbar_wait_warp(&sh.sum_full[t], phase[t], abort_flag, limit))) break;
                const float2 ml = sh.sums[t * kRowTile + r];
                if (!(ok = mbar_wait_warp(&sh.o_full[t], phase[t], abort_flag, limit))) break;
                phase[t] ^= 1u;
                tc_fence_after_sync();
                const size_t row = (size_t)(w.e.row0 + token), h = (size_t)w.h * a.g.G + head;
                __nv_bfloat16* const dst = a.out + row * a.ldo + h * kD;
                const float inv = 1.f / ml.y;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tmem + lanes + 2 * kPromptTile + t * kD + c * 32, o);
                    tmem_ld_wait();
                    if (c == 3) {
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.o_empty[t]);
                    }
                    if (!row_ok) continue;
                    if (part) {                            // [16-byte piece][row]: a warp's stores are whole lines
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            reinterpret_cast<uint4*>(part)[(c * 8 + x) * a.g.rows + r] = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            uint32_t u[4];
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const __nv_bfloat162 hh = __floats2bfloat162_rn(__uint_as_float(o[8 * x + 2 * y]) * inv, __uint_as_float(o[8 * x + 2 * y + 1]) * inv);
                                u[y] = *reinterpret_cast<const uint32_t*>(&hh);
                            }
                            reinterpret_cast<uint4*>(dst)[c * 4 + x] = make_uint4(u[0], u[1], u[2], u[3]);
                        }
                    }
                }
                if (row_ok && part) part_sum[r] = ml;
                if (row_ok && !part && a.lse) a.lse[row * a.p.Hq + h] = (ml.x + log2f(ml.y)) * 0.6931471805599453f;
            }
        }
        if (!ok) {
            if (lane == 0) set_status(status, SD_ERR_TIMEOUT);
            unwind_pause();
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kPTmaWarp) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

// Joins the chunks of the entries that were cut, in the order of the keys.  A thread takes 16 columns of a row.
__global__ void __launch_bounds__(kMergeThreads)
prompt_merge_kernel(const __grid_constant__ PromptArgs a) {
    begin_dependent();
    const int splits = __ldcg(&plan_header(a.p.plan)->splits);
    const PromptSplit* const list = plan_splits(a.p.plan, a.g.cap_entries);
    const int per = (a.g.tiles * a.g.rows * 8 + kMergeThreads - 1) / kMergeThreads;      // CTAs of an entry and KV head, at most
    for (int u = blockIdx.x; u < splits * a.p.Hkv * per; u += gridDim.x) {
        const int4 s = __ldcg(reinterpret_cast<const int4*>(list + u / (a.p.Hkv * per)));
        const int h = u / per % a.p.Hkv, rows = s.y * a.g.G, item = u % per * kMergeThreads + (int)threadIdx.x;
        if (item >= rows * 8) continue;
        const int cg = item / rows, row = item - cg * rows;
        const int tok = row / a.g.G, t = tok >= a.g.tokens ? 1 : 0, r = row - t * a.g.tokens * a.g.G;
        const size_t step = a.g.slot_floats() * a.p.Hkv;
        const float* part = a.partial + (size_t)(s.z + h) * a.g.slot_floats();
        const float2* sums = reinterpret_cast<const float2*>(part + (size_t)a.g.tiles * a.g.rows * kD) + t * a.g.rows + r;
        const float4* o = reinterpret_cast<const float4*>(part + (size_t)t * a.g.rows * kD) + (size_t)cg * 4 * a.g.rows + r;
        float top = -INFINITY;
        for (int c = 0; c < s.w; ++c) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(reinterpret_cast<const float*>(sums) + c * step));
            if (ml.y != 0.f) top = fmaxf(top, ml.x);
        }
        float den = 0.f;
        float4 acc[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c = 0; c < s.w; ++c) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(reinterpret_cast<const float*>(sums) + c * step));
            if (ml.y == 0.f) continue;                     // (no key that the row sees: nothing was written there)
            const float f = exp2f(ml.x - top);
            den = fmaf(f, ml.y, den);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(o + (size_t)x * a.g.rows) + c * step));
                acc[x].x = fmaf(f, v.x, acc[x].x); acc[x].y = fmaf(f, v.y, acc[x].y);
                acc[x].z = fmaf(f, v.z, acc[x].z); acc[x].w = fmaf(f, v.w, acc[x].w);
            }
        }
        const float inv = 1.f / den;
        uint32_t u8[8];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const __nv_bfloat162 h0 = __floats2bfloat162_rn(acc[x].x * inv, acc[x].y * inv), h1 = __floats2bfloat162_rn(acc[x].z * inv, acc[x].w * inv);
            u8[2 * x] = *reinterpret_cast<const uint32_t*>(&h0);
            u8[2 * x + 1] = *reinterpret_cast<const uint32_t*>(&h1);
        }
        const size_t out_row = (size_t)(s.x + tok), out_head = (size_t)h * a.g.G + (row - tok * a.g.G);
        uint4* dst = reinterpret_cast<uint4*>(a.out + out_row * a.ldo + out_head * kD + cg * 16);
        dst[0] = make_uint4(u8[0], u8[1], u8[2], u8[3]);
        dst[1] = make_uint4(u8[4], u8[5], u8[6], u8[7]);
        if (cg == 0 && a.lse) a.lse[out_row * a.p.Hq + out_head] = (top + log2f(den)) * 0.6931471805599453f;
    }
}

int current_sms() {
    int dev = 0;
    cudaGetDevice(&dev);
    return sm_count(dev);
}

size_t prompt_workspace_bytes(const sd_prompts& p) {
    const PromptGeom g = prompt_geom(p, current_sms());
    return ((size_t)g.cap_slots * g.slot_floats() * 4 + 255) & ~(size_t)255;
}

sd_status launch_prompt_attention(const sd_prompts& p, const sd_kv_layer& cache, const void* q, long long ldq, float scale, void* out,
                                  long long ldo, float* lse, void* ws, int32_t* dev_status, cudaStream_t st) {
    const TestKnobs knobs = test_knobs();
    PromptArgs a;
    a.p = p;
    a.g = prompt_geom(p, current_sms());
    a.out = static_cast<__nv_bfloat16*>(out);
    a.ldo = ldo;
    a.lse = lse;
    a.partial = static_cast<float*>(ws);
    a.num_blocks = cache.num_blocks;
    a.scale_log2 = scale * kLog2e;
    a.wait_cycles = knobs.wait_cycles;
    a.withhold = knobs.withhold;
    CUtensorMap qm, km, vm;
    const uint64_t q_dims[3] = {kD, (uint64_t)p.Hq, (uint64_t)p.N}, q_strides[2] = {kD * 2, (uint64_t)ldq * 2};
    const uint32_t q_box[3] = {64, (uint32_t)a.g.G, (uint32_t)a.g.tokens};
    const uint64_t kv_rows = (uint64_t)cache.num_blocks * p.Hkv * kBlock;
    if (!encode_tmap_bf16_3d(&qm, q, q_dims, q_strides, q_box, 128) ||
        !encode_tmap_bf16_2d(&km, cache.k, kv_rows, kD, kD * 2, 64, kBlock, 128) ||
        !encode_tmap_bf16_2d(&vm, cache.v, kv_rows, kD, kD * 2, 64, kBlock, 128))
        return SD_ERR_CUDA;
    if (!allow_dynamic_smem(prompt_kernel, kPSmem)) return SD_ERR_CUDA;
    const long long items = (long long)a.g.cap_entries * p.Hkv;
    const int ctas = (int)(items < a.g.sms ? items : a.g.sms);
    sd_status s = launch_dependent(prompt_kernel, dim3(ctas), kPThreads, kPSmem, 1, st, qm, km, vm, a, dev_status);
    if (s != SD_OK) return s;
    return launch_dependent(prompt_merge_kernel, dim3(2 * a.g.sms), kMergeThreads, 0, 1, st, a);
}

}  // namespace sdv
