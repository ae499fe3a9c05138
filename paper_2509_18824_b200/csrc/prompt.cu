// Causal GQA attention of packed new tokens over the paged cache.
//
// out = softmax(scale q . K^T) V over the keys t <= len + i, a pass over the keys with a row's weights relative to one of its first scores
// (see kSumLimit: the reference moves only where a tile's weights add up to more than 2^40, so that no maximum is looked for and nothing
// is rescaled in the usual tile).
//
// A CTA per SM works through its entries of the plan (prompt_plan.cuh): a row tile of 128 rows - the query heads of a KV head for 128 / G
// tokens - against tiles of 128 keys.  The tiles of all its entries are one stream: the scores of tile g + 2 are computed before the product
// of tile g's weights with V, whatever entries they belong to, in three score buffers of tensor memory beside O.  Weights, in bf16, lie over
// the scores that they come from.  Two groups of four soft-max warps take the tiles in turn; both add to the one O, which works because the
// reference stays (the rare tile that raises it is serialised through a barrier that every tile passes, commit).  Four more warps normalise
// and store an entry's rows while the next one's tiles are under way.
#include "attention_shared.cuh"
#include "prompt_plan.cuh"

namespace sdv {

namespace {
constexpr int kPThreads = 480;                 // warps 0-3, 4-7 soft-max, 8-11 results, 12 products, 13 K and Q copies, 14 V copies
constexpr int kPMmaWarp = 12, kPKeyWarp = 13, kPValueWarp = 14;
constexpr int kPStages = 3;                    // K and V ring slots, score buffers
constexpr int kPWorks = 4;                     // pieces of work that are known ahead
constexpr int kPHalf = kPromptTile * 128;      // bytes of one D-half of a key tile: [128 keys][64] bf16, swizzled (16 KiB)
constexpr int kPStage = 2 * kPHalf;
constexpr int kPQBytes = 2 * kRowTile * 128;
constexpr int kPBars = 512;                    // barriers, two words and the pieces of work
constexpr int kPSmem = kPQBytes + 2 * kPStages * kPStage + kPBars + 5 * kRowTile * 4;
#ifndef POLY
#define POLY 4
#endif
constexpr int kPolyPairs = POLY;
constexpr int kMergeThreads = 256;

struct PromptShared {
    uint8_t *q_smem, *k_smem, *v_smem;
    uint64_t* k_full;       // [3] TMA -> MMA
    uint64_t* v_full;       // [3] TMA -> MMA (and whoever clears V rows)
    uint64_t* s_full;       // [3] MMA -> soft-max, TMA: scores of tile g in buffer g % 3, K slot g % 3 read
    uint64_t* v_empty;      // [3] MMA -> TMA (and whoever raises a reference): O updated by tile g, V slot g % 3 read
    uint64_t* p_full;       // [3] soft-max -> MMA: weights of tile g written over its scores
    uint64_t* commit;       // [4] per TMEM quadrant: tile g's soft-max is final (phase g)
    uint64_t* ref_full;     // [2][4] per TMEM quadrant: the reference that an entry's first tile sets, entries in turn
    uint64_t* q_full;       // TMA -> MMA
    uint64_t* q_empty;      // MMA -> TMA: the entry's last scores are there
    uint64_t* o_full;       // MMA -> results: O updated by the entry's last tile
    uint64_t* o_empty;      // results -> MMA, soft-max: O, references and sums have been read
    uint64_t* sum_full;     // [2] soft-max group -> results: references and sums
    uint64_t* work_full;    // [4] K copies -> the others: a piece of work
    uint64_t* work_empty;   // [4] the others (14 warps) -> K copies: it has been read
    uint64_t* unwound;      // MMA: every product that was issued has completed
    uint32_t* tmem_slot;
    int* abort_flag;
    int* works;             // [4][10]
    float* refs;            // [2][128] reference of a row, entries in turn
    float* sums;            // [2][128] sum of a row over a group's tiles
    float* raised;          // [128] what the entry's last tile has scaled the row by

    __device__ __forceinline__ explicit PromptShared(uint8_t* smem) {
        q_smem = smem;
        k_smem = smem + kPQBytes;
        v_smem = k_smem + kPStages * kPStage;
        uint64_t* bars = reinterpret_cast<uint64_t*>(v_smem + kPStages * kPStage);
        k_full = bars; v_full = bars + 3; s_full = bars + 6; v_empty = bars + 9; p_full = bars + 12; commit = bars + 15; ref_full = bars + 19;
        q_full = bars + 27; q_empty = bars + 28; o_full = bars + 29; o_empty = bars + 30; sum_full = bars + 31;
        work_full = bars + 33; work_empty = bars + 37; unwound = bars + 41;
        tmem_slot = reinterpret_cast<uint32_t*>(bars + 42);
        abort_flag = reinterpret_cast<int*>(bars + 42) + 1;
        works = reinterpret_cast<int*>(bars + 44);
        static_assert(44 * 8 + kPWorks * 40 <= kPBars, "");
        refs = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(bars) + kPBars);
        sums = refs + 2 * kRowTile;
        raised = sums + 2 * kRowTile;
    }
    // (one thread)
    __device__ __forceinline__ void init_barriers() const {
        *abort_flag = 0;
        for (int i = 0; i < kPStages; ++i) {
            mbar_init(&k_full[i], 1); mbar_init(&v_full[i], 1); mbar_init(&s_full[i], 1); mbar_init(&v_empty[i], 1); mbar_init(&p_full[i], 4);
        }
        for (int i = 0; i < 4; ++i) { mbar_init(&commit[i], 1); mbar_init(&ref_full[i], 1); mbar_init(&ref_full[4 + i], 1); }
        mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(o_full, 1); mbar_init(o_empty, 4);
        mbar_init(&sum_full[0], 4); mbar_init(&sum_full[1], 4);
        for (int i = 0; i < kPWorks; ++i) { mbar_init(&work_full[i], 1); mbar_init(&work_empty[i], 14); }
        mbar_init(unwound, 1);
    }
};
static_assert(kPSmem <= 227 * 1024, "");

// position in a ring of n barriers: slot, and parity of the phase
template <int N>
struct RingAt {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() { if (++slot == N) { slot = 0; phase ^= 1u; } }
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

// An entry for one KV head, as PromptEntry; slot is this head's, nb key blocks from kb0 on (0: there is no more work).
struct PromptWork {
    int row0, pos0, tokens, b, kb0, end, slot, h, nb;
    __device__ __forceinline__ int tiles() const { return (nb + 1) / 2; }
};
// the CTA's k-th piece of work, two vectors of its entry, and the head; none: kb1 = 0
struct RawWork { int4 x, y; int h; };
__device__ __forceinline__ RawWork fetch_work(const PromptArgs& a, int k, int entries) {
    const int ctas = gridDim.x, c = blockIdx.x;
    const long long i = (long long)k * ctas + ((k & 1) ? ctas - 1 - c : c);
    RawWork r{make_int4(0, 0, 0, 0), make_int4(0, 0, 0, -1), 0};
    if (i < (long long)entries * a.p.Hkv) {
        const unsigned e = (unsigned)i / (unsigned)a.p.Hkv;                     // (entries x Hkv < 2^32: 2^24 rows of 1024 heads at most, 128 to a tile)
        const int4* src = reinterpret_cast<const int4*>(plan_entries(a.p.plan) + e);
        r.x = __ldcg(src);
        r.y = __ldcg(src + 1);
        r.h = (int)((unsigned)i - e * (unsigned)a.p.Hkv);
    }
    return r;
}
__device__ __forceinline__ PromptWork decode_work(const RawWork& r) {
    return PromptWork{r.x.x, r.x.y, r.x.z, r.x.w, r.y.x, r.y.z, r.y.w < 0 ? -1 : r.y.w + r.h, r.h, r.y.y - r.y.x};
}
// The next piece of work, for every warp but the one that hands them out; false: a wait ran out.  done_with_work: it has been read.
__device__ __forceinline__ bool see_work(const PromptShared& sh, const RingAt<kPWorks>& at, PromptWork& w, long long limit) {
    if (!mbar_wait_warp(&sh.work_full[at.slot], at.phase, sh.abort_flag, limit)) return false;
    const volatile int* src = sh.works + at.slot * 10;
    w.row0 = src[0]; w.pos0 = src[1]; w.tokens = src[2]; w.b = src[3]; w.kb0 = src[4]; w.end = src[5]; w.slot = src[6]; w.h = src[7];
    w.nb = src[8];
    return true;
}
__device__ __forceinline__ void done_with_work(const PromptShared& sh, RingAt<kPWorks>& at, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.work_empty[at.slot]);
    at.next();
}

__device__ __forceinline__ void halves(uint64_t x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t twice(float c) { return pack_f32x2(c, c); }
__device__ __forceinline__ float min3(float a, float b, float c) {
    float d;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 32 raw scores of a row -> 2^(score * scale - reference), packed to bf16 in pairs, and added to the sums.  kPolyPairs of the sixteen pairs go
// through the multiply-add units: x = n + f with n whole and f in [-1/2, 1/2], n by adding 1.5 x 2^23 (Cody and Waite's reduction; the
// reference is a whole number, so that one multiply-add gives it), 2^f by its minimax polynomial of degree 4 (least relative error, 2.6e-6,
// by reweighted least squares), n added to the exponent's bits.  That is right for |n| <= 126; lo, hi: the smallest and largest 1.5 x 2^23 + n.
constexpr float kShift = 12582912.f;
__device__ __forceinline__ void exp_block(const uint32_t (&r)[32], uint64_t scale2, float m, uint32_t* pk, uint64_t (&ps)[2], float& lo, float& hi) {
    const uint64_t neg_m2 = twice(-m), shift = twice(kShift - m);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        const uint64_t s = pack_f32x2(__uint_as_float(r[2 * c]), __uint_as_float(r[2 * c + 1]));
        float y0, y1;
        if (c * kPolyPairs / 16 != (c + 1) * kPolyPairs / 16) {
            const uint64_t t = fma_f32x2(s, scale2, shift);
            const uint64_t f = fma_f32x2(s, scale2, fma_f32x2(t, twice(-1.f), shift));
            uint64_t q = fma_f32x2(f, twice(0x1.3997d4p-7f), twice(0x1.ca1440p-5f));
            q = fma_f32x2(q, f, twice(0x1.ec06dap-3f));
            q = fma_f32x2(q, f, twice(0x1.62e0dcp-1f));
            q = fma_f32x2(q, f, twice(0x1.ffffe8p-1f));
            float t0, t1, q0, q1;
            halves(t, t0, t1);
            halves(q, q0, q1);
            lo = min3(lo, t0, t1);
            hi = max3(hi, t0, t1);
            y0 = __uint_as_float(__float_as_uint(q0) + (__float_as_uint(t0) << 23));
            y1 = __uint_as_float(__float_as_uint(q1) + (__float_as_uint(t1) << 23));
        } else {
            float x0, x1;
            halves(fma_f32x2(s, scale2, neg_m2), x0, x1);
            y0 = ex2_approx(x0);
            y1 = ex2_approx(x1);
        }
        ps[c & 1] = add_f32x2(ps[c & 1], pack_f32x2(y0, y1));
        const __nv_bfloat162 h = __floats2bfloat162_rn(y0, y1);
        pk[c] = *reinterpret_cast<const uint32_t*>(&h);
    }
}

// What the soft-max of a row hands from tile to tile.
struct RowState {
    float m, l;             // reference (a whole number) and sum of the weights relative to it
    float raised;           // what this tile has scaled the row by
    int usual;              // every reference of the warp is small enough for exp_block
    int ok;                 // no wait ran out
};
struct TileAt {
    uint32_t ts, to;        // scores (and weights) and O in tensor memory, at this warp's lanes
    int vis;                // keys of the tile that this row sees
    int blocks;             // of 64 keys, 1 or 2
    int first;              // the first tile of an entry
    uint64_t *ref_full, *commit, *o_done;
    uint32_t commit_phase, o_phase;
    int begun;              // there is a tile before this one in the stream
    int row_ok;
};
// A tile from block hb on, looked at before anything is weighed: masks, the reference of an entry's first tile, references that have to be
// raised (by the largest score, where that is more than 2^32 above), and what exp_block does not take.  (A call: in line it made the usual
// tile's code slower.)
__device__ __noinline__ RowState careful_tile(RowState st, const TileAt t, int hb, float scale_log2, volatile float* my_ref, int* abort_flag,
                                              long long limit) {
    const uint64_t scale2 = twice(scale_log2);
    const int lane = threadIdx.x & 31;
    tmem_ld_wait();
#pragma unroll 1
    for (; hb < t.blocks; ++hb) {
        const uint32_t tb = t.ts + hb * kBlock;
        const int v0 = min(max(t.vis - hb * kBlock, 0), 32), v1 = min(max(t.vis - hb * kBlock - 32, 0), 32);
        const uint32_t mask_lo = v0 == 32 ? ~0u : (1u << v0) - 1u, mask_hi = v1 == 32 ? ~0u : (1u << v1) - 1u;
        float mt = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            uint32_t s[32];
            tmem_ld32(tb + c * 32, s);
            tmem_ld_wait();
            mask_scores(s, c ? mask_hi : mask_lo);
#pragma unroll
            for (int x = 0; x < 32; x += 2) mt = max3(mt, __uint_as_float(s[x]), __uint_as_float(s[x + 1]));
        }
        mt = t.row_ok ? rintf(mt * scale_log2) : -INFINITY;
        if (hb == 0) {
            if (t.first) {
                st.m = mt > -INFINITY ? mt : 0.f;          // (no key: the row has no weight here)
                *my_ref = st.m;
                __syncwarp();
                if (lane == 0) mbar_arrive(t.ref_full);
            }
            // the tile before is final, and so is its reference
            if (t.begun && !mbar_wait_warp(t.commit, t.commit_phase, abort_flag, limit)) { st.ok = 0; return st; }
            const float ref = *my_ref;
            if (ref != st.m) { st.l *= exp2f(st.m - ref); st.m = ref; }
        }
        const bool raise = mt > st.m + kRaiseAbove;
        if (__any_sync(0xffffffffu, raise)) {
            const float alpha = raise ? exp2f(st.m - mt) : 1.f;                // (a power of two: weights of the first block stay exact)
            if (!t.first) {                                // (nothing has been added to O before an entry's first tile)
                if (!mbar_wait_warp(t.o_done, t.o_phase, abort_flag, limit)) { st.ok = 0; return st; }
                tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[32];
                    tmem_ld32(t.to + c * 32, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                    tmem_st32(t.to + c * 32, o);
                }
            }
            if (hb > 0) {
                uint32_t o[32];
                tmem_ld32(t.ts, o);
                tmem_ld_wait();
#pragma unroll
                for (int x = 0; x < 32; ++x) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(bf16lo(o[x]) * alpha, bf16hi(o[x]) * alpha);
                    o[x] = *reinterpret_cast<const uint32_t*>(&h);
                }
                tmem_st32(t.ts, o);
            }
            tmem_st_wait();
            st.l *= alpha;
            st.raised *= alpha;
            if (raise) st.m = mt;
            *my_ref = st.m;
        }
        uint64_t ps[2] = {0ull, 0ull};
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {                      // P of half a block lands on scores that have been read
            uint32_t s[32], part[16];
            tmem_ld32(tb + c * 32, s);
            tmem_ld_wait();
            mask_scores(s, c ? mask_hi : mask_lo);
            exp_pack(s, scale2, twice(-st.m), part, ps);
            tmem_st16(t.ts + hb * 32 + c * 16, part);
        }
        st.l += sum_f32x2(add_f32x2(ps[0], ps[1]));
        tmem_st_wait();
    }
    st.usual = !__any_sync(0xffffffffu, !(fabsf(st.m) < 2097152.f));
    return st;
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
    if (warp == kPKeyWarp) {
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
    const uint32_t tmem = *sh.tmem_slot;                   // O, then three score buffers of 128 columns
    const uint32_t tmem_s = tmem + kD;
    griddep_wait();                                        // global memory from here on

    if (warp == kPKeyWarp || warp == kPValueWarp) {
        // ------------------------------------------------------------ copies (whole warps in uniform control flow)
        const bool keys = warp == kPKeyWarp;
        const CUtensorMap* const map = keys ? &k_map : &v_map;
        uint8_t* const ring = keys ? sh.k_smem : sh.v_smem;
        uint64_t *const full = keys ? sh.k_full : sh.v_full, *const empty = keys ? sh.s_full : sh.v_empty;
        const uint64_t keep = policy_evict_last(), once = policy_evict_first();
        RingAt<kPStages> at;
        RingAt<kPWorks> work_at;
        uint32_t q_phase = 1u;                             // (empty at first)
        bool ok = true;
        RawWork raw;
        int entries = 0;
        if (keys) {
            entries = __ldcg(&plan_header(a.p.plan)->entries);
            raw = fetch_work(a, 0, entries);
        }
        for (int k = 0; ok; ++k) {
            PromptWork w;
            if (keys) {
                w = decode_work(raw);
                if (!(ok = mbar_wait_warp(&sh.work_empty[work_at.slot], work_at.phase ^ 1u, abort_flag, limit))) break;
                if (lane == 0) {
                    int* dst = sh.works + work_at.slot * 10;
                    dst[0] = w.row0; dst[1] = w.pos0; dst[2] = w.tokens; dst[3] = w.b; dst[4] = w.kb0; dst[5] = w.end; dst[6] = w.slot; dst[7] = w.h;
                    dst[8] = w.nb;
                    mbar_arrive(&sh.work_full[work_at.slot]);
                }
                __syncwarp();
                work_at.next();
                if (w.nb == 0) break;
                raw = fetch_work(a, k + 1, entries);       // (on its way while this one's copies are issued)
            } else {
                if (!(ok = see_work(sh, work_at, w, limit))) break;
                done_with_work(sh, work_at, lane);
                if (w.nb == 0) break;
            }
            const int32_t* table = a.p.block_table + (size_t)w.b * a.p.max_blocks_per_seq + w.kb0;
            int held = 0;                                  // 32 entries of the table
            const auto block_of = [&](int i) {
                int blk = __shfl_sync(0xffffffffu, held, i & 31);
                if (blk < 0 || blk >= a.num_blocks) { if (lane == 0) set_status(status, SD_ERR_BOUNDS); blk = 0; }
                return blk;
            };
            for (int j = 0; ok && 2 * j < w.nb; ++j) {
                if ((j & 15) == 0) held = 2 * j + lane < w.nb ? __ldcg(table + 2 * j + lane) : 0;
                const bool two = 2 * j + 1 < w.nb;
                const int y0 = (block_of(2 * j) * a.p.Hkv + w.h) * kBlock, y1 = two ? (block_of(2 * j + 1) * a.p.Hkv + w.h) * kBlock : 0;
                if (!(ok = mbar_wait_warp(&empty[at.slot], at.phase ^ 1u, abort_flag, limit))) break;
                uint8_t* dst = ring + at.slot * kPStage;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&full[at.slot], two ? kPStage : kPStage / 2);
                    tma_load_2d(dst, map, 0, y0, &full[at.slot], keep);
                    tma_load_2d(dst + kPHalf, map, 64, y0, &full[at.slot], keep);
                    if (two) {
                        tma_load_2d(dst + kPHalf / 2, map, 0, y1, &full[at.slot], keep);
                        tma_load_2d(dst + kPHalf + kPHalf / 2, map, 64, y1, &full[at.slot], keep);
                    }
                }
                __syncwarp();
                at.next();
                if (j == 0 && keys) {
                    if (!(ok = mbar_wait_warp(sh.q_empty, q_phase, abort_flag, limit))) break;
                    q_phase ^= 1u;
                    if (elect_one()) {
                        mbar_arrive_expect_tx(sh.q_full, (uint32_t)(a.g.tokens * a.g.G) * kD * 2);
                        tma_load_3d(sh.q_smem, &q_map, 0, w.h * a.g.G, w.row0, sh.q_full, once);
                        tma_load_3d(sh.q_smem + kRowTile * 128, &q_map, 64, w.h * a.g.G, w.row0, sh.q_full, once);
                    }
                    __syncwarp();
                }
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
        const uint64_t k_desc = make_smem_desc(smem_u32(sh.k_smem), 16, 1024, 128);
        const uint64_t v_desc = make_smem_desc(smem_u32(sh.v_smem), kPHalf, 1024, 128);   // [key][d]: N (= d) contiguous
        RingAt<kPStages> s_at, o_at;
        RingAt<kPWorks> s_work, o_work;                    // the scores may be two entries ahead of the products with V
        uint32_t q_phase = 0u, o_phase = 1u;
        int s_nb = 0, s_j = 0, o_nb = 0, o_j = 0;          // blocks and next tile of the entry that either is in
        bool ok = true, more = true;
        PromptWork w;
        const auto scores = [&] {
            if (2 * s_j >= s_nb) {
                if (!(ok = see_work(sh, s_work, w, limit))) return;
                s_work.next();
                s_nb = w.nb;
                s_j = 0;
                if (s_nb == 0) { more = false; return; }
                if (!(ok = mbar_wait_warp(sh.q_full, q_phase, abort_flag, limit))) return;
                q_phase ^= 1u;
            }
            if (!(ok = mbar_wait_warp(&sh.k_full[s_at.slot], s_at.phase, abort_flag, limit))) return;
            tc_fence_after_sync();
            const uint64_t kd = k_desc + (uint64_t)(s_at.slot * (kPStage >> 4));
            const uint32_t d = tmem_s + s_at.slot * kPromptTile;
            const uint32_t idesc = 2 * s_j + 1 < s_nb ? idesc_s : idesc_s_half;
            ++s_j;
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < kD / 16; ++k)
                    mma_ss(d, q_desc + (uint64_t)((k >> 2) * ((kRowTile * 128) >> 4) + (k & 3) * 2),
                           kd + (uint64_t)((k >> 2) * (kPHalf >> 4) + (k & 3) * 2), idesc, k != 0 ? 1u : 0u);
                mma_commit(&sh.s_full[s_at.slot]);
                if (2 * s_j >= s_nb) mma_commit(sh.q_empty);
            }
            __syncwarp();
            s_at.next();
        };
        scores();
        if (ok && more) scores();
        while (ok) {
            // scores two tiles ahead: their buffer held the weights of the tile before this one, whose product was issued before
            if (more) scores();
            if (!ok) break;
            if (2 * o_j >= o_nb) {
                if (o_nb) done_with_work(sh, o_work, lane);
                if (!(ok = see_work(sh, o_work, w, limit))) break;
                o_nb = w.nb;
                o_j = 0;
                if (o_nb == 0) break;
                if (!(ok = mbar_wait_warp(sh.o_empty, o_phase, abort_flag, limit))) break;      // the entry before has left O
                o_phase ^= 1u;
            }
            if (!(ok = mbar_wait_warp(&sh.p_full[o_at.slot], o_at.phase, abort_flag, limit))) break;
            if (!(ok = mbar_wait_warp(&sh.v_full[o_at.slot], o_at.phase, abort_flag, limit))) break;
            tc_fence_after_sync();
            const uint64_t vd = v_desc + (uint64_t)(o_at.slot * (kPStage >> 4));
            const uint32_t pa = tmem_s + o_at.slot * kPromptTile;                      // 16 keys = 8 columns
            const uint32_t first = o_j ? 1u : 0u;
            const bool two = 2 * o_j + 1 < o_nb;
            ++o_j;
            if (elect_one()) {
#pragma unroll
                for (int i = 0; i < 4; ++i) mma_ts(tmem, pa + i * 8, vd + (uint64_t)(i * (2048 >> 4)), idesc_o, i ? 1u : first);
                if (two) {
#pragma unroll
                    for (int i = 4; i < 8; ++i) mma_ts(tmem, pa + i * 8, vd + (uint64_t)(i * (2048 >> 4)), idesc_o, 1u);
                }
                mma_commit(&sh.v_empty[o_at.slot]);
                if (2 * o_j >= o_nb) mma_commit(sh.o_full);
            }
            __syncwarp();
            o_at.next();
        }
        if (elect_one()) mma_commit(sh.unwound);
        __syncwarp();
        if (!ok && lane == 0) set_status(status, SD_ERR_TIMEOUT);
        mbar_wait_plain(sh.unwound, 0, limit);             // (nothing gives tensor memory back while a product runs)
        if (!ok) unwind_pause();
    } else if (warp < 8) {
        // ------------------------------------------------------------ soft-max: one thread per row and group
        const int group = warp >> 2, quad = warp & 3;
        const int r = quad * 32 + lane;                    // TMEM lane, row of the tile
        const int token = a.g.token_of(r);
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint64_t scale2 = twice(a.scale_log2);
        uint64_t* const commit = &sh.commit[quad];
        RingAt<kPStages> at;                               // the stream's next tile
        RingAt<kPWorks> work_at;
        uint32_t n = 0, entry = 0;                         // tiles and entries so far
        bool ok = true;
        while (ok) {
            PromptWork w;
            if (!(ok = see_work(sh, work_at, w, limit))) break;
            done_with_work(sh, work_at, lane);
            if (w.nb == 0) break;
            const bool row_ok = token < w.tokens;
            const int seen = row_ok ? w.pos0 + token + 1 - w.kb0 * kBlock : 0x7fffffff;     // keys from kb0 on that this row sees
            const int all_see = min(w.pos0 + 1 - w.kb0 * kBlock, w.nb * kBlock);            // ... that every row of the tile sees
            const int filled = w.end - w.kb0 * kBlock;     // ... that have been written
            volatile float* const my_ref = sh.refs + (entry & 1) * kRowTile + r;
            uint64_t* const ref_full = sh.ref_full + (entry & 1) * 4 + quad;
            const int nt = w.tiles();
            RowState st{0.f, 0.f, 1.f, 1, 1};
            for (int j = 0; j < nt; ++j, ++n, at.next()) {
                if ((int)(n & 1u) != group) continue;
                const uint32_t ts = tmem_s + lanes + at.slot * kPromptTile;
                if (j == 1) {                              // the reference that the other group found in the first tile
                    if (!(ok = mbar_wait_warp(ref_full, (entry >> 1) & 1u, abort_flag, limit))) break;
                    st.m = *my_ref;
                    st.usual = !__any_sync(0xffffffffu, !(fabsf(st.m) < 2097152.f));
                }
                if (!(ok = mbar_wait_warp(&sh.s_full[at.slot], at.phase, abort_flag, limit))) break;
                tc_fence_after_sync();
                int hb = 0;                                // blocks that are done
                st.raised = 1.f;
                if (j > 0 && all_see >= (j + 1) * kPromptTile && st.usual) {
                    // ---------------------------------------- the usual tile: all keys are visible
                    uint32_t ra[32], rb[32], pk[32];
                    const auto out_of_range = [&](float psum, float lo, float hi) {
                        return row_ok && (!(psum <= kSumLimit) || lo < kShift - 126.f || hi > kShift + 126.f);
                    };
                    uint64_t ps[2] = {0ull, 0ull};
                    float lo = kShift, hi = kShift;
                    tmem_ld32(ts, ra);
                    tmem_ld_wait();
                    tmem_ld32(ts + 32, rb);                // (the next scores are on their way)
                    exp_block(ra, scale2, st.m, pk, ps, lo, hi);
                    tmem_ld_wait();
                    tmem_ld32(ts + 64, ra);
                    exp_block(rb, scale2, st.m, pk + 16, ps, lo, hi);
                    float psum = sum_f32x2(add_f32x2(ps[0], ps[1]));
                    // the tile before is final, and its reference still the one used here
                    if (!(ok = mbar_wait_warp(commit, (n - 1u) & 1u, abort_flag, limit))) break;
                    if (!__any_sync(0xffffffffu, out_of_range(psum, lo, hi) || *my_ref != st.m)) {
                        tmem_st32(ts, pk);                 // over scores that have been read
                        st.l += psum;
                        hb = 1;
                        ps[0] = ps[1] = 0ull;
                        tmem_ld_wait();
                        tmem_ld32(ts + 96, rb);
                        exp_block(ra, scale2, st.m, pk, ps, lo, hi);
                        tmem_ld_wait();
                        exp_block(rb, scale2, st.m, pk + 16, ps, lo, hi);
                        psum = sum_f32x2(add_f32x2(ps[0], ps[1]));
                        if (!__any_sync(0xffffffffu, out_of_range(psum, lo, hi))) {
                            tmem_st32(ts + 32, pk);
                            st.l += psum;
                            hb = 2;
                        }
                    }
                }
                const int blocks = 2 * j + 1 == w.nb ? 1 : 2;
                if (hb < blocks) {
                    // V rows behind the request's last token carry weight 0, but 0 x NaN would still reach O: cleared before P.V reads them
                    if (filled < j * kPromptTile + blocks * kBlock) {
                        if (!(ok = mbar_wait_warp(&sh.v_full[at.slot], at.phase, abort_flag, limit))) break;
                        if (r >= filled - j * kPromptTile) {
                            uint4* z = reinterpret_cast<uint4*>(sh.v_smem + at.slot * kPStage + r * 128);
#pragma unroll
                            for (int c = 0; c < 8; ++c) z[c] = z[c + kPHalf / 16] = make_uint4(0, 0, 0, 0);
                            fence_proxy_async_smem();
                        }
                    }
                    const int last = at.slot == 0 ? kPStages - 1 : at.slot - 1;
                    const TileAt t{ts, tmem + lanes, row_ok ? seen - j * kPromptTile : kPromptTile, blocks, j == 0, ref_full, commit, &sh.v_empty[last],
                                   (n - 1u) & 1u, at.slot == 0 ? at.phase ^ 1u : at.phase, n > 0, row_ok};
                    st = careful_tile(st, t, hb, a.scale_log2, my_ref, abort_flag, limit);
                    if (!(ok = st.ok)) break;
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0 && !a.withhold) { mbar_arrive(&sh.p_full[at.slot]); mbar_arrive(commit); }
            }
            if (!ok) break;
            // the entry before has been read (phase entry - 1)
            if (!(ok = mbar_wait_warp(sh.o_empty, (entry & 1u) ^ 1u, abort_flag, limit))) break;
            ++entry;
            const bool has_last = (int)((n - 1u) & 1u) == group;
            if (nt == 1 && !has_last) continue;            // (no tile of the entry was this group's)
            sh.sums[group * kRowTile + r] = st.l;
            if (has_last) sh.raised[r] = st.raised;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.sum_full[group]);
        }
        if (!ok) {
            if (lane == 0) set_status(status, SD_ERR_TIMEOUT);
            unwind_pause();
        }
    } else if (warp < 12) {
        // ------------------------------------------------------------ results: one thread per row
        const int quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const int token = a.g.token_of(r), head = r - token * a.g.G;
        uint32_t phase = 0u, sum_phase[2] = {0u, 0u}, n = 0, entry = 0;
        RingAt<kPWorks> work_at;
        bool ok = true;
        while (ok) {
            PromptWork w;
            if (!(ok = see_work(sh, work_at, w, limit))) break;
            done_with_work(sh, work_at, lane);
            if (w.nb == 0) break;
            const int nt = w.tiles();
            n += (uint32_t)nt;
            const bool row_ok = token < w.tokens;
            // the sum of the last tile's group is relative to the entry's last reference, the other's to the one before that tile
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const bool last = (int)((n - 1u) & 1u) == g;
                if (!ok || (nt == 1 && !last)) continue;
                ok = mbar_wait_warp(&sh.sum_full[g], sum_phase[g], abort_flag, limit);
                sum_phase[g] ^= 1u;
                sum[g] = sh.sums[g * kRowTile + r];
            }
            if (!ok) break;
            const int last = (int)((n - 1u) & 1u);
            const float l = (last ? sum[1] : sum[0]) + (nt > 1 ? (last ? sum[0] : sum[1]) * sh.raised[r] : 0.f);
            const float m = sh.refs[(entry++ & 1) * kRowTile + r];
            if (!(ok = mbar_wait_warp(sh.o_full, phase, abort_flag, limit))) break;
            phase ^= 1u;
            tc_fence_after_sync();
            float* const part = w.slot < 0 ? nullptr : a.partial + (size_t)w.slot * a.g.slot_floats();
            const size_t row = (size_t)(w.row0 + token), h = (size_t)w.h * a.g.G + head;
            __nv_bfloat16* const dst = a.out + row * a.ldo + h * kD;
            const float inv = 1.f / l;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t o[32];
                tmem_ld32(tmem + lanes + c * 32, o);
                tmem_ld_wait();
                if (c == 3) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sh.o_empty);
                }
                if (!row_ok) continue;
                if (part) {                                // [16-byte piece][row]: a warp's stores are whole lines
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
            if (row_ok && part) reinterpret_cast<float2*>(part + (size_t)a.g.rows * kD)[r] = make_float2(m, l);
            if (row_ok && !part && a.lse) a.lse[row * a.p.Hq + h] = (m + log2f(l)) * 0.6931471805599453f;
        }
        if (!ok) {
            if (lane == 0) set_status(status, SD_ERR_TIMEOUT);
            unwind_pause();
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kPKeyWarp) {
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
    const int per = (a.g.rows * 8 + kMergeThreads - 1) / kMergeThreads;        // CTAs of an entry and KV head, at most
    for (int u = blockIdx.x; u < splits * a.p.Hkv * per; u += gridDim.x) {
        const int4 s = __ldcg(reinterpret_cast<const int4*>(list + u / (a.p.Hkv * per)));
        const int h = u / per % a.p.Hkv, rows = s.y * a.g.G, item = u % per * kMergeThreads + (int)threadIdx.x;
        if (item >= rows * 8) continue;
        const int cg = item / rows, r = item - cg * rows;
        const size_t step = a.g.slot_floats() * a.p.Hkv;
        const float* const part = a.partial + (size_t)(s.z + h) * a.g.slot_floats();
        const float* const sums = part + (size_t)a.g.rows * kD + 2 * r;
        const float* const o = part + ((size_t)cg * 4 * a.g.rows + r) * 4;
        float top = -INFINITY;
        for (int c = 0; c < s.w; ++c) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(sums + c * step));
            if (ml.y != 0.f) top = fmaxf(top, ml.x);
        }
        float den = 0.f;
        float4 acc[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c = 0; c < s.w; ++c) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(sums + c * step));
            if (ml.y == 0.f) continue;                     // (no key that the row sees)
            const float f = exp2f(ml.x - top);
            den = fmaf(f, ml.y, den);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(o + (size_t)x * a.g.rows * 4 + c * step));
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
        const int token = a.g.token_of(r);
        const size_t row = (size_t)(s.x + token), head = (size_t)h * a.g.G + (r - token * a.g.G);
        uint4* dst = reinterpret_cast<uint4*>(a.out + row * a.ldo + head * kD + cg * 16);
        dst[0] = make_uint4(u8[0], u8[1], u8[2], u8[3]);
        dst[1] = make_uint4(u8[4], u8[5], u8[6], u8[7]);
        if (cg == 0 && a.lse) a.lse[row * a.p.Hq + head] = (top + log2f(den)) * 0.6931471805599453f;
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
