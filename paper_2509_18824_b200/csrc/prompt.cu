// Causal GQA attention of packed new tokens over the paged cache.  (The first half of this comment says what is done, the second what bounds it.)
//
// out = softmax(scale q . K^T) V over the keys t <= len + i, a pass over the keys with a row's weights relative to one of its first scores
// (see kSumLimit: the reference moves only where a tile's weights add up to more than 2^40, so that no maximum is looked for and nothing
// is rescaled in the usual tile).  Scores, sums and O are in 32 bits.  A weight is rounded to bf16 (half a step, 2^-8) because V is bf16 and both operands
// of a product have one type; sums are of the weights as they were before.  The output is then 0.0023 of its norm off, 0.0016 with its own rounding alone.
// (Weights of few rows as the sum of two bf16: 0.0017, and 32 single tokens 93 instead of 88 us, a prompt's piece beside single tokens 141 instead of 112.)
//
// A CTA per SM works through its part of the plan (prompt_plan.cuh): entries, a row tile of 128 rows - the query heads of a KV head for 128 / G
// tokens - against tiles of 128 keys.  The tiles of all its entries are one stream: the scores of tile g + 2 are computed before the product
// of tile g's weights with V, whatever entries they belong to, in three score buffers of tensor memory beside O.  Weights, in bf16, lie over
// the scores that they come from.  Two groups of four soft-max warps take the tiles in turn; both add to the one O, which works because the
// reference stays (the rare tile that raises it is serialised through a barrier that every tile passes, commit).  Four more warps normalise
// and store an entry's rows while the next one's tiles are under way.
//
// Eight prompts of 4096 tokens (28 query, 4 KV heads): 792 us, 1215 TFLOP/s, in a few calls (at 1.62 GHz); 920 us, 1046 TFLOP/s, in many, because the
// GPU is at its power cap then (1000 W; a large matrix product sustains 1407 TFLOP/s at 1.36 GHz).  A tile of 128 x 128 takes about 1400 cycles of
// which the tensor pipe is busy for 1024: what passes through shared memory (Q, K and V for the products and the copies, 160 KiB) takes 1280, the
// exponentials (four a cycle and quarter of the SM) 1024 of both groups' time.  An entry costs 500 to 1000 cycles beside its tiles, one of a single
// tile 3000 in all, and a CTA's first 8000 (plan, table, first copies).
// Steps, us for those prompts: two row tiles in a CTA that share K and V and wait for each other 935; this stream 892; scores and products
// with V issued by a warp each (eight instructions take 400 cycles to issue) 862; registers moved to the soft-max warps 842; results
// stored eight rows at a time (a row a thread made thirty-two lines of every store and held up the barriers) 816; the tile before waited for
// behind the weights, not half-way, 792.  A quarter to a third of the exponentials as polynomials on the multiply-add units: 2 % off to 8 % on, left out.
#include <atomic>
#include "attention_shared.cuh"
#include "prompt_plan.cuh"

namespace sdv {

namespace {
constexpr int kPThreads = 512;                 // warps 0-3, 4-7 soft-max, 8-11 results, 12 scores, 13 products with V, 14 K and Q copies, 15 V copies
constexpr int kPScoreWarp = 12, kPKeyWarp = 14, kPValueWarp = 15;
constexpr int kPStages = 3;                    // V ring slots, score buffers
constexpr int kPKeyStages = 2, kPQueryStages = 2;          // K ring slots, and entries whose Q is there
constexpr int kPWorks = 3;                     // pieces of work that are known ahead
constexpr int kPHalf = kPromptTile * 128;      // bytes of one D-half of a key tile: [128 keys][64] bf16, swizzled (16 KiB)
constexpr int kPStage = 2 * kPHalf;
constexpr int kPQBytes = 2 * kRowTile * 128;
constexpr int kPBars = 512;                    // barriers, two words and the pieces of work
constexpr int kPSmem = kPQueryStages * kPQBytes + (kPKeyStages + kPStages) * kPStage + kPBars + 5 * kRowTile * 4;
constexpr int kSoftmaxRegs = 152, kOtherRegs = 104;        // registers of a thread of the eight soft-max warps and the eight others, see setmaxnreg
constexpr int kLaunchRegs = 128;               // ... that the launch brings: 8 x 152 + 8 x 104 = 16 x 128
static_assert(kPThreads / 2 * (kSoftmaxRegs + kOtherRegs) <= kPThreads * kLaunchRegs, "");
constexpr int kMergeThreads = 256;

struct PromptShared {
    uint8_t *q_smem, *k_smem, *v_smem;
    uint64_t* k_full;       // [2] TMA -> MMA
    uint64_t* k_empty;      // [2] MMA -> TMA
    uint64_t* v_full;       // [3] TMA -> MMA (and whoever clears V rows)
    uint64_t* s_full;       // [3] MMA -> soft-max: scores of tile g in buffer g % 3
    uint64_t* v_empty;      // [3] MMA -> TMA (and whoever raises a reference): O updated by tile g, V slot g % 3 read
    uint64_t* p_full;       // [3] soft-max -> MMA: weights of tile g written over its scores
    uint64_t* commit;       // [4] per TMEM quadrant: tile g's soft-max is final (phase g)
    uint64_t* ref_full;     // [2][4] per TMEM quadrant: the reference that an entry's first tile sets, entries in turn
    uint64_t* ref_seen;     // [4] per TMEM quadrant: the group without an entry's first tile has read that reference (phase: the entry)
    uint64_t* q_full;       // [2] TMA -> MMA, entries in turn
    uint64_t* q_empty;      // [2] MMA -> TMA: the entry's last scores are there
    uint64_t* o_full;       // MMA -> results: O updated by the entry's last tile
    uint64_t* o_empty;      // results -> MMA, soft-max: O, references and sums have been read
    uint64_t* other_full;   // soft-max group without an entry's last tile -> results (the other group): its sums
    uint64_t* sum_full;     // soft-max group with an entry's last tile -> results: references and sums
    uint64_t* work_full;    // [3] K copies -> the others: a piece of work
    uint64_t* work_empty;   // [3] the others (15 warps) -> K copies: it has been read
    uint64_t* unwound;      // [2] MMA: everything that either warp has issued has completed
    uint32_t* tmem_slot;
    int* abort_flag;
    int* works;             // [3][9]
    float* refs;            // [2][128] reference of a row, entries in turn
    float* others;          // [128] sum of a row over the tiles of the group without the entry's last one
    float2* sums;           // [128] last reference of an entry's row, and its sum

    __device__ __forceinline__ explicit PromptShared(uint8_t* smem) {
        q_smem = smem;
        k_smem = smem + kPQueryStages * kPQBytes;
        v_smem = k_smem + kPKeyStages * kPStage;
        uint64_t* const bars = reinterpret_cast<uint64_t*>(v_smem + kPStages * kPStage);
        uint64_t* at = bars;
        const auto take = [&](int n) { uint64_t* const got = at; at += n; return got; };
        k_full = take(kPKeyStages); k_empty = take(kPKeyStages);
        v_full = take(kPStages); v_empty = take(kPStages); s_full = take(kPStages); p_full = take(kPStages);
        commit = take(4); ref_full = take(8); ref_seen = take(4);
        q_full = take(kPQueryStages); q_empty = take(kPQueryStages);
        o_full = take(1); o_empty = take(1); other_full = take(1); sum_full = take(1);
        work_full = take(kPWorks); work_empty = take(kPWorks); unwound = take(2);
        tmem_slot = reinterpret_cast<uint32_t*>(take(1));
        abort_flag = reinterpret_cast<int*>(tmem_slot) + 1;
        works = reinterpret_cast<int*>(at);
        static_assert((2 * kPKeyStages + 4 * kPStages + 16 + 2 * kPQueryStages + 4 + 2 * kPWorks + 3) * 8 + kPWorks * 36 <= kPBars, "");
        refs = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(bars) + kPBars);
        others = refs + 2 * kRowTile;
        sums = reinterpret_cast<float2*>(others + kRowTile);
    }
    // (one thread)
    __device__ __forceinline__ void init_barriers() const {
        *abort_flag = 0;
        for (int i = 0; i < kPKeyStages; ++i) { mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1); }
        for (int i = 0; i < kPQueryStages; ++i) { mbar_init(&q_full[i], 1); mbar_init(&q_empty[i], 1); }
        for (int i = 0; i < kPStages; ++i) {
            mbar_init(&v_full[i], 1); mbar_init(&s_full[i], 1); mbar_init(&v_empty[i], 1); mbar_init(&p_full[i], 4);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&commit[i], 1); mbar_init(&ref_full[i], 1); mbar_init(&ref_full[4 + i], 1); mbar_init(&ref_seen[i], 1);
        }
        mbar_init(o_full, 1); mbar_init(o_empty, 4);
        mbar_init(other_full, 4); mbar_init(sum_full, 4);
        for (int i = 0; i < kPWorks; ++i) { mbar_init(&work_full[i], 1); mbar_init(&work_empty[i], 15); }
        mbar_init(&unwound[0], 1); mbar_init(&unwound[1], 1);
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

// A piece of work: (a chunk of) an entry for one KV head; nb key blocks from kb0 on (0: there is no more work), slot of its partial result or -1.
struct PromptWork {
    int row0, pos0, tokens, b, kb0, end, slot, h, nb;
    __device__ __forceinline__ int tiles() const { return (nb + 1) / 2; }
};
// This CTA's pieces, one after the other.
struct PromptWalk {
    int e, h, tile;         // the next piece
    int e1, h1, tile1;      // in parts: where this CTA's ends; dealt out: e is the number of the piece, e1 how many there are
    int slot;               // of the next piece, if that is a chunk
    bool dealt, made;       // how; whether sd_prompt_prepare has made the plan of these prompts
    PromptEntry x;          // its entry
    const PromptEntry* list;
    const int* order;
    int round;
    __device__ __forceinline__ static PromptEntry load(const void* from) {
        const int4* src = static_cast<const int4*>(from);
        const int4 u = __ldcg(src), v = __ldcg(src + 1);
        return PromptEntry{u.x, u.y, u.z, u.w, v.x, v.y, 0, 0};
    }
    __device__ __forceinline__ void begin(const PromptArgs& a) {
        const int4 head = __ldcg(reinterpret_cast<const int4*>(plan_header(a.p.plan)));
        const int entries = head.y;
        const PromptStart* s = plan_starts(a.p.plan) + blockIdx.x;
        const int4 u = __ldcg(reinterpret_cast<const int4*>(s)), v = __ldcg(reinterpret_cast<const int4*>(s + 1));
        x = load(&s->entry);                               // (within the plan whatever stands there)
        list = plan_entries(a.p.plan, a.g.sms);
        order = plan_order(plan_entries(a.p.plan, a.g.sms), a.g.cap);
        made = head.z == plan_stamp(a.p, a.g);
        if (!made) {                                       // (nothing of it is looked at)
            dealt = false;
            e = e1 = h = h1 = tile = tile1 = 0;
            return;
        }
        dealt = entries > 0;
        e = u.x; h = u.y; tile = u.z;
        e1 = v.x; h1 = v.y; tile1 = v.z;
        slot = 2 * (int)blockIdx.x;
        if (dealt) {
            round = tile = 0;
            e1 = entries * a.p.Hkv;                        // (below 2^31: 2^24 rows of 1024 heads at most, 16 or more tokens to a row tile)
            e = (int)blockIdx.x;                           // (its entry stands in the start)
        }
    }
    __device__ __forceinline__ void fetch(int Hkv) {
        x = load(list + __ldcg(order + e / Hkv));
        h = e % Hkv;
    }
    __device__ __forceinline__ PromptWork next(int Hkv) {
        PromptWork w{x.row0, x.pos0, x.tokens, x.b, 2 * tile, x.end, -1, h, 0};
        if (dealt) {
            if (e >= e1) return w;
            w.nb = x.blocks;
            ++round;
            const long long i = (long long)round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
            e = (int)min(i, (long long)e1);
            if (e < e1) fetch(Hkv);                        // (on its way while this piece's copies are issued)
            return w;
        }
        const bool last = e == e1 && h == h1;
        if (e > e1 || (e == e1 && h > h1) || (last && tile >= tile1)) return w;
        const int kb1 = last ? 2 * tile1 : x.blocks;
        w.nb = kb1 - w.kb0;
        if (w.kb0 > 0 || kb1 < x.blocks) w.slot = slot;
        slot = 2 * (int)blockIdx.x + 1;
        tile = 0;
        if (++h == Hkv) {
            h = 0;
            ++e;
            if (e < e1 || (e == e1 && (h1 > 0 || tile1 > 0))) x = load(list + e);
        }
        return w;
    }
};
// The next piece of work, for every warp but the one that hands them out; false: a wait ran out.  done_with_work: it has been read.
__device__ __forceinline__ bool see_work(const PromptShared& sh, const RingAt<kPWorks>& at, PromptWork& w, long long limit) {
    if (!mbar_wait_warp(&sh.work_full[at.slot], at.phase, sh.abort_flag, limit)) return false;
    const volatile int* src = sh.works + at.slot * 9;
    w.row0 = src[0]; w.pos0 = src[1]; w.tokens = src[2]; w.b = src[3]; w.kb0 = src[4]; w.end = src[5]; w.slot = src[6]; w.h = src[7];
    w.nb = src[8];
    return true;
}
__device__ __forceinline__ void done_with_work(const PromptShared& sh, RingAt<kPWorks>& at, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.work_empty[at.slot]);
    at.next();
}

__device__ __forceinline__ uint64_t twice(float c) { return pack_f32x2(c, c); }
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_bf16x2(uint64_t a) {
    float lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a));
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// What the soft-max of a row hands from tile to tile.
struct RowState {
    float m, l;             // reference (a whole number) and sum of the weights relative to it
    float raised;           // what this tile has scaled the row by
    int ok;                 // no wait ran out
};
struct TileAt {
    uint32_t ts, to;        // scores (and weights) and O in tensor memory, at this warp's lanes
    int vis;                // keys of the tile that this row sees
    int blocks;             // of 64 keys, 1 or 2
    int first;              // the first tile of an entry
    uint64_t* hold;         // what a reference is raised behind: O updated by the tile before; for an entry's first tile, if it has more: its
    uint32_t hold_phase;    // reference read by the other group, which would otherwise see it before or after, as it happens
    int row_ok;
};
// A tile whose blocks in front of hb have been weighed (the tile before it is final).  Those get the reference that another tile has raised
// since; the others are looked at before they are weighed, and references raised where they have to be (to the largest score, where that is more than
// 2^32 above).  (A call: in line it made the usual tile's code slower.)
__device__ __noinline__ RowState careful_tile(RowState st, const TileAt t, int hb, float scale_log2, volatile float* my_ref, int* abort_flag,
                                              long long limit) {
    const uint64_t scale2 = twice(scale_log2);
    const auto scale_weights = [&](int block, float by) {
        uint32_t o[32];
        tmem_ld32(t.ts + block * 32, o);
        tmem_ld_wait();
#pragma unroll
        for (int x = 0; x < 32; ++x) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(bf16lo(o[x]) * by, bf16hi(o[x]) * by);
            o[x] = *reinterpret_cast<const uint32_t*>(&h);
        }
        tmem_st32(t.ts + block * 32, o);
        tmem_st_wait();
    };
    tmem_st_wait();
    const float ref = t.row_ok ? *my_ref : st.m;
    if (__any_sync(0xffffffffu, ref != st.m)) {            // (by whole powers of two: the weights' digits stay)
        const float by = ref != st.m ? exp2f(st.m - ref) : 1.f;
#pragma unroll 1
        for (int i = 0; i < hb; ++i) scale_weights(i, by);
        st.l *= by;
        st.m = ref;
    }
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
        const bool raise = mt > st.m + kRaiseAbove;
        if (__any_sync(0xffffffffu, raise)) {
            const float alpha = raise ? exp2f(st.m - mt) : 1.f;                // (a power of two: weights of the first block stay exact)
            if (t.hold && !mbar_wait_warp(t.hold, t.hold_phase, abort_flag, limit)) { st.ok = 0; return st; }
            if (!t.first) {                                // (nothing has been added to O before an entry's first tile)
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
            if (hb > 0) scale_weights(0, alpha);
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

    bool ok = true;                                        // no wait has run out
    if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == kPKeyWarp || warp == kPValueWarp) {
            // ------------------------------------------------------------ copies (whole warps in uniform control flow)
            const bool keys = warp == kPKeyWarp;
            const CUtensorMap* const map = keys ? &k_map : &v_map;
            uint8_t* const ring = keys ? sh.k_smem : sh.v_smem;
            uint64_t *const full = keys ? sh.k_full : sh.v_full, *const empty = keys ? sh.k_empty : sh.v_empty;
            const int stages = keys ? kPKeyStages : kPStages;
            const uint64_t keep = policy_evict_last(), once = policy_evict_first();
            int slot = 0;                                      // of the next K or V
            uint32_t slot_phase = 1u;                          // (empty at first)
            RingAt<kPQueryStages> q_at;
            RingAt<kPWorks> work_at;
            PromptWalk walk;
            if (keys) walk.begin(a);
            if (keys && !walk.made && lane == 0) set_status(status, SD_ERR_INVALID_ARG);
            while (ok) {
                PromptWork w;
                if (keys) {
                    w = walk.next(a.p.Hkv);
                    if (!(ok = mbar_wait_warp(&sh.work_empty[work_at.slot], work_at.phase ^ 1u, abort_flag, limit))) break;
                    if (lane == 0) {
                        int* dst = sh.works + work_at.slot * 9;
                        dst[0] = w.row0; dst[1] = w.pos0; dst[2] = w.tokens; dst[3] = w.b; dst[4] = w.kb0; dst[5] = w.end; dst[6] = w.slot; dst[7] = w.h;
                        dst[8] = w.nb;
                        mbar_arrive(&sh.work_full[work_at.slot]);
                    }
                    __syncwarp();
                    work_at.next();
                    if (w.nb == 0) break;
                } else {
                    if (!(ok = see_work(sh, work_at, w, limit))) break;
                    done_with_work(sh, work_at, lane);
                    if (w.nb == 0) break;
                }
                const uint64_t hint = w.tokens * a.g.G <= 16 ? once : keep;
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
                    if (!(ok = mbar_wait_warp(&empty[slot], slot_phase, abort_flag, limit))) break;
                    uint8_t* dst = ring + slot * kPStage;
                    if (elect_one()) {
                        mbar_arrive_expect_tx(&full[slot], two ? kPStage : kPStage / 2);
                        tma_load_2d(dst, map, 0, y0, &full[slot], hint);
                        tma_load_2d(dst + kPHalf, map, 64, y0, &full[slot], hint);
                        if (two) {
                            tma_load_2d(dst + kPHalf / 2, map, 0, y1, &full[slot], hint);
                            tma_load_2d(dst + kPHalf + kPHalf / 2, map, 64, y1, &full[slot], hint);
                        }
                    }
                    __syncwarp();
                    if (++slot == stages) { slot = 0; slot_phase ^= 1u; }
                    if (j == 0 && keys) {
                        if (!(ok = mbar_wait_warp(&sh.q_empty[q_at.slot], q_at.phase ^ 1u, abort_flag, limit))) break;
                        if (elect_one()) {
                            uint8_t* to = sh.q_smem + q_at.slot * kPQBytes;
                            mbar_arrive_expect_tx(&sh.q_full[q_at.slot], (uint32_t)(a.g.tokens * a.g.G) * kD * 2);
                            tma_load_3d(to, &q_map, 0, w.h * a.g.G, w.row0, &sh.q_full[q_at.slot], once);
                            tma_load_3d(to + kRowTile * 128, &q_map, 64, w.h * a.g.G, w.row0, &sh.q_full[q_at.slot], once);
                        }
                        __syncwarp();
                        q_at.next();
                    }
                }
            }
        } else {                                               // warps 12 and 13
            // ------------------------------------------------------------ products (whole warps in uniform control flow, one lane elected around
            // the instructions).  Eight instructions take about 400 cycles to issue, so that one warp for both products was what the others
            // waited for.
            const bool is_scores = warp == kPScoreWarp;
            RingAt<kPStages> at;
            RingAt<kPKeyStages> k_at;
            RingAt<kPQueryStages> q_at;
            RingAt<kPWorks> work_at;
            uint32_t entry_phase = 1u;
            while (ok) {
                PromptWork w;
                if (!(ok = see_work(sh, work_at, w, limit))) break;
                done_with_work(sh, work_at, lane);
                if (w.nb == 0) break;
                // Q is there; or the entry before has left O
                if (!(ok = is_scores ? mbar_wait_warp(&sh.q_full[q_at.slot], q_at.phase, abort_flag, limit) : mbar_wait_warp(sh.o_empty, entry_phase, abort_flag, limit))) break;
                entry_phase ^= 1u;
                // Products of 64 rows have sixteen in each TMEM quadrant: the first sixteen lie where they do in those of 128.  (Under the power cap what
                // idle rows do costs time: 32 single tokens behind 512 to 16384 100.2 us at 1.46 GHz, 96.7 at 1.64.)
                const bool few = w.tokens * a.g.G <= 16;
                if (is_scores) {
                    const uint32_t idesc_s = make_idesc_bf16(few ? 64 : kRowTile, kPromptTile, false, false), idesc_half = make_idesc_bf16(few ? 64 : kRowTile, kBlock, false, false);
                    const uint64_t q_desc = make_smem_desc(smem_u32(sh.q_smem + q_at.slot * kPQBytes), 16, 1024, 128);
                    const uint64_t k_desc = make_smem_desc(smem_u32(sh.k_smem), 16, 1024, 128);
                    for (int j = 0; 2 * j < w.nb; ++j) {
                        if (!(ok = mbar_wait_warp(&sh.k_full[k_at.slot], k_at.phase, abort_flag, limit))) break;
                        // the buffer held the weights of three tiles before
                        if (!(ok = mbar_wait_warp(&sh.v_empty[at.slot], at.phase ^ 1u, abort_flag, limit))) break;
                        tc_fence_after_sync();
                        const uint64_t kd = k_desc + (uint64_t)(k_at.slot * (kPStage >> 4));
                        const uint32_t d = tmem_s + at.slot * kPromptTile;
                        const uint32_t idesc = 2 * j + 1 < w.nb ? idesc_s : idesc_half;
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kD / 16; ++k)
                                mma_ss(d, q_desc + (uint64_t)((k >> 2) * ((kRowTile * 128) >> 4) + (k & 3) * 2),
                                       kd + (uint64_t)((k >> 2) * (kPHalf >> 4) + (k & 3) * 2), idesc, k != 0 ? 1u : 0u);
                            mma_commit(&sh.s_full[at.slot]);
                            mma_commit(&sh.k_empty[k_at.slot]);
                            if (2 * (j + 1) >= w.nb) mma_commit(&sh.q_empty[q_at.slot]);
                        }
                        __syncwarp();
                        at.next();
                        k_at.next();
                    }
                    q_at.next();
                } else {
                    const uint32_t idesc_o = make_idesc_bf16(few ? 64 : kRowTile, kD, false, true);
                    const uint64_t v_desc = make_smem_desc(smem_u32(sh.v_smem), kPHalf, 1024, 128);   // [key][d]: N (= d) contiguous
                    for (int j = 0; 2 * j < w.nb; ++j) {
                        if (!(ok = mbar_wait_warp(&sh.v_full[at.slot], at.phase, abort_flag, limit))) break;
                        if (!(ok = mbar_wait_warp(&sh.p_full[at.slot], at.phase, abort_flag, limit))) break;
                        tc_fence_after_sync();
                        const uint64_t vd = v_desc + (uint64_t)(at.slot * (kPStage >> 4));
                        const uint32_t pa = tmem_s + at.slot * kPromptTile;                // 16 keys = 8 columns
                        const uint32_t first = j ? 1u : 0u;
                        if (elect_one()) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) mma_ts(tmem, pa + i * 8, vd + (uint64_t)(i * (2048 >> 4)), idesc_o, i ? 1u : first);
                            if (2 * j + 1 < w.nb) {
#pragma unroll
                                for (int i = 4; i < 8; ++i) mma_ts(tmem, pa + i * 8, vd + (uint64_t)(i * (2048 >> 4)), idesc_o, 1u);
                            }
                            mma_commit(&sh.v_empty[at.slot]);
                            if (2 * (j + 1) >= w.nb) mma_commit(sh.o_full);
                        }
                        __syncwarp();
                        at.next();
                    }
                }
            }
            uint64_t* const mine = &sh.unwound[is_scores ? 0 : 1];
            if (elect_one()) mma_commit(mine);
            __syncwarp();
            mbar_wait_plain(mine, 0, limit);                   // (nothing gives tensor memory back while a product runs)
        }
    } else if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
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
        while (ok) {
            PromptWork w;
            if (!(ok = see_work(sh, work_at, w, limit))) break;
            done_with_work(sh, work_at, lane);
            if (w.nb == 0) break;
            const bool row_ok = token < w.tokens;
            const bool idle = !__any_sync(0xffffffffu, row_ok);                // (single tokens: three warps of four)
            const int seen = row_ok ? w.pos0 + token + 1 - w.kb0 * kBlock : 0x7fffffff;     // keys from kb0 on that this row sees
            const int all_see = min(w.pos0 + 1 - w.kb0 * kBlock, w.nb * kBlock);            // ... that every row of the tile sees
            const int filled = w.end - w.kb0 * kBlock;     // ... that have been written
            volatile float* const my_ref = sh.refs + (entry & 1) * kRowTile + r;
            uint64_t* const ref_full = sh.ref_full + (entry & 1) * 4 + quad;
            const int nt = w.tiles();
            RowState st{0.f, 0.f, 1.f, 1};
            const int j0 = (int)(n & 1u) ^ group;          // this group's tiles: every second one of the stream
            uint64_t* const ref_seen = sh.ref_seen + quad;
            if (j0 >= nt && lane == 0) mbar_arrive(ref_seen);                  // (nothing to read)
            RingAt<kPStages> s_at = at;
            if (j0) s_at.next();
            for (int j = j0; j < nt; j += 2, s_at.next(), s_at.next()) {
                const uint32_t ts = tmem_s + lanes + s_at.slot * kPromptTile;
                const bool begun = j > 0 || n > 0;         // there is a tile before this one in the stream
                const uint32_t commit_phase = (n + (uint32_t)j - 1u) & 1u;
                if (j == 1) {                              // the reference that the other group found in the first tile
                    if (!(ok = mbar_wait_warp(ref_full, (entry >> 1) & 1u, abort_flag, limit))) break;
                    st.m = *my_ref;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ref_seen);
                }
                if (!(ok = mbar_wait_warp(&sh.s_full[s_at.slot], s_at.phase, abort_flag, limit))) break;
                tc_fence_after_sync();
                const bool masked = all_see < (j + 1) * kPromptTile;           // some row does not see some key (or there is one block)
                int hb = 0, blocks = 2;                    // blocks that are done, of how many
                int vis = kPromptTile;                     // keys of the tile that this row sees
                const auto weigh = [&] {
                    uint32_t ra[32], rb[32], pk[32];
                    uint64_t ps[2] = {0ull, 0ull};
                    tmem_ld32(ts, ra);
                    st.raised = 1.f;
                    tmem_ld_wait();
                    tmem_ld32(ts + 32, rb);                // (the next scores are on their way)
                    if (j == 0) {                          // the reference: the largest of the first 32 scores that the row sees, as a whole number
                        float mt = fmaxf(__uint_as_float(ra[0]), __uint_as_float(ra[1]));
#pragma unroll
                        for (int c = 2; c < 32; c += 2) mt = max3(mt, __uint_as_float(ra[c]), __uint_as_float(ra[c + 1]));
                        st.m = row_ok && mt > -INFINITY ? rintf(mt * a.scale_log2) : 0.f;      // (no key: the row has no weight here)
                        *my_ref = st.m;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(ref_full);
                    }
                    const uint64_t neg_m2 = twice(-st.m);
                    exp_pack(ra, scale2, neg_m2, pk, ps);
                    tmem_ld_wait();
                    if (blocks == 2) tmem_ld32(ts + 64, ra);
                    exp_pack(rb, scale2, neg_m2, pk + 16, ps);
                    float psum = sum_f32x2(add_f32x2(ps[0], ps[1]));
                    tmem_ld_wait();
                    if (__any_sync(0xffffffffu, row_ok && !(psum <= kSumLimit))) return;
                    tmem_st32(ts, pk);                     // over scores that have been read
                    st.l += psum;
                    hb = 1;
                    if (blocks == 1) return;
                    ps[0] = ps[1] = 0ull;
                    tmem_ld32(ts + 96, rb);
                    exp_pack(ra, scale2, neg_m2, pk, ps);
                    tmem_ld_wait();
                    exp_pack(rb, scale2, neg_m2, pk + 16, ps);
                    psum = sum_f32x2(add_f32x2(ps[0], ps[1]));
                    if (__any_sync(0xffffffffu, row_ok && !(psum <= kSumLimit))) return;
                    tmem_st32(ts + 32, pk);
                    st.l += psum;
                    hb = 2;
                };
                if (masked || idle) {
                    vis = row_ok ? seen - j * kPromptTile : kPromptTile;
                    blocks = 2 * j + 1 == w.nb ? 1 : 2;
                    // V rows behind the request's last token carry weight 0, but 0 x NaN would still reach O: cleared before P.V reads them
                    if (filled < j * kPromptTile + blocks * kBlock) {
                        if (!(ok = mbar_wait_warp(&sh.v_full[s_at.slot], s_at.phase, abort_flag, limit))) break;
                        if (r >= filled - j * kPromptTile) {
                            uint4* z = reinterpret_cast<uint4*>(sh.v_smem + s_at.slot * kPStage + r * 128);
#pragma unroll
                            for (int c = 0; c < 8; ++c) z[c] = z[c + kPHalf / 16] = make_uint4(0, 0, 0, 0);
                            fence_proxy_async_smem();
                        }
                    }
                    // Hidden scores become -inf where they stand, 32 keys at a time where some row does not see them all.  (Sixteen ragged prompts of
                    // up to 2048 tokens 153 us with the masks in a second copy of what follows, 141 so.)
                    const int c0 = __reduce_min_sync(0xffffffffu, vis) & ~31;
#pragma unroll 1
                    for (int c = max(c0, 0); c < blocks * kBlock; c += 32) {
                        uint32_t x[32];
                        tmem_ld32(ts + c, x);
                        tmem_ld_wait();
                        mask_scores(x, vis >= c + 32 ? ~0u : (1u << max(vis - c, 0)) - 1u);
                        tmem_st32(ts + c, x);
                    }
                    tmem_st_wait();
                }
                if (!idle) weigh();                        // (rows that nobody reads only keep their place among the barriers)
                else {
                    if (j == 0 && lane == 0) mbar_arrive(ref_full);
                    hb = blocks;
                }
                // The tile before is final: is its reference still the one used here?  (Looked at behind the weights, not in front of them, so that the groups
                // wait for one another as little as can be.)
                if (begun && !(ok = mbar_wait_warp(commit, commit_phase, abort_flag, limit))) break;
                if (__any_sync(0xffffffffu, hb < blocks || (row_ok && *my_ref != st.m))) {
                    const int last = s_at.slot == 0 ? kPStages - 1 : s_at.slot - 1;
                    const TileAt t{ts, tmem + lanes, vis, blocks, j == 0, j > 0 ? &sh.v_empty[last] : nt > 1 ? ref_seen : nullptr,
                                   j == 0 ? entry & 1u : s_at.slot == 0 ? s_at.phase ^ 1u : s_at.phase, row_ok};
                    st = careful_tile(st, t, hb, a.scale_log2, my_ref, abort_flag, limit);
                    if (!(ok = st.ok)) break;
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0 && !a.withhold) { mbar_arrive(&sh.p_full[s_at.slot]); mbar_arrive(commit); }
            }
            n += (uint32_t)nt;
            {                                              // at += nt
                const int slot = at.slot + nt % kPStages, rounds = nt / kPStages + (slot >= kPStages ? 1 : 0);
                at.slot = slot >= kPStages ? slot - kPStages : slot;
                at.phase ^= (uint32_t)(rounds & 1);
            }
            if (!ok) break;
            // Both groups leave their sums.  The other's is relative to the reference in front of the last tile: where that tile has raised it, the last
            // tile's group adds them up itself.  Every warp waits here for the entry before to have been read, and reports, whether it had a
            // tile of this one or not: nobody is ever two phases away from these barriers, whose waits tell only odd phases from even ones.
            const bool has_last = (int)((n - 1u) & 1u) == group, both = nt > 1;
            const uint32_t phase = entry & 1u;
            ++entry;
            if (!(ok = mbar_wait_warp(sh.o_empty, phase ^ 1u, abort_flag, limit))) break;
            if (!has_last) sh.others[r] = both ? st.l : 0.f;
            if (has_last && __any_sync(0xffffffffu, both && st.raised != 1.f)) {
                if (!(ok = mbar_wait_warp(sh.other_full, phase, abort_flag, limit))) break;
                st.l = fmaf(sh.others[r], st.raised, st.l);
                sh.others[r] = 0.f;
            }
            if (has_last) sh.sums[r] = make_float2(st.m, st.l);
            __syncwarp();
            if (lane == 0) mbar_arrive(has_last ? sh.sum_full : sh.other_full);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        // ------------------------------------------------------------ results: one thread per row
        const int quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const int token = a.g.token_of(r), head = r - token * a.g.G;
        uint32_t phase = 0u;
        RingAt<kPWorks> work_at;
        while (ok) {
            PromptWork w;
            if (!(ok = see_work(sh, work_at, w, limit))) break;
            done_with_work(sh, work_at, lane);
            if (w.nb == 0) break;
            const bool row_ok = token < w.tokens;
            if (!(ok = mbar_wait_warp(sh.sum_full, phase, abort_flag, limit))) break;
            if (!(ok = mbar_wait_warp(sh.other_full, phase, abort_flag, limit))) break;
            const float m = sh.sums[r].x, l = sh.sums[r].y + sh.others[r];
            if (!(ok = mbar_wait_warp(sh.o_full, phase, abort_flag, limit))) break;
            phase ^= 1u;
            tc_fence_after_sync();
            float* const part = w.slot < 0 ? nullptr : a.partial + (size_t)w.slot * a.g.slot_floats();
            const size_t row = (size_t)(w.row0 + token), h = (size_t)w.h * a.g.G + head;
            const float inv = 1.f / l;
            const auto leave = [&] {                       // O has been read: the next entry's first product waits for this
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(sh.o_empty);
            };
            if (part) {
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tmem + lanes + c * 32, o);
                    tmem_ld_wait();
                    if (c == 3) leave();
                    if (!row_ok) continue;
#pragma unroll
                    for (int x = 0; x < 8; ++x)            // [16-byte piece][row]: a warp's stores are whole lines
                        reinterpret_cast<uint4*>(part)[(c * 8 + x) * a.g.rows + r] = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
                }
            } else {
                // A row per thread would make 32 lines of every store, whose passes through the load-store unit hold up the other warps' barriers;
                // so the rows go back to tensor memory in bf16, over columns of O that have been read, and are loaded as eight rows of 32 bytes.
                // (Transposed among four threads instead, with 64 shuffles: 140 us for those prompts, 136 so.  Leaving O with all of it in registers: 153,
                // the soft-max warps spill.)
                const uint64_t inv2 = twice(inv);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[32], pk[16];
                    tmem_ld32(tmem + lanes + c * 32, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int x = 0; x < 16; ++x) pk[x] = pack_bf16x2(mul_f32x2(pack_f32x2(__uint_as_float(o[2 * x]), __uint_as_float(o[2 * x + 1])), inv2));
                    tmem_st16(tmem + lanes + c * 16, pk);
                }
                tmem_st_wait();
                const int q4 = lane & 3;
#pragma unroll
                for (int up = 0; up < 2; ++up) {           // rows 0-15 and 16-31 of the quadrant
                    uint32_t o[2][16];
                    tmem_ld_16x256b_x4(tmem + lanes + ((uint32_t)(up * 16) << 16), o[0]);
                    tmem_ld_16x256b_x4(tmem + lanes + ((uint32_t)(up * 16) << 16) + 32, o[1]);
                    tmem_ld_wait();
                    if (up == 1) leave();
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int rr = quad * 32 + up * 16 + x * 8 + (lane >> 2), t_row = a.g.token_of(rr);
                        if (t_row >= w.tokens) continue;
                        __nv_bfloat16* const to = a.out + (size_t)(w.row0 + t_row) * a.ldo + ((size_t)w.h * a.g.G + (rr - t_row * a.g.G)) * kD + q4 * 4;
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            *reinterpret_cast<uint2*>(to + c * 16) = make_uint2(o[c >> 2][4 * (c & 3) + 2 * x], o[c >> 2][4 * (c & 3) + 2 * x + 1]);
                    }
                }
            }
            if (row_ok && part) reinterpret_cast<float2*>(part + (size_t)a.g.rows * kD)[r] = make_float2(m, l);
            if (row_ok && !part && a.lse) a.lse[row * a.p.Hq + h] = (m + log2f(l)) * 0.6931471805599453f;
        }
    }
    if (!ok) {
        if (lane == 0) set_status(status, SD_ERR_TIMEOUT);
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);  // (as unwind_pause: copies on their way land first; a call would bind every role's registers)
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kPKeyWarp) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

// Joins the chunks of the entries that were cut, in the order of the keys.  A thread takes sixteen columns of a row; sixteen loads are on
// their way together.
__global__ void __launch_bounds__(kMergeThreads)
prompt_merge_kernel(const __grid_constant__ PromptArgs a) {
    begin_dependent();
    const PromptSplit* const list = plan_splits(a.p.plan, a.g.sms);
    const int per = (a.g.rows * 8 + kMergeThreads - 1) / kMergeThreads;        // CTAs of an entry, at most
    int splits = a.g.sms;                                                      // (the most there can be)
    for (int u = blockIdx.x; u < splits * per; u += gridDim.x) {
        const int4* src = reinterpret_cast<const int4*>(list + u / per);
        const int4 s0 = __ldcg(src), s1 = __ldcg(src + 1);
        const int4 of = __ldcg(reinterpret_cast<const int4*>(plan_header(a.p.plan)));
        splits = of.x;
        if (of.z != plan_stamp(a.p, a.g) || u >= splits * per) return;
        const int row0 = s0.x, rows = s0.y * a.g.G, h = s0.z, first = s0.w, cta = s1.x, chunks = s1.y;
        const int item = u % per * kMergeThreads + (int)threadIdx.x;
        if (item >= rows * 8) continue;
        const int cg = item / rows, r = item - cg * rows;
        const auto part = [&](int c) { return a.partial + (size_t)(c == 0 ? first : 2 * (cta + c)) * a.g.slot_floats(); };
        const size_t sums = (size_t)a.g.rows * kD + 2 * r, mine = ((size_t)cg * 4 * a.g.rows + r) * 4, next = (size_t)a.g.rows * 4;
        constexpr int kAhead = 4;
        float top = -INFINITY, den = 0.f;                  // relative to the largest reference so far
        float4 acc[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c0 = 0; c0 < chunks; c0 += kAhead) {
            float2 ml[kAhead];
            float4 v[kAhead][4];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                ml[i] = make_float2(-INFINITY, 0.f);
                if (c0 + i < chunks) {
                    const float* from = part(c0 + i);
                    ml[i] = __ldcg(reinterpret_cast<const float2*>(from + sums));
#pragma unroll
                    for (int x = 0; x < 4; ++x) v[i][x] = __ldcg(reinterpret_cast<const float4*>(from + mine + x * next));
                }
            }
            float high = top;
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (ml[i].y != 0.f) high = fmaxf(high, ml[i].x);               // (0: no key that the row sees)
            if (high == -INFINITY) continue;
            const float scale = exp2f(top - high);
            top = high;
            den *= scale;
#pragma unroll
            for (int x = 0; x < 4; ++x) { acc[x].x *= scale; acc[x].y *= scale; acc[x].z *= scale; acc[x].w *= scale; }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (ml[i].y == 0.f) continue;
                const float f = exp2f(ml[i].x - top);
                den = fmaf(f, ml[i].y, den);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    acc[x].x = fmaf(f, v[i][x].x, acc[x].x); acc[x].y = fmaf(f, v[i][x].y, acc[x].y);
                    acc[x].z = fmaf(f, v[i][x].z, acc[x].z); acc[x].w = fmaf(f, v[i][x].w, acc[x].w);
                }
            }
        }
        const float inv = 1.f / den;
        uint32_t o[8];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const __nv_bfloat162 h0 = __floats2bfloat162_rn(acc[x].x * inv, acc[x].y * inv), h1 = __floats2bfloat162_rn(acc[x].z * inv, acc[x].w * inv);
            o[2 * x] = *reinterpret_cast<const uint32_t*>(&h0);
            o[2 * x + 1] = *reinterpret_cast<const uint32_t*>(&h1);
        }
        const int token = a.g.token_of(r);
        const size_t row = (size_t)(row0 + token), head = (size_t)h * a.g.G + (r - token * a.g.G);
        uint4* dst = reinterpret_cast<uint4*>(a.out + row * a.ldo + head * kD + cg * 16);
        dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
        dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
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
    return ((size_t)2 * g.sms * g.slot_floats() * 4 + 255) & ~(size_t)255;
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
    // (with fewer registers a thread than the split counts on, setmaxnreg would wait for good)
    static std::atomic<int> regs{0};
    if (regs.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes f;
        if (cudaFuncGetAttributes(&f, prompt_kernel) != cudaSuccess) return SD_ERR_CUDA;
        regs.store(f.numRegs, std::memory_order_relaxed);
    }
    if (regs.load(std::memory_order_relaxed) != kLaunchRegs) return SD_ERR_UNSUPPORTED;
    sd_status s = launch_dependent(prompt_kernel, dim3(a.g.sms), kPThreads, kPSmem, 1, st, qm, km, vm, a, dev_status);
    if (s != SD_OK) return s;
    return launch_dependent(prompt_merge_kernel, dim3(4 * a.g.sms), kMergeThreads, 0, 1, st, a);
}

}  // namespace sdv
