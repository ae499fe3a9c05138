// The draft's training loss on rows of logits [M][V] and its gradient (sd_distill_loss, sd_distill_grad).
//
// Memory-bound: a row is read once and, with the gradient, written once.  Persistent clusters of `parts` CTAs take a row at a time,
// each CTA a slice of it, in pieces of 21 KB through a ring of slots.  Fourteen warps sum up the exponentials of a piece; what a row
// needs but once is done by four more, so that it does not stand in their way:
//   copy     issues the pieces' copies as slots become free
//   entries  prepares the next rows' lists: the entries in this CTA's slice, their probabilities
//   pick     takes the listed logits (and the label's) out of a piece that has arrived and puts minus infinity in their place: the others'
//            sums are then those of the rest, without a question per entry (and without the cancellation of a difference)
//   join     brings the warps' sums together, and with stores that report to a barrier the CTAs', and writes the losses
// With the gradient a slice's pieces stay in their slots until the sums are known, the gradient is formed from there, and the next
// row's pieces follow into the slots one by one; the listed entries' gradients (and the label's) are written over the others' afterwards.
// 1024 rows of 152064, K = 64: the loss of bf16 80 us (3.9 TB/s), of f32 124 (5.0 TB/s), loss and gradient of bf16 161 (3.9 TB/s read and
// written), of f32 257 (4.8 TB/s), the gradient alone of bf16 111 (5.6 TB/s), of f32 214 (5.8 TB/s).  The loss of bf16 takes 11 instructions per 32
// entries (the exponentials' pipe at 50 %), its gradient as many again, of which the arithmetic is about four and control the likely rest; f32 is bound by
// HBM, of which the time between a row's last piece and its gradient is lost.  Another temperature than 1 with a label costs a second
// exponential per entry (bf16 129 and 255 us).  The join's code is met once a row and has to stay short: 600 cycles of it more, by the instruction
// caches, took 5 % of the loss.
// (One row per cluster, all warps doing everything, a bitmap of the listed entries: 4096 rows of bf16 790 us, now 640.  Every CTA preparing the
// whole list: no slower at K = 64, but 60 % at K = 427 in short rows.  The exponentials of some entries by a polynomial: slower.)
#include <type_traits>
#include "rows.cuh"

namespace sdv {
namespace rows {

constexpr int kSumWarps = 14;
constexpr int kSumThreads = kSumWarps * 32;
constexpr int kDistillThreads = kSumThreads + 128;
enum { kCopyWarp = kSumWarps, kEntryWarp, kPickWarp, kJoinWarp };
constexpr int kPerThread = 3;
constexpr int kPieceVecs = kPerThread * kSumThreads;       // vectors of a piece
constexpr int kSlots = 5, kMaxSlots = 8;                   // of 21 KB
constexpr int kMaxLists = 4;           // rows whose entries are at hand: as many are prepared ahead
enum { kLoss, kLossGrad, kGrad };      // what a launch computes

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(sm100::smem_u32(dst)), "l"(src), "r"(bytes), "r"(sm100::smem_u32(bar)), "l"(policy) : "memory");
}
// barrier of the fourteen warps, with the disjunction of what they bring
__device__ __forceinline__ bool sum_warps_or(bool v) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}\n"
                 : "=r"(r) : "r"((uint32_t)v), "n"(kSumThreads) : "memory");
    return r != 0;
}

// Exponentials are taken as 2^(x c - R) with R = rint(top c), a whole number: x c - R is one instruction with one rounding (of a small
// number where it matters), and sums with different R are brought together exactly.  R stays above -2^28: what is further down (a
// mask's lowest value, whose R would be minus infinity, and the difference from it NaN) has a power of 0 there.
constexpr double kLn2 = 0.69314718055994530942;
constexpr float kFar = 268435456.f;    // 2^28: up to here 32 bits hold R as near to the logit's power as exponents need
__device__ __forceinline__ float whole_power(float top, float c) { return fmaxf(rintf(top * c), -kFar); }

// What a CTA tells the others of its row: its largest logit and, with its R, the sums of 2^(x c - R) among the entries and of
// 2^(x log2 e - R1); the largest logit outside the entries and, with the R of that, the sum there (a student may be surer of an entry than
// 32 bits have exponents); its entries' sums of p and of p (log p - z c ln 2); the label's logit where it lies in its slice.
struct __align__(16) Message { float top, label, rest, sum1, top_rest, none; double listed, mass, own; };
static_assert(sizeof(Message) == 48, "three stores of 16 bytes");

// A place in the ring of slots and the phase of its barriers
struct Turn {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int slots) { if (++slot == slots) { slot = 0; phase ^= 1u; } }
};

struct RowInfo {                       // prepared ahead
    double mass, plogp;                // sums of p and p log p over them
    float weight, rounding;            // dloss; what top_lse in 32 bits may leave of a p_rest that is 0
    int label, any, count;             // any: the row has entries; count: those that lie in this CTA's slice
};
// What 2^(x c - r_c) is multiplied with at the entries, 2^(x c - r_rest) elsewhere, 2^(x log2 e - r_e) for the cross-entropy, and what
// the list's p are
struct RowFactors { float r_c, r_rest, r_e, listed, tail, one, p; };

struct DistillShared {
    uint64_t full[kMaxSlots], picked[kMaxSlots], free_[kMaxSlots];
    uint64_t info_full[kMaxLists], info_free[kMaxLists], sums_full[kMaxLists], row_ready[2], told[2];
    int abort_flag;
    RowInfo info[kMaxLists];
    float label_z[kMaxLists];
    int dup[kMaxLists], label_listed[kMaxLists];
    float4 sums[2][kSumWarps + 1];     // the warps' (largest logit, sum outside the entries, 0, sum at temperature 1); the entries' last
    double own[2], listed[2];          // sum of p (log p - z c ln 2); the listed entries' sum of 2^(z c - R)
    Message msg[2][8];
    RowFactors row[2];
};

template <typename T>
__device__ __forceinline__ void store_one(void* row, long long v, float g) {
    if constexpr (sizeof(T) == 4) static_cast<float*>(row)[v] = g;
    else static_cast<__nv_bfloat16*>(row)[v] = __float2bfloat16_rn(g);
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&g)[Row<T>::kE]) {
    uint32_t w[4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(g[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(g[2 * e], g[2 * e + 1]);
            w[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}


// RowFactors between two calls, in the four floats that a row has there.  As a rule r_rest is r_c, and that and r_e follow from the row's
// largest logit: (it, listed, tail, one).  Where the entries outside the list lie so far below that their sum has an R of its own (kOwnPower),
// seven numbers in 16 bytes, told by the second one's sign: r_c (r_e at a label and inv_temp < 1; one follows from the other)
// and its distance from r_rest as multiples of 128 in 23 bits each, listed, -tail and one as floats without sign and last four bits (kNoOne:
// no cross-entropy to be had).  Any R near a logit's power will do, with the factors adjusted.
constexpr float kOwnPower = 64.f;      // up to here r_c serves both: factors reach 2^64, what is lost is below 2^-62 of p_rest
constexpr float kStepR = 128.f;
constexpr uint32_t kNoOne = 0x7ffffffu;
__device__ __forceinline__ uint32_t short_float(float x) { return ((__float_as_uint(x) & 0x7fffffffu) + 8u) >> 4; }
__device__ __forceinline__ float long_float(uint32_t u) { return __uint_as_float((u & 0x7ffffffu) << 4); }
__device__ __forceinline__ void stats_powers(float step, bool by_e, float inv_temp, float& r_c, float& r_e) {
    const float r = step * kStepR;
    r_c = by_e ? rintf(r * inv_temp) : r;
    r_e = by_e ? r : rintf(__fdividef(r, inv_temp));
}
__device__ __noinline__ float4 pack_stats(const RowFactors& rf, bool by_e, float inv_temp) {
    const bool none = rf.one != rf.one;
    by_e = by_e && !none;
    const float step = rintf((by_e ? rf.r_e : rf.r_c) / kStepR);
    float r_c, r_e;
    stats_powers(step, by_e, inv_temp, r_c, r_e);
    const int down = (int)rintf((r_c - rf.r_rest) / kStepR);
    const float r_rest = r_c - (float)down * kStepR;
    const uint32_t listed = short_float(rf.listed * ex2(r_c - rf.r_c)), tail = short_float(fmaxf(-rf.tail, 0.f) * ex2(r_rest - rf.r_rest)),
                   one = none ? kNoOne : short_float(rf.one * ex2(r_e - rf.r_e)), at = (uint32_t)(int)step & 0x7fffffu, d = (uint32_t)down;
    return make_float4(__uint_as_float(listed | d << 27), __uint_as_float(0x80000000u | tail | (d >> 5 & 15u) << 27),
                       __uint_as_float(one | (d >> 9 & 31u) << 27), __uint_as_float(at | (d >> 14) << 23));
}
__device__ __forceinline__ RowFactors unpack_stats(const float4& st, bool by_e, float inv_temp) {
    const uint32_t a = __float_as_uint(st.x), b = __float_as_uint(st.y), e = __float_as_uint(st.z), w = __float_as_uint(st.w);
    RowFactors rf{0.f, 0.f, 0.f, st.y, st.z, st.w, 1.f};
    if (!(b >> 31)) {
        rf.r_c = rf.r_rest = whole_power(st.x, inv_temp * kLog2e);
        rf.r_e = whole_power(st.x, kLog2e);
        return rf;
    }
    stats_powers((float)((int)(w << 9) >> 9), by_e && (e & kNoOne) != kNoOne, inv_temp, rf.r_c, rf.r_e);
    rf.r_rest = rf.r_c - (float)(a >> 27 | (b >> 27 & 15u) << 5 | e >> 27 << 9 | w >> 23 << 14) * kStepR;
    rf.listed = long_float(a);
    rf.tail = -long_float(b);
    rf.one = long_float(e);
    return rf;
}

// Gradient factors of a row, with dloss and the weights: an entry x outside the list gets tail * 2^(x c - r_rest) + one *
// 2^(x log2 e - r_e), at temperature 1 in one term.
struct Factors {
    float r_c, r_rest, r_e, c;
    float listed, tail, one;           // `listed` stands for `tail`, and r_c for r_rest, at the listed entries
    float per_p, per_label;            // what a listed entry's p, and the label, take away
    bool two;
    __device__ __forceinline__ Factors(const DistillCall& a, const RowFactors& rf, float g, bool has_label) {
        c = a.inv_temp * kLog2e;
        r_c = rf.r_c;
        r_rest = rf.r_rest;
        r_e = rf.r_e;
        per_p = g * a.kl_weight * a.inv_temp;
        listed = per_p * rf.listed;
        tail = per_p * rf.tail;
        per_p *= rf.p;
        per_label = has_label ? g * a.ce_weight : 0.f;
        one = per_label != 0.f ? per_label * rf.one : 0.f;
        two = a.inv_temp != 1.f && one != 0.f;
        if (!two) { listed += one; tail += one * ex2(r_rest - r_c); }
    }
    __device__ __forceinline__ float at(float x, float factor, float r) const {
        const float e = factor * ex2(fmaf(x, c, -r));
        return two ? fmaf(one, ex2(fmaf(x, kLog2e, -r_e)), e) : e;
    }
    template <typename T, bool TWO>
    __device__ __forceinline__ void vector(const uint4& raw, float (&g)[Row<T>::kE]) const {
        Pair x[Row<T>::kE / 2];
        Row<T>::pairs(raw, x);
#pragma unroll
        for (int e = 0; e < Row<T>::kE / 2; ++e) {
            const Pair w = ex2(fma2(x[e], Pair{c, c}, Pair{-r_rest, -r_rest}));
            Pair o{tail * w.x, tail * w.y};
            if constexpr (TWO) o = fma2(Pair{one, one}, ex2(fma2(x[e], Pair{kLog2e, kLog2e}, Pair{-r_e, -r_e})), o);
            g[2 * e] = o.x;
            g[2 * e + 1] = o.y;
        }
    }
};

// One row's slice as a CTA sees it
template <typename T>
struct SliceOf {
    static constexpr int E = Row<T>::kE;
    Row<T> row;
    int v0, v1, first, pieces;         // vectors [v0, v1); index in the row of the first one's first entry (negative where the row starts inside it)
    __device__ __forceinline__ SliceOf(const DistillCall& a, long long r, int rank, int per) : row(a.logits, a.ld, r, a.V) {
        v0 = min(row.nvec, rank * per);
        v1 = min(row.nvec, v0 + per);
        first = v0 * E - row.lead;
        pieces = (v1 - v0 + kPieceVecs - 1) / kPieceVecs;
    }
};

// Lists of one row in shared memory, the entries in this CTA's slice: probabilities, logits, places in the slice (with kAgain: a place
// that another entry of the list has too, and answers for)
constexpr int kAgain = 1 << 30;
struct Lists { double* p; float* z; int* at; };

// A row's list as it lies in memory, the lane's first two entries of it (the others are loaded when they are needed)
struct RawList {
    const float* val;
    const int32_t* idx;
    int label, i0, i1;
    float weight, t_lse, t0, t1;
    __device__ __forceinline__ RawList(const DistillCall& a, long long r) : val(a.top_val + r * a.K), idx(a.top_idx + r * a.K) {
        const int lane = threadIdx.x & 31;
        i0 = lane < a.K ? __ldcg(idx + lane) : -1;
        t0 = lane < a.K ? __ldcg(val + lane) : 0.f;
        i1 = lane + 32 < a.K ? __ldcg(idx + lane + 32) : -1;
        t1 = lane + 32 < a.K ? __ldcg(val + lane + 32) : 0.f;
        label = a.label ? __ldcg(a.label + r) : -1;
        weight = a.dloss ? __ldcg(a.dloss + r) : 1.f;
        t_lse = a.top_lse ? __ldcg(a.top_lse + r) : 0.f;
    }
    // the entries from the 65th on, into the list's place (the lists in shared memory are written from their front, behind what is read)
    __device__ __forceinline__ void stage(const Lists& li, int K) const {
        const int lane = threadIdx.x & 31;
        for (int k0 = 64 + lane; k0 < K; k0 += 128) {
            int i[4];
            float t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = k0 + 32 * j;
                i[j] = k < K ? __ldcg(idx + k) : -1;
                t[j] = k < K ? __ldcg(val + k) : 0.f;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k0 + 32 * j < K) { li.at[k0 + 32 * j] = i[j]; li.z[k0 + 32 * j] = t[j]; }
        }
        __syncwarp();
    }
    __device__ __forceinline__ int index(const Lists& li, int k) const { return k < 32 ? i0 : (k < 64 ? i1 : li.at[k]); }
    __device__ __forceinline__ float logit(const Lists& li, int k) const { return k < 32 ? t0 : (k < 64 ? t1 : li.z[k]); }
};

// f(k, N values in a row of N * 32) for a list's entries: one each, where they are few, or four side by side (a chain of multiply-adds each)
template <typename F>
__device__ __forceinline__ void each_entry(int count, F f) {
    const int lane = threadIdx.x & 31;
    if (count <= 32) f(lane, std::integral_constant<int, 1>{});
    else
        for (int k = lane; k < count; k += 128) f(k, std::integral_constant<int, 4>{});
}

// By one warp: the entries of row r that lie in the slice (every CTA takes its own, and the join brings their sums together).  Without
// top_lse their p are relative to the row's first one until then (in a launch for the gradient alone, where 32 bits do for p, at once).
template <typename T, int MODE>
__device__ __forceinline__ void prepare_entries(RowInfo& info, const Lists& li, const DistillCall& a, long long r, const RawList& raw,
                                                const SliceOf<T>& sl, bool report) {
    const int lane = threadIdx.x & 31;
    const int count = (sl.v1 - sl.v0) * SliceOf<T>::E;
    raw.stage(li, a.K);
    float top = -INFINITY, norm = 0.f;
    if (!a.top_lse) {                                                              // the entries' own soft-max
        for (int k = lane; k < a.K; k += 32) {
            const int i = raw.index(li, k);
            if (i >= 0 && i < a.V) top = fmaxf(top, raw.logit(li, k));
        }
        top = warp_largest(top);
        if constexpr (MODE == kGrad) {
            for (int k = lane; k < a.K; k += 32) {
                const int i = raw.index(li, k);
                if (i >= 0 && i < a.V) norm += ex2((raw.logit(li, k) - top) * (a.inv_temp * kLog2e));
            }
            norm = warp_add(norm);
        }
    }
    bool any = false;
    int n = 0;
    for (int k0 = 0; k0 < a.K; k0 += 32) {
        const int k = k0 + lane, i = k < a.K ? raw.index(li, k) : -1, at = i - sl.first;
        const float t = k < a.K ? raw.logit(li, k) : 0.f;
        const bool there = i >= 0 && i < a.V, here = there && at >= 0 && at < count;
        const uint32_t all = __ballot_sync(0xffffffffu, here);                     // (all have read their entry of this round)
        if (here) {
            const int to = n + __popc(all & ((1u << lane) - 1));
            li.at[to] = at;
            li.z[to] = t;
        }
        n += __popc(all);
        any = any || there;
        if (i >= a.V && report) set_status(a.status, SD_ERR_BOUNDS);
    }
    __syncwarp();
    const double from = a.top_lse ? 0.0 : (double)top, off = a.top_lse ? (double)raw.t_lse : MODE == kGrad ? (double)logf(norm) : 0.0;
    double mass = 0.0, plogp = 0.0;
    each_entry(n, [&](int k0, auto side) {
        constexpr int N = decltype(side)::value;
        double log_p[N], t[N], p[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = k0 + 32 * j;
            log_p[j] = k < n ? ((double)li.z[k] - from) * (double)a.inv_temp - off : -INFINITY;
            t[j] = log_p[j] * 1.4426950408889634074;
        }
        powers_of_two(t, p);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (k0 + 32 * j < n) li.p[k0 + 32 * j] = p[j];
            mass += p[j];
            if (p[j] != 0.0) plogp += p[j] * log_p[j];
        }
    });
    mass = warp_add(mass);
    plogp = warp_add(plogp);
    any = __any_sync(0xffffffffu, any);
    if (lane == 0) info = RowInfo{mass, plogp, raw.weight, fmaf(fabsf(raw.t_lse), 0x1p-22f, 4e-5f), raw.label, any, n};
    __syncwarp();
}

template <typename T, int MODE>
__global__ void __launch_bounds__(kDistillThreads, 2)
distill_kernel(DistillCall a, long long units, int parts, int per, int slots, int list_bits, int withheld, long long wait_cycles) {
    using namespace sm100;
    using Sl = SliceOf<T>;
    constexpr int E = Row<T>::kE;
    using Number = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
    extern __shared__ __align__(16) uint4 ring[];
    __shared__ DistillShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (tid == 0) {
        sh.abort_flag = 0;
        for (int q = 0; q < slots; ++q) { mbar_init(&sh.full[q], 1); mbar_init(&sh.picked[q], 1); mbar_init(&sh.free_[q], kSumWarps); }
        for (int q = 0; q < kMaxLists; ++q) {
            mbar_init(&sh.info_full[q], 1);
            mbar_init(&sh.info_free[q], kSumWarps + 1 + (MODE != kGrad));
            mbar_init(&sh.sums_full[q], MODE == kGrad ? 1 : kSumWarps + 1);
        }
        for (int q = 0; q < 2; ++q) { mbar_init(&sh.told[q], 1); mbar_init(&sh.row_ready[q], 1); }
        fence_barrier_init();
    }
    const bool talk = MODE != kGrad && parts > 1;                                  // CTAs of a cluster share a row (else every unit is its own)
    const int rank = talk ? (int)cluster_ctarank() : 0;
    if (talk) sync_parts(parts); else __syncthreads();
    begin_dependent(a.logits, a.top_val, a.top_idx, a.top_lse, a.label, a.kl, a.ce, a.stats, a.dloss, a.grad, a.status);
    // units: rows for a cluster; slices where every CTA stands alone
    const long long step = talk ? gridDim.x / parts : gridDim.x, start = talk ? blockIdx.x / parts : blockIdx.x;
    const auto row_of = [&](long long u) { return MODE == kGrad ? u / parts : u; };
    const auto rank_of = [&](long long u) { return MODE == kGrad ? (int)(u % parts) : rank; };
    const auto lists_of = [&](int b) {
        Lists li;
        double* base = reinterpret_cast<double*>(ring + slots * kPieceVecs);
        li.p = base + b * a.K;
        base += a.K << list_bits;
        li.at = reinterpret_cast<int*>(base) + b * a.K;
        li.z = reinterpret_cast<float*>(base) + (a.K << list_bits) + b * a.K;
        return li;
    };
    // the n-th unit's list, and the phase of its barriers; sums alternate between two places
    const auto list_of = [&](long long n) { return (int)(n & ((1 << list_bits) - 1)); };
    const auto phase_of = [&](long long n) { return (uint32_t)((n >> list_bits) & 1); };
    bool ok = true;

    if (warp == kEntryWarp) {
        long long n = 0;
        for (long long u = start; u < units; u += step, ++n) {
            const int b = list_of(n);
            const long long r = row_of(u);
            const Sl sl(a, r, rank_of(u), per);
            const RawList raw(a, r);                                               // (under way while the place is waited for)
            ok = mbar_wait_warp(&sh.info_free[b], phase_of(n) ^ 1u, &sh.abort_flag, wait_cycles);
            if (!ok) break;
            prepare_entries<T, MODE>(sh.info[b], lists_of(b), a, r, raw, sl, rank_of(u) == 0);
            if (lane == 0) mbar_arrive(&sh.info_full[b]);
        }
    } else if (warp == kCopyWarp) {
        const uint64_t pol = policy_evict_first();
        Turn at;
        for (long long u = start; u < units && ok; u += step) {
            const Sl sl(a, row_of(u), rank_of(u), per);
            for (int q = 0; q < sl.pieces && ok; ++q, at.next(slots)) {
                const int slot = at.slot;
                ok = mbar_wait_warp(&sh.free_[slot], at.phase ^ 1u, &sh.abort_flag, wait_cycles);
                if (!ok) break;
                uint4* dst = ring + slot * kPieceVecs;
                const int a0 = sl.v0 + q * kPieceVecs, a1 = min(sl.v1, a0 + kPieceVecs);
                const int i0 = max(sl.row.full0, a0), i1 = min(sl.row.full1, a1);
                // (what lies in the slot from ordinary stores stands behind the copy that comes)
                fence_proxy_async_smem();
                if (lane == 1 && sl.row.full0 > 0 && a0 == 0) dst[0] = sl.row.edge(0);
                const int e = sl.row.nvec - 1;
                if (lane == 2 && e >= max(sl.row.full0, sl.row.full1) && e >= a0 && e < a1) dst[e - a0] = sl.row.edge(e);
                __syncwarp();
                if (lane == 0) {
                    const uint32_t bytes = i1 > i0 ? (uint32_t)(i1 - i0) * 16 : 0;
                    mbar_arrive_expect_tx(&sh.full[slot], bytes + withheld);
                    if (bytes) bulk_load(dst + (i0 - a0), sl.row.vec + i0, bytes, &sh.full[slot], pol);
                }
                __syncwarp();
            }
        }
    } else if (warp == kPickWarp) {
        const float c = a.inv_temp * kLog2e;
        const bool rest_too = a.top_lse != nullptr;
        Turn at;
        long long n = 0;
        for (long long u = start; u < units && ok; u += step, ++n) {
            const int b = list_of(n), h = (int)(n & 1);
            const Sl sl(a, row_of(u), rank_of(u), per);
            const Lists li = lists_of(b);
            ok = mbar_wait_warp(&sh.info_full[b], phase_of(n), &sh.abort_flag, wait_cycles);
            const int label = sh.info[b].label, lj = label - sl.first;
            const bool has_label = label >= 0 && label < a.V;
            const int count = sh.info[b].count;
            const bool away = MODE != kGrad && rest_too;                           // minus infinity takes a listed logit's place
            float label_z = 0.f;
            double part = 0.0;
            bool dup = false, label_listed = false;
            // the lane's first entry (a slice has rarely more than 32)
            const int j0 = ok && lane < count ? li.at[lane] : -1;
            const double p0 = j0 >= 0 ? li.p[lane] : 0.0;
            float z0 = 0.f;
            bool again0 = false;
            for (int q = 0; q < sl.pieces && ok; ++q, at.next(slots)) {
                const int slot = at.slot;
                ok = mbar_wait_warp(&sh.full[slot], at.phase, &sh.abort_flag, wait_cycles);
                if (!ok) break;
                Number* piece = reinterpret_cast<Number*>(ring + slot * kPieceVecs);
                const int e0 = q * kPieceVecs * E, e1 = min(e0 + kPieceVecs * E, (sl.v1 - sl.v0) * E);
                const auto value = [&](int j) { return __uint_as_float(sizeof(T) == 4 ? (uint32_t)piece[j - e0] : (uint32_t)piece[j - e0] << 16); };
                const auto put = [&](int j, float z) { piece[j - e0] = (Number)(sizeof(T) == 4 ? __float_as_uint(z) : __float_as_uint(z) >> 16); };
                if (has_label && lj >= e0 && lj < e1) label_z = value(lj);
                // The same place twice?  Every entry leaves its number there; one of them finds it again.
                const bool here0 = j0 >= e0 && j0 < e1;
                if (count <= 32) {
                    if (__any_sync(0xffffffffu, here0)) {
                        if (here0) z0 = value(j0);
                        __syncwarp();
                        if (here0) piece[j0 - e0] = (Number)lane;
                        __syncwarp();
                        again0 = again0 || (here0 && piece[j0 - e0] != (Number)lane);
                        __syncwarp();
                        if (here0) put(j0, away ? -INFINITY : z0);
                        __syncwarp();
                    }
                } else {
                    const auto here = [&](int k) { const int j = li.at[k]; return j >= e0 && j < e1; };
                    for (int k = lane; k < count; k += 32)
                        if (here(k)) li.z[k] = value(li.at[k]);
                    __syncwarp();
                    for (int k = lane; k < count; k += 32)
                        if (here(k)) piece[li.at[k] - e0] = (Number)k;
                    __syncwarp();
                    uint32_t again = 0;                                            // (at most 1024 entries: a bit per round)
                    for (int k = lane; k < count; k += 32)
                        if (here(k) && piece[li.at[k] - e0] != (Number)k) again |= 1u << (k >> 5);
                    __syncwarp();
                    for (int k = lane; k < count; k += 32)
                        if (here(k)) put(li.at[k], away ? -INFINITY : li.z[k]);
                    __syncwarp();
                    if (again) {
                        dup = true;
                        for (int k = lane; k < count; k += 32) if (again >> (k >> 5) & 1) li.at[k] |= kAgain;
                    }
                }
                if (lane == 0) mbar_arrive(&sh.picked[slot]);
            }
            if (!ok) break;
            if (count <= 32) {
                dup = again0;
                label_listed = j0 >= 0 && j0 == lj;
                part = p0 != 0.0 ? p0 * (double)z0 : 0.0;
                if (j0 >= 0) li.z[lane] = z0;
                if (again0) li.at[lane] = j0 | kAgain;
            } else {
                for (int k = lane; k < count; k += 32) {
                    label_listed = label_listed || (li.at[k] & ~kAgain) == lj;
                    if (li.p[k] != 0.0) part += li.p[k] * (double)li.z[k];
                }
            }
            dup = __any_sync(0xffffffffu, dup);
            label_listed = __any_sync(0xffffffffu, label_listed);
            if constexpr (MODE != kGrad) {
                // the listed entries' own sums, every index once
                // (in 64 bits: a draft that has learned is as near to the target as their rounding in 32)
                float top = -INFINITY, sum1 = 0.f;
                double sum = 0.0;
                if (rest_too) {
                    const auto counts = [&](int k) { return k < 32 ? j0 >= 0 && !again0 : li.at[k] < kAgain; };
                    const auto logit = [&](int k) { return count <= 32 ? z0 : li.z[k]; };
                    if (count > 32) again0 = j0 >= 0 && li.at[lane] >= kAgain;
                    for (int k = lane; k < count; k += 32) if (counts(k)) top = fmaxf(top, logit(k));
                    top = warp_largest(top);
                    const float r_c = whole_power(top, c), r_e = whole_power(top, kLog2e);
                    each_entry(count, [&](int k0, auto side) {
                        constexpr int N = decltype(side)::value;
                        double t[N], m[N];
#pragma unroll
                        for (int j = 0; j < N; ++j) {
                            const int k = k0 + 32 * j;
                            const float z = k < count && counts(k) ? logit(k) : -INFINITY;
                            t[j] = fma((double)z, (double)c, -(double)r_c);
                            sum1 += ex2(fmaf(z, kLog2e, -r_e));
                        }
                        powers_of_two(t, m);
#pragma unroll
                        for (int j = 0; j < N; ++j) sum += m[j];
                    });
                    sum = warp_add(sum);
                    sum1 = warp_add(sum1);
                }
                part = warp_add(part);
                // (the loss alone: the sums of two rows before have been taken over)
                ok = mbar_wait_warp(&sh.row_ready[h], (uint32_t)((n >> 1) & 1) ^ 1u, &sh.abort_flag, wait_cycles);
                if (lane == 0) { sh.sums[h][kSumWarps] = make_float4(top, 0.f, 0.f, sum1); sh.own[h] = sh.info[b].plogp - part * ((double)c * kLn2); sh.listed[h] = sum; }
            }
            if (lane == 0) { sh.label_z[b] = label_z; sh.dup[b] = dup; sh.label_listed[b] = label_listed; }
            __syncwarp();
            if (lane == 0) { mbar_arrive(&sh.sums_full[b]); mbar_arrive(&sh.info_free[b]); }
        }
    } else if (warp == kJoinWarp) {
        const float c = a.inv_temp * kLog2e;
        const bool rest_too = a.top_lse != nullptr;
        const auto weigh = [](float own, float all, float cc) {                    // 2^(R - the row's R)
            return ex2(whole_power(own, cc) - whole_power(all, cc));
        };
        long long n = 0;
        if constexpr (MODE != kGrad)
        for (long long r = start; r < units && ok; r += step, ++n) {
            const int b = list_of(n), h = (int)(n & 1);
            const uint32_t ph = (uint32_t)((n >> 1) & 1);
            ok = mbar_wait_warp(&sh.info_full[b], phase_of(n), &sh.abort_flag, wait_cycles) &&
                 mbar_wait_warp(&sh.sums_full[b], phase_of(n), &sh.abort_flag, wait_cycles);
            if (!ok) break;
            const RowInfo& info = sh.info[b];
            const int label = info.label;
            const bool has_label = label >= 0 && label < a.V, two = has_label && a.inv_temp != 1.f;
            const float4 w = lane <= kSumWarps ? sh.sums[h][lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
            double listed = 0.0, mass = info.mass, own = sh.own[h];
            const float top_rest = lane < kSumWarps ? w.x : -INFINITY, top_listed = __shfl_sync(0xffffffffu, w.x, kSumWarps);
            float label_z = sh.label_z[b], most_rest = warp_largest(top_rest), most = fmaxf(most_rest, top_listed);
            if (rest_too) listed = sh.listed[h] * (double)weigh(top_listed, most, c);
            float rest = warp_add(w.y * weigh(top_rest, most_rest, c)), sum1 = two ? warp_add(w.w * weigh(w.x, most, kLog2e)) : 0.f;
            if (talk) {
                const Message mine{most, label_z, rest, sum1, most_rest, 0.f, listed, mass, own};
                if (lane == rank) {
                    sh.msg[h][rank] = mine;
                    mbar_arrive_expect_tx(&sh.told[h], (parts - 1) * (uint32_t)sizeof(Message));
                } else if (lane < parts) {
                    const uint32_t to = map_dsmem(smem_u32(&sh.msg[h][rank]), lane), bar = map_dsmem(smem_u32(&sh.told[h]), lane);
                    const auto low = [](double x) { return (uint32_t)__double2loint(x); };
                    const auto high = [](double x) { return (uint32_t)__double2hiint(x); };
                    st_async_v4(to, __float_as_uint(most), __float_as_uint(label_z), __float_as_uint(rest), __float_as_uint(sum1), bar);
                    st_async_v4(to + 16, __float_as_uint(most_rest), 0u, low(listed), high(listed), bar);
                    st_async_v4(to + 32, low(mass), high(mass), low(own), high(own), bar);
                }
                ok = mbar_wait_cluster(&sh.told[h], ph, &sh.abort_flag, wait_cycles);
                ok = __all_sync(0xffffffffu, ok);
                Message o{-INFINITY, 0.f, 0.f, 0.f, -INFINITY, 0.f, 0.0, 0.0, 0.0};
                if (lane < parts) o = sh.msg[h][lane];
                most = warp_largest(o.top);
                most_rest = warp_largest(o.top_rest);
                rest = warp_add(o.rest * weigh(o.top_rest, most_rest, c));
                listed = rest_too ? warp_add(o.listed * (double)weigh(o.top, most, c)) : 0.0;
                if (two) sum1 = warp_add(o.sum1 * weigh(o.top, most, kLog2e));
                own = o.own;
                label_z = o.label;
                mass = warp_add(o.mass);
            }
            const double p_unit = rest_too || !(mass > 0.0) ? 1.0 : 1.0 / mass;    // what the list's p are multiples of
            const double p_rest = rest_too ? 1.0 - mass : 0.0;
            const bool has_rest = p_rest > 0.0 && rest > 0.f;
            const bool masked_rest = info.any && rest == 0.f && p_rest > info.rounding;              // mass that the student can have nowhere
            // (beyond 2^28, powers with R as 32 bits hold it are no longer near 1 at the largest logit: such a row has no loss)
            const bool far = !(fabsf(most * c) <= kFar), far1 = !(fabsf(most * kLog2e) <= kFar);
            // the rest has an R of its own where it lies too far below the largest logit, else that one's
            const float r_c = whole_power(most, c), r_e = whole_power(most, kLog2e), r_own = whole_power(most_rest, c);
            const float at_c = ex2(r_own - r_c);
            const bool apart = has_rest && r_c - r_own > kOwnPower && !far;
            const double total = (double)(rest * at_c) + listed;
            const float sum = (float)total;
            if (!apart) rest *= at_c;
            if (!two) sum1 = sum;
            const float all_p = has_rest || masked_rest ? 1.f : (info.any ? (rest_too ? (float)mass : 1.f) : 0.f);
            // tail / sum = (all_p - p_rest / s_rest) / sum with s_rest = rest / sum
            const float inv = far ? __int_as_float(0x7fffffff) : 1.f / sum, tail = has_rest ? (apart ? inv * at_c : inv) - (float)p_rest / rest : all_p * inv;
            const RowFactors rf{r_c, apart ? r_own : r_c, r_e, all_p * inv, tail, two ? (far1 ? __int_as_float(0x7fffffff) : 1.f / sum1) : inv, (float)p_unit};
            if (lane == 0) { sh.row[h] = rf; mbar_arrive(&sh.row_ready[h]); }
            if (rank == 0) {
                if (talk) { own = warp_add(own); label_z = warp_add(label_z); }
                // R belongs to the power with c as 32 bits hold it.  Relative to the largest logit that is a slightly other temperature: ce takes
                // it back at that logit; in kl the entries' logits stand at the same one, so that what is left of it counts by the difference
                // of the two distributions.
                // A logarithm per lane, of one call (four in a row would not stay in the instruction caches from row to row)
                const double log_of = log(lane == 0 ? total : lane == 1 ? (double)sum1 : lane == 2 ? p_rest * total : lane == 3 ? (double)rest : mass);
                const double log_total = __shfl_sync(0xffffffffu, log_of, 0), log_p = __shfl_sync(0xffffffffu, log_of, 2) - __shfl_sync(0xffffffffu, log_of, 3),
                             log_mass = __shfl_sync(0xffffffffu, log_of, 4);
                if (!rest_too) { own = own * p_unit - log_mass; mass = 1.0; }
                if (lane < 2) {                                                    // lane 0: kl; lane 1: ce
                    if (lane == 0) {
                        double kl = info.any ? own + mass * (log_total + (double)r_c * kLn2) : 0.0;
                        if (has_rest && info.any) kl += p_rest * (log_p + ((double)r_c - (double)rf.r_rest) * kLn2);
                        a.kl[r] = far ? inv : masked_rest ? INFINITY : (float)kl;
                        if (a.stats)
                            reinterpret_cast<float4*>(a.stats)[r] = apart ? pack_stats(rf, two && a.inv_temp < 1.f, a.inv_temp)
                                                                          : make_float4(most, rf.listed, rf.tail, rf.one);
                        if (label >= a.V) set_status(a.status, SD_ERR_BOUNDS);
                    } else if (a.ce) {
                        const double lse = (double)most + log_of - ((double)most * (double)kLog2e - (double)r_e) * kLn2;
                        a.ce[r] = !has_label ? 0.f : far1 ? __int_as_float(0x7fffffff) : (float)(lse - (double)label_z);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.info_free[b]);
        }
    } else {
        const float c = a.inv_temp * kLog2e;
        const Pair c2{c, c}, e2{kLog2e, kLog2e};
        Turn at;
        long long n = 0;
        for (long long u = start; u < units; u += step, ++n) {
            const int b = list_of(n), h = (int)(n & 1);
            const long long r = row_of(u);
            const Sl sl(a, r, rank_of(u), per);
            const Lists li = lists_of(b);
            ok = mbar_wait(&sh.info_full[b], phase_of(n), &sh.abort_flag, wait_cycles) && ok;
            const RowInfo& info = sh.info[b];
            const int label = info.label;
            const bool has_label = label >= 0 && label < a.V;
            const bool two = MODE != kGrad && has_label && a.inv_temp != 1.f;
            const Turn at0 = at;

            // ---- sums of the pieces as they come in
            float top = -INFINITY, r_c = -kFar, r_e = -kFar;                        // top: of the lane's entries; the R's are the warp's
            Pair s{0.f, 0.f}, t{0.f, 0.f}, s1{0.f, 0.f};
            for (int q = 0; MODE != kGrad && q < sl.pieces; ++q, at.next(slots)) {
                const int slot = at.slot;
                ok = mbar_wait(&sh.picked[slot], at.phase, &sh.abort_flag, wait_cycles) && ok;
                const uint4* src = ring + slot * kPieceVecs;
                const int len = min(kPieceVecs, sl.v1 - sl.v0 - q * kPieceVecs);
                uint4 raw[kPerThread];
                float m = -INFINITY;
#pragma unroll
                for (int j = 0; j < kPerThread; ++j) {
                    const int i = tid + j * kSumThreads;
                    raw[j] = i < len ? src[i] : Row<T>::nothing();
                    m = Row<T>::largest(raw[j], m);
                }
                // R is that of the first pieces' largest logit until one comes that is 2^32 times as much (exponentials of up to that
                // size are added as exactly)
                if (__any_sync(0xffffffffu, m * c - r_c > 32.f || m * kLog2e - r_e > 32.f)) {
                    const float most = warp_largest(fmaxf(top, m));
                    const float n_c = whole_power(most, c), n_e = whole_power(most, kLog2e);
                    const float f = ex2(r_c - n_c), f1 = ex2(r_e - n_e);
                    s = Pair{s.x * f, s.y * f};
                    t = Pair{t.x * f, t.y * f};
                    s1 = Pair{s1.x * f1, s1.y * f1};
                    r_c = n_c;
                    r_e = n_e;
                }
                top = fmaxf(top, m);
                const Pair from_c{-r_c, -r_c}, from_e{-r_e, -r_e};
                const auto add = [&](auto both) {                                  // (two loops: as one, the second exponentials were issued in either case)
#pragma unroll
                    for (int j = 0; j < kPerThread; ++j) {
                        if (warp * 32 + j * kSumThreads >= len) break;             // (nothing for the whole warp)
                        Pair x[E / 2];
                        Row<T>::pairs(raw[j], x);
#pragma unroll
                        for (int e = 0; e < E / 2; e += 2) {
                            s = add2(s, ex2(fma2(x[e], c2, from_c)));
                            t = add2(t, ex2(fma2(x[e + 1], c2, from_c)));
                        }
                        if constexpr (decltype(both)::value) {
#pragma unroll
                            for (int e = 0; e < E / 2; ++e) s1 = add2(s1, ex2(fma2(x[e], e2, from_e)));
                        }
                    }
                };
                if (two) add(std::true_type{});
                else add(std::false_type{});
                if (MODE == kLoss) {
                    __syncwarp();
                    if (lane == 0 && ok) mbar_arrive(&sh.free_[slot]);             // (a copy that has not come is still expected there)
                }
            }

            RowFactors rf;
            if constexpr (MODE != kGrad) {
                // (handed on relative to the R of the largest logit: the join takes a sum's R from that)
                const float most = warp_largest(top);
                const float rest = warp_add((s.x + s.y) + (t.x + t.y)) * ex2(r_c - whole_power(most, c));
                const float sum1 = two ? warp_add(s1.x + s1.y) * ex2(r_e - whole_power(most, kLog2e)) : 0.f;
                // (the loss alone: the sums of two rows before have been taken over)
                if (MODE == kLoss) ok = mbar_wait(&sh.row_ready[h], (uint32_t)((n >> 1) & 1) ^ 1u, &sh.abort_flag, wait_cycles) && ok;
                if (lane == 0) sh.sums[h][warp] = make_float4(most, rest, 0.f, sum1);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.sums_full[b]);
                if constexpr (MODE == kLossGrad) {
                    ok = mbar_wait(&sh.row_ready[h], (uint32_t)((n >> 1) & 1), &sh.abort_flag, wait_cycles) && ok;
                    rf = sh.row[h];
                }
            } else {
                const float4 st = __ldcg(reinterpret_cast<const float4*>(a.stats) + r);
                rf = unpack_stats(st, has_label && a.inv_temp < 1.f, a.inv_temp);
                if (label >= a.V && tid == 0 && rank_of(u) == 0) set_status(a.status, SD_ERR_BOUNDS);
            }

            // ---- the gradient, piece by piece
            if constexpr (MODE != kLoss) {
                const float weight = info.weight;
                const bool zero = weight == 0.f;
                const Factors f(a, rf, weight, has_label);
                T* grad = static_cast<T*>(a.grad) + r * a.grad_ld;
                const bool same = ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(sl.row.p)) & 15) == 0;
                uint4* out = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(grad) & ~(uintptr_t)15);
                at = at0;
                const int pieces = MODE == kGrad || __all_sync(0xffffffffu, ok) ? sl.pieces : 0;
                for (int q = 0; q < pieces; ++q, at.next(slots)) {
                    const int slot = at.slot;
                    if (MODE == kGrad) ok = mbar_wait(&sh.picked[slot], at.phase, &sh.abort_flag, wait_cycles) && ok;
                    const uint4* src = ring + slot * kPieceVecs;
                    const int len = min(kPieceVecs, sl.v1 - sl.v0 - q * kPieceVecs), a0 = sl.v0 + q * kPieceVecs;
                    const auto one = [&](int i, auto kind) {                       // vector i of the piece
                        constexpr int kind_of = decltype(kind)::value;             // 0: weight 0, 1: one exponential per entry, 2: two
                        float g[E];
                        if constexpr (kind_of == 0) {
#pragma unroll
                            for (int e = 0; e < E; ++e) g[e] = 0.f;
                        } else f.template vector<T, kind_of == 2>(src[i], g);
                        const int v = a0 + i;
                        if (same && v >= sl.row.full0 && v < sl.row.full1) out[v] = pack<T>(g);
                        else
#pragma unroll
                            for (int e = 0; e < E; ++e) {
                                const int at = v * E + e - sl.row.lead;
                                if (at >= 0 && at < a.V) store_one<T>(grad, at, g[e]);
                            }
                    };
                    const auto all = [&](auto kind) {
#pragma unroll
                        for (int j = 0; j < kPerThread; ++j) {
                            const int i = tid + j * kSumThreads;
                            if (i < len) one(i, kind);
                        }
                    };
                    if (zero) all(std::integral_constant<int, 0>{});
                    else if (f.two) all(std::integral_constant<int, 2>{});
                    else all(std::integral_constant<int, 1>{});
                    __syncwarp();
                    if (lane == 0 && (MODE == kLossGrad || ok)) mbar_arrive(&sh.free_[slot]);
                }
                // over what has just been written
                if (MODE == kGrad) ok = mbar_wait(&sh.sums_full[b], phase_of(n), &sh.abort_flag, wait_cycles) && ok;
                ok = !sum_warps_or(!ok);                                           // (all fourteen come here in every row, whatever they waited for)
                if (ok && !zero) {                                                 // (else the list may be another row's)
                    for (int k = tid; k < info.count; k += kSumThreads) {
                        const int j = li.at[k], v = j + sl.first;
                        if (j >= kAgain || v < 0 || v >= a.V) continue;
                        double p = li.p[k];
                        if (sh.dup[b]) {                                           // the same index twice somewhere: all of its masses
                            p = 0.0;
                            for (int x = 0; x < info.count; ++x) p += (li.at[x] & ~kAgain) == j ? li.p[x] : 0.0;
                        }
                        float g = f.at(li.z[k], f.listed, f.r_c) - f.per_p * (float)p;
                        if (v == label) g -= f.per_label;
                        store_one<T>(grad, v, g);
                    }
                    const int lj = label - sl.first;
                    if (tid == kSumThreads - 1 && has_label && !sh.label_listed[b] && lj >= 0 && lj < (sl.v1 - sl.v0) * E)
                        store_one<T>(grad, label, f.at(sh.label_z[b], f.tail, f.r_rest) - f.per_label);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.info_free[b]);
            if (MODE == kLoss) ok = __all_sync(0xffffffffu, ok);                   // (a warp goes on, or leaves, as one: the bound may run out between its lanes)
            if (!ok) break;
        }
    }
    if (!ok) set_status(a.status, SD_ERR_TIMEOUT);                                 // a copy, or another CTA's sums, did not come
    __syncwarp();
    if (talk) sync_parts(parts);                                                   // nobody leaves while another CTA may still send to it
    if (!ok || *reinterpret_cast<volatile int*>(&sh.abort_flag)) unwind_pause();
}

// CTAs per row: slices of at most four pieces (a slot is left for the next row) where eight CTAs are enough for that (172 032 f32; five to
// seven pieces in as many slots beyond), and more of them where the rows leave SMs idle
static int distill_parts(int M, int nvec, int sms) {
    int parts = 1;
    while (parts < 8 && ((nvec + parts - 1) / parts > (kSlots - 1) * kPieceVecs || ((long long)M * parts <= sms && nvec / (parts * 2) >= kSumThreads))) parts *= 2;
    return parts;
}

// Clusters of this kernel that are on the GPU at once, asked once per kind of launch.  (Which GPCs have how many SMs decides: with one cluster
// more, its rows would begin when all the others' are done.)
template <typename Kernel>
static int resident_clusters(Kernel* kern, int dev, int cluster, int smem) {
    struct Known { const void* kern; int dev, cluster, smem, n; };
    static thread_local Known known[32];
    static thread_local int next = 0;
    for (const Known& k : known)
        if (k.kern == reinterpret_cast<const void*>(kern) && k.dev == dev && k.cluster == cluster && k.smem == smem) return k.n;
    int n = 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster);
    cfg.blockDim = dim3(kDistillThreads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) return 0;
    } else {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, kDistillThreads, smem) != cudaSuccess) return 0;
        n *= sm_count(dev);
    }
    if (n < 1) return 0;
    known[next++ % 32] = Known{reinterpret_cast<const void*>(kern), dev, cluster, smem, n};
    return n;
}

template <typename T, int MODE>
static sd_status launch_distill(const DistillCall& call, int M, cudaStream_t st) {
    const int nvec = (int)(((long long)call.V * (int)sizeof(T) + 15) / 16) + 1;                // (a row may lie across one vector more)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SD_ERR_CUDA;
    const int sms = sm_count(dev), parts = distill_parts(M, nvec, sms), per = (nvec + parts - 1) / parts;
    const int pieces = (per + kPieceVecs - 1) / kPieceVecs, slots = pieces > kSlots ? pieces : kSlots;
    const int list_bits = call.K <= 256 ? 2 : 1;                                   // four rows' lists, or two long ones'
    const int smem = slots * kPieceVecs * 16 + (call.K * 16 << list_bits);
    auto kern = distill_kernel<T, MODE>;
    if (slots > kMaxSlots || !allow_dynamic_smem(kern, smem)) return SD_ERR_CUDA;
    const int cluster = MODE == kGrad ? 1 : parts;
    const long long units = MODE == kGrad ? (long long)M * parts : M;
    const int resident = resident_clusters(kern, dev, cluster, smem);
    if (resident < 1) return SD_ERR_CUDA;
    const long long clusters = units < resident ? units : resident;
    const TestKnobs knobs = test_knobs();
    return launch_dependent(kern, dim3((unsigned)(clusters * cluster)), kDistillThreads, smem, cluster, st, call, units, parts, per, slots, list_bits,
                            knobs.withhold ? 16 : 0, knobs.wait_cycles);
}

}  // namespace rows

using namespace rows;

sd_status launch_distill_loss(const DistillCall& call, int dtype, int M, cudaStream_t st) {
    if (call.grad) return dtype == SD_F32 ? launch_distill<float, kLossGrad>(call, M, st) : launch_distill<uint16_t, kLossGrad>(call, M, st);
    return dtype == SD_F32 ? launch_distill<float, kLoss>(call, M, st) : launch_distill<uint16_t, kLoss>(call, M, st);
}

sd_status launch_distill_grad(const DistillCall& call, int dtype, int M, cudaStream_t st) {
    return dtype == SD_F32 ? launch_distill<float, kGrad>(call, M, st) : launch_distill<uint16_t, kGrad>(call, M, st);
}

}  // namespace sdv
