// Top logits, filtered sampling and filtered logits of rows [M][V] (sd_top_logits, sd_sample_logits, sd_filter_logits).
//
// Which entries stay is decided on a list of some hundred entries that one CTA collects and sorts:
//   top-k up to kFewK   entries that reach the k-th largest of 128 groups' largest logits
//   other borders       histograms of the row in bins of a fraction of a factor of two below its largest logit, counts and (to 2e-5)
//                       masses: the bins in which the borders lie are listed, and if there are few, all that is above them
// With all kept entries listed, the borders are prefix lengths of the sorted list and the draws are among its entries.  Otherwise (flat
// rows) the list gives the last entry that stays, and the mass above the listed bins is summed up, in 64 bits, chunk by chunk (32 * kU
// consecutive vectors); a draw looks up the chunk and then the entry.  Lists that overflow (thousands of nearly equal logits) are
// narrowed down by further histograms over the keys.
//
// Few rows: one cluster of up to eight CTAs per row, each with a slice of it in its shared memory (bulk copies; 152064 f32 are eight
// slices of 76 KB, two of which share an SM; of more than 4812 vectors, vocabularies above 154 000 f32, an SM holds one), read once and passed
// over as often as it takes.  One such row, which L2 still holds (from HBM): k = 50 14 us (16), top-p 40 (55), all entries 16 (23); latency bounds it
// (copy 3 us, then barriers of the cluster, sorting, the draw).  The threshold's 128 groups are stretches of the row there: where the large logits
// stand side by side, the list overflows and a k = 50 takes the histograms' time.
// Many rows: passes over L2, as far as the resident rows fit there, with loads ahead in registers, a CTA or a small cluster per row.  Top
// logits then take one pass with the log-sum-exp and one for the list: 2048 rows of 152064 bf16, K = 64 191 us, 3.3 TB/s, of f32 364, 3.4 TB/s
// (its resident rows are 180 MB, more than L2: both passes come from HBM); bound by instructions (63 % of the issue slots, XU pipe 38 %) and by what follows
// a row's passes.  256 rows of 152064 f32: k = 50 70 us, everything 90 (its masses in 64 bits: the fp64 pipe at 39 %), top-p 272 (the
// histograms' atomics).
// (Lists kept in a single pass over global memory, with a threshold that rises, took three times as long: their cutting and their
// barriers, 12 of 30 us for one row, and for flat rows four passes through L2.)
#include <limits.h>
#include <type_traits>
#include "rows.cuh"

namespace sdv {
namespace rows {

constexpr int kFewK = 112;             // of 128 groups: with k near 128 the threshold would be the least of them, and the list long
constexpr int kGroups = 128;
constexpr int kSomeK = 384;            // of 512 threads: 710 entries expected
constexpr int kU = 4;                  // vectors per lane and chunk
constexpr int kMaxChunks = 544;        // of a CTA (a whole row of 2^18 f32: 16 warps' 33)
constexpr int kBins = 1024;
constexpr int kCopies = 8;             // of a row's bins' masses
constexpr int kPieces = 4;             // copies of a slice: four warps' vectors each
constexpr int kComparePairs = 96;      // kept entries up to which the draw compares all pairs instead of sorting again
constexpr double kUnit = 8796093022208.0;          // 2^43: masses as whole numbers
enum { kNone, kList, kWide };          // no entry left; the kept entries are listed; they are those up to a border

struct RowShared {
    uint64_t bar[kPieces];
    int abort_flag;
    uint32_t n;                        // entries in the list
    uint32_t hist[256];
    uint64_t sel_prefix;
    uint32_t sel_left;
    int sel_done;
    float wtop[kWarps], wsum[kWarps];
    int wcnt[kWarps];
    double tmp_d[kWarps];
    uint64_t tmp_u[kWarps];
    uint64_t lo[kWarps], hi[kWarps];
    float groups[kGroups];
    float thr;
    struct { uint32_t bin, n; uint64_t count, mass; } pick;      // a bin, the entries in it, and what stands in front of it
    int found[64];                     // draws
    float edges[4];
    float u[64];
    // what the CTAs of a row read of each other
    float group_top[kGroups], cta_top, cta_sum;
    uint32_t cta_n, cta_m;             // entries in list, in other
    uint64_t cta_lo, cta_hi;
    double cta_mid;
    int cta_count;
    double chunk[kMaxChunks];          // sums of this CTA's chunks
    int chunk_ref[kMaxChunks];         // and what they are relative to, where every chunk has a power of its own
    uint64_t list[kListMax];
    union {
        struct { uint32_t count[kBins], mass[kBins]; } bins;     // of this CTA
        uint64_t other[kListMax];
    };
    // what the first CTA tells the others
    int kind, kept;
    uint64_t border, border_mass;
    double total;
    // the row's, in every CTA: bins, or in the first one chunks or the list's masses, as inclusive sums
    union { double all[kListMax]; uint64_t all_u[kListMax]; };
    __align__(16) uint32_t all_count[kBins];
    uint32_t scan_count[kWarps];
};

// ---------------------------------------------------------------- a slice of a row
// HELD: in the CTA's shared memory.  Otherwise where the row lies (its share of one, two or four): passes over it come from L2, as far as the
// resident rows fit there, and load four vectors ahead of those that they work on.
struct Never {
    __device__ __forceinline__ bool operator()() const { return false; }
};
template <typename T, bool HELD>
struct Slice {
    static constexpr int E = Row<T>::kE;
    Row<T> row;
    uint4* data;
    int parts, rank, per, v0, nv, first, seg, iters;       // first: index in the row of the slice's first entry (negative where the row starts inside it)
    __device__ __forceinline__ Slice(const void* base, long long ld, long long r, int V, int parts_, int rank_, uint4* data_)
        : row(base, ld, r, V), data(data_), parts(parts_), rank(rank_) {
        per = (row.nvec + parts - 1) / parts;
        v0 = min(row.nvec, rank * per);
        nv = min(row.nvec, v0 + per) - v0;
        first = v0 * E - row.lead;
        seg = (per + kWarps - 1) / kWarps;                                         // a warp's consecutive vectors (the same in all parts)
        iters = (seg + 32 * kU - 1) / (32 * kU);                                   // its chunks
    }
    __device__ __forceinline__ uint4 load(int i) const {                           // vector i, or nothing where that is behind the slice
        if constexpr (HELD) return i < nv ? data[i] : Row<T>::nothing();
        else return i < nv ? row.load(v0 + i) : Row<T>::nothing();
    }
    // vectors i0 + lane, + 32, ..
    __device__ __forceinline__ void load_four(int i0, int end, uint4 (&raw)[kU]) const {
        const int lane = threadIdx.x & 31;
        if (!HELD && v0 + i0 >= row.full0 && v0 + i0 + 32 * kU <= row.full1 && i0 + 32 * kU <= end) {
#pragma unroll
            for (int u = 0; u < kU; ++u) raw[u] = __ldcg(row.vec + v0 + i0 + u * 32 + lane);
        } else {
#pragma unroll
            for (int u = 0; u < kU; ++u) raw[u] = i0 + u * 32 + lane < end ? load(i0 + u * 32 + lane) : Row<T>::nothing();
        }
    }
    // f(vectors, index of the first one) for all of the warp's part, four vectors per lane at a time
    template <typename F, typename G = Never>
    __device__ __forceinline__ void each_four(F f, G stop = G()) const {
        const int warp = threadIdx.x >> 5, w0 = min(nv, warp * seg), w1 = min(nv, w0 + seg);
        uint4 raw[kU];
        if constexpr (HELD) {
            for (int i0 = w0; i0 < w1 && !stop(); i0 += 32 * kU) { load_four(i0, w1, raw); f(raw, i0); }
        } else {
            uint4 ahead[kU];
            load_four(w0, w1, ahead);
            for (int i0 = w0; i0 < w1 && !stop(); i0 += 32 * kU) {
#pragma unroll
                for (int u = 0; u < kU; ++u) raw[u] = ahead[u];
                if (i0 + 32 * kU < w1) load_four(i0 + 32 * kU, w1, ahead);
                f(raw, i0);
            }
        }
    }
    // f(vector, its index), for all of the warp's part, or until stop()
    template <typename F, typename G = Never>
    __device__ __forceinline__ void each_vector(F f, G stop = G()) const {
        const int lane = threadIdx.x & 31;
        if constexpr (HELD) {
            const int warp = threadIdx.x >> 5, w0 = min(nv, warp * seg), w1 = min(nv, w0 + seg);
#pragma unroll 2
            for (int i = w0 + lane; i < w1 && !stop(); i += 32) f(data[i], i);
        } else {
            each_four([&](const uint4 (&raw)[kU], int i0) {
#pragma unroll
                for (int u = 0; u < kU; ++u) f(raw[u], i0 + u * 32 + lane);
            }, stop);
        }
    }
    // f(vector, its index) for all lanes of a warp, and end(chunk) behind each of its chunks: for passes with enough to do per vector
    template <typename F, typename G>
    __device__ __forceinline__ void each_chunk(F f, G end) const {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, w0 = min(nv, warp * seg), w1 = min(nv, w0 + seg);
        uint4 ahead = Row<T>::nothing();
        if (!HELD && w0 + lane < w1) ahead = load(w0 + lane);
        for (int c = 0; c < iters; ++c) {
#pragma unroll 1
            for (int u = 0; u < kU; ++u) {
                const int i = w0 + (c * kU + u) * 32 + lane;
                if (i - lane >= w1) break;
                uint4 raw = ahead;
                if constexpr (HELD) raw = i < w1 ? data[i] : Row<T>::nothing();
                else ahead = i + 32 < w1 ? load(i + 32) : Row<T>::nothing();
                f(raw, i);
            }
            end(c);
        }
    }
    __device__ __forceinline__ void copy(RowShared& sh, int withheld) const {      // by the whole CTA; the caller's barrier settles the edges
        const int tid = threadIdx.x;
        if (tid == 0) {
            const uint64_t pol = sm100::policy_evict_first();
            for (int q = 0; q < kPieces; ++q) {
                const int a0 = v0 + min(nv, q * (kWarps / kPieces) * seg), a1 = v0 + min(nv, (q + 1) * (kWarps / kPieces) * seg);
                const int i0 = max(row.full0, a0), i1 = min(row.full1, a1);
                const uint32_t bytes = i1 > i0 ? (uint32_t)(i1 - i0) * 16 : 0;
                sm100::mbar_arrive_expect_tx(&sh.bar[q], bytes + withheld);
                if (bytes)
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                                 ::"r"(sm100::smem_u32(data + (i0 - v0))), "l"(row.vec + i0), "r"(bytes), "r"(sm100::smem_u32(&sh.bar[q])), "l"(pol) : "memory");
            }
        }
        if (tid == 32 && row.full0 > 0 && v0 == 0 && nv > 0) data[0] = row.edge(0);
        const int e = row.nvec - 1;
        if (tid == 64 && e >= max(row.full0, row.full1) && e >= v0 && e < v0 + nv) data[e - v0] = row.edge(e);
    }
    // f(logit, index) for every entry that is not masked
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        each_vector([&](const uint4& raw, int i) {
            float x[E];
            Row<T>::unpack(raw, x);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] > -INFINITY) f(x[e], first + i * E + e);
        });
    }
    // f(logit, index) for every entry from `thr` on
    template <typename F, typename G>
    __device__ __forceinline__ void each_from(float thr, F f, G stop) const {
        each_vector([&](const uint4& raw, int i) {
            if (!(Row<T>::largest(raw, -INFINITY) >= thr)) return;
            float x[E];
            Row<T>::unpack(raw, x);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] >= thr && x[e] > -INFINITY) f(x[e], first + i * E + e);
        }, stop);
    }
    // the chunk that entry `index` of the row belongs to, counted over the parts
    __device__ __forceinline__ int chunk_of(int index) const {
        const int v = (index + row.lead) / E, q = v / per, i = v - q * per, w = i / seg;
        return (q * kWarps + w) * iters + (i - w * seg) / (32 * kU);
    }
};

// ---------------------------------------------------------------- cutting a list down
// Leaves the `keep` first of buf[0..n) in buf[0..keep), in any order (keep < n <= kListMax).  Radix selection from the highest bit
// in which the keys differ.
__device__ __noinline__ void cut_list(RowShared& sh, uint64_t* buf, int n, int keep) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kPer = kListMax / kThreads;
    __syncthreads();
    uint64_t mine[kPer], lo = ~0ull, hi = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = tid + j * kThreads;
        mine[j] = i < n ? buf[i] : ~0ull;
        if (i < n) { lo = min(lo, mine[j]); hi = max(hi, mine[j]); }
    }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    if (lane == 0) { sh.lo[warp] = lo; sh.hi[warp] = hi; }
    if (tid < 256) sh.hist[tid] = 0;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) { lo = min(lo, sh.lo[w]); hi = max(hi, sh.hi[w]); }
    // keys agree above bit `shift`; [prefix, prefix + 2^shift) holds the entry looked for
    int shift = lo == hi ? 0 : 64 - __clzll((long long)(lo ^ hi));
    uint64_t prefix = shift == 64 ? 0 : (lo >> shift) << shift;
    uint32_t left = keep;
    uint64_t last = hi;
    while (shift > 0) {
        const int step = min(8, shift);
        const int down = shift - step;
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (tid + j * kThreads < n && (shift == 64 || (mine[j] >> shift) == (prefix >> shift))) atomicAdd(&sh.hist[(mine[j] >> down) & ((1u << step) - 1)], 1u);
        __syncthreads();
        if (warp == 0) {
            uint32_t s = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += sh.hist[lane * 8 + j];
            uint32_t incl = s;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += o;
            }
            uint32_t before = incl - s;
            if (before < left && left <= incl) {
                int j = lane * 8;
                while (before + sh.hist[j] < left) before += sh.hist[j++];
                sh.sel_prefix = prefix | ((uint64_t)j << down);
                sh.sel_left = left - before;
                sh.sel_done = sh.hist[j] == left - before;                         // all of this bin stay
            }
        }
        __syncthreads();
        prefix = sh.sel_prefix;
        left = sh.sel_left;
        shift = down;
        last = prefix | (down == 0 ? 0 : (~0ull >> (64 - down)));
        if (sh.sel_done) break;
        if (tid < 256) sh.hist[tid] = 0;
        __syncthreads();
    }
    // keys are distinct (the index is part of them): exactly `keep` are at or below `last`
    if (tid == 0) sh.n = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (tid + j * kThreads < n && mine[j] <= last) buf[atomicAdd(&sh.n, 1u)] = mine[j];
    __syncthreads();
}

// ---------------------------------------------------------------- largest logits
// Waits for the slice; the largest logit of every group (4 * parts lanes) and of the CTA, and with LSE the sum of
// 2^((x - cta_top) c).  Returns whether the copies came.
template <bool LSE, typename T, bool HELD>
__device__ __forceinline__ bool first_pass(RowShared& sh, const Slice<T, HELD>& sl, float c, long long wait_cycles) {
    constexpr int E = Row<T>::kE;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    bool ok = true;
    if constexpr (HELD) ok = sm100::mbar_wait_warp(&sh.bar[warp / (kWarps / kPieces)], 0, &sh.abort_flag, wait_cycles);
    float top = -INFINITY;
    sl.each_four([&](const uint4 (&raw)[kU], int) {
#pragma unroll
        for (int u = 0; u < kU; ++u) top = Row<T>::largest(raw[u], top);
    });
    float g = top;
    for (int d = 1; d < 4 * sl.parts; d <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, d));
    if (lane % (4 * sl.parts) == 0) sh.group_top[tid / (4 * sl.parts)] = g;
    top = warp_largest(top);
    float s = 0.f;
    if constexpr (LSE) {
        const float from = top > -INFINITY ? top : 0.f;
        Pair a{0.f, 0.f}, b{0.f, 0.f};
        sl.each_four([&](const uint4 (&raw)[kU], int) {
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                Pair x[E / 2];
                Row<T>::pairs(Row<T>::without_nan(raw[u]), x);
#pragma unroll
                for (int e = 0; e < E / 2; e += 2) {
                    a = add2(a, ex2(mul2(add2(x[e], Pair{-from, -from}), Pair{c, c})));
                    b = add2(b, ex2(mul2(add2(x[e + 1], Pair{-from, -from}), Pair{c, c})));
                }
            }
        });
        s = warp_add((a.x + a.y) + (b.x + b.y));
    }
    if (lane == 0) { sh.wtop[warp] = top; sh.wsum[warp] = s; }
    __syncthreads();
    if (warp == 0) {
        const float t = lane < kWarps ? sh.wtop[lane] : -INFINITY, most = warp_largest(t);
        if constexpr (LSE) {
            s = lane < kWarps && t > -INFINITY ? sh.wsum[lane] * ex2((t - most) * c) : 0.f;
            s = warp_add(s);
        }
        if (lane == 0) { sh.cta_top = most; sh.cta_sum = s; }
    }
    return ok;
}

// Largest logit over the parts (behind a sync_parts).
__device__ __forceinline__ float top_of_parts(RowShared& sh, int parts) {
    const float top = of_parts(&sh.cta_top, parts);
    return warp_largest((threadIdx.x & 31) < parts ? top : -INFINITY);
}

// The k-th largest of the groups' largest logits, k <= kGroups: at least k entries reach it (behind a sync_parts).
__device__ __forceinline__ float kth_group(RowShared& sh, int parts, int k) {
    const int tid = threadIdx.x;
    if (tid < kGroups) {
        const int each = kGroups / parts;
        sh.groups[tid] = *of_rank(&sh.group_top[tid % each], tid / each);
    }
    __syncthreads();
    const int g = tid >> 2;                                                        // four threads count for a group
    const float mine = sh.groups[g];
    int before = 0;
#pragma unroll 8
    for (int j = tid & 3; j < kGroups; j += 4) before += sh.groups[j] > mine || (sh.groups[j] == mine && j < g);
    before += __shfl_xor_sync(0xffffffffu, before, 1);
    before += __shfl_xor_sync(0xffffffffu, before, 2);
    if (before == k - 1) sh.thr = mine;
    __syncthreads();
    return sh.thr;
}

// A threshold that at least k of a row's 512 threads' largest logits reach, and hardly more, in its only CTA (k <= kSomeK): the range of
// keys is halved until the count is near
__device__ __noinline__ float kth_thread(RowShared& sh, float mine, int k) {
    const uint32_t u = __float_as_uint(mine + 0.f), key = u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);           // (upwards with the logit)
    uint32_t lo = 0, hi = 0xffffffffu;                                             // all reach lo; fewer than k reach hi (no logit's key)
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int n = __syncthreads_count(key >= mid);
        if (n >= k) {
            lo = mid;
            if (n <= k + k / 16) break;
        } else hi = mid;
    }
    return __uint_as_float(lo ^ ((lo >> 31) ? 0x80000000u : 0xffffffffu));
}

// ---------------------------------------------------------------- lists
// Entries from `thr` on that `wanted` names into this CTA's list; cta_n counts them, until they find no room.
template <typename S, typename F>
__device__ __forceinline__ void list_entries(RowShared& sh, const S& sl, float thr, F wanted) {
    if (threadIdx.x == 0) sh.cta_n = 0;
    __syncthreads();
    sl.each_from(thr, [&](float x, int index) {
        if (!wanted(x, index)) return;
        const uint32_t at = atomicAdd(&sh.cta_n, 1u);
        if (at < (uint32_t)kListMax) sh.list[at] = order_key(x, index);
    }, [&]() { return *(volatile uint32_t*)&sh.cta_n > (uint32_t)kListMax; });
}
template <typename S>
__device__ __noinline__ void list_from(RowShared& sh, const S sl, float thr) {
    list_entries(sh, sl, thr, [](float, int) { return true; });
}
// how many entries all parts have listed (behind a sync_parts)
__device__ __forceinline__ uint32_t listed(RowShared& sh, int parts) {
    return __reduce_add_sync(0xffffffffu, of_parts(&sh.cta_n, parts));
}
// All parts' entries into the first CTA's list (by the first CTA; they fit): two warps for each part.  Returns how many.
__device__ __forceinline__ int collect(uint64_t* list, uint32_t* count, int parts) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = warp >> 1;
    const uint32_t n = of_parts(count, parts);
    uint32_t upto = n;
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    const int more = __shfl_sync(0xffffffffu, n, r), at = __shfl_sync(0xffffffffu, upto, r) - more;
    if (r > 0 && r < parts) {
        const uint64_t* from = of_rank(list, r);
        for (int i = lane + (warp & 1) * 32; i < more && at + i < kListMax; i += 64) list[at + i] = from[i];
    }
    __syncthreads();
    return min((int)__shfl_sync(0xffffffffu, upto, 7), kListMax);
}
// A list of n entries sorted, cut to the `keep` first ones where that is worth a pass; returns how many there are.
__device__ int sort_list(RowShared& sh, uint64_t* list, int n, int keep) {
    if (n > keep && n > kRankSort) { cut_list(sh, list, n, keep); n = keep; }
    block_sort(list, n);
    return min(n, keep);
}

// first i with a[i] > t (n: none) or, with `or_equal`, a[i] >= t; a ascending
template <typename S>
__device__ __forceinline__ int first_above(const S* a, int n, S t, bool or_equal) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const bool above = or_equal ? a[mid] >= t : a[mid] > t;
        if (above) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// The same over kBins (first index, at most kBins - 1), by the whole CTA: every thread looks at two
template <typename S>
__device__ __forceinline__ void find_bin(const S* a, S t, int* out) {
    const int i = 2 * (int)threadIdx.x;
    const S before = i ? a[i - 1] : a[0], x = a[i], y = a[i + 1];
    if (x >= t && (i == 0 || before < t)) *out = i;
    else if (y >= t && x < t) *out = i + 1;
    else if (i + 2 == kBins && y < t) *out = kBins - 1;
}
// ---------------------------------------------------------------- histograms
// kBins bins of equal widths in the logarithm, counted from the largest logit; what is further off than the last one's beginning belongs to
// that: with 32 bins to a factor of two (for top-p alone: 2^-32, with 2^18 entries at most 6e-5 of the mass) or with 16.  Or, where those
// are too coarse, bins of a window of them.
struct LinearBins {
    float top, per_bin, offset, octaves;           // octaves: a bin's width in powers of two
    bool window;
    __device__ __forceinline__ LinearBins(float top_, const Scale& sc, float per_octave)
        : top(top_), per_bin((float)fmin(per_octave * sc.c, 3.0e38)), offset(0.f), octaves(1.f / per_octave), window(false) {}
    __device__ __forceinline__ void zoom(int from, int to) {                       // to bins from .. to of the coarse ones
        const float f = (float)kBins / (float)(to - from + 1);
        per_bin *= f;
        octaves /= f;
        offset = (float)from * f;
        window = true;
    }
    // (single roundings throughout: a bin's entries are counted in one place and listed in another, and the compiler may fuse a product
    // with a difference in one of them and not in the other)
    __device__ __forceinline__ float distance(float x) const {
        const float d = __fmul_rn(__fsub_rn(top, x), per_bin);
        return window ? fminf(fmaxf(__fsub_rn(d, offset), -1.f), (float)kBins) : fminf(d, (float)(kBins - 1));
    }
    __device__ __forceinline__ int of(float x) const { return (int)floorf(distance(x)); }       // -1, kBins: in front of, behind the window
    // The least logit that falls into bin `bin` or in front of it (minus infinity's successor at least): bins are monotone in the logit,
    // so that this is a search over its bit patterns; a warp's lanes try 32 of them at a time.
    __device__ __forceinline__ float edge(int bin) const {
        if (bin < 0 && !window) return INFINITY;
        const int lane = threadIdx.x & 31;
        const uint32_t t = __float_as_uint(top + 0.f);
        // keys count upwards with the logit; key(top) itself is in bin 0 (or in front of the window)
        uint32_t lo = 0x00800000u, hi = t ^ ((t >> 31) ? 0xffffffffu : 0x80000000u);               // lo: -FLT_MAX
        const auto value = [](uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); };
        if (of(value(hi)) > bin) return INFINITY;
        while (lo < hi) {                                                          // the answer lies in [lo, hi]
            const uint32_t step = (hi - lo) / 33 + 1, k = min(hi, lo + step * lane);
            const uint32_t good = __ballot_sync(0xffffffffu, of(value(k)) <= bin);
            const int first = good ? __ffs(good) - 1 : 32;
            const uint32_t new_hi = first < 32 ? min(hi, lo + step * first) : hi, new_lo = first ? min(hi, lo + step * (first - 1) + 1) : lo;
            hi = new_hi;
            lo = min(new_lo, hi);
        }
        return value(lo);
    }
    __device__ __forceinline__ float at(double octaves_off) const {                // where something so far below the largest entry falls
        return (float)fmin(fmax(octaves_off / (double)octaves - (double)offset, -1.0e6), 1.0e6);
    }
};

template <typename T, bool HELD>
__device__ __noinline__ void bin_entries(RowShared& sh, const Slice<T, HELD> sl, bool counts, bool masses, const LinearBins lin) {
    constexpr int E = Row<T>::kE;
    uint32_t* mass = HELD ? sh.bins.mass : reinterpret_cast<uint32_t*>(sl.data) + (threadIdx.x / 32 % kCopies) * kBins;
    sl.each_vector([&](const uint4& raw, int) {
        float x[E];
        Row<T>::unpack(raw, x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = lin.distance(x[e]), b = floorf(d);
            const int bin = (int)b;
            const bool in = x[e] > -INFINITY && bin >= 0 && bin < kBins;
            // (a far entry of the last coarse bin: one unit, for its count)
            const uint32_t m = (uint32_t)fmaf(ex2(lin.window || bin < kBins - 1 ? (b - d) * lin.octaves : 0.f), 65536.f, 0.5f);
            if (in && masses) atomicAdd(&mass[bin], m);
            if (in && counts) atomicAdd(&sh.bins.count[bin], 1u);
        }
    });
}

// Counts or masses (or both) of the row's bins, in every CTA: all_count and all, inclusive sums that begin with the given ones; masses
// as multiples of the largest entry's.  Without counts, all_count is what the masses allow at most.  A bin's mass is summed up in units
// of 2^-16 of its upper end, in 32 bits, to 2e-5 of it: a slice in shared memory has at most 40960 entries; a row elsewhere has kCopies sums
// for each bin, and two warps' 32784 entries in each.  (The last coarse bin has none.)  Every CTA adds up its share of the bins over the
// parts and hands it to all.
template <typename T, bool HELD>
__device__ void fill_bins(RowShared& sh, const Slice<T, HELD>& sl, bool counts, bool masses, const LinearBins& lin, uint32_t count0, double mass0) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < kBins; i += kThreads) { sh.bins.count[i] = 0; sh.bins.mass[i] = 0; }
    uint32_t* copies = reinterpret_cast<uint32_t*>(sl.data);
    double* folded = reinterpret_cast<double*>(copies + kCopies * kBins);
    if (!HELD && masses)
        for (int i = tid; i < kCopies * kBins; i += kThreads) copies[i] = 0;
    __syncthreads();
    bin_entries(sh, sl, counts, masses, lin);
    if (!HELD && masses) {
        __syncthreads();
        for (int i = tid; i < kBins; i += kThreads) {
            double m = 0.0;
#pragma unroll
            for (int r = 0; r < kCopies; ++r) m += (double)copies[r * kBins + i];
            folded[i] = m;
        }
    }
    sync_parts(sl.parts);
    const int share = kBins / sl.parts;
    for (int j = tid; j < share; j += kThreads) {
        const int i = sl.rank * share + j;
        uint32_t c[8];
        typename std::conditional<HELD, uint32_t, double>::type m[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            c[r] = counts && r < sl.parts ? *of_rank(&sh.bins.count[i], r) : 0;
            if constexpr (HELD) m[r] = masses && r < sl.parts ? *of_rank(&sh.bins.mass[i], r) : 0;
            else m[r] = masses && r < sl.parts ? *of_rank(&folded[i], r) : 0.0;
        }
        uint32_t count = 0;
        double mass = 0.0;
#pragma unroll
        for (int r = 0; r < 8; ++r) { count += c[r]; mass += (double)m[r]; }
        // (a unit of mass is between 2^-octaves and 1 of an entry)
        if (!counts) count = (uint32_t)((float)mass * (1.f / 65535.f) * exp2f(lin.octaves)) + (mass > 0.0);
        if (!lin.window && i == kBins - 1) mass = 0.0;
        mass *= (double)exp2f(-((float)i + lin.offset) * lin.octaves) * (1.0 / 65536.0);
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < sl.parts) {
                *of_rank(&sh.all_count[i], r) = count;
                *of_rank(&sh.all[i], r) = mass;
            }
    }
    sync_parts(sl.parts);
    if (masses) block_scan(sh.all, kBins, sh.tmp_d);
    const uint32_t x = sh.all_count[2 * tid], y = x + sh.all_count[2 * tid + 1];
    uint32_t incl = y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) sh.scan_count[warp] = incl;
    __syncthreads();
    uint32_t before = incl - y + count0;
    for (int w = 0; w < warp; ++w) before += sh.scan_count[w];
    sh.all_count[2 * tid] = before + x;
    sh.all_count[2 * tid + 1] = before + y;
    if (masses && mass0 != 0.0) { sh.all[2 * tid] += mass0; sh.all[2 * tid + 1] += mass0; }
    __syncthreads();
}

// ---------------------------------------------------------------- the general search for a border
// For rows whose border bin holds more than a list does (equal or nearly equal logits): whole-number counts or masses (2^-43 of 2^ref
// as the unit) in bins over ranges of keys, until a list holds what is left.  Slow (a pass and two barriers of the cluster per round of
// ten bits), and right for everything.
template <typename S, typename F>
__device__ void key_bins(RowShared& sh, const S& sl, bool by_mass, const Scale& sc, int ref, F bin_of) {
    const int tid = threadIdx.x;
    sync_parts(sl.parts);
    for (int i = tid; i < kBins; i += kThreads) sh.other[i] = 0;
    __syncthreads();
    sl.each([&](float x, int index) {
        const int bin = bin_of(x, index);
        if (bin >= 0) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.other[bin]), by_mass ? (unsigned long long)(sc.mass(x, ref) * kUnit + 0.5) : 1ull);
    });
    sync_parts(sl.parts);
    for (int i = tid; i < kBins; i += kThreads) {
        uint64_t c = 0;
        for (int r = 0; r < sl.parts; ++r) c += *of_rank(&sh.other[i], r);
        sh.all_u[i] = c;
    }
    block_scan(sh.all_u, kBins, sh.tmp_u);
}
// The key of the last entry, in order, of the shortest prefix whose count (or mass) is at least `target`, and the count or mass with it.
// share: take target as that share of the sum over the keys up to `upto` instead.
template <typename S>
__device__ __noinline__ void search_border(RowShared& sh, const S& sl, bool by_mass, uint64_t target, double share, uint64_t upto, const Scale& sc, int ref,
                              uint64_t* border) {
    uint64_t lo = 0, hi = upto, before = 0;
    bool first = true;
    while (true) {
        const int bits = hi == lo ? 0 : 64 - __clzll((long long)(hi - lo)), shift = max(0, bits - 10);
        key_bins(sh, sl, by_mass, sc, ref, [&](float x, int index) {
            const uint64_t k = order_key(x, index);
            return k >= lo && k <= hi ? (int)((k - lo) >> shift) : -1;
        });
        if (first && share >= 0.0) target = max((uint64_t)1, (uint64_t)ceil(share * (double)sh.all_u[kBins - 1]));
        first = false;
        const int bin = min(first_above(sh.all_u, kBins, target - before, true), kBins - 1);
        before += bin ? sh.all_u[bin - 1] : 0;
        lo += (uint64_t)bin << shift;
        hi = lo + (shift ? (1ull << shift) - 1 : 0);
        if (shift == 0) break;                     // one key
    }
    *border = lo;
}

// ---------------------------------------------------------------- top logits
// (the product stops at f32's range: minus infinity is a row without an entry)
__device__ __forceinline__ float log_sum(float top, float inv_temp, float s) {
    return (float)(fmin(fmax((double)top * (double)inv_temp, -3.4028234663852886e38), 3.4028234663852886e38) + log((double)s));
}

template <typename T, bool HELD>
__global__ void __launch_bounds__(kThreads, 2)
top_kernel(const void* logits, long long ld, int V, int parts, int K, float inv_temp, float* values, int32_t* index, float* lse, int32_t* status,
           int withheld, long long wait_cycles) {
    extern __shared__ __align__(16) uint4 data[];
    __shared__ RowShared sh;
    const int tid = threadIdx.x;
    if (tid == 0) {
        sh.abort_flag = 0;
        for (int q = 0; q < kPieces; ++q) sm100::mbar_init(&sh.bar[q], 1);
        sm100::fence_barrier_init();
    }
    __syncthreads();
    begin_dependent(logits, values, index, lse, status);
    const long long r = blockIdx.x / parts;
    const int rank = parts == 1 ? 0 : (int)sm100::cluster_ctarank();
    const Slice<T, HELD> sl(logits, ld, r, V, parts, rank, data);
    if constexpr (HELD) sl.copy(sh, withheld);
    __syncthreads();
    const float c = inv_temp * kLog2e;
    const bool ok = first_pass<true>(sh, sl, c, wait_cycles);
    sync_parts(parts);
    const float top = top_of_parts(sh, parts);
    uint32_t n = kListMax + 1;
    bool two_lists = false;
    if (K <= kFewK) {
        const float thr = kth_group(sh, parts, K);
        list_from(sh, sl, thr);
        sync_parts(parts);
        n = listed(sh, parts);
    }
    if (n > (uint32_t)kListMax && top > -INFINITY) {
        // the bin of the K-th entry; where it is too full, that bin in finer ones
        LinearBins lin(top, Scale(1.f), 16.f);
        fill_bins(sh, sl, true, false, lin, 0, 0.0);
        const uint32_t n_all = sh.all_count[kBins - 1];
        uint32_t before = 0;
        int bin = min(first_above(sh.all_count, kBins, (uint32_t)K, true), kBins - 1);
        if (n_all > (uint32_t)K && sh.all_count[bin] - (bin ? sh.all_count[bin - 1] : 0) > (uint32_t)kListMax && bin < kBins - 1) {
            before = bin ? sh.all_count[bin - 1] : 0;
            lin.zoom(bin, bin);
            __syncthreads();
            fill_bins(sh, sl, true, false, lin, before, 0.0);
            bin = min(first_above(sh.all_count, kBins, (uint32_t)K, true), kBins - 1);
        }
        // what stands in front of the bin (fewer than K) and the bin's own entries, listed apart; thousands of equal logits there are
        // searched for the K-th's key
        if (bin) before = sh.all_count[bin - 1];
        uint64_t border = ~0ull;
        if (sh.all_count[bin] - before > (uint32_t)kListMax) {
            if (n_all > (uint32_t)K) search_border(sh, sl, false, (uint64_t)K, -1.0, ~0ull, Scale(1.f), 0, &border);
            sync_parts(parts);
            list_entries(sh, sl, -INFINITY, [&](float x, int i) { return order_key(x, i) <= border; });
        } else {
            if (tid == 0) { sh.cta_n = 0; sh.cta_m = 0; }
            __syncthreads();
            sl.each([&](float x, int index) {
                const int b = lin.of(x);
                if (b > bin) return;
                uint64_t* to = b < bin ? sh.list : sh.other;
                const uint32_t at = atomicAdd(b < bin ? &sh.cta_n : &sh.cta_m, 1u);
                if (at < (uint32_t)kListMax) to[at] = order_key(x, index);
            });
            two_lists = true;
        }
        sync_parts(parts);
    }
    if (rank == 0) {
        int have = 0;
        if (top > -INFINITY) {
            have = min(collect(sh.list, &sh.cta_n, parts), kListMax);
            if (two_lists) {
                const int more = collect(sh.other, &sh.cta_m, parts), take = max(0, min(K - have, more));
                sort_list(sh, sh.other, more, max(1, take));
                for (int i = tid; i < take; i += kThreads) sh.list[have + i] = sh.other[i];
                have += take;
            }
            have = sort_list(sh, sh.list, have, K);
        }
        for (int i = tid; i < K; i += kThreads) {
            values[r * K + i] = i < have ? key_logit(sh.list[i]) : -INFINITY;
            index[r * K + i] = i < have ? key_index(sh.list[i]) : -1;
        }
        if (lse && tid == kThreads - 1) {
            float s = 0.f;
            for (int q = 0; q < parts; ++q) {
                const float t = *of_rank(&sh.cta_top, q);
                if (t > -INFINITY) s += *of_rank(&sh.cta_sum, q) * ex2((t - top) * c);
            }
            lse[r] = top > -INFINITY && top < INFINITY ? log_sum(top, inv_temp, s) : top;
        }
    }
    if (!ok) { set_status(status, SD_ERR_TIMEOUT); sm100::unwind_pause(); }
    __syncwarp();
    if (parts > 1) sync_parts(parts);                                              // nobody leaves while the first CTA reads
}

// ---------------------------------------------------------------- top logits of many rows
// Where there are enough rows to fill the GPU, a CTA takes one at a time, twice over: first for the groups' largest logits and the
// sum, then, mostly from L2, for the entries that reach the threshold.  A thread loads four vectors ahead of those that it works on, the
// next pass's and row's first ones too: no warp waits for another within a pass.  Neighbours in the row belong to different threads, and
// so to different groups: vocabularies have their frequent tokens side by side.  (With a sixteenth of the row for every warp, 512 rows of bf16
// whose logits fall along the row took 4900 us, and 59 where they do not.  Clusters that hold a row in shared memory, 4096 rows of 152064
// bf16: 740 us; a ring of copies for all warps of a CTA 580; one for every warp 850; so 377 to 399, by the rows.)
constexpr int kStreamLane = 4;                     // vectors per lane and step
constexpr int kStreamVecs = kStreamLane * 32;

// a whole row where it lies in memory, for the general search
template <typename T>
struct RowInMemory {
    Row<T> row;
    int parts = 1;
    __device__ __forceinline__ explicit RowInMemory(const Row<T>& r) : row(r) {}
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        constexpr int E = Row<T>::kE;
        for (int i = (int)threadIdx.x; i < row.nvec; i += kThreads) {
            float x[E];
            Row<T>::unpack(row.load(i), x);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] > -INFINITY) f(x[e], i * E + e - row.lead);
        }
    }
};

// The logit of the K-th of a full list, K <= kSomeK
__device__ __noinline__ float kth_listed(RowShared& sh, int K) {
    const int tid = threadIdx.x;
    cut_list(sh, sh.list, kListMax, K);
    uint64_t last = tid < K ? sh.list[tid] : 0;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) last = max(last, __shfl_xor_sync(0xffffffffu, last, d));
    if ((tid & 31) == 0) sh.hi[tid >> 5] = last;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) last = max(last, sh.hi[w]);
    return key_logit(last);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
top_stream_kernel(const void* logits, long long ld, int V, int M, int steps, int K, float inv_temp, float* values, int32_t* index, float* lse) {
    constexpr int E = Row<T>::kE;
    __shared__ RowShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    begin_dependent(logits, values, index, lse);
    const float c = inv_temp * kLog2e;
    uint4 ahead[kStreamLane];
    const auto place = [&](int q, int j) { return (q * kStreamLane + j) * kThreads + tid; };         // the thread's vectors of step q
    const auto fetch = [&](const Row<T>& row, int q) {
        if (place(q, 0) - lane >= row.full0 && place(q, kStreamLane - 1) - lane + 32 <= row.full1) {
#pragma unroll
            for (int j = 0; j < kStreamLane; ++j) ahead[j] = __ldcg(row.vec + place(q, j));
        } else {
#pragma unroll
            for (int j = 0; j < kStreamLane; ++j) ahead[j] = place(q, j) < row.nvec ? row.load(place(q, j)) : Row<T>::nothing();
        }
    };
    if (blockIdx.x < M) fetch(Row<T>(logits, ld, blockIdx.x, V), 0);
    for (long long r = blockIdx.x; r < M; r += gridDim.x) {
        const Row<T> row(logits, ld, r, V);
        // ---- the groups' largest logits, and the sum of 2^((x - from) c)
        float top = -INFINITY, from = 0.f;
        Pair a{0.f, 0.f}, b{0.f, 0.f};
        bool begun = false;
        for (int q = 0; q < steps; ++q) {
            uint4 raw[kStreamLane];
            float m = -INFINITY;
#pragma unroll
            for (int j = 0; j < kStreamLane; ++j) raw[j] = ahead[j];
            fetch(row, q + 1 < steps ? q + 1 : 0);                                 // (behind the last one, the second pass's first)
#pragma unroll
            for (int j = 0; j < kStreamLane; ++j) m = Row<T>::largest(raw[j], m);
            if (__any_sync(0xffffffffu, m > -INFINITY && (!begun || (m - from) * c > 32.f))) {
                const float now = warp_largest(fmaxf(top, m));
                if (begun) {
                    const float f = ex2((from - now) * c);
                    a = Pair{a.x * f, a.y * f};
                    b = Pair{b.x * f, b.y * f};
                }
                from = now;
                begun = true;
            }
            top = fmaxf(top, m);
#pragma unroll
            for (int j = 0; j < kStreamLane; ++j) {
                if (place(q, j) - lane >= row.nvec) break;
                Pair x[E / 2];
                Row<T>::pairs(Row<T>::without_nan(raw[j]), x);
#pragma unroll
                for (int e = 0; e < E / 2; e += 2) {
                    a = add2(a, ex2(mul2(add2(x[e], Pair{-from, -from}), Pair{c, c})));
                    b = add2(b, ex2(mul2(add2(x[e + 1], Pair{-from, -from}), Pair{c, c})));
                }
            }
        }
        float g = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
        if ((lane & 3) == 0) sh.group_top[tid >> 2] = g;
        const float mine = top;
        const float sum = warp_add((a.x + a.y) + (b.x + b.y));
        top = warp_largest(top);
        if (lane == 0) { sh.wtop[warp] = top; sh.wsum[warp] = sum; sh.groups[warp] = from; }
        if (tid == 0) sh.cta_n = 0;
        __syncthreads();
        const float wtop = lane < kWarps ? sh.wtop[lane] : -INFINITY, most = warp_largest(wtop);
        if (lse && warp == kWarps - 1) {
            float s = lane < kWarps && wtop > -INFINITY ? sh.wsum[lane] * ex2((sh.groups[lane] - most) * c) : 0.f;
            s = warp_add(s);
            if (lane == 0) lse[r] = most > -INFINITY && most < INFINITY ? log_sum(most, inv_temp, s) : most;
        }
        __syncthreads();                                                           // (groups is written again)
        float thr = K <= kFewK ? kth_group(sh, 1, K) : kth_thread(sh, mine, K);
        uint32_t n;
        // ---- the entries that reach the threshold
        while (true) {
            for (int q = 0; q < steps; ++q) {
                uint4 raw[kStreamLane];
#pragma unroll
                for (int j = 0; j < kStreamLane; ++j) raw[j] = ahead[j];
                if (q + 1 < steps) fetch(row, q + 1);
                else if (r + gridDim.x < M) fetch(Row<T>(logits, ld, r + gridDim.x, V), 0);
#pragma unroll
                for (int j = 0; j < kStreamLane; ++j) {
                    if (!(Row<T>::largest(raw[j], -INFINITY) >= thr)) continue;
                    float x[E];
                    Row<T>::unpack(raw[j], x);
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (x[e] >= thr && x[e] > -INFINITY) {
                            const uint32_t at = atomicAdd(&sh.cta_n, 1u);
                            if (at < (uint32_t)kListMax) sh.list[at] = order_key(x[e], place(q, j) * E + e - row.lead);
                        }
                }
            }
            __syncthreads();
            n = sh.cta_n;
            if (n <= (uint32_t)kListMax) break;
            // Too many.  Where the largest logits stand side by side, the K-th of those listed is a better threshold; behind thousands of
            // equal ones the K-th's key is searched for.
            const float better = kth_listed(sh, K);
            if (tid == 0) sh.cta_n = 0;
            __syncthreads();
            if (better > thr) {
                thr = better;
                fetch(row, 0);
                continue;
            }
            const RowInMemory<T> all(row);
            uint64_t border = ~0ull;
            search_border(sh, all, false, (uint64_t)K, -1.0, ~0ull, Scale(1.f), 0, &border);
            all.each([&](float x, int i) {
                if (order_key(x, i) > border) return;
                const uint32_t at = atomicAdd(&sh.cta_n, 1u);
                if (at < (uint32_t)kListMax) sh.list[at] = order_key(x, i);
            });
            __syncthreads();
            n = min(sh.cta_n, (uint32_t)kListMax);
            break;
        }
        n = sort_list(sh, sh.list, n, K);
        for (int i = tid; i < K; i += kThreads) {
            values[r * K + i] = i < n ? key_logit(sh.list[i]) : -INFINITY;
            index[r * K + i] = i < n ? key_index(sh.list[i]) : -1;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- sampling and filtering
struct SampleCall {
    const void* logits; long long ld; int V, parts;
    const float* inv_temp; const int32_t* top_k; const float* top_p; const float* min_p; const int32_t* n_used; int per_used;
    const float* u; int N; int32_t* tokens; float* prob;       // draws (N = 0: none)
    float* dense; bool scaled;                                 // [M][V]: probabilities, or (scaled) the kept logits times inv_temp
    float* lse; int32_t* kept; int32_t* status;
    int withheld; long long wait_cycles;
};

// Sums of the slice's chunks, relative to 2^ref: of all entries, or (LIST) of those from `above` on, while the entries from `end` to `above`
// and from `end_k` to `above_k` are listed; returns the thread's share of the mass of the others from `above_k` on, and counts the ones above.
template <bool LIST, typename T, bool HELD>
__device__ __noinline__ double sum_chunks(RowShared& sh, const Slice<T, HELD> sl, const Scale sc, int ref, float above, float end, float above_k, float end_k,
                                          int* n_above) {
    constexpr int E = Row<T>::kE;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double mid = 0.0, s = 0.0, t = 0.0;
    int over = 0;
    sl.each_chunk([&](const uint4& raw, int i) {
        float x[E];
        Row<T>::unpack(raw, x);
#pragma unroll
        for (int h = 0; h < E; h += 4) {
            const float y[4] = {x[h], x[h + 1], x[h + 2], x[h + 3]};
            double m[4];
            sc.masses(y, ref, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (LIST) {
                    const bool up = y[e] >= above, here = !up && y[e] > -INFINITY && (y[e] >= end || (y[e] >= end_k && y[e] < above_k));
                    over += up;
                    (e & 1 ? t : s) += up ? m[e] : 0.0;
                    mid += !up && !here && y[e] >= above_k ? m[e] : 0.0;
                    if (here) {
                        const uint32_t at = atomicAdd(&sh.cta_n, 1u);
                        if (at < (uint32_t)kListMax) sh.list[at] = order_key(y[e], sl.first + i * E + h + e);
                    }
                } else {
                    (e & 1 ? t : s) += m[e];
                }
            }
        }
    }, [&](int c) {
        s = warp_add(s + t);
        if (lane == 0) sh.chunk[warp * sl.iters + c] = s;
        s = t = 0.0;
    });
    if constexpr (LIST) *n_above = over;
    return mid;
}
// The same of all entries in a single pass, with the largest logit (cta_top): every chunk relative to a power of its own
template <typename T, bool HELD>
__device__ __noinline__ bool sum_all(RowShared& sh, const Slice<T, HELD> sl, const Scale sc, long long wait_cycles) {
    constexpr int E = Row<T>::kE;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    bool ok = true;
    if constexpr (HELD) ok = sm100::mbar_wait_warp(&sh.bar[warp / (kWarps / kPieces)], 0, &sh.abort_flag, wait_cycles);
    float top = -INFINITY;
    int c = 0, cnt = 0;
    for (int i = lane; i < sl.iters; i += 32) { sh.chunk[warp * sl.iters + i] = 0.0; sh.chunk_ref[warp * sl.iters + i] = INT_MIN; }
    __syncwarp();
    sl.each_four([&](const uint4 (&raw)[kU], int) {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < kU; ++u) m = Row<T>::largest(raw[u], m);
        m = warp_largest(m);
        if (m > -INFINITY) {
            const int ref = sc.whole(m);
            double s = 0.0, t = 0.0;
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                float x[E];
                Row<T>::unpack(raw[u], x);
#pragma unroll
                for (int h = 0; h < E; h += 4) {
                    const float y[4] = {x[h], x[h + 1], x[h + 2], x[h + 3]};
                    double w[4];
                    sc.masses(y, ref, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { (e & 1 ? t : s) += w[e]; cnt += y[e] > -INFINITY; }
                }
            }
            s = warp_add(s + t);
            if (lane == 0) { sh.chunk[warp * sl.iters + c] = s; sh.chunk_ref[warp * sl.iters + c] = ref; }
            top = fmaxf(top, m);
        }
        ++c;
    });
    cnt = __reduce_add_sync(0xffffffffu, cnt);
    if (lane == 0) { sh.wtop[warp] = top; sh.wcnt[warp] = cnt; }
    __syncthreads();
    if (warp == 0) {
        const float most = warp_largest(lane < kWarps ? sh.wtop[lane] : -INFINITY);
        cnt = __reduce_add_sync(0xffffffffu, lane < kWarps ? sh.wcnt[lane] : 0);
        if (lane == 0) { sh.cta_top = most; sh.cta_count = cnt; }
    }
    return ok;
}
// The sums of the entries up to the key `last` with a mass of at least `least`, and (the thread's) how many there are
template <typename T, bool HELD>
__device__ __noinline__ void sum_kept(RowShared& sh, const Slice<T, HELD> sl, const Scale sc, int ref, uint64_t last, double least, int* kept) {
    constexpr int E = Row<T>::kE;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double s = 0.0;
    int cnt = 0;
    sl.each_chunk([&](const uint4& raw, int i) {
        float x[E];
        Row<T>::unpack(raw, x);
#pragma unroll
        for (int h = 0; h < E; h += 4) {
            const float y[4] = {x[h], x[h + 1], x[h + 2], x[h + 3]};
            double m[4];
            sc.masses(y, ref, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = y[e] > -INFINITY && order_key(y[e], sl.first + i * E + h + e) <= last && m[e] >= least;
                s += in ? m[e] : 0.0;
                cnt += in;
            }
        }
    }, [&](int c) {
        s = warp_add(s);
        if (lane == 0) sh.chunk[warp * sl.iters + c] = s;
        s = 0.0;
    });
    *kept = cnt;
}

// The entry of a chunk at which the mass in vocabulary order exceeds `over`; kept(x, index, mass): whether an entry counts.  A warp
// calls it; the chunk may lie in another CTA's slice.  Sums that fall short by rounding end at the last entry with mass.
template <typename T, bool HELD, typename F>
__device__ int chunk_crossing(const Slice<T, HELD>& sl, int g, double over, const Scale& sc, int ref, F kept, double* its_mass) {
    constexpr int E = Row<T>::kE;
    const int lane = threadIdx.x & 31, per_part = kWarps * sl.iters, q = g / per_part, at = g - q * per_part, w = at / sl.iters, c = at - w * sl.iters;
    const uint4* data = HELD && sl.parts > 1 ? of_rank(sl.data, q) : sl.data;
    const int v0 = min(sl.row.nvec, q * sl.per), nv = min(sl.row.nvec, v0 + sl.per) - v0, first = v0 * E - sl.row.lead;
    const int w0 = min(nv, w * sl.seg), w1 = min(nv, w0 + sl.seg);
    uint4 raw[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const int i = w0 + (c * kU + u) * 32 + lane;
        if constexpr (HELD) raw[u] = i < w1 ? data[i] : Row<T>::nothing();
        else raw[u] = i < w1 ? sl.row.load(v0 + i) : Row<T>::nothing();
    }
    const auto masses_of = [&](const uint4& now, int u, double (&m)[E]) {
        float x[E];
        Row<T>::unpack(now, x);
        sc.masses(x, ref, m);
#pragma unroll
        for (int e = 0; e < E; ++e) if (!kept(x[e], first + (w0 + (c * kU + u) * 32 + lane) * E + e, m[e])) m[e] = 0.0;
    };
    // the sums of the kU steps, and in which of them the mark is passed (else the last with mass)
    double sum[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        double m[E], s = 0.0;
        masses_of(raw[u], u, m);
#pragma unroll
        for (int e = 0; e < E; ++e) s += m[e];
        sum[u] = warp_add(s);
    }
    double before = 0.0, run = 0.0;
    int step = -1;
    bool passed = false;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        if (!passed && sum[u] > 0.0) { step = u; before = run; passed = run + sum[u] > over; }
        run += sum[u];
    }
    int last = -1;
    double last_mass = 0.0;
    if (step >= 0) {
        uint4 now = raw[0];
#pragma unroll
        for (int j = 1; j < kU; ++j) if (step == j) now = raw[j];
        double m[E], s = 0.0;
        masses_of(now, step, m);
#pragma unroll
        for (int e = 0; e < E; ++e) s += m[e];
        double incl = s;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const double o = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += o;
        }
        const uint32_t over_here = __ballot_sync(0xffffffffu, s > 0.0 && before + incl > over);
        const uint32_t with_mass = __ballot_sync(0xffffffffu, s > 0.0);
        // within the lane: the first entry at which the sum exceeds `over`, else the last with mass
        int found = -1;
        double found_mass = 0.0;
        bool crossed = false;
        run = before + (incl - s);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            run += m[e];
            if (m[e] > 0.0 && !crossed) { found = first + (w0 + (c * kU + step) * 32 + lane) * E + e; found_mass = m[e]; crossed = run > over; }
        }
        const int src = over_here ? __ffs(over_here) - 1 : 31 - __clz(with_mass);
        last = __shfl_sync(0xffffffffu, found, src);
        last_mass = __shfl_sync(0xffffffffu, found_mass, src);
    }
    *its_mass = last_mass;
    return last;
}

// a scaled logit as it is given back: products beyond the type's range stop there, so that what is not masked stays finite
__device__ __forceinline__ float scaled_logit(float x, float inv_temp) { return fminf(fmaxf(x * inv_temp, -3.4028234663852886e38f), 3.4028234663852886e38f); }
// log of a mass that is given relative to 2^ref; the largest logit belongs to it
__device__ __forceinline__ float log_mass(const Scale& sc, float top, float inv_temp, int ref, double total) {
    const double z = fmin(fmax((double)top * (double)inv_temp, -3.4028234663852886e38), 3.4028234663852886e38);
    return (float)(z + log(total / sc.mass(top, ref)));
}

// dst[0..n) = value, by the whole CTA
__device__ void fill_floats(float* dst, int n, float value) {
    const int lead = min(n, (int)(((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) & 15) / 4)), vecs = (n - lead) / 4;
    const int tid = threadIdx.x;
    if (tid < lead) dst[tid] = value;
    for (int i = tid; i < vecs; i += kThreads) reinterpret_cast<float4*>(dst + lead)[i] = make_float4(value, value, value, value);
    if (tid < n - lead - vecs * 4) dst[lead + vecs * 4 + tid] = value;
}

// Draws among the `kept` first entries of the sorted list (by the first CTA; sh.all: the list's masses as inclusive sums)
__device__ void draw_from_list(RowShared& sh, const SampleCall& a, long long r, const Scale& sc, int ref, int kept) {
    const int tid = threadIdx.x;
    const auto report = [&](int i, bool fine, int token, double share) {
        if (!fine) set_status(a.status, SD_ERR_INVALID_ARG);
        a.tokens[r * a.N + i] = fine ? token : -1;
        if (a.prob) a.prob[r * a.N + i] = fine ? (float)share : 0.f;
    };
    if (kept <= kComparePairs) {
        // every entry sums up the masses of those in front of it in the vocabulary; of the entries past the mark the first is drawn
        const double total = sh.all[kept - 1];
        double* mass = reinterpret_cast<double*>(sh.other);
        double mine = 0.0, cum = 0.0;
        if (tid < kept) mass[tid] = mine = sc.mass(key_logit(sh.list[tid]), ref);
        if (tid < a.N) sh.found[tid] = INT_MAX;
        __syncthreads();
        int index = 0;
        if (tid < kept) {
            index = key_index(sh.list[tid]);
#pragma unroll 4
            for (int j = 0; j < kept; ++j) cum += key_index(sh.list[j]) <= index ? mass[j] : 0.0;
            for (int i = 0; i < a.N; ++i)
                if (mine > 0.0 && cum > (double)sh.u[i] * total) atomicMin(&sh.found[i], index);
        }
        __syncthreads();
        // rounding may leave all sums at or below the mark: the last entry with mass then
        for (int i = 0; i < a.N; ++i) {
            const float u = sh.u[i];
            const bool fine = u >= 0.f && u < 1.f, none = sh.found[i] == INT_MAX;
            if (none) {
                int last = tid < kept && mine > 0.0 ? index : -1;
                last = __reduce_max_sync(0xffffffffu, last);
                if ((tid & 31) == 0) sh.wcnt[tid >> 5] = last;
                __syncthreads();
                for (int w = 0; w < kWarps; ++w) last = max(last, sh.wcnt[w]);
                __syncthreads();
                if (tid == 0) sh.found[i] = last;
                __syncthreads();
            }
            if (fine ? tid < kept && index == sh.found[i] : tid == 0) report(i, fine, index, sc.mass(key_logit(sh.list[tid < kept ? tid : 0]), ref) / total);
        }
        __syncthreads();
        return;
    }
    // the kept entries in vocabulary order, and where the uniform numbers fall among them
    uint64_t* by_index = sh.other;
    for (int i = tid; i < kept; i += kThreads) by_index[i] = ((uint64_t)(uint32_t)key_index(sh.list[i]) << 32) | (uint32_t)i;
    block_sort(by_index, kept);
    for (int i = tid; i < kept; i += kThreads) sh.all[i] = sc.mass(key_logit(sh.list[(uint32_t)by_index[i]]), ref);
    block_scan(sh.all, kept, sh.tmp_d);
    for (int i = tid; i < a.N; i += kThreads) {
        const float u = sh.u[i];
        const double total = sh.all[kept - 1];
        int at = first_above(sh.all, kept, (double)u * total, false);
        while (at >= kept || (at > 0 && !(sh.all[at] > sh.all[at - 1]))) --at;       // (none above: the last with mass)
        report(i, u >= 0.f && u < 1.f, (int)(by_index[at] >> 32), sc.mass(key_logit(sh.list[(uint32_t)by_index[at]]), ref) / total);
    }
}

template <typename T, bool HELD>
__global__ void __launch_bounds__(kThreads, 2)
sample_kernel(SampleCall a) {
    extern __shared__ __align__(16) uint4 data[];
    __shared__ RowShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        sh.abort_flag = 0;
        for (int q = 0; q < kPieces; ++q) sm100::mbar_init(&sh.bar[q], 1);
        sm100::fence_barrier_init();
    }
    __syncthreads();
    begin_dependent(a.logits, a.inv_temp, a.top_k, a.top_p, a.min_p, a.n_used, a.u, a.tokens, a.prob, a.dense, a.lse, a.kept, a.status);
    const int parts = a.parts, V = a.V;
    const long long r = blockIdx.x / parts;
    const int rank = parts == 1 ? 0 : (int)sm100::cluster_ctarank();
    const Slice<T, HELD> sl(a.logits, a.ld, r, V, parts, rank, data);
    if constexpr (HELD) sl.copy(sh, a.withheld);

    // ---- what the row asks for
    float it = a.inv_temp ? a.inv_temp[r] : 1.f;
    int k = a.top_k ? a.top_k[r] : 0;
    float p = a.top_p ? a.top_p[r] : 1.f;
    float mp = a.min_p ? a.min_p[r] : 0.f;
    const bool used = !a.n_used || (int)(r % a.per_used) < a.n_used[r / a.per_used];
    if (!used) it = 1.f;
    bool bad = !(it >= 1e-6f);
    if (bad || it > 1e30f) { if (!bad) k = 1; it = 1.f; }                          // infinite: the first entry alone
    if (k >= V) k = 0;
    const bool by_k = k >= 1, by_p = p < 1.f, by_mp = mp > 0.f;
    p = fmaxf(p, 0.f);
    mp = by_mp ? fminf(mp, 1.f) : 0.f;
    if (tid < a.N) sh.u[tid] = a.u[r * a.N + tid];
    Scale sc(it);
    __syncthreads();

    bool all_stay = !by_k && !by_p && !by_mp;
    const bool ok = all_stay ? sum_all(sh, sl, sc, a.wait_cycles) : first_pass<false>(sh, sl, 0.f, a.wait_cycles);
    sync_parts(parts);
    float top = top_of_parts(sh, parts);
    bad = bad || (used && top == INFINITY);                                        // (no distribution)
    if (bad || !used) top = -INFINITY;
    if (top > -INFINITY) sc.from(top);
    if (sc.base != 0.f) all_stay = false;                                          // (its sums are with another base)
    const int ref = top > -INFINITY ? sc.whole(top) : 0;
    const double top_mass = sc.mass(top, ref), least = (double)mp * top_mass;
    float* dense = a.dense ? a.dense + r * (long long)V : nullptr;
    const int per = ((V + parts - 1) / parts + 3) & ~3;                            // this CTA's share of the output row
    const int o0 = min(V, rank * per), o1 = min(V, o0 + per);

    int kind = kNone;
    uint64_t border = ~0ull;                                                       // kWide: the key of the last entry that stays
    double total = 0.0;
    int kept = 0;
    if (top > -INFINITY) {
        kind = kWide;
        bool summed = false;                                                       // sh.chunk has what the draws need, but for the listed entries
        bool narrow = false;                                                       // the list has all that can stay
        // ---- the list
        if (by_k && k <= kFewK) {
            const float thr = kth_group(sh, parts, k);
            list_from(sh, sl, thr);
            sync_parts(parts);
            narrow = listed(sh, parts) <= (uint32_t)kListMax;
        }
        if (!narrow && (by_k || by_p)) {
            LinearBins lin(top, sc, by_k ? 16.f : 32.f);
            fill_bins(sh, sl, by_k, by_p, lin, 0, 0.0);
            const uint32_t n_all = sh.all_count[kBins - 1];
            const double m_all = sh.all[kBins - 1], m_far = (double)(n_all - sh.all_count[kBins - 2]) * exp2(-(double)lin.octaves * (kBins - 1));
            const bool cut_k = by_k && (uint32_t)k < n_all;
            uint32_t count0 = 0;                                                   // what stands in front of the bins
            double mass0 = 0.0;
            int bk, b_lo, b_hi, m_lo;
            bool p_counts;
            uint32_t n_list, n_down;
            const auto count_to = [&](int b) { return b >= 0 ? sh.all_count[b] : count0; };
            const auto mass_to = [&](int b) { return b >= 0 ? sh.all[b] : mass0; };
            const auto find = [&]() {
                // bin of the k-th entry; bins between which the border of top_p must lie: masses are known to 2e-5 (2^-17 from the units,
                // 3e-6 from a distance in 32 bits) and to what the last bin may hold, and M, the mass of the k first entries, to that of the k-th's bin
                bk = kBins - 1;
                if (cut_k) {
                    find_bin(sh.all_count, (uint32_t)k, &sh.found[0]);
                    __syncthreads();
                    bk = sh.found[0];
                }
                b_lo = b_hi = bk;
                if (by_p) {
                    const double lo = cut_k ? fmax(mass_to(bk - 1), 1.0) : m_all, hi = (cut_k ? mass_to(bk) : m_all) + m_far;
                    find_bin(sh.all, (double)p * lo * (1.0 - 4e-5), &sh.found[1]);
                    find_bin(sh.all, (double)p * hi * (1.0 + 4e-5), &sh.found[2]);
                    __syncthreads();
                    b_lo = min(sh.found[1], bk);
                    b_hi = min(sh.found[2], bk);
                }
                // min_p's border: above, among or below the listed bins
                m_lo = b_lo;
                p_counts = by_p;
                if (by_mp) {
                    const int bm = (int)floorf(lin.at(-log2((double)mp)));
                    if (bm + 1 < b_lo) { p_counts = false; m_lo = -1; }
                    else m_lo = min(m_lo, max(0, bm - 1));
                }
                const int to = p_counts ? b_hi : bk;
                n_list = count_to(to) - count_to(max(m_lo, 0) - 1) + (cut_k && bk > to ? count_to(bk) - count_to(bk - 1) : 0);
                n_down = count_to(cut_k ? bk : b_hi);                              // all down to the border
            };
            find();
            if ((cut_k || by_p) && m_lo >= 0 && n_list > (uint32_t)kListMax && n_down > (uint32_t)kListMax) {
                const int from = m_lo, to = max(bk * cut_k, b_hi);
                if (to < kBins - 1) {
                    count0 = count_to(from - 1);
                    mass0 = mass_to(from - 1);
                    lin.zoom(from, to);
                    __syncthreads();
                    fill_bins(sh, sl, by_k, by_p, lin, count0, mass0);
                    find();
                }
            }
            const int end = by_p ? b_hi : bk;
            if ((cut_k || by_p) && n_down <= (uint32_t)kListMax) {
                // everything down to the border is few: listed (with top-k and top-p, down to the k-th)
                const int down = cut_k ? bk : end;
                __syncthreads();
                list_from(sh, sl, lin.edge(down));
                if (!cut_k) {                                                      // top_p of the whole row: its mass
                    sum_chunks<false>(sh, sl, sc, ref, 0.f, 0.f, 0.f, 0.f, nullptr);
                    summed = true;
                }
                sync_parts(parts);
                narrow = true;
            } else if (cut_k || by_p) {
                // flat: the borders' bins are listed, what is above them is summed up
                if (m_lo >= 0) {
                    const int above_k = cut_k ? count_to(bk - 1) : 0, in_bk = cut_k ? (int)count_to(bk) - above_k : 0;
                    const int to = p_counts ? b_hi : bk;
                    if (n_list <= (uint32_t)kListMax) {
                        if (tid == 0) sh.cta_n = 0;
                        __syncthreads();
                        int n_over = 0;
                        // the bins' borders as logits: above the listed ones, down to their end, and the k-th's bin (a warp each)
                        if (warp < 4) {
                            const float e = warp < 2 || cut_k ? lin.edge(warp == 0 ? m_lo - 1 : warp == 1 ? to : warp == 2 ? bk - 1 : bk) : -INFINITY;
                            if (lane == 0) sh.edges[warp] = e;
                        }
                        __syncthreads();
                        const float above_them = sh.edges[0], end_them = sh.edges[1], above_k_bin = sh.edges[2], end_k_bin = sh.edges[3];
                        // (without top-k, above_k_bin is minus infinity and nothing lies below it)
                        double mid = sum_chunks<true>(sh, sl, sc, ref, above_them, end_them, above_k_bin, end_k_bin, &n_over);
                        n_over = __reduce_add_sync(0xffffffffu, n_over);
                        if (lane == 0) sh.wcnt[warp] = n_over;
                        mid = warp_add(mid);
                        if (lane == 0) sh.tmp_d[warp] = mid;
                        __syncthreads();
                        if (tid == 0) {
                            for (int w = 1; w < kWarps; ++w) { mid += sh.tmp_d[w]; n_over += sh.wcnt[w]; }
                            sh.cta_mid = mid;
                            sh.cta_count = n_over;
                        }
                        sync_parts(parts);
                        if (rank == 0) {
                            // masses above the listed bins, chunk by chunk; the listed entries in order
                            const int n = collect(sh.list, &sh.cta_n, parts), per_part = kWarps * sl.iters, chunks = parts * per_part;
                            block_sort(sh.list, n);
                            double above = 0.0;
                            mid = 0.0;
                            mid = warp_add(of_parts(&sh.cta_mid, parts));
                            const int n_above = __reduce_add_sync(0xffffffffu, of_parts(&sh.cta_count, parts));
                            for (int i = tid; i < chunks; i += kThreads) above += *of_rank(&sh.chunk[i % per_part], i / per_part);
                            above = warp_add(above);
                            __syncthreads();
                            if (lane == 0) sh.tmp_d[warp] = above;
                            __syncthreads();
                            above = 0.0;
                            for (int w = 0; w < kWarps; ++w) above += sh.tmp_d[w];
                            for (int i = tid; i < n; i += kThreads) sh.all[i] = sc.mass(key_logit(sh.list[i]), ref);
                            block_scan(sh.all, n, sh.tmp_d);
                            // how many of the list belong to the k first; the listed ones in front of the k-th's bin stand before them
                            int len = n;
                            const bool apart = cut_k && bk > to;
                            if (cut_k) len = (apart ? n - in_bk : above_k - n_above) + (k - above_k);
                            len = min(len, n);
                            if (p_counts) {
                                const double listed_mass = len ? sh.all[len - 1] : 0.0;
                                const double m_k = above + listed_mass + mid;
                                const int span = apart ? n - in_bk : len;                            // the border of top_p is not among the k-th's bin alone
                                len = min(len, min(first_above(sh.all, span, (double)p * m_k - above, true) + 1, span));
                            }
                            if (by_mp) {
                                int l = 0, h = len;
                                while (l < h) {
                                    const int m = (l + h) >> 1;
                                    if (sc.mass(key_logit(sh.list[m]), ref) < least) h = m; else l = m + 1;
                                }
                                len = l;
                            }
                            if (tid == 0) {
                                sh.border = len ? sh.list[len - 1] : sh.list[0] - 1;                 // (none of the list: all above its bins)
                                sh.kept = n_above + len;
                                sh.total = above + (len ? sh.all[len - 1] : 0.0);
                            }
                            // the draws' chunks: with the listed entries that stay
                            __syncthreads();
                            if (a.N) {
                                const int stays = len;
                                for (int i = tid; i < kBins; i += kThreads) sh.other[i] = 0;
                                __syncthreads();
                                for (int i = tid; i < stays; i += kThreads) {
                                    const int id = sl.chunk_of(key_index(sh.list[i]));
                                    if (id >= 0 && id < chunks)
                                        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.other[id]),
                                                  (unsigned long long)(sc.mass(key_logit(sh.list[i]), ref) * kUnit + 0.5));
                                    else set_status(a.status, SD_ERR_BOUNDS);
                                }
                                __syncthreads();
                                for (int i = tid; i < chunks; i += kThreads)
                                    sh.all[i] = *of_rank(&sh.chunk[i % per_part], i / per_part) + (double)sh.other[i] / kUnit;
                                block_scan(sh.all, chunks, sh.tmp_d);
                            }
                        }
                        sync_parts(parts);
                        border = *of_rank(&sh.border, 0);
                        total = *of_rank(&sh.total, 0);
                        kind = -1;                                                 // (done: borders, count and mass are known)
                    } else {
                        // more than a list holds in the borders' bins
                        if (cut_k) search_border(sh, sl, false, (uint64_t)k, -1.0, ~0ull, sc, ref, &border);
                        if (p_counts) search_border(sh, sl, true, 0, (double)p, border, sc, ref, &border);
                    }
                }
            }
        } else if (!narrow && by_mp) {
            // min_p alone: the entries that stay, listed if they are few
            const float d = (float)(-log2((double)mp) * 1.0001 / sc.c), from = top - d - fabsf(top) * 1e-6f - d * 1e-4f;
            list_from(sh, sl, from);                                               // (the few that are too small are cut off below)
            sync_parts(parts);
            narrow = listed(sh, parts) <= (uint32_t)kListMax;
        }

        // ---- the row is decided on the list
        if (narrow) {
            if (dense) fill_floats(dense + o0, o1 - o0, a.scaled ? -INFINITY : 0.f);
            if (rank == 0) {
                int n = collect(sh.list, &sh.cta_n, parts);
                double all = 0.0;
                if (summed) {
                    const int per_part = kWarps * sl.iters, chunks = parts * per_part;
                    for (int i = tid; i < chunks; i += kThreads) all += *of_rank(&sh.chunk[i % per_part], i / per_part);
                    all = warp_add(all);
                    if (lane == 0) sh.tmp_d[warp] = all;
                    __syncthreads();
                    all = 0.0;
                    for (int w = 0; w < kWarps; ++w) all += sh.tmp_d[w];
                }
                // the other CTAs' parts of the output are filled, and they are not needed any more
                sync_parts(parts);
                if (n == 0) {                                                      // (a slice that did not come: what follows needs an entry)
                    if (tid == 0) sh.list[0] = order_key(top, 0);
                    n = 1;
                    __syncthreads();
                }
                n = sort_list(sh, sh.list, n, by_k ? min(k, kListMax) : kListMax);
                for (int i = tid; i < n; i += kThreads) sh.all[i] = sc.mass(key_logit(sh.list[i]), ref);
                block_scan(sh.all, n, sh.tmp_d);
                int len = n;
                if (by_p) len = min(len, first_above(sh.all, len, (double)p * (summed ? all : sh.all[len - 1]), true) + 1);
                if (by_mp) {
                    int l = 0, h = len;
                    while (l < h) {
                        const int m = (l + h) >> 1;
                        if (sc.mass(key_logit(sh.list[m]), ref) < least) h = m; else l = m + 1;
                    }
                    len = l;
                }
                len = max(len, 1);
                kept = len;
                total = sh.all[len - 1];
            } else {
                sync_parts(parts);
            }
            kind = kList;
        } else if (kind == kWide) {
            // ---- everything up to a border (or all, or by min_p): its mass chunk by chunk
            if (!all_stay) {
                int cnt = 0;
                sum_kept(sh, sl, sc, ref, border, least, &cnt);
                cnt = __reduce_add_sync(0xffffffffu, cnt);
                if (lane == 0) sh.wcnt[warp] = cnt;
                __syncthreads();
                if (tid == 0) {
                    for (int w = 1; w < kWarps; ++w) cnt += sh.wcnt[w];
                    sh.cta_count = cnt;
                }
            }
            if (!all_stay) sync_parts(parts);
            if (rank == 0) {
                const int per_part = kWarps * sl.iters, chunks = parts * per_part;
                for (int i = tid; i < chunks; i += kThreads) {
                    double m = *of_rank(&sh.chunk[i % per_part], i / per_part);
                    if (all_stay) {
                        const int e = *of_rank(&sh.chunk_ref[i % per_part], i / per_part);
                        m = e == INT_MIN ? 0.0 : times_pow2(m, e - ref);
                    }
                    sh.all[i] = m;
                }
                block_scan(sh.all, chunks, sh.tmp_d);
                const int cnt = __reduce_add_sync(0xffffffffu, of_parts(&sh.cta_count, parts));
                if (tid == 0) { sh.total = sh.all[chunks - 1]; sh.kept = cnt; }
                __syncthreads();
            }
        }
        if (kind == -1) kind = kWide;
    }

    // ---- outputs
    if (kind == kNone) {
        if (dense) fill_floats(dense + o0, o1 - o0, a.scaled ? -INFINITY : 0.f);
        if (rank == 0) {
            if (bad && tid == 0) set_status(a.status, SD_ERR_INVALID_ARG);
            for (int i = tid; i < a.N; i += kThreads) { a.tokens[r * a.N + i] = -1; if (a.prob) a.prob[r * a.N + i] = 0.f; }
            if (tid == 0) { if (a.lse) a.lse[r] = -INFINITY; if (a.kept) a.kept[r] = 0; }
        }
        if (parts > 1) sync_parts(parts);
    } else if (kind == kList) {
        if (rank == 0) {                                                           // (alone by now)
            if (tid == kThreads - 1) {
                if (a.lse) a.lse[r] = log_mass(sc, top, it, ref, total);
                if (a.kept) a.kept[r] = kept;
            }
            if (dense)
                for (int i = tid; i < kept; i += kThreads) {
                    const float x = key_logit(sh.list[i]);
                    dense[key_index(sh.list[i])] = a.scaled ? scaled_logit(x, it) : (float)(sc.mass(x, ref) / total);
                }
            if (a.N) draw_from_list(sh, a, r, sc, ref, kept);
        }
    } else {
        if (dense) sync_parts(parts);                                              // the total is known
        else __syncthreads();
        if (dense) total = *of_rank(&sh.total, 0);
        if (rank == 0) {
            total = sh.total;
            if (tid == kThreads - 1) {
                if (a.lse) a.lse[r] = log_mass(sc, top, it, ref, total);
                if (a.kept) a.kept[r] = sh.kept;
            }
            const int chunks = parts * kWarps * sl.iters;
            for (int d = warp; d < a.N; d += kWarps) {                             // a warp per draw
                const float u = sh.u[d];
                const bool fine = u >= 0.f && u < 1.f;
                int token = -1;
                double mass = 0.0;
                if (fine) {
                    const double target = (double)u * sh.all[chunks - 1];
                    int g = first_above(sh.all, chunks, target, false);
                    while (g >= chunks || (g > 0 && !(sh.all[g] > sh.all[g - 1]))) --g;
                    token = chunk_crossing(sl, g, target - (g ? sh.all[g - 1] : 0.0), sc, ref,
                                           [&](float x, int index, double m) { return x > -INFINITY && order_key(x, index) <= border && m >= least; }, &mass);
                } else if (lane == 0) set_status(a.status, SD_ERR_INVALID_ARG);
                if (lane == 0) { a.tokens[r * a.N + d] = token; if (a.prob) a.prob[r * a.N + d] = (float)(mass / total); }
            }
        }
        if (dense) {
            const float c32 = (float)fmin(sc.c, 3.4028234663852886e38), at_top = (float)(top_mass / total);
            constexpr int E = Row<T>::kE;
            // the borders as logits; masses are compared where the distance in 32 bits leaves them open
            const float border_at = border == ~0ull ? -INFINITY : key_logit(border);
            const float d = by_mp ? (float)(-log2((double)mp) / sc.c) : 0.f, slack = fabsf(top) * 1e-6f + d * 1e-4f;
            const float surely = by_mp ? top - d + slack : -INFINITY, never = by_mp ? top - d - slack : -INFINITY;
            const auto value = [&](float x, int v) {
                bool in = x > border_at || (x == border_at && border != ~0ull && order_key(x, v) <= border);
                if (by_mp && !(x > surely)) in = in && x >= never && sc.mass(x, ref) >= least;
                return a.scaled ? (in ? scaled_logit(x, it) : -INFINITY) : (in ? at_top * exp2f((x - top) * c32) : 0.f);
            };
            if (((reinterpret_cast<uintptr_t>(dense) + (uintptr_t)((long long)sl.first * 4)) & 15) == 0) {
                sl.each_chunk([&](const uint4& raw, int i) {
                    const int v = sl.first + i * E;
                    if (i >= min(sl.nv, (warp + 1) * sl.seg)) return;
                    float x[E];
                    Row<T>::unpack(raw, x);
                    if (v >= 0 && v + E <= V) {
#pragma unroll
                        for (int e = 0; e < E; e += 4)
                            __stcs(reinterpret_cast<float4*>(dense + v + e), make_float4(value(x[e], v + e), value(x[e + 1], v + e + 1),
                                                                                         value(x[e + 2], v + e + 2), value(x[e + 3], v + e + 3)));
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (v + e >= 0 && v + e < V) dense[v + e] = value(x[e], v + e);
                    }
                }, [](int) {});
            } else {
                const T* entries = reinterpret_cast<const T*>(data);
                const int lo = max(0, sl.first), hi = min(V, sl.first + sl.nv * E);
#pragma unroll 4
                for (int v = lo + tid; v < hi; v += kThreads) {
                    float x;
                    if constexpr (!HELD) x = sl.row.at(v);
                    else if constexpr (sizeof(T) == 4) x = (float)entries[v - sl.first];
                    else x = __uint_as_float((uint32_t)entries[v - sl.first] << 16);
                    dense[v] = value(x, v);
                }
            }
        }
        __syncwarp();
        if (parts > 1) sync_parts(parts);                                          // nobody leaves while another CTA reads
    }
    if (!ok) { set_status(a.status, SD_ERR_TIMEOUT); sm100::unwind_pause(); }
}

// A row's shares where it lies in memory: as many as still run at once, and two where rows differ in what they ask for (256 rows, all
// kinds mixed: 235 us in one, 199 in two, 209 in four; 2048 rows: 920, 1026, 1309 us).
static int shares_of(int M, int sms) { return 4LL * M <= 2 * sms ? 4 : M <= 2 * sms ? 2 : 1; }

// CTAs per row: slices of at most 80 KB while eight are enough for that, and more of them while all run at once, and a warp's
// lanes have a vector each (80 rows of 32003 bf16, top-p: 79 us in one, 60 in two)
static int parts_for(int M, int nvec, int sms) {
    int parts = 1;
    while (parts < 8 && ((nvec + parts - 1) / parts > 5120 || ((long long)M * parts <= sms && nvec / (parts * 2) >= kThreads - 32))) parts *= 2;
    return parts;
}

}  // namespace rows

using namespace rows;

sd_status launch_top_logits(const void* logits, int dtype, long long ld, int M, int V, int K, float inv_temp, float* values, int32_t* index,
                            float* lse, int32_t* dev_status, cudaStream_t st) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SD_ERR_CUDA;
    const int nvec = (int)(((long long)V * (dtype == SD_F32 ? 4 : 2) + 15) / 16) + 1;
    const TestKnobs knobs = test_knobs();
    const int sms = sm_count(dev), fit = parts_for(M, nvec, sms);
    // (GPCs whose SMs are no multiple of a cluster's leave some: 33 clusters of eight run at once, 71 of four)
    const bool all_at_once = (long long)M * fit <= 2 * sms - 32;
    if (K <= kSomeK && (M >= sms / 2 || !all_at_once)) {
        auto kern = dtype == SD_F32 ? top_stream_kernel<float> : top_stream_kernel<uint16_t>;
        // (up to one row per SM: so much shared memory that no SM takes two; 80 rows of f32 27 -> 20 to 25 us, by the rows)
        const int ctas = 2 * sms, steps = (nvec + kWarps * kStreamVecs - 1) / (kWarps * kStreamVecs), alone = M <= sms ? 96 * 1024 : 0;
        if (!allow_dynamic_smem(kern, 96 * 1024)) return SD_ERR_CUDA;
        return launch_dependent(kern, dim3((unsigned)(M < ctas ? M : ctas)), kThreads, alone, 1, st, logits, ld, V, M, steps, K, inv_temp, values, index, lse);
    }
    // (long lists: as sampled rows, below; K = 1000 of 148 rows of 152064 f32 136 -> 76 us, of 2048 1697 -> 892)
    const bool held = nvec <= 5120 || all_at_once;
    const int parts = held ? fit : shares_of(M, sms);
    const int smem = held ? (nvec + parts - 1) / parts * 16 : kCopies * kBins * 4 + kBins * 8;
    auto kern = dtype == SD_F32 ? (held ? top_kernel<float, true> : top_kernel<float, false>)
                                : (held ? top_kernel<uint16_t, true> : top_kernel<uint16_t, false>);
    if (!allow_dynamic_smem(kern, smem)) return SD_ERR_CUDA;
    return launch_dependent(kern, dim3((unsigned)M * parts), kThreads, smem, parts, st, logits, ld, V, parts, K, inv_temp, values, index, lse, dev_status,
                            knobs.withhold ? 16 : 0, knobs.wait_cycles);
}

sd_status launch_sample(const void* logits, int dtype, long long ld, int M, int V, const sd_sampling& how, const float* u, int N, int32_t* tokens,
                        float* prob, float* dense, bool scaled, float* lse, int32_t* kept, int32_t* dev_status, cudaStream_t st) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SD_ERR_CUDA;
    const int nvec = (int)(((long long)V * (dtype == SD_F32 ? 4 : 2) + 15) / 16) + 1;
    // One reading into shared memory where the SMs hold all clusters at once, two CTAs each (slices above 77 KB, of which an SM holds one, then take
    // two waves), and where one CTA holds a row.  Beyond that the waves of
    // clusters wait for their own copies, and passes through L2 by CTAs of which two are resident are faster.  152064 f32, k = 50 / top_p:
    // 64 rows 36 -> 21 / 108 -> 90 us, 256 rows 101 -> 72 / 368 -> 270 us; 32 rows are as fast, but 57 -> 88 us.
    const int fit = parts_for(M, nvec, sm_count(dev)), sms = sm_count(dev);
    const bool held = nvec <= 5120 || (long long)M * fit <= 2 * sms;
    const int parts = held ? fit : shares_of(M, sms);
    const int smem = held ? (nvec + parts - 1) / parts * 16 : kCopies * kBins * 4 + kBins * 8;
    auto kern = dtype == SD_F32 ? (held ? sample_kernel<float, true> : sample_kernel<float, false>)
                                : (held ? sample_kernel<uint16_t, true> : sample_kernel<uint16_t, false>);
    if (!allow_dynamic_smem(kern, smem)) return SD_ERR_CUDA;
    const TestKnobs knobs = test_knobs();
    const SampleCall call{logits, ld, V, parts, how.inv_temp, how.top_k, how.top_p, how.min_p, how.n_used, how.per, u, N, tokens, prob, dense, scaled, lse, kept, dev_status,
                          knobs.withhold ? 16 : 0, knobs.wait_cycles};
    return launch_dependent(kern, dim3((unsigned)M * parts), kThreads, smem, parts, st, call);
}

}  // namespace sdv
