// Top logits, filtered sampling and filtered logits of rows [M][V] (sd_top_logits, sd_sample_logits, sd_filter_logits).
//
// One cluster of `parts` CTAs per row; every warp reads one consecutive piece of it.  A row is read once: a warp keeps what its
// lanes see above a threshold that only rises (at least `keep` entries are known to reach it), so that of 152064 entries a few
// hundred ever enter the list in shared memory, and where the row's whole mass is needed it is summed up beside that, one sum
// per chunk of kU * 32 vectors.  The lists meet in the first CTA, are cut to the `keep` first entries in order and sorted; on
// the sorted list top-k, top-p and min-p are prefix lengths.  Only where a border lies behind the listed entries (flat rows)
// the row is read again (it is in L2 by then): histograms of counts and masses, over the cluster's CTAs, narrow the border down to
// one entry.  The draw is by inverse CDF in vocabulary order: over the list, or over the chunks' sums and then one chunk.
#include <limits.h>
#include "rows.cuh"

namespace sdv {
namespace rows {

constexpr int kKeepMax = 1024;         // entries of a sorted list
constexpr int kCap = 8192;             // entries that a CTA's list holds before it is cut
constexpr int kU = 4;                  // vectors in flight per lane
constexpr int kMaxChunks = 1024;       // of a row: 2^18 entries in chunks of 512, and one broken one for each of 128 warps
constexpr int kBins = 1024;

struct Plan {                          // what the first CTA found out about its row
    int kind;                          // kNone: no entry left; kList: the kept entries are listed; kWide: they are not
    int n;                             // entries kept (kList)
    int ref;
    float top;                         // largest logit
    double total;                      // mass of the kept entries (kList)
};
enum { kNone, kList, kWide };

struct RowShared {
    uint32_t n;                        // entries in the list
    float thr;                         // a logit that at least `keep` entries seen so far reach
    uint64_t thr_key;                  // and the key of the last of them, where it is known
    uint32_t hist[256];
    uint64_t sel_prefix;
    uint32_t sel_left;
    int sel_done;
    float wmax[kWarps], wsum[kWarps];
    int wcnt[kWarps];
    float cta_top, cta_sum;
    int cta_count;
    double tmp_d[kWarps];
    uint64_t tmp_u[kWarps];
    uint64_t lo[kWarps], hi[kWarps], cta_lo, cta_hi;
    struct { uint32_t bin, n; uint64_t count, mass; } pick;      // a bin, the entries in it, and what stands in front of it
    uint64_t border, border_mass;
    Plan plan;
    double chunk[kMaxChunks];          // sums of this CTA's chunks, relative to 2^chunk_ref
    int chunk_ref[kMaxChunks];
    double all[kMaxChunks];            // the row's
};

// ---------------------------------------------------------------- cutting a list down
// Leaves the `keep` first of buf[0..n) in buf[0..keep), in any order, and their last key in thr_key (keep < n <= kCap).  Radix
// selection from the highest bit in which the keys differ.
__device__ void cut_list(RowShared& sh, uint64_t* buf, int n, int keep) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __syncthreads();
    uint64_t lo = ~0ull, hi = 0;
    for (int i = tid; i < n; i += kThreads) { const uint64_t k = buf[i]; lo = min(lo, k); hi = max(hi, k); }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    if (lane == 0) { sh.lo[warp] = lo; sh.hi[warp] = hi; }
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
        if (tid < 256) sh.hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t k = buf[i];
            if (shift == 64 || (k >> shift) == (prefix >> shift)) atomicAdd(&sh.hist[(k >> down) & ((1u << step) - 1)], 1u);
        }
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
        __syncthreads();
    }
    // keys are distinct (the index is part of them): exactly `keep` are at or below `last`
    constexpr int kPer = kCap / kThreads;
    uint64_t mine[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = tid + j * kThreads;
        mine[j] = i < n ? buf[i] : ~0ull;
    }
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
    uint64_t worst = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (mine[j] <= last && mine[j] != ~0ull) {
            const uint32_t at = atomicAdd(&sh.n, 1u);
            if (at < (uint32_t)kCap) buf[at] = mine[j];
            worst = max(worst, mine[j]);
        }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) worst = max(worst, __shfl_xor_sync(0xffffffffu, worst, d));
    if (lane == 0) sh.hi[warp] = worst;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kWarps; ++w) worst = max(worst, sh.hi[w]);
        sh.thr_key = worst;
        sh.thr = key_logit(worst);
    }
    __syncthreads();
}

// ---------------------------------------------------------------- the first pass
// This CTA's part of the row: the entries that may be among its `keep` first ones into buf, the largest logit, and either the
// chunks' masses (need_mass) or (LSE) the sum of exp((x - largest) inv_temp).
template <typename T, bool LSE>
__device__ void scan_part(RowShared& sh, uint64_t* buf, const Row<T>& row, int v0, int v1, int seg, int iters, int keep, bool need_mass,
                          const Scale& sc, float c32) {
    constexpr int E = Row<T>::kE;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int w0 = min(v1, v0 + warp * seg), w1 = min(v1, w0 + seg);
    if (tid == 0) { sh.n = 0; sh.thr = -INFINITY; sh.thr_key = ~0ull; }
    __syncthreads();
    float thr = -INFINITY, top = -INFINITY, sum = 0.f;
    uint64_t thr_key = ~0ull;
    uint32_t bound = 0;                                                            // entries in the list, at most
    for (int it = 0; it < iters; ++it) {
        uint4 raw[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int i = w0 + (it * kU + u) * 32 + lane;
            raw[u] = i < w1 ? row.load(i) : Row<T>::nothing();
        }
        float m_lo = -INFINITY, m_hi = -INFINITY;                                  // largest of either half
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            float x[E];
            Row<T>::unpack(raw[u], x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (u < kU / 2) m_lo = fmaxf(m_lo, x[e]);
                else m_hi = fmaxf(m_hi, x[e]);
            }
        }
        const float vmax = fmaxf(m_lo, m_hi);
        if constexpr (LSE) {
            const float now = fmaxf(top, vmax);
            if (now > -INFINITY) {
                sum *= ex2((top - now) * c32);
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    float x[E];
                    Row<T>::unpack(raw[u], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) sum += ex2((fmaxf(x[e], -INFINITY) - now) * c32);
                }
            }
        } else if (need_mass) {
            const int ref = __reduce_max_sync(0xffffffffu, vmax > -INFINITY ? sc.whole(vmax) : INT_MIN);
            double s = 0.0;
            if (ref != INT_MIN) {
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    float x[E];
                    Row<T>::unpack(raw[u], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) s += sc.mass(x[e], ref);
                }
                s = warp_add(s);
            }
            if (lane == 0) { sh.chunk[warp * iters + it] = s; sh.chunk_ref[warp * iters + it] = ref; }
        }
        top = fmaxf(top, vmax);
        if (keep == 0) continue;
        if (it == 0) {
            // a first threshold: the least of as many groups' largest entries as there are entries to keep
            float g = keep > kThreads ? fminf(m_lo, m_hi) : vmax;
            for (int d = 1; d < 32 && (kThreads >> __ffs(d)) >= keep; d <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, d));
#pragma unroll
            for (int d = 16; d >= 1; d >>= 1) g = fminf(g, __shfl_xor_sync(0xffffffffu, g, d));
            if (lane == 0) sh.wmax[warp] = g;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWarps; ++w) g = fminf(g, sh.wmax[w]);
            thr = g;
        }
        bool any = vmax >= thr && vmax > -INFINITY;
        uint32_t threads = __syncthreads_count(any);
        bool one_by_one = false;
        if (bound + threads * (kU * E) > (uint32_t)kCap) {
            bound = sh.n;                                                          // (nothing is added until all have seen it)
            __syncthreads();
            if (bound > (uint32_t)max(2 * keep, 512) || bound + threads * (kU * E) > (uint32_t)kCap) {
                if (bound > (uint32_t)keep) {
                    cut_list(sh, buf, bound, keep);
                    bound = keep;
                    thr = sh.thr;
                    thr_key = sh.thr_key;
                    any = vmax >= thr && vmax > -INFINITY;
                    threads = __syncthreads_count(any);
                }
                one_by_one = bound + threads * (kU * E) > (uint32_t)kCap;
            }
        }
        if (threads == 0) continue;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            if (any) {
                float x[E];
                Row<T>::unpack(raw[u], x);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (x[e] >= thr && x[e] > -INFINITY) {
                        const uint64_t key = order_key(x[e], (w0 + (it * kU + u) * 32 + lane) * E + e - row.lead);
                        if (key <= thr_key) {
                            const uint32_t at = atomicAdd(&sh.n, 1u);
                            if (at < (uint32_t)kCap) buf[at] = key;
                        }
                    }
            }
            if (one_by_one) {                                                      // at most kThreads * E more each time
                __syncthreads();
                bound = sh.n;
                __syncthreads();
                if (bound > (uint32_t)(kCap - kThreads * E)) {
                    cut_list(sh, buf, bound, keep);
                    bound = keep;
                    thr = sh.thr;
                    thr_key = sh.thr_key;
                }
            }
        }
        if (!one_by_one) bound += threads * (kU * E);
    }
    // the CTA's largest logit, and sum
    const float wtop = warp_fmax(top);
    __syncthreads();
    if (lane == 0) sh.wmax[warp] = wtop;
    __syncthreads();
    float all = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all = fmaxf(all, sh.wmax[w]);
    if constexpr (LSE) {
        sum = top > -INFINITY ? sum * ex2((top - all) * c32) : 0.f;
        sum = warp_add(sum);
        if (lane == 0) sh.wsum[warp] = sum;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += sh.wsum[w];
        if (tid == 0) sh.cta_sum = s;
    }
    if (tid == 0) sh.cta_top = all;
    __syncthreads();
}

// The lists of all parts into the first CTA's, cut to the `keep` first entries and sorted (a list that travels holds at most
// kCap / parts entries).  Returns the entries there are (in the first CTA).
__device__ int meet(RowShared& sh, uint64_t* buf, int parts, int rank, int keep) {
    const int tid = threadIdx.x;
    __syncthreads();
    const uint32_t have = sh.n;
    if (have > (uint32_t)(kCap / parts) || (parts == 1 && have > (uint32_t)kKeepMax)) cut_list(sh, buf, min(have, (uint32_t)kCap), keep);
    sync_parts(parts);
    if (rank != 0) return 0;
    int n = sh.n;
    for (int r = 1; r < parts; ++r) {
        const int more = *of_rank(&sh.n, r);
        const uint64_t* from = of_rank(buf, r);
        for (int i = tid; i < more; i += kThreads) buf[n + i] = from[i];
        n += more;
    }
    __syncthreads();
    if (n > kKeepMax) { cut_list(sh, buf, n, keep); n = keep; }
    block_sort(buf, n);
    return min(n, keep);
}

// Largest logit over the parts (behind a sync_parts).
__device__ __forceinline__ float top_of_parts(RowShared& sh, int parts) {
    float top = -INFINITY;
    for (int r = 0; r < parts; ++r) top = fmaxf(top, *of_rank(&sh.cta_top, r));
    return top;
}

// The chunks of all parts as inclusive sums in sh.all, relative to 2^ref (behind a sync_parts).  Returns how many.
__device__ int scan_chunks(RowShared& sh, int parts, int per_part, int ref) {
    const int n = parts * per_part;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int r = i / per_part, at = i - r * per_part;
        const double s = *of_rank(&sh.chunk[at], r);
        const int e = *of_rank(&sh.chunk_ref[at], r);
        sh.all[i] = e == INT_MIN ? 0.0 : times_pow2(s, e - ref);
    }
    block_scan(sh.all, n, sh.tmp_d);
    return n;
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

template <typename T>
struct Part {                          // this CTA's share of a row
    Row<T> row;
    int parts, rank, v0, v1, seg, iters;
    __device__ __forceinline__ Part(const void* base, long long ld, long long r, int V, int parts_, int rank_) : row(base, ld, r, V), parts(parts_), rank(rank_) {
        const int per = (row.nvec + parts - 1) / parts;
        v0 = min(row.nvec, rank * per);
        v1 = min(row.nvec, v0 + per);
        seg = (per + kWarps - 1) / kWarps;                                         // (the same in all parts: chunks are numbered alike)
        iters = (seg + 32 * kU - 1) / (32 * kU);
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {                              // f(logit, index), entries of minus infinity and NaN left out
        constexpr int E = Row<T>::kE;
        for (int i = v0 + (int)threadIdx.x; i < v1; i += kThreads) {
            const uint4 raw = row.load(i);
            float x[E];
            Row<T>::unpack(raw, x);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] > -INFINITY) f(x[e], i * E + e - row.lead);
        }
    }
};

// ---------------------------------------------------------------- flat rows: the border by histograms
// Counts and masses (2^-43 of 2^ref as the unit; whole numbers, so that the order of additions is of no matter) of
// kBins bins, in buf; merged over the parts into inclusive sums.
struct Bins {
    uint32_t* count; uint64_t* mass;               // this CTA's
    uint64_t* sum_count; uint64_t* sum_mass;       // of all parts
    __device__ __forceinline__ explicit Bins(uint64_t* buf)
        : count(reinterpret_cast<uint32_t*>(buf)), mass(buf + kBins / 2), sum_count(buf + 3 * kBins / 2), sum_mass(buf + 5 * kBins / 2) {}
};
constexpr int kListAt = 4096;                      // where lists start in buf while the bins are in use
static_assert(7 * kBins / 2 <= kListAt && kListAt + kKeepMax <= kCap, "bins, then a list");

__device__ __forceinline__ uint64_t unit_mass(const Scale& sc, float x, int ref) { return (uint64_t)(sc.mass(x, ref) * 8796093022208.0 + 0.5); }

// bin_of(x, index): the entry's bin, or -1
template <typename T, typename F>
__device__ void fill_bins(RowShared& sh, const Bins& b, const Part<T>& part, bool masses, const Scale& sc, int ref, F bin_of) {
    const int tid = threadIdx.x;
    sync_parts(part.parts);                        // (nobody reads the bins any more)
    for (int i = tid; i < kBins; i += kThreads) { b.count[i] = 0; b.mass[i] = 0; }
    __syncthreads();
    part.each([&](float x, int index) {
        const int bin = bin_of(x, index);
        if (bin < 0) return;
        atomicAdd(&b.count[bin], 1u);
        if (masses) atomicAdd(reinterpret_cast<unsigned long long*>(&b.mass[bin]), (unsigned long long)unit_mass(sc, x, ref));
    });
    sync_parts(part.parts);
    for (int i = tid; i < kBins; i += kThreads) {
        uint64_t c = 0, m = 0;
        for (int r = 0; r < part.parts; ++r) {
            c += *of_rank(&b.count[i], r);
            if (masses) m += *of_rank(&b.mass[i], r);
        }
        b.sum_count[i] = c;
        b.sum_mass[i] = m;
    }
    block_scan(b.sum_count, kBins, sh.tmp_u);
    block_scan(b.sum_mass, kBins, sh.tmp_u);
}

// The bin in which the counts (or masses) reach `target`, at least 1 and at most their sum.
__device__ void pick_bin(RowShared& sh, const Bins& b, bool by_mass, uint64_t target) {
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint64_t* sums = by_mass ? b.sum_mass : b.sum_count;
        const int bin = min(first_above(sums, kBins, target, true), kBins - 1);
        sh.pick.bin = bin;
        sh.pick.count = bin ? b.sum_count[bin - 1] : 0;
        sh.pick.mass = bin ? b.sum_mass[bin - 1] : 0;
        sh.pick.n = (uint32_t)(b.sum_count[bin] - sh.pick.count);
    }
    __syncthreads();
}

// The last entry, in order, of the shortest prefix whose count (or mass) is at least `target`: its key, and the mass up to and
// with it.  The bins hold the row's linear histogram with pick_bin's answer in sh.pick; they are used up.
template <typename T, typename F>
__device__ void find_border(RowShared& sh, uint64_t* buf, const Bins& b, const Part<T>& part, bool by_mass, bool masses, uint64_t target,
                            const Scale& sc, int ref, F linear_bin, uint64_t* border, uint64_t* border_mass) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bin = sh.pick.bin;
    uint64_t before_n = sh.pick.count, before_m = sh.pick.mass;
    uint32_t n = sh.pick.n;
    uint64_t lo = 0, hi = ~0ull;                   // and among the bin's entries those with keys in [lo, hi]
    if (n > (uint32_t)kKeepMax) {
        // more than a list holds: equal or nearly equal logits.  The range of the keys, then bins of equal widths in it.
        uint64_t l = ~0ull, h = 0;
        part.each([&](float x, int index) {
            if (linear_bin(x) != bin) return;
            const uint64_t k = order_key(x, index);
            l = min(l, k);
            h = max(h, k);
        });
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) {
            l = min(l, __shfl_xor_sync(0xffffffffu, l, d));
            h = max(h, __shfl_xor_sync(0xffffffffu, h, d));
        }
        if (lane == 0) { sh.lo[warp] = l; sh.hi[warp] = h; }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kWarps; ++w) { l = min(l, sh.lo[w]); h = max(h, sh.hi[w]); }
            sh.cta_lo = l;
            sh.cta_hi = h;
        }
        sync_parts(part.parts);
        lo = ~0ull;
        hi = 0;
        for (int r = 0; r < part.parts; ++r) { lo = min(lo, *of_rank(&sh.cta_lo, r)); hi = max(hi, *of_rank(&sh.cta_hi, r)); }
        while (n > (uint32_t)kKeepMax) {           // (keys differ: a range of up to kBins keys leaves one entry to a bin)
            const int bits = 64 - __clzll((long long)(hi - lo));
            const int shift = max(0, bits - 10);
            fill_bins(sh, b, part, masses, sc, ref, [&](float x, int index) {
                if (linear_bin(x) != bin) return -1;
                const uint64_t k = order_key(x, index);
                return k >= lo && k <= hi ? (int)((k - lo) >> shift) : -1;
            });
            pick_bin(sh, b, by_mass, target - (by_mass ? before_m : before_n));
            before_n += sh.pick.count;
            before_m += sh.pick.mass;
            n = sh.pick.n;
            lo += (uint64_t)sh.pick.bin << shift;
            hi = lo + ((1ull << shift) - 1);
        }
    }
    // the few that are left: listed, sorted, and counted or summed up
    uint64_t* list = buf + kListAt;
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
    part.each([&](float x, int index) {
        if (linear_bin(x) != bin) return;
        const uint64_t k = order_key(x, index);
        if (k >= lo && k <= hi) {
            const uint32_t at = atomicAdd(&sh.n, 1u);
            if (at < (uint32_t)kKeepMax) list[at] = k;
        }
    });
    sync_parts(part.parts);
    if (part.rank == 0) {
        int m = min(sh.n, (uint32_t)kKeepMax);
        for (int r = 1; r < part.parts; ++r) {
            const int more = min(*of_rank(&sh.n, r), (uint32_t)(kKeepMax - m));
            const uint64_t* from = of_rank(list, r);
            for (int i = tid; i < more; i += kThreads) list[m + i] = from[i];
            m += more;
        }
        block_sort(list, m);
        uint64_t* sums = b.sum_mass;               // (its histogram is not needed any more)
        for (int i = tid; i < m; i += kThreads) sums[i] = unit_mass(sc, key_logit(list[i]), ref);
        block_scan(sums, m, sh.tmp_u);
        if (tid == 0) {
            int j = by_mass ? first_above(sums, m, target - before_m, true) : (int)(target - before_n) - 1;
            j = max(0, min(j, m - 1));
            sh.border = list[j];
            sh.border_mass = before_m + sums[j];
        }
    }
    sync_parts(part.parts);
    *border = *of_rank(&sh.border, 0);
    *border_mass = *of_rank(&sh.border_mass, 0);
}

// ---------------------------------------------------------------- top logits
template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
top_kernel(const void* logits, long long ld, int V, int parts, int K, float inv_temp, float* values, int32_t* index, float* lse) {
    extern __shared__ __align__(16) uint64_t buf[];
    __shared__ RowShared sh;
    begin_dependent(logits, values, index, lse);
    const long long r = blockIdx.x / parts;
    const int rank = parts == 1 ? 0 : (int)sm100::cluster_ctarank();
    const Part<T> part(logits, ld, r, V, parts, rank);
    const float c32 = inv_temp * kLog2e;
    scan_part<T, true>(sh, buf, part.row, part.v0, part.v1, part.seg, part.iters, K, false, Scale(1.f), c32);
    const int n = meet(sh, buf, parts, rank, K);
    if (rank == 0) {
        for (int i = threadIdx.x; i < K; i += kThreads) {
            values[r * K + i] = i < n ? key_logit(buf[i]) : -INFINITY;
            index[r * K + i] = i < n ? key_index(buf[i]) : -1;
        }
        if (lse && threadIdx.x == 0) {
            const float top = top_of_parts(sh, parts);
            float s = 0.f;
            for (int q = 0; q < parts; ++q) {
                const float t = *of_rank(&sh.cta_top, q);
                if (t > -INFINITY) s += *of_rank(&sh.cta_sum, q) * ex2((t - top) * c32);
            }
            lse[r] = top > -INFINITY && top < INFINITY ? (float)((double)top * inv_temp + log((double)s)) : top;
        }
    }
    if (parts > 1) sync_parts(parts);                                              // nobody leaves while the first CTA reads
}

// ---------------------------------------------------------------- sampling and filtering
struct SampleCall {
    const void* logits; long long ld; int V, parts;
    const float* inv_temp; const int32_t* top_k; const float* top_p; const float* min_p;
    const float* u; int N; int32_t* tokens; float* prob;       // draws (N = 0: none)
    float* dense; bool scaled;                                 // [M][V]: probabilities, or (scaled) the kept logits times inv_temp
    float* lse; int32_t* kept; int32_t* status;
};

// The entry of a chunk at which the mass in vocabulary order exceeds `over`; kept(x, index): whether an entry counts.  A warp
// calls it.  Sums that fall short by rounding end at the last entry with mass.
template <typename T, typename F>
__device__ int chunk_crossing(const Part<T>& part, int warp_of, int it, double over, const Scale& sc, int ref, F kept, double* its_mass) {
    constexpr int E = Row<T>::kE;
    const int lane = threadIdx.x & 31;
    const int w0 = min(part.v1, part.v0 + warp_of * part.seg), w1 = min(part.v1, w0 + part.seg);
    double before = 0.0, last_mass = 0.0;
    int last = -1;
    for (int u = 0; u < kU; ++u) {
        const int i = w0 + (it * kU + u) * 32 + lane;
        const uint4 raw = i < w1 ? part.row.load(i) : Row<T>::nothing();
        float x[E];
        Row<T>::unpack(raw, x);
        double m[E], s = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int index = i * E + e - part.row.lead;
            m[e] = x[e] > -INFINITY && kept(x[e], index) ? sc.mass(x[e], ref) : 0.0;
            s += m[e];
        }
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
        double found_mass = 0.0, run = before + (incl - s);
        bool crossed = false;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            run += m[e];
            if (m[e] > 0.0 && !crossed) { found = i * E + e - part.row.lead; found_mass = m[e]; crossed = run > over; }
        }
        if (over_here | with_mass) {
            const int src = over_here ? __ffs(over_here) - 1 : 31 - __clz(with_mass);
            last = __shfl_sync(0xffffffffu, found, src);
            last_mass = __shfl_sync(0xffffffffu, found_mass, src);
            if (over_here) break;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
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

template <typename T>
__global__ void __launch_bounds__(kThreads, 2)
sample_kernel(SampleCall a) {
    extern __shared__ __align__(16) uint64_t buf[];
    __shared__ RowShared sh;
    begin_dependent(a.logits, a.inv_temp, a.top_k, a.top_p, a.min_p, a.u, a.tokens, a.prob, a.dense, a.lse, a.kept, a.status);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int parts = a.parts, V = a.V;
    const long long r = blockIdx.x / parts;
    const int rank = parts == 1 ? 0 : (int)sm100::cluster_ctarank();
    const Part<T> part(a.logits, a.ld, r, V, parts, rank);

    // ---- what the row asks for
    float it = a.inv_temp ? a.inv_temp[r] : 1.f;
    int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.f;
    float mp = a.min_p ? a.min_p[r] : 0.f;
    const bool bad = !(it >= 1e-6f);
    if (bad || it > 3.4e38f) { if (!bad) k = 1; it = 1.f; }                        // infinite: the first entry alone
    if (k >= V) k = 0;
    const bool by_k = k >= 1, by_p = p < 1.f, by_mp = mp > 0.f;
    mp = by_mp ? fminf(mp, 1.f) : 0.f;
    const bool short_k = by_k && k <= kKeepMax;
    const int keep = short_k ? k : (by_k || by_p || by_mp ? kKeepMax : 0);
    const bool need_mass = !short_k;
    const Scale sc(it);

    scan_part<T, false>(sh, buf, part.row, part.v0, part.v1, part.seg, part.iters, keep, need_mass, sc, 0.f);
    const int n = meet(sh, buf, parts, rank, keep);                                // (keep = 0: only the parts' meeting)

    if (rank == 0) {
        const float top = bad ? -INFINITY : top_of_parts(sh, parts);
        const int ref = top > -INFINITY ? sc.whole(top) : 0;
        double total = 0.0;
        int kept = -1;
        if (top > -INFINITY) {
            double* sums = sh.all;
            if (need_mass) {
                const int chunks = scan_chunks(sh, parts, kWarps * part.iters, ref);
                total = sh.all[chunks - 1];
                __syncthreads();
            }
            if (keep) {
                const bool whole = short_k || n < keep;                            // every entry that can stay is listed
                for (int i = tid; i < n; i += kThreads) sums[i] = sc.mass(key_logit(buf[i]), ref);
                block_scan(sums, n, sh.tmp_d);
                const int in_k = by_k ? min(k, n) : n;
                // the listed entries whose mass min_p lets pass: a prefix
                int in_mp = n;
                if (by_mp) {
                    const double least = (double)mp * sc.mass(top, ref);
                    int lo = 0, hi = n;
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (sc.mass(key_logit(buf[mid]), ref) < least) hi = mid; else lo = mid + 1;
                    }
                    in_mp = lo;
                }
                if (whole) {
                    kept = in_k;
                    if (by_p) kept = min(kept, first_above(sums, in_k, (double)p * sums[in_k - 1], true) + 1);
                    kept = min(kept, in_mp);
                } else {
                    // entries may follow behind the list
                    const bool known = !(by_p && by_k);                            // (the mass of the k first ones is not at hand)
                    int len = n + 1;
                    if (by_p && !by_k) {
                        const int at = first_above(sums, n, (double)p * total, true);
                        if (at < n) len = at + 1;
                    }
                    if (in_mp < n) len = min(len, in_mp);
                    if (known && len <= n) kept = len;
                }
                if (kept >= 0) { kept = max(kept, 1); total = sums[kept - 1]; }
            }
        }
        __syncthreads();
        if (tid == 0) sh.plan = Plan{!(top > -INFINITY) ? kNone : (kept >= 0 ? kList : kWide), kept, ref, top, total};
    }
    sync_parts(parts);
    const Plan plan = *of_rank(&sh.plan, 0);
    float* dense = a.dense ? a.dense + r * (long long)V : nullptr;
    const int per = ((V + parts - 1) / parts + 3) & ~3;                            // this CTA's share of the output row
    const int o0 = min(V, rank * per), o1 = min(V, o0 + per);

    if (plan.kind == kNone) {
        if (dense) fill_floats(dense + o0, o1 - o0, a.scaled ? -INFINITY : 0.f);
        if (rank == 0) {
            if (bad && tid == 0) set_status(a.status, SD_ERR_INVALID_ARG);
            for (int i = tid; i < a.N; i += kThreads) { a.tokens[r * a.N + i] = -1; if (a.prob) a.prob[r * a.N + i] = 0.f; }
            if (tid == 0) { if (a.lse) a.lse[r] = -INFINITY; if (a.kept) a.kept[r] = 0; }
        }
        if (parts > 1) sync_parts(parts);
        return;
    }
    if (plan.kind == kList) {
        if (dense) {
            fill_floats(dense + o0, o1 - o0, a.scaled ? -INFINITY : 0.f);
            sync_parts(parts);                                                     // all parts are filled before entries go in
        }
        if (rank == 0) {
            if (dense)
                for (int i = tid; i < plan.n; i += kThreads) {
                    const float x = key_logit(buf[i]);
                    dense[key_index(buf[i])] = a.scaled ? scaled_logit(x, it) : (float)(sc.mass(x, plan.ref) / plan.total);
                }
            if (tid == 0) {
                if (a.lse) a.lse[r] = log_mass(sc, plan.top, it, plan.ref, plan.total);
                if (a.kept) a.kept[r] = plan.n;
            }
            if (a.N) {
                // the kept entries in vocabulary order, and where the uniform numbers fall among them
                uint64_t* by_index = buf + kListAt;
                for (int i = tid; i < plan.n; i += kThreads) by_index[i] = ((uint64_t)(uint32_t)key_index(buf[i]) << 32) | (uint32_t)i;
                block_sort(by_index, plan.n);
                for (int i = tid; i < plan.n; i += kThreads) sh.all[i] = sc.mass(key_logit(buf[(uint32_t)by_index[i]]), plan.ref);
                block_scan(sh.all, plan.n, sh.tmp_d);
                for (int i = tid; i < a.N; i += kThreads) {
                    const float u = a.u[r * a.N + i];
                    const double total = sh.all[plan.n - 1];
                    int at = first_above(sh.all, plan.n, (double)u * total, false);
                    while (at >= plan.n || (at > 0 && !(sh.all[at] > sh.all[at - 1]))) --at;       // (none above: the last with mass)
                    const bool fine = u >= 0.f && u < 1.f;
                    if (!fine) set_status(a.status, SD_ERR_INVALID_ARG);
                    a.tokens[r * a.N + i] = fine ? (int)(by_index[at] >> 32) : -1;
                    if (a.prob) a.prob[r * a.N + i] = fine ? (float)(sc.mass(key_logit(buf[(uint32_t)by_index[at]]), plan.ref) / total) : 0.f;
                }
            }
        }
        if (parts > 1) sync_parts(parts);
        return;
    }

    // ---- the kept entries are not all listed: borders by histograms, where there is one, then the kept mass chunk by chunk
    const int ref = plan.ref;
    uint64_t border = ~0ull;
    if (by_k || by_p) {
        // bins of a sixteenth of a factor of two, counted from the largest logit; what is further off than 2^-64 shares the last
        const float per_bin = (float)fmin(16.0 * sc.c, 3.0e38), top = plan.top;
        const auto linear_bin = [&](float x) { return (int)fminf((top - x) * per_bin, (float)(kBins - 1)); };
        const Bins b(buf);
        fill_bins(sh, b, part, by_p, sc, ref, [&](float x, int) { return linear_bin(x); });
        uint64_t mass_k = b.sum_mass[kBins - 1];
        const uint64_t count = b.sum_count[kBins - 1];
        if (by_k && (uint64_t)k < count) {
            pick_bin(sh, b, false, (uint64_t)k);
            find_border(sh, buf, b, part, false, by_p, (uint64_t)k, sc, ref, linear_bin, &border, &mass_k);
            if (by_p) fill_bins(sh, b, part, true, sc, ref, [&](float x, int) { return linear_bin(x); });
        }
        if (by_p) {
            uint64_t target = (uint64_t)ceil((double)fmaxf(p, 0.f) * (double)mass_k), last, last_mass;
            target = max((uint64_t)1, min(target, mass_k));
            pick_bin(sh, b, true, target);
            find_border(sh, buf, b, part, true, true, target, sc, ref, linear_bin, &last, &last_mass);
            border = min(border, last);
        }
    }
    const double least = by_mp ? (double)mp * sc.mass(plan.top, ref) : 0.0;
    const auto stays = [&](float x, int index) { return order_key(x, index) <= border && (!by_mp || sc.mass(x, ref) >= least); };
    const bool everything = border == ~0ull && !by_mp;
    if (!everything || a.kept) {
        // (chunk sums of the first pass are this CTA's own until here; the first CTA has read them)
        constexpr int E = Row<T>::kE;
        const int w0 = min(part.v1, part.v0 + warp * part.seg), w1 = min(part.v1, w0 + part.seg);
        int cnt = 0;
        for (int c = 0; c < part.iters; ++c) {
            double s = 0.0;
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int i = w0 + (c * kU + u) * 32 + lane;
                const uint4 raw = i < w1 ? part.row.load(i) : Row<T>::nothing();
                float x[E];
                Row<T>::unpack(raw, x);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (x[e] > -INFINITY && order_key(x[e], i * E + e - part.row.lead) <= border) {
                        const double mass = sc.mass(x[e], ref);
                        if (!by_mp || mass >= least) { s += mass; ++cnt; }
                    }
            }
            s = warp_add(s);
            if (lane == 0) { sh.chunk[warp * part.iters + c] = s; sh.chunk_ref[warp * part.iters + c] = ref; }
        }
        cnt = warp_add(cnt);
        if (lane == 0) sh.wcnt[warp] = cnt;
        __syncthreads();
        if (tid == 0) {
            cnt = 0;
            for (int w = 0; w < kWarps; ++w) cnt += sh.wcnt[w];
            sh.cta_count = cnt;
        }
    }
    sync_parts(parts);
    const int chunks = scan_chunks(sh, parts, kWarps * part.iters, ref);
    const double total = sh.all[chunks - 1];
    if (rank == 0 && tid == 0) {
        if (a.lse) a.lse[r] = log_mass(sc, plan.top, it, ref, total);
        if (a.kept) {
            int all = 0;
            for (int q = 0; q < parts; ++q) all += *of_rank(&sh.cta_count, q);
            a.kept[r] = all;
        }
    }
    for (int d = warp; d < a.N; d += kWarps) {                                     // a warp per draw, in the CTA whose part it falls into
        const float u = a.u[r * a.N + d];
        if (!(u >= 0.f && u < 1.f)) {
            if (rank == 0 && lane == 0) { set_status(a.status, SD_ERR_INVALID_ARG); a.tokens[r * a.N + d] = -1; if (a.prob) a.prob[r * a.N + d] = 0.f; }
            continue;
        }
        const double target = (double)u * total;
        int g = first_above(sh.all, chunks, target, false);
        while (g >= chunks || (g > 0 && !(sh.all[g] > sh.all[g - 1]))) --g;
        const int per_part = kWarps * part.iters;
        if (g / per_part != rank) continue;
        const int at = g - rank * per_part;
        double mass = 0.0;
        const int token = chunk_crossing(part, at / part.iters, at % part.iters, target - (g ? sh.all[g - 1] : 0.0), sc, ref, stays, &mass);
        if (lane == 0) { a.tokens[r * a.N + d] = token; if (a.prob) a.prob[r * a.N + d] = (float)(mass / total); }
    }
    sync_parts(parts);                                                             // the last reading of other CTAs' memory, and of the row for draws
    if (dense) {
        const float top = plan.top, c32 = (float)sc.c, at_top = (float)(sc.mass(top, ref) / total);
        for (int v = o0 + tid; v < o1; v += kThreads) {
            const float x = part.row.at(v);
            const bool in = x > -INFINITY && stays(x, v);
            dense[v] = a.scaled ? (in ? scaled_logit(x, it) : -INFINITY) : (in ? at_top * exp2f((x - top) * c32) : 0.f);
        }
    }
}

// CTAs per row: as many as leave every warp a few vectors, while all of them fit on the GPU at once
static int parts_for(int M, int V, int elem) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    const long long slots = 2ll * sm_count(dev);
    const int vecs = (int)(((long long)V * elem + 15) / 16);
    int parts = 1;
    while (parts < 8 && (long long)M * parts * 2 <= slots && vecs / (parts * 2) >= kThreads) parts *= 2;
    return parts;
}

}  // namespace rows

using namespace rows;

sd_status launch_top_logits(const void* logits, int dtype, long long ld, int M, int V, int K, float inv_temp, float* values, int32_t* index,
                            float* lse, cudaStream_t st) {
    const int parts = parts_for(M, V, dtype == SD_F32 ? 4 : 2);
    auto kern = dtype == SD_F32 ? top_kernel<float> : top_kernel<uint16_t>;
    if (!allow_dynamic_smem(kern, kCap * 8)) return SD_ERR_CUDA;
    return launch_dependent(kern, dim3((unsigned)M * parts), kThreads, kCap * 8, parts, st, logits, ld, V, parts, K, inv_temp, values, index, lse);
}

sd_status launch_sample(const void* logits, int dtype, long long ld, int M, int V, const sd_sampling& how, const float* u, int N, int32_t* tokens,
                        float* prob, float* dense, bool scaled, float* lse, int32_t* kept, int32_t* dev_status, cudaStream_t st) {
    const int parts = parts_for(M, V, dtype == SD_F32 ? 4 : 2);
    auto kern = dtype == SD_F32 ? sample_kernel<float> : sample_kernel<uint16_t>;
    if (!allow_dynamic_smem(kern, kCap * 8)) return SD_ERR_CUDA;
    const SampleCall call{logits, ld, V, parts, how.inv_temp, how.top_k, how.top_p, how.min_p, u, N, tokens, prob, dense, scaled, lse, kept, dev_status};
    return launch_dependent(kern, dim3((unsigned)M * parts), kThreads, kCap * 8, parts, st, call);
}

}  // namespace sdv
