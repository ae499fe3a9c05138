// The draft's training loss on rows of logits [M][V] and its gradient (sd_distill_loss, sd_distill_grad).
//
// Memory-bound: a row is read once and, with the gradient, written once.  For that a cluster of CTAs holds the whole row in its
// shared memory (bulk copies; 152064 bf16 are eight slices of 38 KB, five of which share an SM at different stages), so that
// the gradient, which needs the row's sums, is formed from there.  One exchange between the CTAs: largest logit, sums, and the
// entries' part of the loss.  Which entries of a slice the target lists is a bitmap, one byte of which goes with each vector; their
// gradients (and the label's) are written over the others' afterwards, by one thread each.
#include "rows.cuh"

namespace sdv {
namespace rows {

constexpr int kDistillThreads = 256;
constexpr int kDistillWarps = kDistillThreads / 32;
constexpr int kPieces = 4;             // copies of a slice, each with a barrier of its own

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(sm100::smem_u32(dst)), "l"(src), "r"(bytes), "r"(sm100::smem_u32(bar)), "l"(policy) : "memory");
}

// Exponentials are taken as 2^(x c - R) with R = rint(top c), a whole number: x c - R is one instruction with one rounding (of a small
// number where it matters), and sums with different R are brought together exactly.
//
// What the CTAs of a row tell each other: for each warp its largest logit and, with its R, the sums of 2^(x c - R) outside
// and among the entries and of 2^(x log2 e - R); and the CTA's part of sum p (log p - z inv_temp), and the label's logit where
// it lies in its slice.
struct Published {
    float4 warp[kDistillWarps];
    double entries;
    float label;
};

// The row's factors: largest logit, and what an exponential is multiplied with at the entries, elsewhere, and for the cross-entropy
struct RowFactors { float top, listed, tail, one, label_z; };

struct DistillShared {
    uint64_t bar[kPieces];
    int abort_flag, dup, label_listed, any;
    float wf[kDistillWarps];
    double wd[kDistillWarps];
    double we[kDistillWarps];
    Published pub;
    RowFactors row;
};

__device__ __forceinline__ double block_add(DistillShared& sh, double v) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_add(v);
    __syncthreads();
    if (lane == 0) sh.wd[warp] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kDistillWarps; ++w) v += sh.wd[w];
    return v;
}
__device__ __forceinline__ float block_max(DistillShared& sh, float v) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_largest(v);
    __syncthreads();
    if (lane == 0) sh.wf[warp] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kDistillWarps; ++w) v = fmaxf(v, sh.wf[w]);
    return v;
}

__device__ __forceinline__ float whole_power(float top, float c) { return top > -INFINITY ? rintf(top * c) : 0.f; }

// The target's entries of one row as the kernels keep them in shared memory: probability and place in this CTA's slice (entries
// from the slice's first one on; -1: elsewhere, or no entry), and the slice's bitmap.
struct Entries {
    double* p;
    int* at;
    uint32_t* bits;
    double log_norm;                   // log p = t inv_temp - log_norm
};
// `first`: index in the row of the slice's first entry (negative where the row starts inside vector 0); `count`: entries of the slice.
// Leaves the warps' sums of p in sh.wd; the caller's barrier settles everything but log_norm.
__device__ __forceinline__ void load_entries(DistillShared& sh, Entries& en, const DistillCall& a, long long r, int first, int count, bool report) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float* val = a.top_val + r * a.K;
    const int32_t* idx = a.top_idx + r * a.K;
    const int label = a.label ? __ldg(a.label + r) : -1;
    int i0 = -1;                                                                   // the thread's first entry (most calls have no more)
    float t0 = 0.f;
    if (tid < a.K) { i0 = __ldg(idx + tid); t0 = __ldg(val + tid); }
    if (a.top_lse) en.log_norm = (double)__ldg(a.top_lse + r);
    const int words = (count + 31) / 32;
    for (int i = tid; i < words; i += kDistillThreads) en.bits[i] = 0;
    if (tid == 0) { sh.dup = 0; sh.label_listed = 0; sh.any = 0; }
    __syncthreads();
    if (!a.top_lse) {                                                              // the entries' own soft-max
        float top = -INFINITY;
        for (int k = tid; k < a.K; k += kDistillThreads) {
            const int i = k == tid ? i0 : __ldg(idx + k);
            if (i >= 0 && i < a.V) top = fmaxf(top, k == tid ? t0 : __ldg(val + k));
        }
        top = block_max(sh, top);
        double norm = 0.0;
        for (int k = tid; k < a.K; k += kDistillThreads) {
            const int i = k == tid ? i0 : __ldg(idx + k);
            if (i >= 0 && i < a.V) norm += exp(((double)(k == tid ? t0 : __ldg(val + k)) - (double)top) * (double)a.inv_temp);
        }
        norm = block_add(sh, norm);
        en.log_norm = (double)top * (double)a.inv_temp + log(norm);
        __syncthreads();                                                           // (sh.wd is written again below)
    }
    double mass = 0.0;
    if (warp * 32 < a.K) {
        for (int k = tid; k < a.K; k += kDistillThreads) {
            const int i = k == tid ? i0 : __ldg(idx + k), at = i - first;
            const bool there = i >= 0 && i < a.V, here = there && at >= 0 && at < count;
            const double p = there ? exp((double)(k == tid ? t0 : __ldg(val + k)) * (double)a.inv_temp - en.log_norm) : 0.0;
            mass += p;
            en.p[k] = p;
            en.at[k] = here ? at : -1;
            if (there) sh.any = 1;
            if (i >= a.V && report) set_status(a.status, SD_ERR_BOUNDS);
            if (here) {
                if (i == label) sh.label_listed = 1;
                const uint32_t bit = 1u << (at & 31);
                if (atomicOr(&en.bits[at >> 5], bit) & bit) sh.dup = 1;
            }
        }
        __syncwarp();
        mass = warp_add(mass);
    }
    if (lane == 0) sh.wd[warp] = mass;
}

// Gradient factors of a row, with dloss and the weights: an entry x outside the list gets tail * 2^(x c - R) + one *
// 2^(x log2 e - R1), at temperature 1 in one term.
struct Factors {
    float top_c, top_e, c;             // R, R1
    float listed, tail, one;           // `listed` stands for `tail` at the listed entries
    float per_p, per_label;            // what a listed entry's p, and the label, take away
    bool two;
    __device__ __forceinline__ float plain(float x) const {
        const float e = ex2(fmaf(x, c, -top_c));
        return two ? fmaf(one, ex2(fmaf(x, kLog2e, -top_e)), tail * e) : tail * e;
    }
    __device__ __forceinline__ float entry(float x) const {
        const float e = ex2(fmaf(x, c, -top_c));
        return two ? fmaf(one, ex2(fmaf(x, kLog2e, -top_e)), listed * e) : listed * e;
    }
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

// The gradient of vectors [v0, v1) of a row.  load(i): vector i; at(j): entry j of the slice; listed_at(k, j): the same for the list's
// k-th entry, and label_z the label's logit, as they were before anything was written (the gradient may take the logits' place)
template <typename T, typename L, typename A, typename B>
__device__ __forceinline__ void write_gradient(DistillShared& sh, const DistillCall& a, const Entries& en, const Row<T>& row, long long r, int v0, int v1,
                                               const Factors& f, bool zero, L load, A at, B listed_at, float label_z) {
    constexpr int E = Row<T>::kE;
    const int tid = threadIdx.x;
    T* grad = static_cast<T*>(a.grad) + r * a.grad_ld;
    const int first = v0 * E - row.lead;
    if (((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(row.p)) & 15) == 0) {
        uint4* out = reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(grad) & ~(uintptr_t)15);
#pragma unroll 4
        for (int i = v0 + tid; i < v1; i += kDistillThreads) {
            float g[E];
            if (zero) {
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] = 0.f;
            } else {
                Pair x[E / 2];
                Row<T>::pairs(load(i), x);
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    const Pair w = ex2(fma2(x[e], Pair{f.c, f.c}, Pair{-f.top_c, -f.top_c}));
                    Pair o{f.tail * w.x, f.tail * w.y};
                    if (f.two) o = fma2(Pair{f.one, f.one}, ex2(fma2(x[e], Pair{kLog2e, kLog2e}, Pair{-f.top_e, -f.top_e})), o);
                    g[2 * e] = o.x;
                    g[2 * e + 1] = o.y;
                }
            }
            if (i >= row.full0 && i < row.full1) out[i] = pack<T>(g);
            else
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int v = i * E + e - row.lead;
                    if (v >= 0 && v < a.V) store_one<T>(grad, v, g[e]);
                }
        }
    } else {                                                                       // rows that start at different places in their 16 bytes
        const int lo = max(0, first), hi = min(a.V, v1 * E - row.lead);
        for (int v = lo + tid; v < hi; v += kDistillThreads) store_one<T>(grad, v, zero ? 0.f : f.plain(at(v - first)));
    }
    if (zero) return;
    __syncthreads();                                                               // over what has just been written
    const int label = a.label ? a.label[r] : -1;
    for (int k = tid; k < a.K; k += kDistillThreads) {
        const int j = en.at[k];
        if (j < 0) continue;
        double p = en.p[k];
        if (sh.dup) {                                                              // the same index twice somewhere: all of its masses
            p = 0.0;
            for (int q = 0; q < a.K; ++q) p += en.at[q] == j ? en.p[q] : 0.0;
        }
        float g = f.entry(listed_at(k, j)) - f.per_p * (float)p;
        if (j + first == label) g -= f.per_label;
        store_one<T>(grad, j + first, g);
    }
    if (tid == 0 && label >= 0 && label < a.V && !sh.label_listed) {
        const int j = label - first;
        if (j >= 0 && j < (v1 - v0) * E) store_one<T>(grad, label, f.plain(label_z) - f.per_label);
    }
}

__device__ __forceinline__ Factors factors_of(const DistillCall& a, float g, bool has_label, float top, float listed, float tail, float one) {
    Factors f;
    f.c = a.inv_temp * kLog2e;
    f.top_c = whole_power(top, f.c);
    f.top_e = whole_power(top, kLog2e);
    f.per_p = g * a.kl_weight * a.inv_temp;
    f.listed = f.per_p * listed;
    f.tail = f.per_p * tail;
    f.per_label = has_label ? g * a.ce_weight : 0.f;
    f.one = f.per_label != 0.f ? f.per_label * one : 0.f;
    f.two = a.inv_temp != 1.f && f.one != 0.f;
    if (!f.two) { f.listed += f.one; f.tail += f.one; }
    return f;
}

template <typename T>
__global__ void __launch_bounds__(kDistillThreads)
distill_loss_kernel(DistillCall a, int parts, int per, int withheld, long long wait_cycles) {
    using namespace sm100;
    constexpr int E = Row<T>::kE;
    extern __shared__ __align__(16) uint4 slice[];
    __shared__ DistillShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        sh.abort_flag = 0;
        for (int q = 0; q < kPieces; ++q) mbar_init(&sh.bar[q], 1);
        fence_barrier_init();
    }
    __syncthreads();
    begin_dependent(a.logits, a.top_val, a.top_idx, a.top_lse, a.label, a.kl, a.ce, a.stats, a.dloss, a.grad, a.status);
    const long long r = blockIdx.x / parts;
    const int rank = parts == 1 ? 0 : (int)cluster_ctarank();
    const Row<T> row(a.logits, a.ld, r, a.V);
    const int v0 = min(row.nvec, rank * per), v1 = min(row.nvec, v0 + per);
    // (a piece is whole rounds of the threads: a warp then sums up the vectors of which it has taken the largest entry)
    const int piece = (per + kPieces * kDistillThreads - 1) / (kPieces * kDistillThreads) * kDistillThreads;
    if (tid == 0) {
        const uint64_t pol = policy_evict_first();
        for (int q = 0; q < kPieces; ++q) {
            const int i0 = max(row.full0, min(v1, v0 + q * piece)), i1 = min(row.full1, min(v1, v0 + (q + 1) * piece));
            const uint32_t bytes = i1 > i0 ? (uint32_t)(i1 - i0) * 16 : 0;
            mbar_arrive_expect_tx(&sh.bar[q], bytes + withheld);
            if (bytes) bulk_load(slice + (i0 - v0), row.vec + i0, bytes, &sh.bar[q], pol);
        }
    }
    if (tid == 32 && row.full0 > 0 && v0 == 0 && v1 > 0) slice[0] = row.edge(0);
    if (tid == 64 && row.nvec - 1 >= max(row.full0, row.full1) && row.nvec - 1 >= v0 && row.nvec - 1 < v1) slice[row.nvec - 1 - v0] = row.edge(row.nvec - 1);

    Entries en;
    en.p = reinterpret_cast<double*>(slice + per);
    en.at = reinterpret_cast<int*>(en.p + a.K);
    en.bits = reinterpret_cast<uint32_t*>(en.at + a.K);
    const int first = v0 * E - row.lead;
    load_entries(sh, en, a, r, first, (v1 - v0) * E, rank == 0);

    __syncthreads();
    // ---- largest logit of the warp's vectors, as they come in
    const float c = a.inv_temp * kLog2e;
    float top = -INFINITY;
    bool ok = true;
    for (int q = 0; q < kPieces; ++q) {
        ok = mbar_wait(&sh.bar[q], 0, &sh.abort_flag, wait_cycles) && ok;
        const int i1 = min(v1, v0 + (q + 1) * piece);
        for (int i = v0 + q * piece + tid; i < i1; i += kDistillThreads) top = Row<T>::largest(slice[i - v0], top);
    }
    top = warp_largest(top);
    // ---- sums relative to it
    const int label = a.label ? __ldg(a.label + r) : -1;
    const bool has_label = label >= 0 && label < a.V;
    const bool two = has_label && a.inv_temp != 1.f, rest_too = a.top_lse != nullptr;
    const float r_c = whole_power(top, c), r_e = whole_power(top, kLog2e);
    const Pair c2{c, c}, from_c{-r_c, -r_c}, e2{kLog2e, kLog2e}, from_e{-r_e, -r_e};
    Pair s{0.f, 0.f}, t{0.f, 0.f}, s1{0.f, 0.f};
    float s_listed = 0.f;
    const uint8_t* bytes = reinterpret_cast<const uint8_t*>(en.bits);
#pragma unroll 2
    for (int j = tid; j < v1 - v0; j += kDistillThreads) {
        Pair x[E / 2], w[E / 2];
        Row<T>::pairs(slice[j], x);
        const uint32_t mask = E == 8 ? bytes[j] : (bytes[j >> 1] >> ((j & 1) * 4)) & 15u;
        if (two) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) s1 = add2(s1, ex2(fma2(x[e], e2, from_e)));
        }
#pragma unroll
        for (int e = 0; e < E / 2; ++e) w[e] = ex2(fma2(x[e], c2, from_c));
        if (mask != 0 && rest_too) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                if (mask >> (2 * e) & 1) { s_listed += w[e].x; w[e].x = 0.f; }
                if (mask >> (2 * e + 1) & 1) { s_listed += w[e].y; w[e].y = 0.f; }
            }
        }
#pragma unroll
        for (int e = 0; e < E / 2; e += 2) { s = add2(s, w[e]); t = add2(t, w[e + 1]); }
    }
    const T* entries = reinterpret_cast<const T*>(slice);
    const auto at = [&](int j) {
        if constexpr (sizeof(T) == 4) return (float)entries[j];
        else return __uint_as_float((uint32_t)entries[j] << 16);
    };
    double part = 0.0;
    if (warp * 32 < a.K) {
        for (int k = tid; k < a.K; k += kDistillThreads) {
            const int j = en.at[k];
            const double p = en.p[k];
            if (j >= 0 && p != 0.0) part += p * ((double)__ldg(a.top_val + r * a.K + k) * (double)a.inv_temp - en.log_norm - (double)at(j) * (double)a.inv_temp);
        }
        __syncwarp();
        part = warp_add(part);
    }
    {
        const float rest = warp_add((s.x + s.y) + (t.x + t.y)), listed = rest_too ? warp_add(s_listed) : 0.f, sum1 = two ? warp_add(s1.x + s1.y) : 0.f;
        if (lane == 0) { sh.pub.warp[warp] = make_float4(top, rest, listed, sum1); sh.we[warp] = part; }
    }
    __syncthreads();
    if (tid == 0) {
        const int j = label - first;
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < kDistillWarps; ++w) all += sh.we[w];
        sh.pub.entries = all;
        sh.pub.label = has_label && j >= 0 && j < (v1 - v0) * E ? at(j) : 0.f;
    }
    sync_parts(parts);

    // ---- the row's: one warp brings the parts together
    if (warp == 0) {
        float4 w[2];
        float most = -INFINITY;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = lane + q * 32, rk = i / kDistillWarps;
            w[q] = rk < parts ? *of_rank(&sh.pub.warp[i % kDistillWarps], rk) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
            most = fmaxf(most, w[q].x);
        }
        double entries_part = lane < parts ? *of_rank(&sh.pub.entries, lane) : 0.0;
        float z_label = lane < parts ? *of_rank(&sh.pub.label, lane) : 0.f;
        double mass = lane < kDistillWarps ? sh.wd[lane] : 0.0;
        most = warp_largest(most);
        const float r_row = whole_power(most, c), r_row1 = whole_power(most, kLog2e);
        double rest = 0.0, sum = 0.0, sum1 = 0.0;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const bool some = w[q].x > -INFINITY;
            const double f = some ? times_pow2(1.0, (int)fmaxf(whole_power(w[q].x, c) - r_row, -2000.f)) : 1.0;
            rest += (double)w[q].y * f;
            sum += ((double)w[q].y + (double)w[q].z) * f;
            if (two) sum1 += (double)w[q].w * (some ? times_pow2(1.0, (int)fmaxf(whole_power(w[q].x, kLog2e) - r_row1, -2000.f)) : 1.0);
        }
        rest = warp_add(rest);
        sum = warp_add(sum);
        sum1 = two ? warp_add(sum1) : sum;
        // (R belongs to the power with c as 32 bits hold it: log sum = R ln 2 + log(sum), but for top's own rounding)
        const double lse = (double)most * (double)a.inv_temp + log(sum) - ((double)most * (double)c - (double)r_row) * 0.69314718055994530942;
        const double lse1 = two ? (double)most + log(sum1) - ((double)most * (double)kLog2e - (double)r_row1) * 0.69314718055994530942 : lse;
        entries_part = warp_add(entries_part);
        mass = warp_add(mass);
        z_label = warp_add(z_label);
        const bool any = sh.any != 0;
        const double p_rest = rest_too ? 1.0 - mass : 0.0, s_rest = rest / sum;
        const bool has_rest = p_rest > 0.0 && rest > 0.0;
        const double all_p = has_rest ? 1.0 : (any ? mass : 0.0);
        const double tail = all_p - (has_rest ? p_rest / s_rest : 0.0);
        if (lane == 0) {
            sh.row = RowFactors{most, (float)(all_p / sum), (float)(tail / sum), (float)(1.0 / sum1), z_label};
            if (rank == 0) {
                double kl = any ? entries_part + mass * lse : 0.0;
                if (has_rest && any) kl += p_rest * (log(p_rest) - log(s_rest));
                a.kl[r] = (float)kl;
                if (a.ce) a.ce[r] = has_label ? (float)(lse1 - (double)z_label) : 0.f;
                if (a.stats) reinterpret_cast<float4*>(a.stats)[r] = make_float4(sh.row.top, sh.row.listed, sh.row.tail, sh.row.one);
                if (label >= a.V) set_status(a.status, SD_ERR_BOUNDS);
            }
        }
    }
    __syncwarp();
    if (parts > 1) cluster_arrive_relaxed();                                       // this CTA has read the others' (the wait is at the end)
    if (a.grad) {
        const float g = a.dloss ? __ldg(a.dloss + r) : 1.f;
        __syncthreads();
        const RowFactors rf = sh.row;
        const Factors f = factors_of(a, g, has_label, rf.top, rf.listed, rf.tail, rf.one);
        write_gradient<T>(sh, a, en, row, r, v0, v1, f, g == 0.f, [&](int i) { return slice[i - v0]; }, at, [&](int, int j) { return at(j); }, rf.label_z);
    }
    if (parts > 1) cluster_wait_acquire();
    if (!ok) {                                                                     // a copy did not come
        set_status(a.status, SD_ERR_TIMEOUT);
        unwind_pause();
    }
}

template <typename T>
__global__ void __launch_bounds__(kDistillThreads)
distill_grad_kernel(DistillCall a, int parts, int per) {
    constexpr int E = Row<T>::kE;
    extern __shared__ __align__(16) uint4 lists[];
    __shared__ DistillShared sh;
    begin_dependent(a.logits, a.top_val, a.top_idx, a.top_lse, a.label, a.stats, a.dloss, a.grad, a.status);
    const long long r = blockIdx.x / parts;
    const int part = (int)(blockIdx.x - r * parts);
    const Row<T> row(a.logits, a.ld, r, a.V);
    const int v0 = min(row.nvec, part * per), v1 = min(row.nvec, v0 + per);
    const int first = v0 * E - row.lead;
    Entries en;
    en.p = reinterpret_cast<double*>(lists);
    en.at = reinterpret_cast<int*>(en.p + a.K);
    float* z = reinterpret_cast<float*>(en.at + a.K);                              // the listed logits, and the label's, read before they are overwritten
    en.bits = reinterpret_cast<uint32_t*>(z + a.K + 1);
    load_entries(sh, en, a, r, first, (v1 - v0) * E, part == 0);
    __syncthreads();
    const int label = a.label ? a.label[r] : -1;
    const bool has_label = label >= 0 && label < a.V;
    for (int k = threadIdx.x; k < a.K; k += kDistillThreads) z[k] = en.at[k] >= 0 ? row.at(en.at[k] + first) : 0.f;
    if (threadIdx.x == 0) {
        const bool here = has_label && label >= first && label < first + (v1 - v0) * E;
        z[a.K] = here ? row.at(label) : 0.f;
        if (label >= a.V && part == 0) set_status(a.status, SD_ERR_BOUNDS);
    }
    __syncthreads();
    const float4 st = reinterpret_cast<const float4*>(a.stats)[r];
    const float g = a.dloss ? a.dloss[r] : 1.f;
    const Factors f = factors_of(a, g, has_label, st.x, st.y, st.z, st.w);
    write_gradient<T>(sh, a, en, row, r, v0, v1, f, g == 0.f, [&](int i) { return row.load(i); }, [&](int j) { return row.at(j + first); },
                      [&](int k, int) { return z[k]; }, z[a.K]);
}

// CTAs per row: slices of at most 40 KB while eight are enough for that, and more of them where the rows leave SMs idle
static int loss_parts(int M, int nvec, int sms) {
    int parts = 1;
    while (parts < 8 && ((nvec + parts - 1) / parts * 16 > 40 * 1024 || ((long long)M * parts * 2 <= sms && nvec / (parts * 2) >= kDistillThreads))) parts *= 2;
    return parts;
}

}  // namespace rows

using namespace rows;

sd_status launch_distill_loss(const DistillCall& call, int dtype, int M, cudaStream_t st) {
    const int elem = dtype == SD_F32 ? 4 : 2, nvec = (call.V * elem + 15) / 16 + 1;            // (a row may lie across one vector more)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SD_ERR_CUDA;
    const int parts = loss_parts(M, nvec, sm_count(dev)), per = (nvec + parts - 1) / parts;
    const int smem = per * 16 + call.K * 12 + (per * (16 / elem) + 31) / 32 * 4;
    auto kern = dtype == SD_F32 ? distill_loss_kernel<float> : distill_loss_kernel<uint16_t>;
    if (!allow_dynamic_smem(kern, smem)) return SD_ERR_CUDA;
    const TestKnobs knobs = test_knobs();
    return launch_dependent(kern, dim3((unsigned)M * parts), kDistillThreads, smem, parts, st, call, parts, per, knobs.withhold ? 16 : 0, knobs.wait_cycles);
}

sd_status launch_distill_grad(const DistillCall& call, int dtype, int M, cudaStream_t st) {
    const int elem = dtype == SD_F32 ? 4 : 2, nvec = (call.V * elem + 15) / 16 + 1;
    const int parts = (nvec + 2047) / 2048, per = (nvec + parts - 1) / parts;
    const int smem = call.K * 16 + 4 + (per * (16 / elem) + 31) / 32 * 4;
    auto kern = dtype == SD_F32 ? distill_grad_kernel<float> : distill_grad_kernel<uint16_t>;
    if (!allow_dynamic_smem(kern, smem)) return SD_ERR_CUDA;
    return launch_dependent(kern, dim3((unsigned)M * parts), kDistillThreads, smem, 1, st, call, parts, per);
}

}  // namespace sdv
