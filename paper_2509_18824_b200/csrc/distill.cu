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

struct Published {                     // what the CTAs of a row tell each other
    double sum, rest, sum1, entries;   // sums of 2^((x - top) c), of those outside the entries, at temperature 1; sum p (log p - z inv_temp)
    float top, label;                  // label: its logit, where it lies in this CTA's slice
};

struct DistillShared {
    uint64_t bar[kPieces];
    int abort_flag, dup, label_listed;
    float wf[kDistillWarps];
    double wd[4][kDistillWarps];
    Published pub, all[8];
};

// Sums of N doubles over the CTA, in every thread
template <int N>
__device__ __forceinline__ void block_add(DistillShared& sh, double (&v)[N]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = warp_add(v[j]);
    __syncthreads();
    if (lane == 0)
#pragma unroll
        for (int j = 0; j < N; ++j) sh.wd[j][warp] = v[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) {
        v[j] = 0.0;
#pragma unroll
        for (int w = 0; w < kDistillWarps; ++w) v[j] += sh.wd[j][w];
    }
}
__device__ __forceinline__ float block_max(DistillShared& sh, float v) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = warp_fmax(v);
    __syncthreads();
    if (lane == 0) sh.wf[warp] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kDistillWarps; ++w) v = fmaxf(v, sh.wf[w]);
    return v;
}

// The target's entries of one row as the kernels keep them in shared memory: probability and place in this CTA's slice (entries
// from the slice's first one on; -1: elsewhere, or no entry), and the slice's bitmap.
struct Entries {
    double* p;
    int* at;
    uint32_t* bits;
    double mass;                       // sum of p
    double log_norm;                   // log p = t inv_temp - log_norm
    bool any;
};
// `first`: index in the row of the slice's first entry (negative where the row starts inside vector 0); `count`: entries of the slice
__device__ __forceinline__ void load_entries(DistillShared& sh, Entries& en, const DistillCall& a, long long r, int first, int count, bool report) {
    const int tid = threadIdx.x;
    const float* val = a.top_val + r * a.K;
    const int32_t* idx = a.top_idx + r * a.K;
    const int words = (count + 31) / 32;
    for (int i = tid; i < words; i += kDistillThreads) en.bits[i] = 0;
    if (tid == 0) { sh.dup = 0; sh.label_listed = 0; }
    float top = -INFINITY;
    bool any = false;
    for (int k = tid; k < a.K; k += kDistillThreads) {
        const int i = __ldg(idx + k);
        if (i >= a.V && report) set_status(a.status, SD_ERR_BOUNDS);
        if (i >= 0 && i < a.V) { any = true; top = fmaxf(top, __ldg(val + k)); }
    }
    en.any = __syncthreads_or(any);
    double norm[1] = {0.0};
    if (!a.top_lse) {
        top = block_max(sh, top);
        for (int k = tid; k < a.K; k += kDistillThreads) {
            const int i = __ldg(idx + k);
            if (i >= 0 && i < a.V) norm[0] += exp(((double)__ldg(val + k) - (double)top) * (double)a.inv_temp);
        }
        block_add(sh, norm);
        en.log_norm = (double)top * (double)a.inv_temp + log(norm[0]);
    } else {
        en.log_norm = (double)a.top_lse[r];
    }
    double mass[1] = {0.0};
    const int label = a.label ? a.label[r] : -1;
    for (int k = tid; k < a.K; k += kDistillThreads) {
        const int i = __ldg(idx + k), at = i - first;
        const bool there = i >= 0 && i < a.V, here = there && at >= 0 && at < count;
        const double p = there ? exp((double)__ldg(val + k) * (double)a.inv_temp - en.log_norm) : 0.0;
        mass[0] += p;
        en.p[k] = p;
        en.at[k] = here ? at : -1;
        if (here) {
            if (i == label) sh.label_listed = 1;
            const uint32_t bit = 1u << (at & 31);
            if (atomicOr(&en.bits[at >> 5], bit) & bit) sh.dup = 1;
        }
    }
    block_add(sh, mass);
    en.mass = mass[0];
}

// Gradient factors of a row: an entry x outside the list gets tail * 2^((x - top) c) + one * 2^((x - top) log2 e)
struct Factors {
    float top, c;
    float listed, tail, one;           // with dloss and the weights; `listed` stands for `tail` at the listed entries
    float per_p, per_label;            // what a listed entry's p, and the label, take away
};
__device__ __forceinline__ float gradient(const Factors& f, float x, bool two) {
    const float d = x - f.top;
    return two ? f.tail * ex2(d * f.c) + f.one * ex2(d * kLog2e) : (f.tail + f.one) * ex2(d * f.c);
}
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
    const bool two = f.one != 0.f && a.inv_temp != 1.f;
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
                float x[E];
                Row<T>::unpack(load(i), x);
                if (two) {
#pragma unroll
                    for (int e = 0; e < E; ++e) g[e] = gradient(f, x[e], true);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) g[e] = gradient(f, x[e], false);
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
        for (int v = lo + tid; v < hi; v += kDistillThreads) store_one<T>(grad, v, zero ? 0.f : gradient(f, at(v - first), two));
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
        const float d = listed_at(k, j) - f.top;
        float g = f.listed * ex2(d * f.c) - f.per_p * (float)p;
        if (f.one != 0.f) g += f.one * ex2(d * kLog2e);
        if (j + first == label) g -= f.per_label;
        store_one<T>(grad, j + first, g);
    }
    if (tid == 0 && label >= 0 && label < a.V && !sh.label_listed) {
        const int j = label - first;
        if (j >= 0 && j < (v1 - v0) * E) store_one<T>(grad, label, gradient(f, label_z, two) - f.per_label);
    }
}

__device__ __forceinline__ Factors factors_of(const DistillCall& a, float g, bool has_label, float top, float listed, float tail, float one) {
    Factors f;
    f.top = top;
    f.c = a.inv_temp * kLog2e;
    f.per_p = g * a.kl_weight * a.inv_temp;
    f.listed = f.per_p * listed;
    f.tail = f.per_p * tail;
    f.per_label = has_label ? g * a.ce_weight : 0.f;
    f.one = has_label ? f.per_label * one : 0.f;
    return f;
}

template <typename T>
__global__ void __launch_bounds__(kDistillThreads)
distill_loss_kernel(DistillCall a, int parts, int per, int withheld, long long wait_cycles) {
    using namespace sm100;
    constexpr int E = Row<T>::kE;
    extern __shared__ __align__(16) uint4 slice[];
    __shared__ DistillShared sh;
    const int tid = threadIdx.x;
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
    const int piece = (per + kPieces - 1) / kPieces;
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
    load_entries(sh, en, a, r, first, (v1 - v0) * E, rank == 0);                   // (its barriers also settle the edges)

    // ---- largest logit
    const float c = a.inv_temp * kLog2e;
    float top = -INFINITY;
    bool ok = true;
    for (int q = 0; q < kPieces; ++q) {
        ok = mbar_wait(&sh.bar[q], 0, &sh.abort_flag, wait_cycles) && ok;
        const int i1 = min(v1, v0 + (q + 1) * piece);
        for (int i = v0 + q * piece + tid; i < i1; i += kDistillThreads) {
            float x[E];
            Row<T>::unpack(slice[i - v0], x);
#pragma unroll
            for (int e = 0; e < E; ++e) top = fmaxf(top, x[e]);
        }
    }
    top = block_max(sh, top);
    // ---- sums relative to it
    const float from = top > -INFINITY ? top : 0.f;
    const int label = a.label ? a.label[r] : -1;
    const bool has_label = label >= 0 && label < a.V;
    const bool two = has_label && a.inv_temp != 1.f, rest_too = a.top_lse != nullptr;
    float s = 0.f, s_listed = 0.f, s1 = 0.f;
    const uint8_t* bytes = reinterpret_cast<const uint8_t*>(en.bits);
    for (int i = v0 + tid; i < v1; i += kDistillThreads) {
        float x[E];
        Row<T>::unpack(slice[i - v0], x);
        const int j = i - v0;
        const uint32_t mask = E == 8 ? bytes[j] : (bytes[j >> 1] >> ((j & 1) * 4)) & 15u;
        if (two) {
#pragma unroll
            for (int e = 0; e < E; ++e) s1 += ex2((x[e] - from) * kLog2e);
        }
        if (mask == 0 || !rest_too) {
#pragma unroll
            for (int e = 0; e < E; ++e) s += ex2((x[e] - from) * c);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float v = ex2((x[e] - from) * c);
                if (mask >> e & 1) s_listed += v; else s += v;
            }
        }
    }
    const T* entries = reinterpret_cast<const T*>(slice);
    const auto at = [&](int j) {
        if constexpr (sizeof(T) == 4) return (float)entries[j];
        else return __uint_as_float((uint32_t)entries[j] << 16);
    };
    double sums[4] = {(double)s + (double)s_listed, (double)s, (double)s1, 0.0};
    for (int k = tid; k < a.K; k += kDistillThreads) {
        const int j = en.at[k];
        const double p = en.p[k];
        if (j >= 0 && p != 0.0) sums[3] += p * ((double)__ldg(a.top_val + r * a.K + k) * (double)a.inv_temp - en.log_norm - (double)at(j) * (double)a.inv_temp);
    }
    block_add(sh, sums);
    if (tid == 0) {
        const int j = label - first;
        sh.pub = Published{sums[0], sums[1], sums[2], sums[3], top, has_label && j >= 0 && j < (v1 - v0) * E ? at(j) : 0.f};
    }
    sync_parts(parts);
    if (tid < parts) sh.all[tid] = *of_rank(&sh.pub, tid);
    __syncthreads();
    if (parts > 1) cluster_arrive_relaxed();                                       // this CTA has read the others' (the wait is at the end)

    // ---- the row's
    float most = -INFINITY;
    for (int q = 0; q < parts; ++q) most = fmaxf(most, sh.all[q].top);
    double sum = 0.0, rest = 0.0, sum1 = 0.0, entries_part = 0.0, z_label = 0.0;
    for (int q = 0; q < parts; ++q) {
        const Published& o = sh.all[q];
        const double d = o.top > -INFINITY ? (double)o.top - (double)most : 0.0;
        const double w = (double)ex2((float)d * c);
        sum += o.sum * w;
        rest += o.rest * w;
        if (two) sum1 += o.sum1 * (double)ex2((float)d * kLog2e);
        entries_part += o.entries;
        z_label += o.label;
    }
    if (!two) sum1 = sum;
    const double p_rest = rest_too ? 1.0 - en.mass : 0.0, s_rest = rest / sum;
    const bool has_rest = p_rest > 0.0 && rest > 0.0;
    const double all_p = has_rest ? 1.0 : (en.any ? en.mass : 0.0);
    const double tail = all_p - (has_rest ? p_rest / s_rest : 0.0);
    if (rank == 0 && tid == 0) {
        const double lse = (double)most * (double)a.inv_temp + log(sum);
        double kl = en.any ? entries_part + en.mass * lse : 0.0;
        if (has_rest && en.any) kl += p_rest * (log(p_rest) - log(s_rest));
        a.kl[r] = (float)kl;
        if (a.ce) a.ce[r] = has_label ? (float)((double)most + log(sum1) - z_label) : 0.f;
        if (a.stats) reinterpret_cast<float4*>(a.stats)[r] = make_float4(most, (float)(all_p / sum), (float)(tail / sum), (float)(1.0 / sum1));
        if (label >= a.V) set_status(a.status, SD_ERR_BOUNDS);
    }
    if (a.grad) {
        const float g = a.dloss ? a.dloss[r] : 1.f;
        const Factors f = factors_of(a, g, has_label, most, (float)(all_p / sum), (float)(tail / sum), (float)(1.0 / sum1));
        write_gradient<T>(sh, a, en, row, r, v0, v1, f, g == 0.f, [&](int i) { return slice[i - v0]; }, at, [&](int, int j) { return at(j); }, (float)z_label);
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
