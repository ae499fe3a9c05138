// Rows of logits: 16-byte vectors of a row that may start anywhere, masses in 64 bits, the order of a row's entries, and the
// block-wide steps (sums, scans, sorting) that the kernels on rows share.
#pragma once
#include "common.cuh"
#include "sm100.cuh"

namespace sdv {
namespace rows {

constexpr int kThreads = 512;          // threads of a CTA of sample.cu
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

// ---------------------------------------------------------------- arithmetic
// 2^x, to about 2^-22 of it
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two 32-bit operations in one instruction
struct Pair { float x, y; };
__device__ __forceinline__ uint64_t as_u64(Pair a) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y)); return r; }
__device__ __forceinline__ Pair as_pair(uint64_t v) { Pair a; asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(v)); return a; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(as_u64(a)), "l"(as_u64(b)), "l"(as_u64(c)));
    return as_pair(d);
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(as_u64(a)), "l"(as_u64(b)));
    return as_pair(d);
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(as_u64(a)), "l"(as_u64(b)));
    return as_pair(d);
}
__device__ __forceinline__ Pair ex2(Pair a) { return Pair{ex2(a.x), ex2(a.y)}; }

// largest over the warp (NaN left out), by one reduction of integers that are ordered as the values are
__device__ __forceinline__ float warp_largest(float v) {
    const int i = __float_as_int(fmaxf(v, -INFINITY));
    const int m = __reduce_max_sync(0xffffffffu, i ^ ((i >> 31) & 0x7fffffff));
    return __int_as_float(m ^ ((m >> 31) & 0x7fffffff));
}

// ---------------------------------------------------------------- a row as 16-byte vectors
// Vector 0 is the aligned one that holds the row's first entry; `lead` entries of it lie in front of the row, and the last
// one may reach behind the row.  Those two are put together from single entries, so that nothing outside the row is read.
template <typename T>
struct Row {
    static constexpr int kE = 16 / (int)sizeof(T);
    const T* p;
    const uint4* vec;
    int lead, V, nvec, full0, full1;
    __device__ __forceinline__ Row(const void* base, long long ld, long long r, int V_) : p(static_cast<const T*>(base) + r * ld), V(V_) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p);
        vec = reinterpret_cast<const uint4*>(a & ~(uintptr_t)15);
        lead = (int)((a & 15) / sizeof(T));
        nvec = (lead + V + kE - 1) / kE;
        full0 = lead ? 1 : 0;
        full1 = (lead + V) / kE;
    }
    static __device__ __forceinline__ uint4 nothing() {                            // entries of minus infinity
        const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
        return make_uint4(w, w, w, w);
    }
    __device__ __forceinline__ uint4 edge(int i) const {
        const uint4 r = nothing();
        uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const int v = i * kE + e - lead;
            if (v < 0 || v >= V) continue;
            if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(__ldcg(reinterpret_cast<const float*>(p) + v));
            else {
                const uint32_t h = __ldcg(reinterpret_cast<const unsigned short*>(p) + v);
                w[e >> 1] = (e & 1) ? ((w[e >> 1] & 0xffffu) | (h << 16)) : ((w[e >> 1] & 0xffff0000u) | h);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // (through L2, never the read-only path: a filter's output may be the row itself)
    __device__ __forceinline__ uint4 load(int i) const { return i >= full0 && i < full1 ? __ldcg(vec + i) : edge(i); }
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[kE]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(w[e]);
            else x[e] = (e & 1) ? bf16hi(w[e >> 1]) : bf16lo(w[e >> 1]);
        }
    }
    // the vector's entries two by two
    static __device__ __forceinline__ void pairs(const uint4& r, Pair (&x)[kE / 2]) {
        float f[kE];
        unpack(r, f);
#pragma unroll
        for (int e = 0; e < kE / 2; ++e) x[e] = Pair{f[2 * e], f[2 * e + 1]};
    }
    static __device__ __forceinline__ uint4 without_nan(const uint4& r) {           // minus infinity instead
        if constexpr (sizeof(T) == 4) {
            const auto f = [](uint32_t w) { return __float_as_uint(fmaxf(__uint_as_float(w), -INFINITY)); };
            return make_uint4(f(r.x), f(r.y), f(r.z), f(r.w));
        } else {
            const auto f = [](uint32_t w) {
                const uint32_t none = 0xff80ff80u;
                const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w), *reinterpret_cast<const __nv_bfloat162*>(&none));
                return *reinterpret_cast<const uint32_t*>(&m);
            };
            return make_uint4(f(r.x), f(r.y), f(r.z), f(r.w));
        }
    }
    // largest entry of a vector and `m` (NaN left out)
    static __device__ __forceinline__ float largest(const uint4& r, float m) {
        if constexpr (sizeof(T) == 4) {
            return fmaxf(fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w))), m);
        } else {
            const auto h = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
            const __nv_bfloat162 t = __hmax2(__hmax2(h(r.x), h(r.y)), __hmax2(h(r.z), h(r.w)));
            return fmaxf(fmaxf(__low2float(t), __high2float(t)), m);
        }
    }
    __device__ __forceinline__ float at(int v) const {
        if constexpr (sizeof(T) == 4) return __ldcg(reinterpret_cast<const float*>(p) + v);
        else return __uint_as_float((uint32_t)__ldcg(reinterpret_cast<const unsigned short*>(p) + v) << 16);
    }
};

// ---------------------------------------------------------------- masses
// mass(x) = 2^(x c - ref) with c = inv_temp log2 e and a whole number ref, in 64 bits: which token a uniform number falls on, and
// where a sum passes top_p of another, must not depend on the rounding of single masses (with 2^-24 in each of 152064 equal masses
// one draw in forty thousand would).  2^f for |f| <= 1/2 is its Taylor series up to f^9 (the rest is below 7e-12 of it); ref
// being whole, sums taken with different ones are brought together exactly. (So far as they stay below
// 2^28: beyond, logits are taken relative to the largest one.)
struct Scale {
    double c;
    float lim, base;                   // base: what logits are relative to
    __device__ __forceinline__ explicit Scale(float inv_temp) : c((double)inv_temp * 1.4426950408889634073599), base(0.f) {
        lim = (float)fmin(536870912.0 / c, 3.4028234663852886e38);
    }
    __device__ __forceinline__ double clamped(float x) const { return __dmul_rn((double)fminf(fmaxf(__fsub_rn(x, base), -lim), lim), c); }
    // Where exponents would leave 2^28, logits count from the largest one.  (Differences of nearby ones are exact, the others' masses 0.)
    __device__ __forceinline__ void from(float top) { base = fabs((double)top * c) > 268435456.0 ? top : 0.f; }
    __device__ __forceinline__ int whole(float x) const { return __double2int_rn(clamped(x)); }
    // N masses side by side: their chains of multiply-adds hide one another's latency
    template <int N>
    __device__ __forceinline__ void masses(const float (&x)[N], int ref, double (&m)[N]) const {
        const double big = 6755399441055744.0;                                     // 1.5 * 2^52: adding it rounds to a whole number
        constexpr double kC[10] = {1.0, 6.9314718055994531e-01, 2.4022650695910072e-01, 5.5504108664821580e-02, 9.6181291076284772e-03,
                                   1.3333558146428443e-03, 1.5403530393381609e-04, 1.5252733804059841e-05, 1.3215486790144309e-06,
                                   1.0178086009239699e-07};                        // (ln 2)^k / k!
        double f[N];
        int e[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            // (single roundings: the same entry has the same mass wherever it is computed, to the last bit)
            const double t = clamped(x[j]), r = __dadd_rn(t, big);
            e[j] = __double2loint(r) - ref;
            f[j] = __dsub_rn(t, __dsub_rn(r, big));
            m[j] = kC[9];
        }
#pragma unroll
        for (int k = 8; k >= 0; --k)
#pragma unroll
            for (int j = 0; j < N; ++j) m[j] = fma(m[j], f[j], kC[k]);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const bool none = !(x[j] > -INFINITY) || e[j] < -1000;                 // masked entries and NaN have none
            m[j] = __hiloint2double(none ? 0 : __double2hiint(m[j]) + (e[j] << 20), none ? 0 : __double2loint(m[j]));
        }
    }
    __device__ __forceinline__ double mass(float x, int ref) const {
        const float a[1] = {x};
        double m[1];
        masses(a, ref, m);
        return m[0];
    }
};
// 2^t, by the same series, N of them side by side; 0 below 2^-1000, NaN of NaN
template <int N>
__device__ __forceinline__ void powers_of_two(const double (&t)[N], double (&m)[N]) {
    const double big = 6755399441055744.0;
    constexpr double kC[10] = {1.0, 6.9314718055994531e-01, 2.4022650695910072e-01, 5.5504108664821580e-02, 9.6181291076284772e-03,
                               1.3333558146428443e-03, 1.5403530393381609e-04, 1.5252733804059841e-05, 1.3215486790144309e-06,
                               1.0178086009239699e-07};                            // (ln 2)^k / k!
    double f[N];
    int e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const double x = fmin(fmax(t[j], -2000.0), 1000.0), r = x + big;
        e[j] = __double2loint(r);
        f[j] = x - (r - big);
        m[j] = kC[9];
    }
#pragma unroll
    for (int k = 8; k >= 0; --k)
#pragma unroll
        for (int j = 0; j < N; ++j) m[j] = fma(m[j], f[j], kC[k]);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const bool none = e[j] < -1000;
        m[j] = t[j] != t[j] ? t[j] : __hiloint2double(none ? 0 : __double2hiint(m[j]) + (e[j] << 20), none ? 0 : __double2loint(m[j]));
    }
}
// v * 2^e
__device__ __forceinline__ double times_pow2(double v, int e) {
    if (e < -1000) return 0.0;
    return v * __hiloint2double((1023 + min(e, 1000)) << 20, 0);
}

// ---------------------------------------------------------------- the order of a row's entries
// Entries stand in the order (logit descending, index ascending); the smaller key comes first.  Zeros of both signs are equal.
__device__ __forceinline__ uint64_t order_key(float x, int index) {
    const uint32_t u = __float_as_uint(x + 0.f);
    const uint32_t up = u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
    return ((uint64_t)(~up) << 32) | (uint32_t)index;
}
__device__ __forceinline__ float key_logit(uint64_t key) {
    const uint32_t up = ~(uint32_t)(key >> 32);
    return __uint_as_float(up ^ ((up >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int key_index(uint64_t key) { return (int)(uint32_t)key; }

// ---------------------------------------------------------------- clusters of one to eight CTAs
// (Not the aligned form of the barrier: what stands in front of it is code in which a warp's lanes part, loops with a condition per
// entry, and an aligned barrier that a warp reaches in pieces is an illegal instruction.)
__device__ __forceinline__ void sync_parts(int parts) {
    if (parts == 1) { __syncthreads(); return; }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
// the same variable of shared memory in CTA `rank` of the cluster
template <typename P>
__device__ __forceinline__ P* of_rank(P* mine, int rank) {
    uint64_t r;
    asm volatile("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<uint64_t>(mine)), "r"(rank));
    return reinterpret_cast<P*>(r);
}

// the same variable of every part, part r's in lane r (0 in the others)
template <typename P>
__device__ __forceinline__ P of_parts(P* mine, int parts) {
    const int lane = threadIdx.x & 31;
    return lane < parts ? *of_rank(mine, lane) : P(0);
}

// ---------------------------------------------------------------- block-wide steps
template <typename S>
__device__ __forceinline__ S warp_add(S v) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float warp_fmax(float v) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

// Inclusive sums of a[0..n), n <= kListMax, in place and in a fixed order.  `tmp`: kWarps values.
constexpr int kListMax = 2 * kThreads;
template <typename S>
static __device__ __noinline__ void block_scan(S* a, int n, S* tmp) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, i = 2 * tid;
    __syncthreads();
    const S x = i < n ? a[i] : S(0), y = x + (i + 1 < n ? a[i + 1] : S(0));
    S incl = y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const S o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) tmp[warp] = incl;
    __syncthreads();
    S before = S(0);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) before += w < warp ? tmp[w] : S(0);
    const S own = __shfl_up_sync(0xffffffffu, incl, 1);
    if (lane > 0) before += own;
    if (i < n) a[i] = before + x;
    if (i + 1 < n) a[i + 1] = before + y;
    __syncthreads();
}

// a[0..n) in ascending order; n <= kListMax, room for the next power of two.  Distinct keys.
constexpr int kRankSort = 160;         // up to which every key counts those in front of it (128 keys: 0.5 us, the network 0.9)
static __device__ __noinline__ void block_sort(uint64_t* a, int n) {
    const int tid = threadIdx.x;
    if (n <= kRankSort) {
        __syncthreads();
        const uint64_t mine = tid < n ? a[tid] : 0;
        int at = 0;
        if (tid < n) {
#pragma unroll 8
            for (int j = 0; j < n; ++j) at += a[j] < mine;
        }
        __syncthreads();
        if (tid < n) a[at] = mine;
        __syncthreads();
        return;
    }
    // A bitonic network.  A warp holds 64 consecutive keys, lane l keys l and l + 32: distances below 64 stay in its registers (through
    // shared memory, step by step, 1024 keys took 13000 cycles).
    const int lane = tid & 31, warp = tid >> 5, base = warp * 64;
    int size = 64;
    while (size < n) size <<= 1;
    const bool in = base < size;
    __syncthreads();
    uint64_t x = in && base + lane < n ? a[base + lane] : ~0ull, y = in && base + lane + 32 < n ? a[base + lane + 32] : ~0ull;
    const auto swap_in_warp = [&](int k, int from) {                               // distances from, from / 2 .. 1 of stage k
        if (from >= 32) {
            const bool up = ((base + lane) & k) == 0;                              // (k > 32: the same for both keys)
            if ((x > y) == up) { const uint64_t t = x; x = y; y = t; }
        }
#pragma unroll
        for (int j = 16; j >= 1; j >>= 1) {
            if (j > from) continue;
            const uint64_t ox = __shfl_xor_sync(0xffffffffu, x, j), oy = __shfl_xor_sync(0xffffffffu, y, j);
            const bool low = (lane & j) == 0;
            const bool upx = ((base + lane) & k) == 0, upy = ((base + lane + 32) & k) == 0;
            x = (low == upx) == (ox < x) ? ox : x;
            y = (low == upy) == (oy < y) ? oy : y;
        }
    };
    if (in) for (int k = 2; k <= 64; k <<= 1) swap_in_warp(k, k >> 1);
    for (int k = 128; k <= size; k <<= 1) {
        if (in) { a[base + lane] = x; a[base + lane + 32] = y; }
        __syncthreads();
        for (int j = k >> 1; j >= 64; j >>= 1) {
            if (tid < size / 2) {
                const int i = 2 * tid - (tid & (j - 1)), o = i + j;
                const uint64_t p = a[i], q = a[o];
                if ((p > q) == ((i & k) == 0)) { a[i] = q; a[o] = p; }
            }
            __syncthreads();
        }
        if (in) {
            x = a[base + lane];
            y = a[base + lane + 32];
            swap_in_warp(k, 32);
        }
    }
    if (in) { a[base + lane] = x; a[base + lane + 32] = y; }
    __syncthreads();
}

}  // namespace rows
}  // namespace sdv
