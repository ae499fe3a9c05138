// Causal GQA attention of packed new tokens over the paged cache: one warp per row and query head.
#include "prompt_plan.cuh"

namespace sdv {

constexpr float kPromptLog2e = 1.4426950408889634f;

__global__ void __launch_bounds__(256)
prompt_rows_kernel(sd_prompts p, sd_kv_layer cache, const __nv_bfloat16* q, long long ldq, float scale_log2, __nv_bfloat16* out,
                   long long ldo, float* lse, int32_t* status) {
    begin_dependent(p.block_table, p.n_blocks, p.len, p.n_new, p.start, cache.k, cache.v, q, out, lse);
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int row = (int)(w / p.Hq), h = (int)(w % p.Hq);
    if (row >= __ldcg(p.start + p.B)) return;
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (__ldcg(p.start + m) <= row) lo = m; else hi = m;
    }
    const int first = __ldcg(p.start + lo);
    const RequestSpan r = request_span(p, lo, first, __ldcg(p.start + lo + 1));
    if (!r.covered) return;
    const int keys = r.len + row - first + 1, kvh = h / (p.Hq / p.Hkv);
    float4 x;
    {
        const uint2 u = *reinterpret_cast<const uint2*>(q + row * ldq + h * kD + lane * 4);
        x = make_float4(bf16lo(u.x), bf16hi(u.x), bf16lo(u.y), bf16hi(u.y));
    }
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int t = 0; t < keys; ++t) {
        const int block = __ldcg(p.block_table + (size_t)lo * p.max_blocks_per_seq + t / kBlock);
        if (block < 0 || block >= cache.num_blocks) { if (lane == 0) set_status(status, SD_ERR_BOUNDS); return; }
        const size_t at = ((((size_t)block * p.Hkv + kvh) * kBlock + t % kBlock) * kD) / 4 + lane;
        const uint2 k = static_cast<const uint2*>(cache.k)[at], v = static_cast<const uint2*>(cache.v)[at];
        float s = x.x * bf16lo(k.x) + x.y * bf16hi(k.x) + x.z * bf16lo(k.y) + x.w * bf16hi(k.y);
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= scale_log2;
        const float top = fmaxf(m, s), a = exp2f(m - top), e = exp2f(s - top);
        m = top;
        l = l * a + e;
        o.x = o.x * a + e * bf16lo(v.x); o.y = o.y * a + e * bf16hi(v.x);
        o.z = o.z * a + e * bf16lo(v.y); o.w = o.w * a + e * bf16hi(v.y);
    }
    const float inv = 1.f / l;
    const __nv_bfloat162 a = __floats2bfloat162_rn(o.x * inv, o.y * inv), b = __floats2bfloat162_rn(o.z * inv, o.w * inv);
    *reinterpret_cast<uint2*>(out + row * ldo + h * kD + lane * 4) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    if (lse && lane == 0) lse[(size_t)row * p.Hq + h] = (m + log2f(l)) * 0.6931471805599453f;
}

size_t prompt_plan_bytes(const sd_prompts&) { return 256; }
size_t prompt_workspace_bytes(const sd_prompts&) { return 256; }

sd_status launch_prompt_attention(const sd_prompts& p, const sd_kv_layer& cache, const void* q, long long ldq, float scale, void* out,
                                  long long ldo, float* lse, void*, int32_t* dev_status, cudaStream_t st) {
    const long long warps = (long long)p.N * p.Hq;
    return launch_dependent(prompt_rows_kernel, dim3((unsigned)((warps + 7) / 8)), 256, 0, 1, st, p, cache,
                            static_cast<const __nv_bfloat16*>(q), ldq, scale * kPromptLog2e, static_cast<__nv_bfloat16*>(out), ldo, lse, dev_status);
}

}  // namespace sdv
