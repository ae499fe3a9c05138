// C-ABI entry points: argument validation, then the kernel launchers.
#include "common.cuh"
#include "prompt_plan.cuh"

#include <atomic>
#include <mutex>
#include <math.h>
#include <stdlib.h>
#include <string.h>
#include <unistd.h>

using namespace sdv;

namespace sdv {
int sm_count(int dev) {
    constexpr int kDevs = 64;
    static std::atomic<int> cache[kDevs];
    const bool cached = dev >= 0 && dev < kDevs;
    if (cached)
        if (const int v = cache[dev].load(std::memory_order_relaxed)) return v;
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) return 148;
    if (cached) cache[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

bool raise_dynamic_smem(const void* kern, int bytes) {
    static std::mutex lock;
    const std::lock_guard<std::mutex> hold(lock);
    cudaFuncAttributes now;
    if (cudaFuncGetAttributes(&now, kern) != cudaSuccess) return false;
    return now.maxDynamicSharedSizeBytes >= bytes || cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
}

// (One pass over the environment: three getenv calls took 0.35 us with 200 variables, a tenth of what the smallest
// calls take on the host; this 0.15.)
TestKnobs test_knobs() {
    TestKnobs k{1ll << 31, 0, 0};
    for (char** e = environ; e && *e; ++e) {
        if ((*e)[0] != 'S' || (*e)[1] != 'D' || strncmp(*e, "SDV_TEST_", 9) != 0) continue;
        const char* name = *e + 9;
        const auto value = [&](const char* n) -> const char* {             // behind "n=", if that is the variable
            const size_t l = strlen(n);
            return strncmp(name, n, l) == 0 && name[l] == '=' ? name + l + 1 : nullptr;
        };
        if (const char* v = value("WAIT_CYCLES")) { if (atoll(v) >= 1000) k.wait_cycles = atoll(v); }
        else if (const char* v = value("WITHHOLD")) k.withhold = atoi(v) == 1 ? 1 : 0;
        else if (const char* v = value("CHUNKS")) { if (atoi(v) >= 1 && atoi(v) <= 8) k.chunks = atoi(v); }
    }
    return k;
}
}  // namespace sdv

namespace {

sd_status check_geometry(const sd_batch* bt, bool need_pointers) {
    if (!bt) return SD_ERR_INVALID_ARG;
    if (bt->B < 1 || bt->T_max < 1 || bt->Hq < 1 || bt->Hkv < 1 || bt->max_blocks_per_seq < 1)
        return SD_ERR_INVALID_ARG;
    if (bt->D != kD || bt->block_size != kBlock || bt->T_max > kMaxT) return SD_ERR_UNSUPPORTED;
    if (bt->Hq % bt->Hkv != 0 || bt->Hq / bt->Hkv > 8) return SD_ERR_UNSUPPORTED;
    if (need_pointers) {
        if (!bt->block_table || !bt->len || !bt->n_nodes || !bt->parents) return SD_ERR_INVALID_ARG;
        if (!aligned16(bt->block_table) || !aligned16(bt->len) || !aligned16(bt->n_nodes) ||
            !aligned16(bt->parents))
            return SD_ERR_INVALID_ARG;
    }
    return SD_OK;
}

bool ok_ptr(const void* p) { return p && aligned16(p); }
bool ok_4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

sd_status check_rows(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V) {
    if (M < 0 || V < 1 || ld < V) return SD_ERR_INVALID_ARG;
    if (dtype != SD_F32 && dtype != SD_BF16) return SD_ERR_UNSUPPORTED;
    if (V > 262144 || M > (1 << 24)) return SD_ERR_UNSUPPORTED;
    if (M > 0 && !ok_ptr(logits)) return SD_ERR_INVALID_ARG;
    return SD_OK;
}
bool ok_sampling(const sd_sampling* how) {
    return how && ok_4(how->inv_temp) && ok_4(how->top_k) && ok_4(how->top_p) && ok_4(how->min_p) && ok_4(how->n_used) &&
           (!how->n_used || how->per >= 1);
}
// the arguments that the two distillation calls share
sd_status check_distill(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V, const float* top_val, const int32_t* top_idx,
                        int32_t K, const float* top_lse, const int32_t* label, float inv_temp, const float* dloss, const void* grad,
                        int64_t grad_ld, const int32_t* dev_status) {
    const sd_status s = check_rows(logits, dtype, ld, M, V);
    if (s != SD_OK) return s;
    if (K < 1 || !(inv_temp > 0.f) || !(inv_temp < INFINITY)) return SD_ERR_INVALID_ARG;
    if (K > 1024) return SD_ERR_UNSUPPORTED;
    if (M == 0) return SD_OK;
    if (!top_val || !top_idx || !dev_status) return SD_ERR_INVALID_ARG;
    if (!ok_4(top_val) || !ok_4(top_idx) || !ok_4(top_lse) || !ok_4(label) || !ok_4(dloss)) return SD_ERR_INVALID_ARG;
    if (grad && (!aligned16(grad) || grad_ld < V)) return SD_ERR_INVALID_ARG;
    if (grad == logits && grad_ld != ld) return SD_ERR_INVALID_ARG;
    return SD_OK;
}

sd_status check_prompts(const sd_prompts* p, bool need_pointers) {
    if (!p) return SD_ERR_INVALID_ARG;
    if (p->B < 1 || p->N < 0 || p->Hq < 1 || p->Hkv < 1 || p->max_blocks_per_seq < 1 || p->num_blocks < 1) return SD_ERR_INVALID_ARG;
    if (p->D != kD || p->block_size != kBlock || p->B > kMaxRequests || p->N > (1 << 24) || p->num_blocks > kMaxPoolBlocks)
        return SD_ERR_UNSUPPORTED;
    if (p->Hq % p->Hkv != 0 || p->Hq / p->Hkv > 8 || p->Hq > 1024) return SD_ERR_UNSUPPORTED;
    if (need_pointers) {
        if (!p->block_table || !p->len || !p->n_new || !p->start || !p->slot || !p->position || !ok_ptr(p->plan)) return SD_ERR_INVALID_ARG;
        if (!ok_4(p->block_table) || !ok_4(p->n_blocks) || !ok_4(p->len) || !ok_4(p->n_new) || !ok_4(p->start) || !ok_4(p->slot) ||
            !ok_4(p->position))
            return SD_ERR_INVALID_ARG;
    }
    return SD_OK;
}
// rows of `heads` heads, ld elements apart
bool ok_heads(const void* x, int64_t ld, int heads) { return ok_ptr(x) && ld >= (int64_t)heads * kD && ld % 8 == 0 && ld < (1ll << 31); }

}  // namespace

extern "C" {

int sd_version(void) { return 100; }

const char* sd_status_string(sd_status s) {
    switch (s) {
        case SD_OK: return "SD_OK";
        case SD_ERR_INVALID_ARG: return "SD_ERR_INVALID_ARG";
        case SD_ERR_INVALID_TREE: return "SD_ERR_INVALID_TREE";
        case SD_ERR_UNSUPPORTED: return "SD_ERR_UNSUPPORTED";
        case SD_ERR_WORKSPACE: return "SD_ERR_WORKSPACE";
        case SD_ERR_CUDA: return "SD_ERR_CUDA";
        case SD_ERR_TIMEOUT: return "SD_ERR_TIMEOUT";
        case SD_ERR_BOUNDS: return "SD_ERR_BOUNDS";
    }
    return "SD_ERR_UNKNOWN";
}

size_t sd_workspace_bytes(const sd_batch* geom, int32_t M, int32_t V) {
    size_t a = 0, l = 0;
    if (geom && check_geometry(geom, false) == SD_OK) a = attention_workspace_bytes(*geom);
    if (M > 0 && V > 0) l = stats_workspace_bytes(M, V);    // covers sd_lmhead_argmax, the fused tail and sd_lmhead_stats
    if (geom && V > 0 && check_geometry(geom, false) == SD_OK) {
        const size_t sw = sampled_workspace_bytes(geom->B, geom->T_max, V, 16384);   // sd_accept_tree_sampled (Hd <= 16384)
        if (sw > l) l = sw;
    }
    size_t n = a > l ? a : l;
    return (n + 255) & ~(size_t)255;
}

sd_status sd_tree_prepare(const sd_batch* batch, int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!ok_ptr(batch->anc_mask) || !dev_status) return SD_ERR_INVALID_ARG;
    return launch_tree_prepare(*batch, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_verify_attention(const sd_batch* batch, const sd_kv_layer* cache,
                              const void* q, const void* k_tree, const void* v_tree,
                              float scale, void* out, float* lse,
                              void* workspace, size_t workspace_bytes,
                              int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!cache || !ok_ptr(cache->k) || !ok_ptr(cache->v) || cache->num_blocks < 1) return SD_ERR_INVALID_ARG;
    if (!ok_ptr(q) || !ok_ptr(k_tree) || !ok_ptr(v_tree) || !ok_ptr(out) || !ok_ptr(batch->anc_mask))
        return SD_ERR_INVALID_ARG;
    if (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) return SD_ERR_INVALID_ARG;
    if (!ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (!(scale > 0.f)) return SD_ERR_INVALID_ARG;
    return launch_attention(*batch, *cache, q, k_tree, v_tree, scale, out, lse, workspace,
                            workspace_bytes, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_verify_attention_layers(const sd_batch* batch, const sd_kv_layer* caches, int32_t L,
                                     const void* const* q_layers, const void* const* k_tree_layers,
                                     const void* const* v_tree_layers, float scale,
                                     void* const* out_layers, float* const* lse_layers,
                                     void* workspace, size_t workspace_bytes,
                                     int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!caches || L < 1 || !q_layers || !k_tree_layers || !v_tree_layers || !out_layers) return SD_ERR_INVALID_ARG;
    if (!ok_ptr(batch->anc_mask) || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (!(scale > 0.f)) return SD_ERR_INVALID_ARG;
    for (int l = 0; l < L; ++l) {
        if (!ok_ptr(caches[l].k) || !ok_ptr(caches[l].v) || caches[l].num_blocks < 1) return SD_ERR_INVALID_ARG;
        if (!ok_ptr(q_layers[l]) || !ok_ptr(k_tree_layers[l]) || !ok_ptr(v_tree_layers[l]) || !ok_ptr(out_layers[l]))
            return SD_ERR_INVALID_ARG;
        if (lse_layers && lse_layers[l] && (reinterpret_cast<uintptr_t>(lse_layers[l]) & 3u)) return SD_ERR_INVALID_ARG;
    }
    if (workspace_bytes < attention_workspace_bytes(*batch)) return SD_ERR_WORKSPACE;
    return launch_attention_layers(*batch, caches, L, q_layers, k_tree_layers, v_tree_layers, scale, out_layers,
                                   lse_layers, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_lmhead_argmax(const void* hidden, const void* W, int32_t M, int32_t Hd, int32_t V,
                           int32_t* argmax, float* maxlogit, void* workspace, size_t workspace_bytes,
                           int32_t* dev_status, void* stream) {
    if (!ok_ptr(hidden) || !ok_ptr(W) || !argmax || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (M < 1 || V < 1 || Hd < 1) return SD_ERR_INVALID_ARG;
    if (Hd % 64 != 0) return SD_ERR_UNSUPPORTED;
    return launch_lmhead(hidden, W, M, Hd, V, argmax, maxlogit, workspace, workspace_bytes, dev_status,
                         static_cast<cudaStream_t>(stream));
}

sd_status sd_accept_tree(const sd_batch* batch, const int32_t* draft_tok, const int32_t* target_argmax,
                         int32_t* n_acc, int32_t* path, int32_t* out_tok, int32_t* new_len,
                         int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!draft_tok || !target_argmax || !n_acc || !path || !out_tok || !new_len || !dev_status)
        return SD_ERR_INVALID_ARG;
    return launch_accept(*batch, draft_tok, target_argmax, n_acc, path, out_tok, new_len, dev_status,
                         static_cast<cudaStream_t>(stream));
}

sd_status sd_compact_kv(const sd_batch* batch, const sd_kv_layer* layers, int32_t L,
                        const void* const* k_tree_layers, const void* const* v_tree_layers,
                        const int32_t* n_acc, const int32_t* path, int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!layers || L < 1 || !k_tree_layers || !v_tree_layers || !n_acc || !path || !dev_status)
        return SD_ERR_INVALID_ARG;
    for (int l = 0; l < L; ++l) {
        if (!ok_ptr(layers[l].k) || !ok_ptr(layers[l].v) || layers[l].num_blocks < 1) return SD_ERR_INVALID_ARG;
        if (!ok_ptr(k_tree_layers[l]) || !ok_ptr(v_tree_layers[l])) return SD_ERR_INVALID_ARG;
    }
    return launch_compact(*batch, layers, L, k_tree_layers, v_tree_layers, n_acc, path, dev_status,
                          static_cast<cudaStream_t>(stream));
}

sd_status sd_lmhead_accept_compact(const sd_batch* batch, const void* hidden, const void* W, int32_t Hd, int32_t V,
                                   const int32_t* draft_tok, const sd_kv_layer* layers, int32_t L,
                                   const void* const* k_tree_layers, const void* const* v_tree_layers,
                                   int32_t* argmax, float* maxlogit,
                                   int32_t* n_acc, int32_t* path, int32_t* out_tok, int32_t* new_len,
                                   void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!ok_ptr(hidden) || !ok_ptr(W) || !argmax || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (V < 1 || Hd < 1) return SD_ERR_INVALID_ARG;
    if (Hd % 64 != 0) return SD_ERR_UNSUPPORTED;
    if (!draft_tok || !n_acc || !path || !out_tok || !new_len) return SD_ERR_INVALID_ARG;
    if (!layers || L < 1 || !k_tree_layers || !v_tree_layers) return SD_ERR_INVALID_ARG;
    for (int l = 0; l < L; ++l) {
        if (!ok_ptr(layers[l].k) || !ok_ptr(layers[l].v) || layers[l].num_blocks < 1) return SD_ERR_INVALID_ARG;
        if (!ok_ptr(k_tree_layers[l]) || !ok_ptr(v_tree_layers[l])) return SD_ERR_INVALID_ARG;
    }
    return launch_lmhead_accept_compact(*batch, hidden, W, Hd, V, draft_tok, layers, L, k_tree_layers, v_tree_layers,
                                        argmax, maxlogit, n_acc, path, out_tok, new_len, workspace, workspace_bytes,
                                        dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_lmhead_stats(const void* hidden, const void* W, int32_t M, int32_t Hd, int32_t V, float inv_temp,
                          int32_t* argmax, float* maxlogit, float* lse, float* group_stats,
                          void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    if (group_stats && (reinterpret_cast<uintptr_t>(group_stats) & 7u)) return SD_ERR_INVALID_ARG;
    if (!ok_ptr(hidden) || !ok_ptr(W) || !lse || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (M < 1 || V < 1 || Hd < 1 || !(inv_temp > 0.f)) return SD_ERR_INVALID_ARG;
    if (Hd % 64 != 0) return SD_ERR_UNSUPPORTED;
    return launch_lmhead_stats(hidden, W, M, Hd, V, inv_temp, argmax, maxlogit, lse, group_stats, workspace,
                               workspace_bytes, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_accept_tree_sampled(const sd_batch* batch, const void* hidden, const void* W, int32_t Hd, int32_t V,
                                 float inv_temp, const float* lse, const float* group_stats, const int32_t* draft_tok,
                                 const float* u, const float* w,
                                 int32_t* n_acc, int32_t* path, int32_t* out_tok, int32_t* new_len,
                                 void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!ok_ptr(hidden) || !ok_ptr(W) || !lse || !draft_tok || !u || !w) return SD_ERR_INVALID_ARG;
    if (!n_acc || !path || !out_tok || !new_len || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (V < 1 || Hd < 1 || !(inv_temp > 0.f)) return SD_ERR_INVALID_ARG;
    if (Hd % 64 != 0) return SD_ERR_UNSUPPORTED;
    return launch_accept_sampled(*batch, hidden, W, Hd, V, inv_temp, lse, group_stats, draft_tok, u, w, n_acc, path, out_tok,
                                 new_len, workspace, workspace_bytes, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_lmhead_stats_logits(const void* hidden, const void* W, int32_t M, int32_t Hd, int32_t V, float inv_temp,
                                 int32_t* argmax, float* maxlogit, float* lse, float* logits,
                                 void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    if (!ok_ptr(hidden) || !ok_ptr(W) || !lse || !logits || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(logits) & 3u) return SD_ERR_INVALID_ARG;
    if (M < 1 || V < 1 || Hd < 1 || !(inv_temp > 0.f)) return SD_ERR_INVALID_ARG;
    if (Hd % 64 != 0) return SD_ERR_UNSUPPORTED;
    return launch_lmhead_stats(hidden, W, M, Hd, V, inv_temp, argmax, maxlogit, lse, nullptr, workspace, workspace_bytes,
                               dev_status, static_cast<cudaStream_t>(stream), logits);
}

sd_status sd_accept_chain_sampled(const sd_batch* batch, const void* hidden, const void* W, int32_t Hd, int32_t V,
                                  float inv_temp, const float* lse, const float* logits,
                                  const int32_t* draft_tok, const float* q_tok,
                                  const float* q_rows, const float* u, const float* w,
                                  int32_t* n_acc, int32_t* path, int32_t* out_tok, int32_t* new_len,
                                  void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!ok_ptr(hidden) || !ok_ptr(W) || !lse || !draft_tok || !q_tok || !q_rows || !u || !w) return SD_ERR_INVALID_ARG;
    if (!n_acc || !path || !out_tok || !new_len || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (V < 1 || Hd < 1 || !(inv_temp > 0.f)) return SD_ERR_INVALID_ARG;
    if (Hd % 64 != 0) return SD_ERR_UNSUPPORTED;
    return launch_accept_chain_sampled(*batch, hidden, W, Hd, V, inv_temp, lse, logits, draft_tok, q_tok, q_rows, u, w, n_acc, path,
                                       out_tok, new_len, workspace, workspace_bytes, dev_status,
                                       static_cast<cudaStream_t>(stream));
}

sd_status sd_accept_tree_sampled_q(const sd_batch* batch, int32_t V, float inv_temp, const float* lse, const float* logits,
                                   const int32_t* draft_tok, const float* q_rows, const float* u, const float* w,
                                   int32_t* n_acc, int32_t* path, int32_t* out_tok, int32_t* new_len,
                                   int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!lse || !logits || !draft_tok || !q_rows || !u || !w) return SD_ERR_INVALID_ARG;
    if (!n_acc || !path || !out_tok || !new_len || !dev_status) return SD_ERR_INVALID_ARG;
    if (V < 1 || !(inv_temp > 0.f)) return SD_ERR_INVALID_ARG;
    return launch_accept_tree_sampled_q(*batch, V, inv_temp, lse, logits, draft_tok, q_rows, u, w, n_acc, path, out_tok,
                                        new_len, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_lmhead_accept_sampled_compact(const sd_batch* batch, const void* hidden, const void* W, int32_t Hd, int32_t V,
                                           float inv_temp, const int32_t* draft_tok, const float* u, const float* w,
                                           const sd_kv_layer* layers, int32_t L,
                                           const void* const* k_tree_layers, const void* const* v_tree_layers,
                                           float* lse, float* group_stats,
                                           int32_t* n_acc, int32_t* path, int32_t* out_tok, int32_t* new_len,
                                           void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
    sd_status s = check_geometry(batch, true);
    if (s != SD_OK) return s;
    if (!ok_ptr(hidden) || !ok_ptr(W) || !lse || !group_stats || !draft_tok || !u || !w) return SD_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(group_stats) & 7u) return SD_ERR_INVALID_ARG;
    if (!n_acc || !path || !out_tok || !new_len || !ok_ptr(workspace) || !dev_status) return SD_ERR_INVALID_ARG;
    if (V < 1 || Hd < 1 || !(inv_temp > 0.f)) return SD_ERR_INVALID_ARG;
    if (Hd % 64 != 0) return SD_ERR_UNSUPPORTED;
    if (!layers || L < 1 || !k_tree_layers || !v_tree_layers) return SD_ERR_INVALID_ARG;
    for (int l = 0; l < L; ++l) {
        if (!ok_ptr(layers[l].k) || !ok_ptr(layers[l].v) || layers[l].num_blocks < 1) return SD_ERR_INVALID_ARG;
        if (!ok_ptr(k_tree_layers[l]) || !ok_ptr(v_tree_layers[l])) return SD_ERR_INVALID_ARG;
    }
    return launch_lmhead_accept_sampled_compact(*batch, hidden, W, Hd, V, inv_temp, draft_tok, u, w, layers, L, k_tree_layers,
                                                v_tree_layers, lse, group_stats, n_acc, path, out_tok, new_len, workspace,
                                                workspace_bytes, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_draft_feature_attention(const void* qp, const void* k, const void* v, int32_t S, int32_t L, int32_t Q,
                                     int32_t H, int32_t D, float scale, void* out, void* stream) {
    if (!ok_ptr(qp) || !ok_ptr(k) || !ok_ptr(v) || !ok_ptr(out)) return SD_ERR_INVALID_ARG;
    if (S < 1 || L < 1 || Q < 1 || H < 1 || !(scale > 0.f)) return SD_ERR_INVALID_ARG;
    if (D != H * 128 || L > 32 || Q > 8) return SD_ERR_UNSUPPORTED;
    return launch_draft_feature_attention(qp, k, v, S, L, Q, H, scale, out, static_cast<cudaStream_t>(stream));
}

sd_status sd_top_logits(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V, int32_t K, float inv_temp,
                        float* values, int32_t* index, float* lse, int32_t* dev_status, void* stream) {
    const sd_status s = check_rows(logits, dtype, ld, M, V);
    if (s != SD_OK) return s;
    if (K < 1 || !(inv_temp > 0.f) || !(inv_temp < INFINITY)) return SD_ERR_INVALID_ARG;
    if (K > 1024) return SD_ERR_UNSUPPORTED;
    if (M == 0) return SD_OK;
    if (!values || !index || !ok_4(values) || !ok_4(index) || !ok_4(lse) || !dev_status) return SD_ERR_INVALID_ARG;
    return launch_top_logits(logits, dtype, ld, M, V, K, inv_temp, values, index, lse, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_sample_logits(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V, const sd_sampling* how,
                           const float* u, int32_t N, int32_t* tokens, float* prob, float* probs, float* lse,
                           int32_t* dev_status, void* stream) {
    const sd_status s = check_rows(logits, dtype, ld, M, V);
    if (s != SD_OK) return s;
    if (!ok_sampling(how) || N < 1) return SD_ERR_INVALID_ARG;
    if (N > 64) return SD_ERR_UNSUPPORTED;
    if (M == 0) return SD_OK;
    if (!u || !tokens || !dev_status) return SD_ERR_INVALID_ARG;
    if (!ok_4(u) || !ok_4(tokens) || !ok_4(prob) || !ok_4(lse) || (probs && !aligned16(probs)) || probs == logits) return SD_ERR_INVALID_ARG;
    return launch_sample(logits, dtype, ld, M, V, *how, u, N, tokens, prob, probs, false, lse, nullptr, dev_status,
                         static_cast<cudaStream_t>(stream));
}

sd_status sd_filter_logits(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V, const sd_sampling* how,
                           float* out, float* lse, int32_t* kept, int32_t* dev_status, void* stream) {
    const sd_status s = check_rows(logits, dtype, ld, M, V);
    if (s != SD_OK) return s;
    if (!ok_sampling(how)) return SD_ERR_INVALID_ARG;
    if (M == 0) return SD_OK;
    if (!ok_ptr(out) || !lse || !ok_4(lse) || !ok_4(kept) || !dev_status) return SD_ERR_INVALID_ARG;
    if (out == logits && (dtype != SD_F32 || ld != V)) return SD_ERR_INVALID_ARG;
    return launch_sample(logits, dtype, ld, M, V, *how, nullptr, 0, nullptr, nullptr, out, true, lse, kept, dev_status,
                         static_cast<cudaStream_t>(stream));
}

sd_status sd_distill_loss(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V, const float* top_val,
                          const int32_t* top_idx, int32_t K, const float* top_lse, const int32_t* label, float inv_temp,
                          float kl_weight, float ce_weight, float* kl, float* ce, float* stats, const float* dloss, void* grad,
                          int64_t grad_ld, int32_t* dev_status, void* stream) {
    const sd_status s = check_distill(logits, dtype, ld, M, V, top_val, top_idx, K, top_lse, label, inv_temp, dloss, grad, grad_ld, dev_status);
    if (s != SD_OK || M == 0) return s;
    if (!kl || !ok_4(kl) || (label && !ce) || !ok_4(ce) || (stats && !aligned16(stats))) return SD_ERR_INVALID_ARG;
    return launch_distill_loss(DistillCall{logits, ld, V, top_val, top_idx, K, top_lse, label, inv_temp, kl_weight, ce_weight, kl, ce, stats, dloss,
                                           grad, grad_ld, dev_status}, dtype, M, static_cast<cudaStream_t>(stream));
}

sd_status sd_distill_grad(const void* logits, int32_t dtype, int64_t ld, int32_t M, int32_t V, const float* top_val,
                          const int32_t* top_idx, int32_t K, const float* top_lse, const int32_t* label, float inv_temp,
                          float kl_weight, float ce_weight, const float* stats, const float* dloss, void* grad, int64_t grad_ld,
                          int32_t* dev_status, void* stream) {
    const sd_status s = check_distill(logits, dtype, ld, M, V, top_val, top_idx, K, top_lse, label, inv_temp, dloss, grad, grad_ld, dev_status);
    if (s != SD_OK || M == 0) return s;
    if (!grad || !ok_ptr(stats)) return SD_ERR_INVALID_ARG;
    return launch_distill_grad(DistillCall{logits, ld, V, top_val, top_idx, K, top_lse, label, inv_temp, kl_weight, ce_weight, nullptr, nullptr,
                                           const_cast<float*>(stats), dloss, grad, grad_ld, dev_status}, dtype, M, static_cast<cudaStream_t>(stream));
}

sd_status sd_assign_blocks(const sd_block_pool* pool, int32_t B, int32_t max_blocks_per_seq, int32_t* block_table,
                           int32_t* n_blocks, const int32_t* len, const int32_t* n_new, int32_t* granted,
                           int32_t* dev_status, void* stream) {
    if (!pool || B < 1 || max_blocks_per_seq < 1 || pool->num_blocks < 1) return SD_ERR_INVALID_ARG;
    if (B > kMaxRequests || pool->num_blocks > kMaxPoolBlocks || (int64_t)B * max_blocks_per_seq >= 1 << 29) return SD_ERR_UNSUPPORTED;
    if (!pool->free_blocks || !pool->n_free || !block_table || !n_blocks || !len || !n_new || !dev_status) return SD_ERR_INVALID_ARG;
    if (!ok_4(pool->free_blocks) || !ok_4(pool->n_free) || !ok_4(block_table) || !ok_4(n_blocks) || !ok_4(len) || !ok_4(n_new) || !ok_4(granted))
        return SD_ERR_INVALID_ARG;
    return launch_assign_blocks(*pool, B, max_blocks_per_seq, block_table, n_blocks, len, n_new, granted, dev_status,
                                static_cast<cudaStream_t>(stream));
}

size_t sd_prompt_plan_bytes(const sd_prompts* prompts) { return check_prompts(prompts, false) == SD_OK ? prompt_plan_bytes(*prompts) : 0; }
size_t sd_prompt_workspace_bytes(const sd_prompts* prompts) {
    return check_prompts(prompts, false) == SD_OK ? prompt_workspace_bytes(*prompts) : 0;
}

sd_status sd_prompt_prepare(const sd_prompts* prompts, int32_t* dev_status, void* stream) {
    const sd_status s = check_prompts(prompts, true);
    if (s != SD_OK) return s;
    if (!dev_status) return SD_ERR_INVALID_ARG;
    return launch_prompt_prepare(*prompts, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_append_kv(const sd_prompts* prompts, const sd_kv_layer* cache, const void* k, int64_t ldk, const void* v, int64_t ldv,
                       int32_t* dev_status, void* stream) {
    const sd_status s = check_prompts(prompts, true);
    if (s != SD_OK) return s;
    if (!cache || !ok_ptr(cache->k) || !ok_ptr(cache->v) || cache->num_blocks != prompts->num_blocks || !dev_status) return SD_ERR_INVALID_ARG;
    if (prompts->N == 0) return SD_OK;
    if (!ok_heads(k, ldk, prompts->Hkv) || !ok_heads(v, ldv, prompts->Hkv)) return SD_ERR_INVALID_ARG;
    return launch_append_kv(*prompts, *cache, k, ldk, v, ldv, dev_status, static_cast<cudaStream_t>(stream));
}

sd_status sd_prompt_attention(const sd_prompts* prompts, const sd_kv_layer* cache, const void* q, int64_t ldq, float scale,
                              void* out, int64_t ldo, float* lse, void* workspace, size_t workspace_bytes,
                              int32_t* dev_status, void* stream) {
    const sd_status s = check_prompts(prompts, true);
    if (s != SD_OK) return s;
    if (!cache || !ok_ptr(cache->k) || !ok_ptr(cache->v) || cache->num_blocks != prompts->num_blocks || !dev_status) return SD_ERR_INVALID_ARG;
    if (!(scale > 0.f) || !(scale < INFINITY) || !ok_4(lse)) return SD_ERR_INVALID_ARG;
    if (prompts->N == 0) return SD_OK;                     // (which needs no scratch either)
    if (!ok_ptr(workspace)) return SD_ERR_INVALID_ARG;
    if (workspace_bytes < prompt_workspace_bytes(*prompts)) return SD_ERR_WORKSPACE;
    if (!ok_heads(q, ldq, prompts->Hq) || !ok_heads(out, ldo, prompts->Hq) || out == q) return SD_ERR_INVALID_ARG;
    if ((int64_t)cache->num_blocks * prompts->Hkv * kBlock > INT32_MAX) return SD_ERR_UNSUPPORTED;             // (rows of the copies' coordinates)
    return launch_prompt_attention(*prompts, *cache, q, ldq, scale, out, ldo, lse, workspace, dev_status,
                                   static_cast<cudaStream_t>(stream));
}

}  // extern "C"
