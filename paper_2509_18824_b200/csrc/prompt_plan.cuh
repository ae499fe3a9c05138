// Packed new tokens of several requests: what the calls on them share, and how the attention's work is laid out.
#pragma once
#include "common.cuh"

namespace sdv {

constexpr int kMaxRequests = 8192;             // requests of a call: their prefix sums stand in shared memory
constexpr int kMaxPoolBlocks = 1 << 25;        // so that a slot (64 x block + offset) is an int32

// Request b's new tokens (packed rows start .. end) behind its cached ones, and whether its blocks hold them all.
struct RequestSpan { int len, n; bool covered; };
__device__ __forceinline__ RequestSpan request_span(const sd_prompts& p, int b, int start, int end) {
    RequestSpan r;
    r.len = __ldcg(p.len + b);
    r.n = end - start;
    const long long blocks = ((long long)r.len + r.n + kBlock - 1) / kBlock;
    const int held = p.n_blocks ? min(__ldcg(p.n_blocks + b), p.max_blocks_per_seq) : p.max_blocks_per_seq;
    r.covered = r.len >= 0 && r.n == __ldcg(p.n_new + b) && blocks <= held && blocks < kMaxPoolBlocks;       // (places are int32)
    return r;
}

// ---------------------------------------------------------------- the attention's work
// A row tile is the query heads of one KV head for whole tokens, at most 128 rows; an entry is a row tile and the key blocks [kb0, kb1) of
// its request; every KV head has the same entries.  Entries are in order of their length, the longest first; CTA c of the attention's grid
// takes number c, then 2 G - 1 - c, 2 G + c, ...
constexpr int kPromptTile = 128;               // keys per tile: two cache blocks
struct alignas(16) PromptEntry {
    int row0, pos0;        // packed row and place in the sequence of the entry's first token
    int tokens;
    int b;
    int kb0, kb1;          // key blocks (kb0 even)
    int end;               // len + n_new of the request
    int slot;              // first partial result (KV head 0), or -1: the entry has all the keys of its rows
};
struct alignas(16) PromptSplit { int row0, tokens, slot, chunks; };     // partial results slot + chunk * Hkv + KV head
struct alignas(16) PromptHeader { int entries, splits, slots, unused; };

struct PromptGeom {
    int G;                 // query heads of a KV head
    int tokens;            // of a row tile
    int cap_entries, cap_splits, cap_slots;
    int rows;              // of a partial result
    int sms;
    int g_magic;           // ceil(65536 / G): row / G for rows below 128
    __host__ __device__ __forceinline__ int token_of(int row) const { return (row * g_magic) >> 16; }
    __host__ __device__ __forceinline__ size_t slot_floats() const { return (size_t)rows * (kD + 2); }
};
inline PromptGeom prompt_geom(const sd_prompts& p, int sms) {
    PromptGeom g;
    g.G = p.Hq / p.Hkv;
    g.tokens = 128 / g.G;
    g.sms = sms;
    g.g_magic = (65536 + g.G - 1) / g.G;
    // (chunk_tiles: a chunk is at least a 2 sms-th of all key tiles of all heads, and what is cut at least two of them long)
    g.cap_slots = 4 * sms + p.Hkv;
    g.cap_splits = 2 * sms / p.Hkv + 2;
    g.cap_entries = p.N / g.tokens + (p.B < p.N ? p.B : p.N) + 4 * sms / p.Hkv + 4;
    const long long rows = (long long)p.N * g.G;
    g.rows = rows >= 128 ? 128 : (int)((rows + 7) / 8 * 8);
    return g;
}
__host__ __device__ __forceinline__ PromptHeader* plan_header(void* plan) { return static_cast<PromptHeader*>(plan); }
__host__ __device__ __forceinline__ PromptEntry* plan_entries(void* plan) { return reinterpret_cast<PromptEntry*>(plan_header(plan) + 1); }
__host__ __device__ __forceinline__ PromptSplit* plan_splits(void* plan, int cap_entries) {
    return reinterpret_cast<PromptSplit*>(plan_entries(plan) + cap_entries);
}
int current_sms();

}  // namespace sdv
