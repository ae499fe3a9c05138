// Packed new tokens of several requests: what the calls on them share, and how the attention's work is laid out.
#pragma once
#include "common.cuh"

namespace sdv {

constexpr int kMaxRequests = 8192;             // requests of a call: their prefix sums stand in shared memory
constexpr int kMaxPoolBlocks = 1 << 25;        // so that a slot (64 x block + offset) is an int32

// Request b's n new tokens behind its cached ones, and whether its blocks hold them all.
struct RequestSpan { int len, n; bool covered; };
__device__ __forceinline__ RequestSpan request_span(const sd_prompts& p, int b, int n) {
    RequestSpan r;
    r.len = __ldcg(p.len + b);
    r.n = n;
    const long long blocks = ((long long)r.len + n + kBlock - 1) / kBlock;
    const int held = p.n_blocks ? min(__ldcg(p.n_blocks + b), p.max_blocks_per_seq) : p.max_blocks_per_seq;
    r.covered = r.len >= 0 && n >= 0 && blocks <= held && blocks < kMaxPoolBlocks;       // (places are int32)
    return r;
}

// ---------------------------------------------------------------- the attention's work
// A row tile is the query heads of one KV head for whole tokens, at most 128 rows; an entry is a row tile with all the keys that it sees; every
// KV head has the same entries.  They are handed to the CTAs in one of two ways.
//   Dealt out: entries in order of their length, the longest first, each for all heads; CTA c of G takes number c, then 2 G - 1 - c, 2 G + c ..
//   In parts: all entries of all heads stand in one line, entry by entry and head by head, each as long as its key tiles and kEntryTiles; the
//   line is cut into G equal parts.  An entry that a cut goes through is computed in chunks of whole key tiles and joined.  Every
//   CTA has at most two such chunks, its first and its last piece.
// Parts are even, but their ends have to be joined (about 5 us), and what an entry costs beside its tiles is not known well (it overlaps its
// neighbours); dealt out, every CTA has as many entries as the others.  So entries are dealt out where every CTA gets kDealFrom times the
// longest.  Us, dealt out and in parts (28 query, 4 KV heads): 16 prompts of up to 2048 tokens 137 and 148, three of up to 6000 with twelve heads 189 and
// 198, eight of 4096 799 and 811, one of 32749 5660 and 5735; in parts by the rule: 1000 tokens behind 7000 beside 24 single ones 112 and 114, 32 single
// tokens behind 512 to 16384 121 and 94, one behind 2047 20 and 12, 61 tokens behind 16000 104 and 30.
constexpr int kPromptTile = 128;               // keys per tile: two cache blocks
constexpr int kEntryTiles = 2;                 // what an entry costs beside its key tiles, in key tiles (1 and 3: the same within 1 %)
constexpr int kPartMin = 2;                    // the shortest part of a CTA
constexpr int kDealFrom = 4;
constexpr int kSnap = 3;                       // a cut so few key tiles from an entry's end is made there
struct alignas(16) PromptEntry {
    int row0, pos0;        // packed row and place in the sequence of the entry's first token
    int tokens;
    int b;
    int blocks;            // key blocks that its last token sees
    int end;               // len + n_new of the request
    int unused0, unused1;
};
struct alignas(16) PromptStart { int e, h, tile, unused; PromptEntry entry; };  // where a CTA's part begins (and the one's before ends); dealt out: its first piece
struct alignas(16) PromptSplit {
    int row0, tokens, h;
    int slot, cta, chunks;                     // partial results: slot, then 2 (cta + 1), 2 (cta + 2) ..
    int unused0, unused1;
};
struct alignas(16) PromptHeader { int splits, dealt, stamp, unused; };          // dealt: how many entries, 0: in parts

struct PromptGeom {
    int G;                 // query heads of a KV head
    int tokens;            // of a row tile
    int sms;               // CTAs
    int rows;              // of a partial result
    int g_magic;           // ceil(65536 / G): row / G for rows below 128
    int cap;               // entries that the plan has room for
    __host__ __device__ __forceinline__ int token_of(int row) const { return (row * g_magic) >> 16; }
    __host__ __device__ __forceinline__ size_t slot_floats() const { return (size_t)rows * (kD + 2); }
};
inline PromptGeom prompt_geom(const sd_prompts& p, int sms) {
    PromptGeom g;
    g.G = p.Hq / p.Hkv;
    g.tokens = 128 / g.G;
    g.sms = sms;
    g.g_magic = (65536 + g.G - 1) / g.G;
    const long long rows = (long long)p.N * g.G;
    g.rows = rows >= 128 ? 128 : (int)((rows + 7) / 8 * 8);
    g.cap = p.N / g.tokens + (p.B < p.N ? p.B : p.N) + 1;
    return g;
}
// Tells a plan that sd_prompt_prepare has made for these sizes from other memory.
__host__ __device__ __forceinline__ int plan_stamp(const sd_prompts& p, const PromptGeom& g) {
    uint32_t x = 0x9e3779b9u;
    for (const int v : {p.B, p.N, p.Hq, p.Hkv, p.max_blocks_per_seq, p.num_blocks, g.sms}) x = (x ^ (uint32_t)v) * 0x01000193u + 0x7f4a7c15u;
    return (int)x;
}
// the plan: header, starts [sms + 1], splits [sms], entries [cap], and for entries that are dealt out their order [cap]
__host__ __device__ __forceinline__ PromptHeader* plan_header(void* plan) { return static_cast<PromptHeader*>(plan); }
__host__ __device__ __forceinline__ PromptStart* plan_starts(void* plan) { return reinterpret_cast<PromptStart*>(plan_header(plan) + 1); }
__host__ __device__ __forceinline__ PromptSplit* plan_splits(void* plan, int sms) { return reinterpret_cast<PromptSplit*>(plan_starts(plan) + sms + 1); }
__host__ __device__ __forceinline__ PromptEntry* plan_entries(void* plan, int sms) { return reinterpret_cast<PromptEntry*>(plan_splits(plan, sms) + sms); }
__host__ __device__ __forceinline__ int* plan_order(PromptEntry* entries, size_t cap) { return reinterpret_cast<int*>(entries + cap); }
int current_sms();

}  // namespace sdv
