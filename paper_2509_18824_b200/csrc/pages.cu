// Block tables, slot maps and the cache's new rows: what stands between a request's length and the attention over its cache.
//
// Lengths are known on the device first (acceptance leaves new_len there), so tables that are made on the host cost a round trip per
// step.  Both calls on lengths are scans over the requests; every CTA repeats the scan (8192 requests: 32 KB of lengths through L2), so
// that nothing has to be handed from one to another.
#include "prompt_plan.cuh"
#include "sm100.cuh"

namespace sdv {
using namespace sm100;

namespace {
constexpr int kPageThreads = 1024;
constexpr int kSlotRows = 4096;                // packed rows of one CTA of the slot map

// Sums of a value over the threads in front of this one, and over all; two values at a time.
struct Pair { long long a, b; };
__device__ __forceinline__ Pair block_scan(Pair v, Pair* warp_sums, Pair* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Pair in = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, in.a, d), b = __shfl_up_sync(0xffffffffu, in.b, d);
        if (lane >= d) { in.a += a; in.b += b; }
    }
    if (lane == 31) warp_sums[warp] = in;
    __syncthreads();
    if (warp == 0) {
        Pair w = warp_sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long a = __shfl_up_sync(0xffffffffu, w.a, d), b = __shfl_up_sync(0xffffffffu, w.b, d);
            if (lane >= d) { w.a += a; w.b += b; }
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    const Pair before = warp > 0 ? warp_sums[warp - 1] : Pair{0, 0};
    *total = warp_sums[31];
    __syncthreads();                           // (warp_sums may be written again)
    return Pair{before.a + in.a - v.a, before.b + in.b - v.b};
}
__device__ __forceinline__ int cut(long long x) { return (int)min(x, 1ll << 30); }

// the last of n ascending numbers that is at most x (the first one is)
__device__ __forceinline__ int last_at_most(const int* a, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (a[m] <= x) lo = m; else hi = m;
    }
    return lo;
}
}  // namespace

// One cluster.  Blocks that come free stand in front of the stack, in order of the requests; the t-th block that is taken is the t-th of
// this list.  So giving back what was taken leaves the stack as it was.
__global__ void __launch_bounds__(kPageThreads)
assign_blocks_kernel(sd_block_pool pool, int B, int W, int32_t* table, int32_t* n_blocks, const int32_t* len, const int32_t* n_new,
                     int32_t* granted, int32_t* status) {
    extern __shared__ int page_smem[];
    int *const grow_at = page_smem, *const free_at = page_smem + B, *const held_of = page_smem + 2 * B;      // prefix sums; blocks held
    __shared__ Pair warp_sums[32];
    __shared__ int taken_smem;
    // (Tables are read through the read-only path by the attention calls, so no kernel behind this one begins before it has ended.)
    griddep_wait();
    settle(pool.free_blocks); settle(pool.n_free); settle(table); settle(n_blocks); settle(len); settle(n_new);
    const int cta = blockIdx.x, ctas = gridDim.x;
    const bool first = cta == 0;
    if (threadIdx.x == 0) taken_smem = 0;
    int n_free = __ldcg(pool.n_free);
    if (n_free < 0 || n_free > pool.num_blocks) {
        if (first && threadIdx.x == 0) set_status(status, SD_ERR_BOUNDS);
        n_free = 0;
    }
    Pair sum{0, 0};
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + (int)threadIdx.x;
        Pair mine{0, 0};
        int held = 0;
        if (b < B) {
            held = __ldcg(n_blocks + b);
            const int l = __ldcg(len + b), n = __ldcg(n_new + b);
            const long long want = ((long long)l + n + kBlock - 1) / kBlock;
            int bad = 0;
            if (l < 0 || n < 0) bad = SD_ERR_INVALID_ARG;
            else if (held < 0 || held > W || want > W) bad = SD_ERR_BOUNDS;
            if (bad) { if (first) set_status(status, bad); }                    // (and the request keeps what it has)
            else if (want > held) mine.a = want - held;
            else mine.b = held - want;
        }
        Pair all;
        const Pair before = block_scan(mine, warp_sums, &all);
        if (b < B) { grow_at[b] = cut(sum.a + before.a); free_at[b] = cut(sum.b + before.b); held_of[b] = held; }
        sum.a += all.a; sum.b += all.b;
    }
    const int come_free = cut(sum.b), needed = cut(sum.a);
    const long long supply = (long long)n_free + come_free;
    const auto grow_end = [&](int b) { return b + 1 < B ? grow_at[b + 1] : needed; };
    const auto free_end = [&](int b) { return b + 1 < B ? free_at[b + 1] : come_free; };
    __syncthreads();
    // what is taken: the needs of the requests in front of the first that goes short
    int taken = 0;
    for (int b = threadIdx.x; b < B; b += kPageThreads)
        if (grow_end(b) <= supply && grow_end(b) < (1 << 30)) taken = max(taken, grow_end(b));
    if (taken) atomicMax(&taken_smem, taken);
    __syncthreads();
    taken = taken_smem;
    if (ctas > 1) cluster_arrive_release();    // everybody has read the counts

    const auto released = [&](int t) {
        const int b = last_at_most(free_at, B, t), want = held_of[b] - (free_end(b) - free_at[b]);
        return __ldcg(table + (size_t)b * W + want + (t - free_at[b]));
    };
    const int tid = cta * kPageThreads + (int)threadIdx.x, threads = ctas * kPageThreads;
    for (int t = tid; t < taken; t += threads) {
        const int b = last_at_most(grow_at, B, t);
        const int block = t < come_free ? released(t) : __ldcg(pool.free_blocks + n_free - 1 - (t - come_free));
        table[(size_t)b * W + held_of[b] + (t - grow_at[b])] = block;
    }
    for (int t = taken + tid; t < come_free; t += threads) {
        const long long at = (long long)n_free + come_free - 1 - t;
        if (at < pool.num_blocks) pool.free_blocks[at] = released(t);
        else set_status(status, SD_ERR_BOUNDS);                                 // (more than the pool has: given back twice)
    }
    if (ctas > 1) cluster_wait_acquire();
    for (int b = tid; b < B; b += threads) {
        const int grow = grow_end(b) - grow_at[b], shrink = free_end(b) - free_at[b];
        const bool ok = grow == 0 || grow_end(b) <= taken;
        if (grow && ok) n_blocks[b] = held_of[b] + grow;
        if (shrink) n_blocks[b] = held_of[b] - shrink;
        if (granted) granted[b] = ok ? 1 : 0;
    }
    if (tid == 0) *pool.n_free = (int)min((long long)n_free + come_free - taken, (long long)pool.num_blocks);
}

sd_status launch_assign_blocks(const sd_block_pool& pool, int B, int W, int32_t* table, int32_t* n_blocks, const int32_t* len,
                               const int32_t* n_new, int32_t* granted, int32_t* dev_status, cudaStream_t st) {
    const int smem = 3 * B * 4;
    if (!allow_dynamic_smem(assign_blocks_kernel, smem)) return SD_ERR_CUDA;
    const int ctas = B <= 64 ? 1 : 8;
    return launch_dependent(assign_blocks_kernel, dim3(ctas), kPageThreads, smem, ctas, st, pool, B, W, table, n_blocks, len, n_new,
                            granted, dev_status);
}

// First rows of the requests; slot and position of each packed row (all CTAs but the first); the attention's entries (the first).
namespace {
constexpr int kOrderBins = 1024;
constexpr int kEntryTiles = 2;                 // what an entry costs beside its key tiles, in key tiles
constexpr int kChunkMin = 2;                   // key tiles of the shortest chunk
}  // namespace

__global__ void __launch_bounds__(kPageThreads)
prompt_prepare_kernel(sd_prompts p, PromptGeom geom, int32_t* status) {
    extern __shared__ int page_smem[];
    int* const start = page_smem;              // [B + 1]
    int* const first_entry = page_smem + p.B + 1;        // [B + 1] (the first CTA)
    __shared__ Pair warp_sums[32];
    __shared__ int bins[kOrderBins];
    __shared__ int n_splits, n_slots, n_entries;
    begin_dependent(p.block_table, p.n_blocks, p.len, p.n_new, p.start, p.slot, p.position, p.plan);
    const int B = p.B, W = p.max_blocks_per_seq;
    const bool planner = blockIdx.x == 0;
    Pair sum{0, 0};
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + (int)threadIdx.x;
        Pair mine{0, 0};
        if (b < B) {
            const int n = __ldcg(p.n_new + b), l = __ldcg(p.len + b);
            if ((n < 0 || l < 0) && planner) set_status(status, SD_ERR_INVALID_ARG);
            mine.a = max(n, 0);
        }
        Pair all;
        const Pair before = block_scan(mine, warp_sums, &all);
        if (b < B) start[b] = (int)min(sum.a + before.a, (long long)p.N);       // (rows behind the packed ones belong to nobody)
        sum.a += all.a;
    }
    if (threadIdx.x == 0) start[B] = (int)min(sum.a, (long long)p.N);
    if (planner && threadIdx.x == 0 && sum.a > p.N) set_status(status, SD_ERR_BOUNDS);
    __syncthreads();
    if (!planner) {
        const int total = start[B];
        const int r0 = ((int)blockIdx.x - 1) * kSlotRows, r1 = min(r0 + kSlotRows, p.N);
        for (int r = r0 + (int)threadIdx.x; r < r1; r += kPageThreads) {
            int slot = -1, position = 0;
            if (r < total) {
                const int b = last_at_most(start, B, r);
                const RequestSpan q = request_span(p, b, start[b], start[b + 1]);
                position = max(q.len, 0) + r - start[b];
                if (q.covered) {
                    const int block = __ldcg(p.block_table + (size_t)b * W + position / kBlock);
                    if (block >= 0 && block < p.num_blocks) slot = block * kBlock + position % kBlock;
                    else set_status(status, SD_ERR_BOUNDS);
                } else if (!p.n_blocks) {
                    set_status(status, SD_ERR_BOUNDS);
                }
            }
            p.slot[r] = slot;
            p.position[r] = position;
        }
        return;
    }
    // ------------------------------------------------------------ entries
    int at = 0;
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + (int)threadIdx.x;
        Pair mine{0, 0};
        if (b < B) {
            p.start[b] = start[b];
            const RequestSpan q = request_span(p, b, start[b], start[b + 1]);
            if (q.covered) mine.a = (q.n + geom.tokens - 1) / geom.tokens;
        }
        Pair all;
        const Pair before = block_scan(mine, warp_sums, &all);
        if (b < B) first_entry[b] = at + (int)before.a;
        at += (int)all.a;
    }
    if (threadIdx.x == 0) {
        p.start[B] = start[B];
        first_entry[B] = at;
        n_splits = n_slots = n_entries = 0;
    }
    for (int i = threadIdx.x; i < kOrderBins; i += kPageThreads) bins[i] = 0;
    __syncthreads();
    const int total = min(at, geom.cap_entries);
    // entry e with all its keys
    const auto whole = [&](int e) {
        PromptEntry x;
        x.b = last_at_most(first_entry, B, e);
        const int len = __ldcg(p.len + x.b), n = start[x.b + 1] - start[x.b], t0 = (e - first_entry[x.b]) * geom.tokens;
        x.row0 = start[x.b] + t0;
        x.pos0 = len + t0;
        x.tokens = min(geom.tokens, n - t0);
        x.kb0 = 0;
        x.kb1 = (x.pos0 + x.tokens + kBlock - 1) / kBlock;
        x.end = len + n;
        x.slot = -1;
        return x;
    };
    Pair cost{0, 0};
    for (int e = threadIdx.x; e < total; e += kPageThreads) cost.a += (whole(e).kb1 + 1) / 2 + kEntryTiles;
    Pair all;
    block_scan(cost, warp_sums, &all);
    // An entry is cut where it is longer than a CTA's share of all of them; into chunks of half a share, so that what the CTAs take adds
    // up more evenly.
    const long long share = (all.a * p.Hkv + 2 * geom.sms - 1) / (2 * geom.sms);
    const int chunk = (int)min(max(share, (long long)kChunkMin), 1ll << 24);
    const auto chunks_of = [&](int tiles) { return tiles >= 2 * chunk ? (tiles + chunk - 1) / chunk : 1; };
    const auto bin_of = [&](int tiles) { return kOrderBins - 1 - min(tiles, kOrderBins - 1); };
    for (int e = threadIdx.x; e < total; e += kPageThreads) {
        const int tiles = (whole(e).kb1 + 1) / 2, n = chunks_of(tiles), per = (tiles + n - 1) / n;
        for (int c = 0; c < n; ++c) atomicAdd(&bins[bin_of(min(per, tiles - c * per))], 1);
    }
    __syncthreads();
    {
        static_assert(kOrderBins == kPageThreads, "");
        const Pair here{bins[threadIdx.x], 0};
        const Pair before = block_scan(here, warp_sums, &all);
        bins[threadIdx.x] = (int)before.a;
    }
    __syncthreads();
    PromptEntry* const entries = plan_entries(p.plan);
    PromptSplit* const splits = plan_splits(p.plan, geom.cap_entries);
    for (int e = threadIdx.x; e < total; e += kPageThreads) {
        PromptEntry x = whole(e);
        const int tiles = (x.kb1 + 1) / 2, n = chunks_of(tiles), per = (tiles + n - 1) / n, last = x.kb1;
        int slot = -1;
        if (n > 1) {
            slot = atomicAdd(&n_slots, n * p.Hkv);
            splits[atomicAdd(&n_splits, 1)] = PromptSplit{x.row0, x.tokens, slot, n};
        }
        for (int c = 0; c < n; ++c) {
            x.kb0 = 2 * c * per;
            x.kb1 = min(2 * (c + 1) * per, last);
            x.slot = n > 1 ? slot + c * p.Hkv : -1;
            entries[atomicAdd(&bins[bin_of(min(per, tiles - c * per))], 1)] = x;
            atomicAdd(&n_entries, 1);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *plan_header(p.plan) = PromptHeader{n_entries, n_splits, n_slots, 0};
}

size_t prompt_plan_bytes(const sd_prompts& p) {
    const PromptGeom g = prompt_geom(p, current_sms());
    return sizeof(PromptHeader) + (size_t)g.cap_entries * sizeof(PromptEntry) + (size_t)g.cap_splits * sizeof(PromptSplit);
}

sd_status launch_prompt_prepare(const sd_prompts& p, int32_t* dev_status, cudaStream_t st) {
    const int smem = 2 * (p.B + 1) * 4;
    if (!allow_dynamic_smem(prompt_prepare_kernel, smem)) return SD_ERR_CUDA;
    return launch_dependent(prompt_prepare_kernel, dim3(1 + (p.N + kSlotRows - 1) / kSlotRows), kPageThreads, smem, 1, st, p,
                            prompt_geom(p, current_sms()), dev_status);
}

// A token's K and V rows of all KV heads (256 bytes a head) into its slot; unit of work = one 16-byte vector of each.
__global__ void __launch_bounds__(256)
append_kernel(sd_prompts p, sd_kv_layer cache, const uint4* k, long long ldk, const uint4* v, long long ldv, int32_t* status) {
    begin_dependent(p.slot, cache.k, cache.v, k, v);
    const int per = p.Hkv * 16;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(i / per), vec = (int)(i - (long long)row * per);
    if (row >= p.N) return;
    const int slot = __ldcg(p.slot + row);
    if (slot < 0) return;
    const int block = slot / kBlock;
    if (block >= cache.num_blocks) { set_status(status, SD_ERR_BOUNDS); return; }
    const size_t at = (((size_t)block * p.Hkv + vec / 16) * kBlock + slot % kBlock) * 16 + vec % 16;
    static_cast<uint4*>(cache.k)[at] = __ldcs(k + row * ldk + vec);
    static_cast<uint4*>(cache.v)[at] = __ldcs(v + row * ldv + vec);
}

sd_status launch_append_kv(const sd_prompts& p, const sd_kv_layer& cache, const void* k, long long ldk, const void* v, long long ldv,
                           int32_t* dev_status, cudaStream_t st) {
    const long long threads = (long long)p.N * p.Hkv * 16;
    return launch_dependent(append_kernel, dim3((unsigned)((threads + 255) / 256)), 256, 0, 1, st, p, cache,
                            static_cast<const uint4*>(k), ldk / 8, static_cast<const uint4*>(v), ldv / 8, dev_status);
}

}  // namespace sdv
