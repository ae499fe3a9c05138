// Block tables, slot maps and the cache's new rows: what stands between a request's length and the attention over its cache.
//
// Lengths are known on the device first (acceptance leaves new_len there), so tables that are made on the host cost a round trip per
// step.  Both calls on lengths are scans over the requests; every CTA repeats the scan (8192 requests: 32 KB of lengths through L2), so
// that nothing has to be handed from one to another.  They are bound by latencies: launches, one or two trips to L2, and the scans.
#include "prompt_plan.cuh"
#include "sm100.cuh"

namespace sdv {
using namespace sm100;

namespace {
// Threads of a CTA: a pass of the scans is shorter with few, and with many there are fewer passes.  Us, 256 threads and 1024 (blocks: in a cluster
// of eight), blocks / slots and plan: 64 requests of 60 new tokens 3.4 and 4.2 / 6.1 and 7.4, 256 of one 3.6 and 4.5 / 6.4 and 7.7, 256 of 60 (15360 rows) 3.8
// and 4.7 / 7.8 and 6.8, 400 of 30 4.5 and 4.5 / 8.7 and 6.5, 2000 of 50 15.4 and 6.7 / 39 and 16.5.
constexpr int kFewThreads = 256, kManyThreads = 1024;
constexpr int kOrderBins = 1024;
constexpr int kNotHeld = -1;                   // in place of the blocks of a request whose numbers are out of range

// Sums of whole numbers from 0 up stop at 2^29, which no count of rows or blocks reaches: what is behind that does not fit anyway.
constexpr int kMost = 1 << 29;
__device__ __forceinline__ int add_up(int a, int b) { return min(a + b, kMost); }
__device__ __forceinline__ long long add_up(long long a, long long b) { return a + b; }

// v: K values of this thread -> their sums over the threads in front of it; total: over all.  sums: room for two scans of K x 32 numbers; scans
// that follow one another take the two in turn (buf), so that one barrier is enough.
template <int THREADS, int K, typename T>
__device__ __forceinline__ void block_scan(T (&v)[K], T (&total)[K], T* sums, int& buf) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T* const here = sums + buf * K * 32;
    buf ^= 1;
    const auto scan = [&](T (&x)[K]) {
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const T below = __shfl_up_sync(0xffffffffu, x[k], d);
                if (lane >= d) x[k] = add_up(x[k], below);
            }
        }
    };
    scan(v);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (lane == 31) here[k * 32 + warp] = v[k];
    __syncthreads();
    T w[K];
#pragma unroll
    for (int k = 0; k < K; ++k) w[k] = lane < THREADS / 32 ? here[k * 32 + lane] : T(0);
    scan(w);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const T before = __shfl_sync(0xffffffffu, w[k], max(warp - 1, 0)), below = __shfl_up_sync(0xffffffffu, v[k], 1);
        total[k] = __shfl_sync(0xffffffffu, w[k], 31);
        v[k] = add_up(warp > 0 ? before : T(0), lane > 0 ? below : T(0));
    }
}

// the last of n ascending numbers that is at most x (the first one is)
__device__ __forceinline__ int last_at_most(const int* a, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (a[m] <= x) lo = m; else hi = m;
    }
    return lo;
}
// The same for the 32 lanes of a warp, whose x follow one another: thirty-two numbers are looked at together.  (A search per lane is eleven steps for 2000
// numbers, each with bank conflicts: searching and writing 6000 row tiles of 2000 requests took 15200 cycles, 13200 so.)
__device__ __forceinline__ int last_at_most_warp(const int* a, int n, int x) {
    const int lane = threadIdx.x & 31, x0 = x - lane;
    int lo = 0;
    for (int left = n; left > 1;) {                        // of lane 0
        const int step = (left + 31) / 32, at = lane * step;
        const int k = __popc(__ballot_sync(0xffffffffu, at < left && a[lo + min(at, left - 1)] <= x0)) - 1;    // (a[lo] is at most x0)
        lo += k * step;
        left = min(step, left - k * step);
    }
    int mine = lo;
    for (int base = lo + 1;; base += 32) {                 // and how many of those behind it each lane passes
        const int next = base + lane < n ? a[base + lane] : 0x7fffffff;
        int c = 0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
            if (__shfl_sync(0xffffffffu, next, c + d - 1) <= x) c += d;
        if (__shfl_sync(0xffffffffu, next, c) <= x) ++c;
        mine += c;
        if (!__any_sync(0xffffffffu, c == 32)) return mine;
    }
}
}  // namespace

// One cluster.  Blocks that come free stand in front of the stack, in order of the requests; the t-th block that is taken is the t-th of
// this list.  So giving back what was taken leaves the stack as it was.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
assign_blocks_kernel(sd_block_pool pool, int B, int W, int32_t* table, int32_t* n_blocks, const int32_t* len, const int32_t* n_new,
                     int32_t* granted, int32_t* status) {
    extern __shared__ int page_smem[];
    int *const grow_at = page_smem, *const free_at = page_smem + B + 1, *const held_of = page_smem + 2 * B + 2;      // sums in front [B + 1]; blocks held [B]
    __shared__ int sums[2 * 2 * 32];
    // (Tables are read through the read-only path by the attention calls, so no kernel behind this one begins before it has ended.)
    griddep_wait();
    settle(pool.free_blocks); settle(pool.n_free); settle(table); settle(n_blocks); settle(len); settle(n_new);
    const int cta = blockIdx.x, ctas = gridDim.x;
    const bool first = cta == 0;
    int n_free = __ldcg(pool.n_free), buf = 0;
    int so_far[2] = {0, 0};
    for (int b0 = 0; b0 < B; b0 += THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int move[2] = {0, 0}, all[2];                      // blocks to take and to give back
        int held = 0;
        if (b < B) {
            held = __ldcg(n_blocks + b);
            const int l = __ldcg(len + b), n = __ldcg(n_new + b);
            const long long want = ((long long)l + n + kBlock - 1) / kBlock;
            int bad = 0;
            if (l < 0 || n < 0) bad = SD_ERR_INVALID_ARG;
            else if (held < 0 || held > W || want > W) bad = SD_ERR_BOUNDS;
            if (bad) {                                                          // (and the request keeps what it has)
                if (first) set_status(status, bad);
                held = kNotHeld;
            }
            else if (want > held) move[0] = (int)want - held;
            else move[1] = held - (int)want;
        }
        block_scan<THREADS>(move, all, sums, buf);
        if (b < B) {
            grow_at[b] = add_up(so_far[0], move[0]);
            free_at[b] = add_up(so_far[1], move[1]);
            held_of[b] = held;
        }
        so_far[0] = add_up(so_far[0], all[0]);
        so_far[1] = add_up(so_far[1], all[1]);
    }
    if (threadIdx.x == 0) { grow_at[B] = so_far[0]; free_at[B] = so_far[1]; }
    if (n_free < 0 || n_free > pool.num_blocks) {
        if (first && threadIdx.x == 0) set_status(status, SD_ERR_BOUNDS);
        n_free = 0;
    }
    const int come_free = so_far[1];
    __syncthreads();
    // what is taken: the needs of the requests in front of the first that goes short
    const int taken = grow_at[last_at_most(grow_at, B + 1, min(n_free + come_free, kMost - 1))];
    if (ctas > 1) cluster_arrive_release();                // everybody has read the counts

    const auto released = [&](int t) {
        const int b = last_at_most(free_at, B, t), want = held_of[b] - (free_at[b + 1] - free_at[b]);
        return __ldcg(table + (size_t)b * W + want + (t - free_at[b]));
    };
    const int tid = cta * THREADS + (int)threadIdx.x, threads = ctas * THREADS;
    for (int t = tid; t < taken; t += threads) {
        const int b = last_at_most(grow_at, B, t);
        const int block = t < come_free ? released(t) : __ldcg(pool.free_blocks + n_free - 1 - (t - come_free));
        table[(size_t)b * W + held_of[b] + (t - grow_at[b])] = block;
        if (block < 0 || block >= pool.num_blocks) set_status(status, SD_ERR_BOUNDS);
    }
    for (int t = taken + tid; t < come_free; t += threads) {
        const int at = n_free + come_free - 1 - t;
        const int block = released(t);
        if (at < pool.num_blocks) pool.free_blocks[at] = block;
        if (at >= pool.num_blocks || block < 0 || block >= pool.num_blocks) set_status(status, SD_ERR_BOUNDS);     // (more than the pool has: given back twice)
    }
    if (ctas > 1) cluster_wait_acquire();
    for (int b = tid; b < B; b += threads) {
        const int grow = grow_at[b + 1] - grow_at[b], shrink = free_at[b + 1] - free_at[b];
        const bool ok = held_of[b] != kNotHeld && (grow_at[b + 1] <= taken || grow == 0);
        if (grow && ok) n_blocks[b] = held_of[b] + grow;
        if (shrink) n_blocks[b] = held_of[b] - shrink;
        if (granted) granted[b] = ok ? 1 : 0;
    }
    if (tid == 0) *pool.n_free = min(n_free + come_free - taken, pool.num_blocks);
}

sd_status launch_assign_blocks(const sd_block_pool& pool, int B, int W, int32_t* table, int32_t* n_blocks, const int32_t* len,
                               const int32_t* n_new, int32_t* granted, int32_t* dev_status, cudaStream_t st) {
    const int smem = (3 * B + 2) * 4;
    if (B <= kFewThreads)
        return launch_dependent(assign_blocks_kernel<kFewThreads>, dim3(1), kFewThreads, smem, 1, st, pool, B, W, table, n_blocks, len, n_new,
                                granted, dev_status);
    if (!allow_dynamic_smem(assign_blocks_kernel<kManyThreads>, smem)) return SD_ERR_CUDA;
    return launch_dependent(assign_blocks_kernel<kManyThreads>, dim3(8), kManyThreads, smem, 8, st, pool, B, W, table, n_blocks, len, n_new,
                            granted, dev_status);
}

// First rows of the requests and the attention's work (the first CTA); slot and position of each packed row (the others, `rows` rows each).
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
prompt_prepare_kernel(sd_prompts p, PromptGeom geom, int rows, int32_t* status) {
    extern __shared__ int page_smem[];
    int* const start = page_smem;              // [B + 1]
    int* const len_of = page_smem + p.B + 1;   // [B] cached tokens; ~cached tokens of a request that is left out
    int* const first_entry = len_of + p.B;     // [B + 1] (the first CTA)
    __shared__ int sums[2 * 32];
    __shared__ long long line_sums[2 * 32];
    __shared__ int bins[kOrderBins];
    __shared__ int n_splits, longest_smem;
    begin_dependent(p.block_table, p.n_blocks, p.len, p.n_new, p.start, p.slot, p.position, p.plan);
    const int B = p.B, W = p.max_blocks_per_seq;
    const bool planner = blockIdx.x == 0;
    int buf = 0, so_far = 0, entries = 0;
    if (planner) {
        for (int i = threadIdx.x; i < kOrderBins; i += THREADS) bins[i] = 0;
        if (threadIdx.x == 0) { n_splits = longest_smem = 0; }
    }
    for (int b0 = 0; b0 < B; b0 += THREADS) {
        const int b = b0 + (int)threadIdx.x;
        RequestSpan q{0, 0, false};
        if (b < B) {
            q = request_span(p, b, __ldcg(p.n_new + b));
            if ((q.n < 0 || q.len < 0) && planner) set_status(status, SD_ERR_INVALID_ARG);
            if (q.n > 0 && !q.covered && !p.n_blocks && q.len >= 0 && planner) set_status(status, SD_ERR_BOUNDS);
        }
        const int n = min(max(q.n, 0), kMost);
        int at[1] = {n}, all[1];
        block_scan<THREADS>(at, all, sums, buf);
        at[0] = add_up(so_far, at[0]);
        so_far = add_up(so_far, all[0]);
        // (rows behind the packed ones belong to nobody, and a request that has some there is left out)
        const bool there = q.covered && add_up(at[0], n) <= p.N;
        if (b < B) {
            start[b] = min(at[0], p.N);
            len_of[b] = there ? q.len : ~max(q.len, 0);
        }
        if (planner) {
            at[0] = there ? (n + geom.tokens - 1) / geom.tokens : 0;
            block_scan<THREADS>(at, all, sums, buf);
            if (b < B) first_entry[b] = entries + at[0];
            entries += all[0];
        }
    }
    if (threadIdx.x == 0) {
        start[B] = min(so_far, p.N);
        if (planner) first_entry[B] = entries;
        if (planner && so_far > p.N) set_status(status, SD_ERR_BOUNDS);
    }
    __syncthreads();
    if (!planner) {
        const int total = start[B];
        const int r0 = ((int)blockIdx.x - 1) * rows, r1 = min(r0 + rows, p.N);
        int b = 0, next = 0;                   // the request of the last row, and the next one's first
        for (int r = r0 + (int)threadIdx.x; r < r1; r += THREADS) {
            int slot = -1, position = 0;
            if (r < total) {
                if (r >= next) {
                    b = last_at_most(start, B, r);
                    next = start[b + 1];
                }
                const int len = len_of[b];
                position = (len < 0 ? ~len : len) + r - start[b];
                if (len >= 0) {
                    const int block = __ldcg(p.block_table + (size_t)b * W + position / kBlock);
                    if (block >= 0 && block < p.num_blocks) slot = block * kBlock + position % kBlock;
                    else set_status(status, SD_ERR_BOUNDS);
                }
            }
            p.slot[r] = slot;
            p.position[r] = position;
        }
        return;
    }
    // ------------------------------------------------------------ the attention's work
    for (int b = threadIdx.x; b <= B; b += THREADS) p.start[b] = start[b];
    const int Hkv = p.Hkv;
    PromptEntry* const list = plan_entries(p.plan, geom.sms);
    PromptStart* const starts = plan_starts(p.plan);
    PromptSplit* const splits = plan_splits(p.plan, geom.sms);
    const auto entry_of = [&](int b, int e) {
        PromptEntry x;
        x.b = b;
        const int len = len_of[x.b], n = start[x.b + 1] - start[x.b], t0 = (e - first_entry[x.b]) * geom.tokens;
        x.row0 = start[x.b] + t0;
        x.pos0 = len + t0;
        x.tokens = min(geom.tokens, n - t0);
        x.blocks = (x.pos0 + x.tokens + kBlock - 1) / kBlock;
        x.end = len + n;
        x.unused0 = x.unused1 = 0;
        return x;
    };
    const auto entry = [&](int e) { return entry_of(last_at_most(first_entry, B, e), e); };
    // All entries are made once; the first lengths of each thread stay in shared memory.  (In registers the loops below have to be written out, and one
    // CTA's cold code is slower than its loads: a request 6.3 us, 5.7 so; 2000 of 50 tokens 15.2, 16.5 so.)
    constexpr int kHeld = 8;
    __shared__ int held[kHeld * THREADS];
    const auto for_own = [&](auto&& use) {     // use(e, key tiles): for all threads together, -1 where there is no entry
#pragma unroll 1
        for (int e0 = 0; e0 < entries; e0 += THREADS) {
            const int e = e0 + (int)threadIdx.x;
            use(e, e >= entries ? -1 : e < kHeld * THREADS ? held[e] : (list[e].blocks + 1) / 2);
        }
    };
    long long cost[1] = {0}, all_cost[1];
    int longest = 0;
    const auto make = [&](int e) {             // (whole warps)
        if (e - (int)(threadIdx.x & 31) >= entries) return -1;
        const int b = last_at_most_warp(first_entry, B, e);
        if (e >= entries) return -1;
        const PromptEntry x = entry_of(b, e);
        list[e] = x;
        const int tiles = (x.blocks + 1) / 2;
        longest = max(longest, tiles);
        cost[0] += tiles + kEntryTiles;
        return tiles;
    };
#pragma unroll 1
    for (int e0 = 0; e0 < entries; e0 += THREADS) {
        const int e = e0 + (int)threadIdx.x, tiles = make(e);
        if (e < kHeld * THREADS) held[e] = tiles;
    }
    longest = __reduce_max_sync(0xffffffffu, longest);
    if ((threadIdx.x & 31) == 0 && longest) atomicMax(&longest_smem, longest);
    buf = 0;
    block_scan<THREADS>(cost, all_cost, line_sums, buf);       // (its barrier is behind the atomics)
    const long long line = all_cost[0] * Hkv, part = max((line + geom.sms - 1) / geom.sms, (long long)kPartMin);
    if (part >= (long long)kDealFrom * (longest_smem + kEntryTiles)) {
        // ---------------------------------------- dealt out: sorted by counting.  (A warp of one length counts as one.)
        const auto put = [&](int tiles) {                                      // the place that each lane's entry gets in its bin
            const int bin = tiles < 0 ? -1 : kOrderBins - 1 - min(tiles, kOrderBins - 1), lane = threadIdx.x & 31;
            int alike = 0, first = 0;
            __match_all_sync(0xffffffffu, bin, &alike);
            if (!alike) return bin < 0 ? 0 : atomicAdd(&bins[bin], 1);
            if (lane == 0 && bin >= 0) first = atomicAdd(&bins[bin], 32);
            return __shfl_sync(0xffffffffu, first, 0) + lane;
        };
        for_own([&](int, int tiles) { put(tiles); });
        __syncthreads();
        constexpr int kOwn = kOrderBins / THREADS;                             // bins of a thread
        int own[1] = {0}, all[1];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) own[0] += bins[threadIdx.x * kOwn + i];
        buf = 0;
        block_scan<THREADS>(own, all, sums, buf);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int n = bins[threadIdx.x * kOwn + i];
            bins[threadIdx.x * kOwn + i] = own[0];
            own[0] += n;
        }
        __syncthreads();
        int* const order = plan_order(list, geom.cap);
        for_own([&](int e, int tiles) {
            const int at = put(tiles);
            if (tiles >= 0) order[at] = e;
        });
        __syncthreads();
        // every CTA's first piece, so that it need not look for it
        for (int c = threadIdx.x; c < geom.sms && c < (long long)entries * Hkv; c += THREADS) starts[c] = PromptStart{c, c % Hkv, 0, 0, list[order[c / Hkv]]};
        if (threadIdx.x == 0) *plan_header(p.plan) = PromptHeader{0, entries, plan_stamp(p, geom), 0};
        return;
    }
    // ------------------------------------------------ in parts
    // where part c begins, given the entry that its cut lies in and where that begins in the line
    const auto cut_at = [&](long long c, int e, int tiles, long long from) {
        const int one = tiles + kEntryTiles;
        const long long off = min(c * part - from, (long long)Hkv * one);
        int h = off < kMost ? (int)off / one : (int)(off / one), tile = max((int)(off - (long long)h * one) - kEntryTiles, 0);
        // (a chunk of a few tiles is not worth joining, unless the parts are not much longer)
        if (part > 32 * kSnap && tile <= kSnap) tile = 0;
        else if (part > 32 * kSnap && tile >= tiles - kSnap) { tile = 0; ++h; }
        if (h == Hkv) { h = 0; ++e; }
        starts[c] = PromptStart{e, h, tile, 0, entry(min(e, entries - 1))};
    };
    const bool few = entries <= kOrderBins && line < kMost;                    // (then there may be many cuts to an entry: a thread for each of them)
    long long at = 0;
    for_own([&](int e, int tiles) {
        const long long one = tiles < 0 ? 0 : tiles + kEntryTiles;             // of one head
        long long before[1] = {one}, all[1];
        block_scan<THREADS>(before, all, line_sums, buf);
        const long long from = at + before[0];
        if (few && tiles >= 0) bins[e] = (int)from;
        if (!few && tiles >= 0)
            for (long long c = (from * Hkv + part - 1) / part; c * part < (from + one) * Hkv; ++c) cut_at(c, e, tiles, from * Hkv);
        at += all[0];
    });
    __syncthreads();
    if (few)
        for (int c = threadIdx.x; c * part < line; c += THREADS) {
            const int e = last_at_most(bins, entries, (int)((unsigned)(c * (int)part) / (unsigned)Hkv));
            cut_at(c, e, (list[e].blocks + 1) / 2, (long long)bins[e] * Hkv);
        }
    const int used = (int)((line + part - 1) / part);
    for (int c = used + (int)threadIdx.x; c <= geom.sms; c += THREADS) starts[c] = PromptStart{entries, 0, 0, 0, PromptEntry{0, 0, 0, 0, 0, 0, 0, 0}};
    __syncthreads();
    // what was cut: found at its first cut
    for (int c = 1 + (int)threadIdx.x; c < used; c += THREADS) {
        const PromptStart s = starts[c];
        if (s.tile == 0) continue;
        const auto through = [&](int d) { return starts[d].e == s.e && starts[d].h == s.h && starts[d].tile > 0; };
        if (through(c - 1)) continue;
        int chunks = 2;
        while (c + chunks - 1 < used && through(c + chunks - 1)) ++chunks;
        // the first chunk is the last piece of CTA c - 1, and its first one too if its part begins with the entry
        const bool only = starts[c - 1].e == s.e && starts[c - 1].h == s.h;
        splits[atomicAdd(&n_splits, 1)] = PromptSplit{s.entry.row0, s.entry.tokens, s.h, 2 * (c - 1) + (only ? 0 : 1), c - 1, chunks, 0, 0};
    }
    __syncthreads();
    if (threadIdx.x == 0) *plan_header(p.plan) = PromptHeader{n_splits, 0, plan_stamp(p, geom), 0};
}

size_t prompt_plan_bytes(const sd_prompts& p) {
    const PromptGeom g = prompt_geom(p, current_sms());
    return sizeof(PromptHeader) + (g.sms + 1) * sizeof(PromptStart) + g.sms * sizeof(PromptSplit) + (size_t)g.cap * (sizeof(PromptEntry) + sizeof(int));
}

template <int THREADS>
static sd_status launch_prepare(const sd_prompts& p, int32_t* dev_status, cudaStream_t st) {
    const int smem = (3 * p.B + 2) * 4;
    if (!allow_dynamic_smem(prompt_prepare_kernel<THREADS>, smem)) return SD_ERR_CUDA;
    const PromptGeom geom = prompt_geom(p, current_sms());
    // (one row a thread until the CTAs fill the GPU: every CTA repeats the scan over the requests)
    const int others = geom.sms > 1 ? geom.sms - 1 : 1;
    const int rows = ((p.N + others - 1) / others + THREADS - 1) / THREADS * THREADS;
    const int ctas = 1 + (p.N > 0 ? (p.N + rows - 1) / rows : 0);
    return launch_dependent(prompt_prepare_kernel<THREADS>, dim3(ctas), THREADS, smem, 1, st, p, geom, rows, dev_status);
}
sd_status launch_prompt_prepare(const sd_prompts& p, int32_t* dev_status, cudaStream_t st) {
    return p.B <= kFewThreads && p.N <= 32 * kFewThreads ? launch_prepare<kFewThreads>(p, dev_status, st) : launch_prepare<kManyThreads>(p, dev_status, st);
}

// A token's K and V rows of all KV heads (256 bytes a head) into its slot, a 16-byte vector of each per thread.  Bound by HBM: 47195 rows of four
// heads 31.1 us, 6.2 TB/s (four vectors of each per thread, their loads together: 31.5, and 16 rows 3.3 instead of 2.1).
__global__ void __launch_bounds__(256)
append_kernel(sd_prompts p, sd_kv_layer cache, const uint4* k, long long ldk, const uint4* v, long long ldv, int32_t* status) {
    begin_dependent(p.slot, cache.k, cache.v, k, v);
    const unsigned per = (unsigned)p.Hkv * 16u;
    const unsigned long long units = (unsigned long long)p.N * per, i = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= units) return;
    const unsigned row = units < 0xffffffffull ? (unsigned)i / per : (unsigned)(i / per), vec = (unsigned)(i - (unsigned long long)row * per);
    const int slot = __ldcg(p.slot + row);
    const uint4 kx = __ldcs(k + row * ldk + vec), vx = __ldcs(v + row * ldv + vec);                // (without waiting for the slot)
    if (slot < 0) return;
    const int block = slot / kBlock;
    if (block >= cache.num_blocks) { set_status(status, SD_ERR_BOUNDS); return; }
    const size_t at = (((size_t)block * p.Hkv + vec / 16) * kBlock + slot % kBlock) * 16 + vec % 16;
    static_cast<uint4*>(cache.k)[at] = kx;
    static_cast<uint4*>(cache.v)[at] = vx;
}

sd_status launch_append_kv(const sd_prompts& p, const sd_kv_layer& cache, const void* k, long long ldk, const void* v, long long ldv,
                           int32_t* dev_status, cudaStream_t st) {
    const long long units = (long long)p.N * p.Hkv * 16;
    return launch_dependent(append_kernel, dim3((unsigned)((units + 255) / 256)), 256, 0, 1, st, p, cache, static_cast<const uint4*>(k), ldk / 8,
                            static_cast<const uint4*>(v), ldv / 8, dev_status);
}

}  // namespace sdv
