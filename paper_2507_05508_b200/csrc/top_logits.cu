// Messages of top logits: the k largest of every row, in order, and the mass of all others.
//
// One pass over the row.  A block takes it in groups of 64 bytes per thread (more in long rows) and keeps of each group its largest
// logit m and s = sum exp((z - m) / T).  The k-th largest of such maxima is a floor under the row's k-th largest logit, so only the
// groups that reach it, hardly more than k of them, are looked at again, entry by entry: what reaches the floor becomes a
// candidate, the candidates are ranked, and all else is rest.  The rest's mass is summed from what is rest, never as a difference: where
// it is 1e-6 of the row it keeps its digits.
// Rows with more candidates than there is room for (many equal logits) find the k-th largest by four digit counts instead.
// Few long rows are cut into sections, the blocks of a cluster: they agree on a floor, and the first block ranks all candidates.
//
// What bounds it: the pass runs at what the blocks have in flight, and a quarter of a block's time (floor, list, second look, ranking) asks
// for nothing.  Calls: 4096 x 65,536 bf16 117 us, 4.6 TB/s (0.71 of a copy's rate); 1024 x 131,072 fp32 125 us, 4.3 TB/s: the groups' numbers take
// 35 KB of shared memory per row, which leaves four rows per SM; 999 x 50,257 bf16 31 us, 3.3 TB/s: all rows run at once, so what follows
// their passes overlaps with nothing; one row 8.4 us: 1.4 in the pass, the rest a chain of two cluster and five block barriers.
// (Choices below compare GPU times in replayed graphs, which are up to a tenth below a call's.)  Clusters of two blocks for 999 and 1024
// rows: 40 and 140 us.
#include <algorithm>

#include "logits.cuh"

namespace mlmc {
namespace {

namespace cg = cooperative_groups;

struct TopPlan {
    const void* logits;
    int V;
    int64_t N, ld;
    const uint8_t* skip;
    double inv_T;
    float c;            // log2(e) / T
    int k;
    uint32_t* idx;
    float* val;
    int32_t* count;
    float* rest;
    int* status;
    int groups;         // per thread, of the longest section
    int log_span;       // of the trips of a group
    int room;           // candidates and listed groups
};

constexpr int kTopPlaces = 2;
// Threads per SM.  (64 registers and a fourth block of 256 threads: 2048 x 32,000 fp32, k = 512, 167 us, 184 with 72 registers; clusters, which
// run where there is room, are 0.3 us slower with fewer registers.)
template <bool CLUSTER, int THREADS>
constexpr int kResident = !CLUSTER && THREADS == 256 ? 1024 : 896;
constexpr int kGroupsMost = 32;    // per thread, where the span can be chosen so; with two for what is around the trips, 64 at most
// Trips of 64 bytes per thread in a row, from 128-byte lines, so that the groups' second reads are pieces of that size: rows of a block of 64
// threads are still in the caches then, and have a longer head instead (4000 x 1000 fp32: 12 us, 14 us packed; 1024 x 131,072 fp32: 124
// us, 117 us packed).
template <int THREADS>
constexpr bool kPacked = THREADS > 64;
template <int THREADS>
constexpr int kLine = kPacked<THREADS> ? 8 : 1;
constexpr int kTops = 4;           // largest logits that a thread offers for the floor, of every kTops-th group each

template <int THREADS>
struct TopShared {
    ExpSum warp_sum[THREADS / 32];
    uint32_t warp_n[2][THREADS / 32];
    uint32_t warp_floor[THREADS / 32];
    uint32_t hist[256];            // before that: every thread's largest logit
    uint32_t n;                    // candidates
    uint32_t digit, need, total;
    uint64_t best;                 // the row's first entry
    // of a cluster: the first block's are in use
    int received[kRowClusterMost];
    uint32_t floor[kRowClusterMost];
    ExpSum part[kRowClusterMost];
    int bad[kRowClusterMost];
};

// Sum over the block, the same in every thread; calls in a row alternate between the two halves of `shared`.
template <int WARPS>
__device__ __forceinline__ uint32_t block_count(uint32_t x, uint32_t (*shared)[WARPS], int half) {
    x = __reduce_add_sync(0xFFFFFFFFu, x);
    if ((threadIdx.x & 31) == 0) shared[half][threadIdx.x >> 5] = x;
    __syncthreads();
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) r += shared[half][i];
    return r;
}

// The nth largest of n <= 32 numbers in shared memory, the same in every lane.
__device__ __forceinline__ uint32_t nth_largest(const uint32_t* x, int n, int nth) {
    const int lane = threadIdx.x & 31;
    const uint32_t mine = lane < n ? x[lane] : 0;
    int before = 0;
    for (int i = 0; i < n; ++i) before += x[i] > mine || (x[i] == mine && i < lane);
    return __shfl_sync(0xFFFFFFFFu, mine, __ffs((int)__ballot_sync(0xFFFFFFFFu, lane < n && before == nth - 1)) - 1);
}

// What `share` of a warp's numbers reach, 1 <= share <= 16 N: two bits at a time from the top 16, ten bits for each of three counts.
template <int N>
__device__ __forceinline__ uint32_t warp_floor(const uint32_t (&mine)[N], uint32_t share) {
    uint32_t floor = 0;
    for (int shift = 30; shift >= 16; shift -= 2) {
        const uint32_t x1 = floor + (1u << shift), x2 = floor + (2u << shift), x3 = floor + (3u << shift);
        uint32_t reached = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) reached += (mine[i] >= x1 ? 1u : 0u) + (mine[i] >= x2 ? 1u << 10 : 0u) + (mine[i] >= x3 ? 1u << 20 : 0u);
        reached = __reduce_add_sync(0xFFFFFFFFu, reached);
        floor = reached >> 20 >= share ? x3 : (reached >> 10 & 1023u) >= share ? x2 : (reached & 1023u) >= share ? x1 : floor;
    }
    return floor;
}

// How many x the threads before this one have; total: all of them.  `shared` as above.
template <int WARPS>
__device__ __forceinline__ uint32_t block_before(uint32_t x, uint32_t (*shared)[WARPS], int half, uint32_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t upto = x;
#pragma unroll
    for (int i = 1; i < 32; i *= 2) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, upto, i);
        if (lane >= i) upto += y;
    }
    if (lane == 31) shared[half][warp] = upto;
    __syncthreads();
    uint32_t before = upto - x, all = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        if (i < warp) before += shared[half][i];
        all += shared[half][i];
    }
    *total = all;
    return before;
}

// What `share` entries of a section reach, rounded down to the upper half of a key: eight passes over it, two bits in each.
template <typename T, int THREADS>
__device__ __noinline__ uint32_t floor_of_entries(RowSlots<T> r, int s0, int s1, uint32_t share, uint32_t* shared) {
    constexpr int E = ElemTraits<T>::kVec, U = kSlots, WARPS = THREADS / 32;
    uint4 q[U];  // all of a short section
    auto ask = [&](int at) {
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = load_slot<T>(r, at + u * THREADS < s1 ? at + u * THREADS : r.n);
    };
    ask(s0 + (int)threadIdx.x);
    uint32_t floor = 0;
    for (int shift = 30; shift >= 16; shift -= 2) {
        const uint32_t step = 1u << shift;
        const float x[3] = {key_logit(floor + step), key_logit(floor + 2 * step), key_logit(floor + 3 * step)};  // NaN below -inf: not reached
        uint32_t n[3] = {0, 0, 0};
        for (int s = s0; s < s1; s += U * THREADS) {
            if (s1 - s0 > U * THREADS) ask(s + (int)threadIdx.x);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (s + u * THREADS >= s1) break;
                float v[E];
                slot_values<T>(q[u], v);
#pragma unroll
                for (int e = 0; e < E; ++e)
#pragma unroll
                    for (int i = 0; i < 3; ++i) n[i] += v[e] >= x[i];
            }
        }
        uint32_t* mine = shared + (shift >> 1 & 1) * 3 * WARPS;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            n[i] = __reduce_add_sync(0xFFFFFFFFu, n[i]);
            if ((threadIdx.x & 31) == 0) mine[i * WARPS + (threadIdx.x >> 5)] = n[i];
        }
        __syncthreads();
        uint32_t digits = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            uint32_t all = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) all += mine[i * WARPS + w];
            if (all >= share) digits = i + 1;
        }
        floor += digits * step;
    }
    return floor;
}

// Hands f(rank, entry) every one of the n distinct entries.  e has room for the next multiple of 32.
template <int THREADS, typename F>
__device__ __forceinline__ void rank_entries(uint64_t* e, int n, F&& f) {
    if (n <= 128) {  // each is compared with all others, by as many neighbouring threads as there are
        const int threads = n > THREADS / 2 ? 1 : n > THREADS / 4 ? 2 : n > THREADS / 8 ? 4 : 8;
        const int sub = threadIdx.x & (threads - 1);
        for (int first = 0; first < n; first += THREADS) {  // (whole warps)
            const int i = first + threadIdx.x / threads;
            const uint64_t x = i < n ? e[i] : 0;
            int rank = 0;
#pragma unroll 4
            for (int j = sub; j < n; j += threads) rank += e[j] > x;
            for (int step = threads / 2; step; step /= 2) rank += __shfl_xor_sync(0xFFFFFFFFu, rank, step);
            if (i < n && sub == 0) f(rank, x);
        }
        return;
    }
    if (n <= 512) {
        // runs of 32 are sorted, a run per warp; an entry's rank is its place in its run and how many of every other run are larger
        const int lane = threadIdx.x & 31, runs = (n + 31) / 32;
        for (int i = threadIdx.x >> 5; i < runs; i += THREADS / 32) {
            uint64_t x = i * 32 + lane < n ? e[i * 32 + lane] : 0;
#pragma unroll
            for (int size = 2; size <= 32; size *= 2)
#pragma unroll
                for (int step = size / 2; step; step /= 2) {
                    const uint64_t y = __shfl_xor_sync(0xFFFFFFFFu, x, step);
                    const bool larger = ((lane & step) == 0) == ((lane & size) == 0 || size == 32);  // this lane keeps the larger
                    x = (x > y) == larger ? x : y;
                }
            e[i * 32 + lane] = x;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const uint64_t x = e[i];
            int rank = i & 31;
            for (int run = 0; run < runs; ++run) {
                if (run == i / 32) continue;
                const uint64_t* other = e + run * 32;
                int above = 0;  // entries of the run that are larger: 0..32
#pragma unroll
                for (int step = 16; step; step /= 2)
                    if (other[above + step - 1] > x) above += step;
                if (other[above] > x) ++above;
                rank += above;
            }
            f(rank, x);
        }
        return;
    }
    int width = 1024;
    while (width < n) width *= 2;
    for (int i = n + threadIdx.x; i < width; i += THREADS) e[i] = 0;
    for (int size = 2; size <= width; size *= 2)
        for (int step = size / 2; step; step /= 2) {
            __syncthreads();
            for (int i = threadIdx.x; i < width / 2; i += THREADS) {
                const int a = 2 * i - (i & (step - 1)), b = a + step;
                const uint64_t x = e[a], y = e[b];
                if ((x < y) == ((a & size) == 0)) {
                    e[a] = y;
                    e[b] = x;
                }
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) f(i, e[i]);
}

// The section's min(k, entries above -inf) best entries into `cand`, everything else into `rest`; by four counts of key digits from the
// top and a collecting pass in index order.  Returns how many.
template <typename T, int THREADS>
__device__ __noinline__ int select_by_digits(RowSlots<T> r, int s0, int s1, int k, float c, uint64_t* cand, TopShared<THREADS>& sh,
                                             ExpSum& rest) {
    constexpr int E = ElemTraits<T>::kVec;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t prefix = 0, need = (uint32_t)k;
    bool all = false;
    for (int shift = 24; shift >= 0 && !all; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += THREADS) sh.hist[i] = 0;
        __syncthreads();
        // equal digits in a row are added at once: rows that get here are full of them
        uint32_t last = 0, run = 0;
        for (int s = s0 + (int)threadIdx.x; s < s1; s += THREADS) {
            float v[E];
            slot_values<T>(load_slot<T>(r, s), v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t key = logit_key(v[e]);
                if (key < kLowestKey || (shift < 24 && (key >> (shift + 8)) != prefix)) continue;
                const uint32_t digit = key >> shift & 255u;
                if (digit != last && run) {
                    atomicAdd(&sh.hist[last], run);
                    run = 0;
                }
                last = digit;
                ++run;
            }
        }
        if (run) atomicAdd(&sh.hist[last], run);
        __syncthreads();
        if (warp == 0) {  // lane l: digits 8 l .. 8 l + 7
            uint32_t h[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += h[i] = sh.hist[8 * lane + i];
            uint32_t above = sum;  // entries of this lane's digits and the ones above
#pragma unroll
            for (int i = 1; i < 32; i *= 2) {
                const uint32_t x = __shfl_down_sync(0xFFFFFFFFu, above, i);
                if (lane + i < 32) above += x;
            }
            if (lane == 0) sh.total = above;
            above -= sum;
            if (above < need && above + sum >= need) {
                uint32_t left = need - above, digit = 0;
                bool found = false;
#pragma unroll
                for (int i = 7; i >= 0; --i) {
                    if (!found && h[i] >= left) {
                        found = true;
                        digit = 8 * lane + i;
                    }
                    if (!found) left -= h[i];
                }
                sh.digit = digit;
                sh.need = left;
            }
        }
        __syncthreads();
        if (shift == 24 && sh.total <= need) {
            all = true;  // everything above -inf
        } else {
            prefix = prefix << 8 | sh.digit;
            need = sh.need;
        }
    }
    // keys above the threshold, and the first `need` that equal it
    const uint32_t threshold = all ? kLowestKey - 1 : prefix;
    uint32_t ties = all ? 0 : need;  // left to find
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    int half = 0;
    for (int tile = s0; tile < s1; tile += THREADS) {
        const int s = tile + (int)threadIdx.x;
        uint4 one[1] = {load_slot<T>(r, s < s1 ? s : r.n)};
        float v[E];
        slot_values<T>(one[0], v);
        uint32_t mine = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) mine += logit_key(v[e]) == threshold;
        uint32_t before = 0, found = 0;
        if (ties) {
            before = block_before(mine, sh.warp_n, half, &found);
            half ^= 1;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t key = logit_key(v[e]);
            const bool tie = key == threshold;
            if (key > threshold || (tie && before < ties)) {
                cand[atomicAdd(&sh.n, 1u)] = entry_of(key, s * E + e - r.phase);
                drop_element<T>(one[0], e);
                v[e] = -CUDART_INF_F;
            }
            before += tie;
        }
        ties -= min(ties, found);
        float m = -CUDART_INF_F;
#pragma unroll
        for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
        if (m > -CUDART_INF_F) rest.add(m, exp_sum<T, 1>(one, m, c), c);
    }
    __syncthreads();
    return (int)sh.n;
}

// Dynamic shared memory: {m, s} of every group; places of trips, and where they were the candidates, in a cluster what the first block
// receives, the list of groups.
template <int THREADS>
size_t top_smem(int groups, int room, bool cluster) {
    const size_t later = (size_t)room * ((cluster ? 2 : 1) * sizeof(uint64_t) + sizeof(uint32_t)), trips = kTopPlaces > 1 ? kTopPlaces * kPlaceBytes<THREADS> : 0;
    return (size_t)groups * THREADS * sizeof(float2) + (later > trips ? later : trips);
}

template <typename T, bool CLUSTER, int THREADS>
__global__ void __launch_bounds__(THREADS, kResident<CLUSTER, THREADS> / THREADS) top_logits_kernel(const TopPlan p) {
    constexpr int E = ElemTraits<T>::kVec, U = kSlots, WARPS = THREADS / 32, TOPS = kTops;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ TopShared<THREADS> sh;
    float2* group = reinterpret_cast<float2*>(dyn);
    uint64_t* cand = reinterpret_cast<uint64_t*>(group + (size_t)p.groups * THREADS);
    uint64_t* received = cand + (CLUSTER ? p.room : 0);
    uint32_t* list = reinterpret_cast<uint32_t*>(received + p.room);
    float* over = reinterpret_cast<float*>(list);          // when the list is done with: logits of the entries behind the k best, in order
    cg::cluster_group cluster = cg::this_cluster();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int blocks = CLUSTER ? (int)cluster.num_blocks() : 1, part = CLUSTER ? (int)cluster.block_rank() : 0;
    const float c = p.c;
    pdl_enter();
    if (CLUSTER) cluster.barrier_arrive();  // this block runs: its shared memory can be written

    const int64_t row = blockIdx.x / blocks;
    if (p.skip && p.skip[row]) {  // every block of the row
        if (CLUSTER) cluster.barrier_wait();
        if (part == 0 && t == 0) {
            p.count[row] = 0;
            p.rest[row] = -CUDART_INF_F;
        }
        return;
    }
    const Section<T> x = section_of<T, THREADS, kLine<THREADS>>(p.logits, row, p.ld, p.V, part, blocks);
    TripStream<T, THREADS, kTopPlaces, kPacked<THREADS>> stream(cand);
    stream.start(x, x.trips);
    const RowSlots<T>& r = x.r;
    const int s0 = x.head ? 0 : x.s0, s1 = x.s1;  // all its slots
    if (t == 0) sh.n = 0;

    // the pass over the section: groups of trips, one of what lies behind them, one of the head
    float top = -CUDART_INF_F, m_group = -CUDART_INF_F, s_group = 0.0f;
    const int span = 1 << p.log_span, trip_groups = (x.trips + span - 1) >> p.log_span;
    int groups = 0, left = span;
    float tops[TOPS];
#pragma unroll
    for (int i = 0; i < TOPS; ++i) tops[i] = -CUDART_INF_F;
    auto put = [&] {
#pragma unroll
        for (int i = 0; i < TOPS; ++i) tops[i] = fmaxf(tops[i], groups % TOPS == i ? m_group : -CUDART_INF_F);
        group[groups++ * THREADS + t] = make_float2(m_group, s_group);
        top = max_nan(top, m_group);
        m_group = -CUDART_INF_F;
        s_group = 0.0f;
        left = span;
    };
    auto add = [&](const uint4 (&q)[U]) {
        const float m = max_nan(m_group, batch_max<T>(q)), ref = reference(m);
        s_group = s_group * exp2_approx((m_group - ref) * c) + exp_sum<T, U>(q, ref, c);
        m_group = m;
    };
    stream.run(x, [&](int, const uint4* slots) {
        uint4 q[U];
        stream.take(slots, q);
        add(q);
        if (--left == 0) put();
    });
    if (left != span) put();
    const bool head = x.head && warp == 0;
    if (x.rest > 0 || head) {
        uint4 q[U], one[1];
        load_rest<T, THREADS>(x, q);
        one[0] = load_head<T>(x);
        add(q);
        put();
        if (head) {
            float v[E];
            slot_values<T>(one[0], v);
#pragma unroll
            for (int e = 0; e < E; ++e) m_group = max_nan(m_group, v[e]);
            s_group = exp_sum<T, 1>(one, reference(m_group), c);
            put();
        }
    }
    // the i-th slot of a thread's group, r.n: there is none
    auto slot_of = [&](uint32_t id, int i) {
        const int g = (int)(id / THREADS), thread = (int)(id % THREADS), trip = (g << p.log_span) + (i >> 2);
        if (g < trip_groups) return trip < x.trips ? x.s0 + trip * U * THREADS + slot_in_trip<THREADS, kPacked<THREADS>>(thread, i & 3) : r.n;
        if (g == trip_groups + 1) return i == 0 && thread < x.s0 ? thread : r.n;
        const int s = x.s0 + (x.trips * U + i) * THREADS + thread;
        return i < U && s < x.s1 ? s : r.n;
    };
    // The floor, rounded down to the upper half of a key, so that k entries of the row reach it: what a section's share of the threads'
    // largest logits reach, found by one warp, and in a cluster the least of the sections'.  If there are too few threads for that, a warp
    // looks at TOPS logits of each of its own, for its part of the share, and the least of the warps' floors is taken.  The largest k
    // count all groups.
    const uint32_t share = (uint32_t)((p.k + blocks - 1) / blocks), lot = (share + WARPS - 1) / WARPS;
    // A section with few groups for its share looks at its entries (649 x 1244 bf16, k = 64: 17 us, 34 without).
    const bool entries = 2 * (trip_groups * THREADS + min(x.rest, THREADS)) < 3 * (int)share;
    const bool one = !entries && share <= THREADS / 2;
    uint32_t floor = 0;
    if (one) {
        sh.hist[t] = logit_key(top);
    } else if (!entries && lot <= 16 * TOPS) {
        uint32_t mine[TOPS];
#pragma unroll
        for (int i = 0; i < TOPS; ++i) mine[i] = logit_key(tops[i]);
        floor = warp_floor(mine, lot);
        if (lane == 0) sh.warp_floor[warp] = floor;
    }
    bool bad = __syncthreads_or(!(top < CUDART_INF_F));  // NaN or +inf
    if (one) {
        if (warp == 0) {
            uint32_t mine[WARPS];
#pragma unroll
            for (int i = 0; i < WARPS; ++i) mine[i] = sh.hist[i * 32 + lane];
            floor = warp_floor(mine, share);
            if (!CLUSTER && lane == 0) sh.warp_floor[0] = floor;
        }
        if constexpr (!CLUSTER) {
            __syncthreads();
            floor = sh.warp_floor[0];
        }
    } else if (entries) {
        floor = floor_of_entries<T, THREADS>(r, s0, s1, share, sh.hist);
    } else if (lot <= 16 * TOPS) {
        floor = nth_largest(sh.warp_floor, WARPS, (int)((share + lot - 1) / lot));
    } else {
        for (uint32_t bit = 0x80000000u; bit > 0xFFFFu; bit >>= 1) {
            const uint32_t x = floor | bit;
            uint32_t own = 0;
            for (int g = 0; g < groups; ++g) own += logit_key(group[g * THREADS + t].x) >= x;
            if (block_count(own, sh.warp_n, bit & 0x55550000u ? 0 : 1) >= share) floor = x;
        }
    }
    if constexpr (CLUSTER) {
        cluster.barrier_wait();
        if (t < blocks) {  // (the first warp)
            cluster.map_shared_rank(sh.floor, t)[part] = floor;
            cluster.map_shared_rank(sh.bad, t)[part] = bad;
        }
        cluster.sync();
        floor = nth_largest(sh.floor, blocks, (int)((p.k + share - 1) / share));
        bad = __any_sync(0xFFFFFFFFu, lane < blocks && sh.bad[lane % kRowClusterMost] != 0);
    }
    if (bad) {  // every block of the row
        if (part == 0 && t == 0) {
            set_status(p.status, MLMC_ERR_NONFINITE);
            p.count[row] = 0;
            p.rest[row] = -CUDART_INF_F;
        }
        return;
    }
    const float least = key_logit(max(floor, kLowestKey));

    // The groups that reach it, listed in the threads' order, so that every run adds up the rest alike.  What does not reach it is summed
    // next to the floor where it is near, `far` holds what is not.
    uint32_t marks[2] = {0, 0}, total;
    float near = 0.0f;
    ExpSum far = {-CUDART_INF_F, 0.0f};
    constexpr float kNear = -16.0f;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int end = min(groups, 32 * half + 32);
#pragma unroll 4
        for (int g = 32 * half; g < end; ++g) {
            const float2 b = group[g * THREADS + t];
            const float y = (b.x - least) * c;
            if (b.x >= least)
                marks[half] |= 1u << (g & 31);
            else if (y >= kNear)
                near += b.y * exp2_approx(y);
            else if (b.y > 0.0f)
                far.add(b.x, b.y, c);
        }
    }
    uint32_t place = block_before((uint32_t)(__popc(marks[0]) + __popc(marks[1])), sh.warp_n, 1, &total);
#pragma unroll
    for (int half = 0; half < 2; ++half)
        for (; marks[half]; marks[half] &= marks[half] - 1u, ++place)
            if (place < (uint32_t)p.room) list[place] = (uint32_t)((32 * half + __ffs((int)marks[half]) - 1) * THREADS + t);
    __syncthreads();
    const int listed = (int)total, shift = p.log_span + 2;
    static_assert(kSlots == 4, "two bits of a slot's number in its batch");
    if (listed <= p.room) {
        // The listed groups' slots are copied where the groups' numbers were, as many at a time as fit: a long row has left L2, and asking
        // for all at once takes one wait (1024 x 131,072 fp32, k = 128: 37,000 cycles with eight loads per thread at a time).
        uint4* stage = reinterpret_cast<uint4*>(group);
        const int fit = p.groups * THREADS / 2, end = listed << shift;
        for (int base = 0; base < end; base += fit) {
            const int n = min(fit, end - base);
            for (int i = t; i < n; i += THREADS) {
                const int s = slot_of(list[(base + i) >> shift], (base + i) & ((1 << shift) - 1));
                if (whole_slot<T>(r, s))
                    cp_async_16(stage + i, r.first + (int64_t)s * 16);
                else
                    stage[i] = load_slot<T>(r, s);
            }
            cp_async_commit();
            cp_async_wait<0>();
            for (int i = t; i < n; i += THREADS) {  // a thread's own copies
                float v[E], m = -CUDART_INF_F;
                uint32_t in = 0;
                slot_values<T>(stage[i], v);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (v[e] >= least) {
                        in |= 1u << e;
                        v[e] = -CUDART_INF_F;
                    }
                    m = fmaxf(m, v[e]);
                }
                if (in) {
                    const int first = slot_of(list[(base + i) >> shift], (base + i) & ((1 << shift) - 1)) * E - r.phase;
                    uint32_t to = atomicAdd(&sh.n, (uint32_t)__popc(in));
                    for (; in; in &= in - 1u, ++to) {
                        const int e = __ffs((int)in) - 1;
                        const float x = load_logit<T>(stage + i, 0, 0, e);
                        if (to < (uint32_t)p.room) cand[to] = entry_of(logit_key(x), first + e);
                    }
                }
                const bool close = (m - least) * c >= kNear;
                const float ref = close ? least : reference(m);
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) sum += exp2_approx((v[e] - ref) * c);
                if (close)
                    near += sum;
                else if (sum > 0.0f)
                    far.add(m, sum, c);
            }
        }
        __syncthreads();
    }
    ExpSum rest = far;
    if (near > 0.0f) rest.add(least, near, c);
    int found = (int)sh.n;
    if (listed > p.room || found > p.room / blocks) {  // a section sends its share of the room at most
        __syncthreads();
        ExpSum others = {-CUDART_INF_F, 0.0f};
        found = select_by_digits<T, THREADS>(r, s0, s1, p.k, c, cand, sh, others);
        rest = others;
    }
    if constexpr (CLUSTER) {  // the first block gets all candidates, hardly more than k
        rest = warp_exp_sum(rest, c);
        if (lane == 0) sh.warp_sum[warp] = rest;
        const int each = p.room / blocks;
        uint64_t* to = cluster.map_shared_rank(received, 0) + part * each;
        for (int i = t; i < found; i += THREADS) to[i] = cand[i];
        __syncthreads();
        if (warp == 0) {
            rest = warp_exp_sum(lane < WARPS ? sh.warp_sum[lane % WARPS] : ExpSum{-CUDART_INF_F, 0.0f}, c);
            if (lane == 0) {
                cluster.map_shared_rank(sh.part, 0)[part] = rest;
                cluster.map_shared_rank(sh.received, 0)[part] = found;
            }
        }
        cluster.sync();
        if (part != 0) return;
        found = 0;
        for (int q = 0; q < blocks; ++q) {  // side by side
            const int n = sh.received[q];
            if (q % WARPS == warp)
                for (int i = lane; i < n; i += 32) cand[found + i] = received[q * each + i];
            found += n;
        }
        __syncthreads();
        rest = {-CUDART_INF_F, 0.0f};
    }
    const int n = min(found, p.k);
    rank_entries<THREADS>(cand, found, [&](int rank, uint64_t e) {
        if (rank >= p.k) {
            over[rank - p.k] = key_logit(entry_key(e));
        } else {
            if (rank == 0) sh.best = e;
            p.idx[row * p.k + rank] = entry_index(e);
            p.val[row * p.k + rank] = key_logit(entry_key(e));
        }
    });
    __syncthreads();
    for (int i = t; i < found - p.k; i += THREADS) rest.add(over[i], 1.0f, c);
    rest = warp_exp_sum(rest, c);
    if (lane == 0) sh.warp_sum[warp] = rest;
    __syncthreads();
    if (warp == 0) {
        ExpSum sum = lane < WARPS ? sh.warp_sum[lane % WARPS] : ExpSum{-CUDART_INF_F, 0.0f};
        if constexpr (CLUSTER) {
            if (lane >= WARPS && lane < WARPS + blocks) sum = sh.part[lane - WARPS];
        }
        sum = warp_exp_sum(sum, c);
        if (lane != 0) return;
        p.count[row] = n;
        const Two ln = log_of(sum.s);
        p.rest[row] = n && sum.s > 0.0f ? (float)(((double)sum.m - (double)key_logit(entry_key(sh.best))) * p.inv_T + (double)ln.hi + (double)ln.lo)
                                         : -CUDART_INF_F;
    }
}

constexpr int kTopSmemMost = 200 * 1024;

template <typename T, int THREADS>
void launch_threads(Workspace& ws, TopPlan& p, cudaStream_t s) {
    // As many blocks per row, a power of two, as are resident at a time for all rows, while each has a batch per thread (64 x 131,072 fp32,
    // 256 threads: 20 us with one, 14 with four, 17 with six, 16 with eight).  A section may send k entries, and all together have to fit.
    // Rows of 1 MB and more whose k is large have sections of 2^17 logits at most, whatever their number: the second look at k groups of
    // several trips is long (700 x 262,144 fp32, k = 256: 192 us so, 228 with a block per row; 160 x 2^20 bf16, k = 500: 116 and 150).  For
    // others it is not worth a cluster's barriers (700 x 300,000 bf16, k = 700: 262 us with two blocks, 187 with one; 400 x 262,144 fp32,
    // k = 128: 107 and 91; 2048 x 160,000 bf16, k = 100: 169 and 149; but 300 x 2^20 fp32, k = 20: 233 with eight, 243 with one).
    int most = 1;
    while (most < kRowClusterMost && 2 * most * p.k <= 2048) most *= 2;
    const bool large = p.V * (int64_t)sizeof(T) >= 1 << 20 && p.k >= 256;
    size_t smem;
    int blocks = most;
    for (;; blocks /= 2) {
        const int64_t needed = (int64_t)p.k * blocks;
        p.room = needed <= (blocks > 1 ? 128 : 64) ? 512 : needed <= (blocks > 1 ? 512 : 256) ? 1024 : 2048;
        const int trips = (int)(section_slots<T, kLine<THREADS>>(p.V, blocks) / (kSlots * THREADS));
        // groups of one trip as far as kGroupsMost of them go; about twice as many where all of them are counted for the floor
        const int most_groups = (p.k + blocks - 1) / blocks > THREADS * kTops / 2 ? 62 : kGroupsMost;
        p.log_span = 0;
        while (trips > most_groups << p.log_span) ++p.log_span;
        p.groups = ((trips + (1 << p.log_span) - 1) >> p.log_span) + 2;
        smem = top_smem<THREADS>(p.groups, p.room, blocks > 1);
        const int per_sm = std::min<int>(kResident<true, THREADS> / THREADS, (int)(227 * 1024 / (smem + sizeof(TopShared<THREADS>) + 1024)));
        if (blocks == 1 || (large && p.V > (int64_t)(blocks / 2) << 17)) break;
        if (p.N * blocks <= (int64_t)per_sm * ws.sm_count && p.V > (int64_t)(blocks / 2) * THREADS * kBatch<T>) break;
    }
    const unsigned grid = (unsigned)(p.N * blocks);
    if (blocks > 1)
        launch_kernel_cluster(ws, K_TOP_LOGITS, blocks, top_logits_kernel<T, true, THREADS>, dim3(grid), THREADS, smem, s, p);
    else
        launch_kernel(ws, K_TOP_LOGITS, top_logits_kernel<T, false, THREADS>, dim3(grid), THREADS, smem, s, p);
}

// Short rows take blocks of 64 threads (4000 x 1000 fp32: 15 us, 22 us with 128), unless k is large (335 x 3877 bf16, k = 256: 34 us, 21
// with 128); longer ones of 128, whose pauses between two passes
// overlap (600 x 50,257 fp32: 32 us, 53 with 64, 39 with 256); few rows, which leave room, and large k, whose floor takes more
// groups, of 256 (64 x 131,072 fp32: 18 us with 128, 16 with 256; 2048 x 32,000 fp32, k = 512: 182 and 167 us).
template <typename T>
void launch_typed(Workspace& ws, TopPlan& p, cudaStream_t s) {
    if (p.V * (int64_t)sizeof(T) <= 16 * 1024 && p.k <= 64)
        launch_threads<T, 64>(ws, p, s);
    else if (p.N >= 2 * ws.sm_count && p.k <= 256)
        launch_threads<T, 128>(ws, p, s);
    else
        launch_threads<T, 256>(ws, p, s);
}

template <typename K>
bool allow_smem(K kernel) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kTopSmemMost) == cudaSuccess &&
           cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) == cudaSuccess;
}

template <typename T, int THREADS>
bool allow_threads() {
    return allow_smem(top_logits_kernel<T, false, THREADS>) && allow_smem(top_logits_kernel<T, true, THREADS>);
}
template <typename T>
bool allow_typed() {
    return allow_threads<T, 64>() && allow_threads<T, 128>() && allow_threads<T, 256>();
}

}  // namespace

int configure_top_logits() { return allow_typed<float>() && allow_typed<bf16_t>() ? MLMC_OK : MLMC_ERR_CUDA; }

void launch_top_logits(Workspace& ws, const void* logits, int dtype, int64_t V, int64_t N, int64_t ld, const uint8_t* skip, double T,
                       const mlmc_logit_msgs& out, cudaStream_t s) {
    TopPlan p = {};
    p.logits = logits;
    p.V = (int)V;
    p.N = N;
    p.ld = ld;
    p.skip = skip;
    p.inv_T = 1.0 / T;
    p.c = (float)(1.4426950408889634 / T);
    p.k = out.k;
    p.idx = out.idx;
    p.val = out.val;
    p.count = out.count;
    p.rest = out.rest;
    p.status = ws.status;
    if (dtype == MLMC_BF16)
        launch_typed<bf16_t>(ws, p, s);
    else
        launch_typed<float>(ws, p, s);
}

}  // namespace mlmc
