// Distillation from messages of top logits: the loss of every row, its gradient, both in one call.
//
//   loss = T^2 sum_b q_b ln(q_b / p_b)     buckets b: the message's indices S and, if asked for, all others as one (r)
//   dz_i = w T (p_i - q_i), i in S;        w T p_i (1 - q_r / p_r) for the others (w T p_i without their bucket)
//
// The others' largest logit m_r and s_r = sum exp((z_j - m_r) / T) come from one pass that leaves out S by a bit per logit, so that
// p_r keeps its digits however small it is.  An entry outside S then is exp((z_i - m_r) / T) times one factor of the row; the pass that
// writes the gradient gives every entry that, and the entries of S are written over it after a barrier.  Between the two passes there is
// nothing but the row's sums: rows lie in L2 for the second, or in shared memory.
//
// What bounds it (calls): loss of 1000 x 131,072 fp32 96 us, 5.5 TB/s (0.85 of a copy's rate), of 4096 x 32,000 bf16 59 us, 4.4 TB/s: 7 instructions
// for 32 logits, issue 54 % busy, and a row's beginning and end (message, sums, loss) around 64 KB.  Loss and gradient of 2048 x 131,072 bf16
// 253 us, 4.3 TB/s: half of the second reads miss L2; of 1000 x 131,072 fp32 217 us, 4.8 TB/s: clusters wait for all of a row before they
// write any of it.  The gradient by itself, 4096 x 32,000 bf16: 88 us, 6.0 TB/s.  16 rows 6 us, 4.9 of them on the GPU: a chain of
// dependent loads (count, index, logit), barriers, the loss.  (Choices below compare GPU times in replayed graphs, up to a tenth below a call's.)
#include <algorithm>

#include "logits.cuh"

namespace mlmc {
namespace {

namespace cg = cooperative_groups;

// Logits, and so differences of them, may be 3e38: what is computed from differences is in units of 2^16.
constexpr float kUnit = 0x1.0p16f, kPerUnit = 0x1.0p-16f;

struct DistillPlan {
    const void* logits;
    int V;
    int64_t N, ld;
    const uint32_t* idx;
    const float* val;
    const int32_t* count;
    const float* rest;
    int k;
    int use_rest;
    float T, T2;        // the temperature, and its square
    float c;            // log2(e) / T
    Two by_T;           // 1 / T, of the temperature that the exponentials have: c rounded
    const float* weight;
    float* loss;
    float* stat;
    void* grad;
    int64_t ldg;
    int* status;
    int batches;        // per thread, of the longest section
    uint32_t* counter;  // of rows handed out
};

// What the gradient of a row needs.
struct RowStat {
    float m_r, others;  // entries outside S: others exp((z - m_r) / T)
    float m, inv_p;     // p_i = inv_p exp((z - m) / T)
    float t_max, inv_q; // q_i = inv_q exp((t - t_max) / T)
    float pad[2];
};

// An entry of the message: its index, the teacher's logit, the student's.
struct Sent {
    int j;
    float t, z;
};

// What one block of a row finds out.
struct RowPart {
    float m;            // the others' largest logit and sum
    int wrong;          // 1: the message is not one, 2: a number that is not finite
    float s;
    float u, p;         // of the message's entries: sum exp((t - t_max) / T), sum exp((z - z_max) / T)
};

template <int THREADS>
struct DistillShared {
    RowPart part[2][kRowClusterMost];
    ExpSum warp_sum[THREADS / 32];
    float sums[2][THREADS / 32];
    float tops[2][THREADS / 32];
    int wrong, broken;
    int64_t rows[2];    // handed out
    RowStat stat;
};

// What a bucket adds to sum q ln(q / p), d = ln(q / p) in units: q d + (p - q), as the buckets' sums of p and q are both 1.  It is never
// negative, and an error that all d share has no first order in the sum; near d = 0, q (d + exp(-d) - 1) by its series, to 4e-8 of itself.
struct Loss {
    float near, far;  // far in units
    __device__ __forceinline__ void add(float q, float p, float d) {
        const float x = d * kUnit;
        if (!(q > 0.0f)) {
            near += p;
        } else if (fabsf(x) >= 0.5f) {
            far += q * d + (p - q) * kPerUnit;
        } else {
            float g = 1.0f / 40320.0f;
            g = g * x - 1.0f / 5040.0f;
            g = g * x + 1.0f / 720.0f;
            g = g * x - 1.0f / 120.0f;
            g = g * x + 1.0f / 24.0f;
            g = g * x - 1.0f / 6.0f;
            g = g * x + 0.5f;
            near += q * x * x * g;
        }
    }
};

template <typename T>
__device__ __forceinline__ uint4 pack_slot(const float (&v)[ElemTraits<T>::kVec]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4)
            w[i] = __float_as_uint(v[i]);
        else
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Writes slot s of a gradient row (grad: its first element), v[e] for its elements; `aligned`: the row starts like the row of logits.
template <typename T>
__device__ __forceinline__ void store_slot(const RowSlots<T>& r, char* grad, bool aligned, int s, const float (&v)[ElemTraits<T>::kVec]) {
    constexpr int E = ElemTraits<T>::kVec;
    const int j = s * E - r.phase;
    const uint4 q = pack_slot<T>(v);
    if (aligned && whole_slot<T>(r, s)) {
        *reinterpret_cast<uint4*>(grad + (int64_t)j * (int)sizeof(T)) = q;
        return;
    }
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (E == 4) {
            if (j + i >= 0 && j + i < r.V) reinterpret_cast<uint32_t*>(grad)[j + i] = w[i];
        } else {
            if (j + 2 * i >= 0 && j + 2 * i < r.V) reinterpret_cast<uint16_t*>(grad)[j + 2 * i] = (uint16_t)w[i];
            if (j + 2 * i + 1 >= 0 && j + 2 * i + 1 < r.V) reinterpret_cast<uint16_t*>(grad)[j + 2 * i + 1] = (uint16_t)(w[i] >> 16);
        }
    }
}

template <typename T>
__device__ __forceinline__ void store_value(char* grad, int j, float v) {
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float*>(grad)[j] = v;
    } else {
        uint32_t w;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(0.0f), "f"(v));
        reinterpret_cast<uint16_t*>(grad)[j] = (uint16_t)w;
    }
}

template <typename T, int THREADS>
__device__ __forceinline__ void write_zeros(const Section<T>& x, char* grad, bool aligned) {
    float v[ElemTraits<T>::kVec] = {};
    for (int s = (x.head ? 0 : x.s0) + (int)threadIdx.x; s < x.s1; s += THREADS) store_slot<T>(x.r, grad, aligned, s, v);
}

// The gradient's entries outside the message: one slot's.
template <typename T>
__device__ __forceinline__ void others_of(const uint4& q, float m_r, float c, float factor, float (&v)[ElemTraits<T>::kVec]) {
    const uint64_t minus = pair(-m_r, -m_r), scale = pair(c, c), times = pair(factor, factor);
    slot_values<T>(q, v);
#pragma unroll
    for (int e = 0; e < ElemTraits<T>::kVec; e += 2) {
        const uint64_t x = mul_pair(add_pair(pair(v[e], v[e + 1]), minus), scale);
        const uint64_t y = mul_pair(pair(exp2_approx(__uint_as_float((uint32_t)x)), exp2_approx(__uint_as_float((uint32_t)(x >> 32)))), times);
        v[e] = __uint_as_float((uint32_t)y);
        v[e + 1] = __uint_as_float((uint32_t)(y >> 32));
    }
}
// Of a trip (g), to a row that starts like the row of logits or elsewhere.
template <typename T, int THREADS>
__device__ __forceinline__ void write_trip(const Section<T>& x, char* grad, bool aligned, int g, const uint4* slots, float m_r, float c, float factor) {
    const int at = x.s0 + g * kSlots * THREADS + (int)threadIdx.x;
    char* to = grad + (int64_t)(at * ElemTraits<T>::kVec - x.r.phase) * (int)sizeof(T);
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
        float v[ElemTraits<T>::kVec];
        others_of<T>(slots[u * THREADS], m_r, c, factor, v);
        if (aligned)
            __stcs(reinterpret_cast<uint4*>(to) + u * THREADS, pack_slot<T>(v));
        else
            store_slot<T>(x.r, grad, false, at + u * THREADS, v);
    }
}
// Of what lies behind the trips and before them.
template <typename T, int THREADS>
__device__ __forceinline__ void write_rest(const Section<T>& x, char* grad, bool aligned, float m_r, float c, float factor) {
    float v[ElemTraits<T>::kVec];
    if (x.rest > 0) {
        uint4 q[kSlots];
        load_rest<T, THREADS>(x, q);
        const int at = x.s0 + x.trips * kSlots * THREADS + (int)threadIdx.x;
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
            others_of<T>(q[u], m_r, c, factor, v);
            if (at + u * THREADS < x.s1) store_slot<T>(x.r, grad, aligned, at + u * THREADS, v);
        }
    }
    if (x.head && (int)threadIdx.x < x.s0) {
        others_of<T>(load_slot<T>(x.r, threadIdx.x), m_r, c, factor, v);
        store_slot<T>(x.r, grad, aligned, threadIdx.x, v);
    }
}

// The message's entries in the section; their student logits were read before anything was written (the gradient may lie over them).
template <typename T, int THREADS>
__device__ __forceinline__ void write_sent(const Section<T>& x, char* grad, int n, const RowStat& st, float w, float c, const Sent* sent) {
    const int first = x.head ? 0 : x.s0 * ElemTraits<T>::kVec - x.r.phase, end = min(x.s1 * ElemTraits<T>::kVec - x.r.phase, x.r.V);
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const Sent e = sent[i];
        if (e.j < first || e.j >= end) continue;  // in another section (or no index: the row's gradient is NaN)
        const float pj = st.inv_p * exp2_approx((e.z - st.m) * c), qj = st.inv_q * exp2_approx((e.t - st.t_max) * c);
        store_value<T>(grad, e.j, w * (pj - qj));
    }
}

// Dynamic shared memory: places of trips; a bit per logit, a word per batch; the message.
template <int THREADS>
size_t distill_smem(int places, int batches, int k) {
    return places * kPlaceBytes<THREADS> + (size_t)batches * THREADS * sizeof(uint32_t) + (size_t)k * sizeof(Sent);
}

// What a call computes, and how.
constexpr int kLoss = 0;
constexpr int kReread = 1;  // the gradient too: the section is read again for it, a block (cluster) per row
constexpr int kHeld = 2;    // the gradient too: the section's trips stay in shared memory; clusters take one row after the other
template <int MODE>
constexpr int kPlaces = MODE == kHeld ? 4 : 3;
constexpr int kHeldThreads = 256;
template <int MODE>
constexpr int kResident = MODE == kLoss ? 1024 : MODE == kReread ? 896 : 768;  // threads per SM

template <typename T, int MODE, bool CLUSTER, int THREADS>
__global__ void __launch_bounds__(THREADS, kResident<MODE> / THREADS) distill_kernel(const DistillPlan p) {
    constexpr int E = ElemTraits<T>::kVec, U = kSlots, WARPS = THREADS / 32, kTrip = U * THREADS;
    constexpr bool HELD = MODE == kHeld, GRAD = MODE != kLoss;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ DistillShared<THREADS> sh;
    uint32_t* bits = reinterpret_cast<uint32_t*>(dyn + kPlaces<MODE> * kPlaceBytes<THREADS>);  // all 0 between two rows
    Sent* sent = reinterpret_cast<Sent*>(bits + (size_t)p.batches * THREADS);
    cg::cluster_group cluster = cg::this_cluster();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int blocks = CLUSTER ? (int)cluster.num_blocks() : 1, part = CLUSTER ? (int)cluster.block_rank() : 0;
    const float c = p.c;
    pdl_enter();

    // Rows that are held are handed out, by the first block of a cluster; else the block (cluster) has one.  (Clusters do not get on at the
    // same pace, and fewer are resident than their blocks would be: every 55th row for each, 1000 x 131,072 fp32 took 332 us instead of
    // 217, with as many clusters as are resident 235.)
    int64_t taken = p.N;  // in the first thread of the first block: a row that the others do not know yet
    int64_t row = blockIdx.x / blocks, next = p.N;
    auto tell = [&](int64_t x, int half) {
        for (int i = 0; i < blocks; ++i) *cluster.map_shared_rank(&sh.rows[half], i) = x;
    };
    if constexpr (HELD) {
        cluster.sync();  // every block runs: its shared memory can be written
        if (part == 0 && t == 0) {
            tell((int64_t)atomicAdd(p.counter, 1u), 0);
            tell((int64_t)atomicAdd(p.counter, 1u), 1);
            taken = (int64_t)atomicAdd(p.counter, 1u);
        }
    } else if constexpr (CLUSTER) {
        cluster.barrier_arrive();
    }
    for (int i = t; i < p.batches * THREADS; i += THREADS) bits[i] = 0;
    if (t == 0) sh.wrong = 0;
    if constexpr (HELD) {
        cluster.sync();
        row = sh.rows[0];
        next = sh.rows[1];
        cluster.sync();
    }

    // Of the (next) row: count and a thread's first entry, its student logit, the first trips (all, if they are held).
    TripStream<T, THREADS, kPlaces<MODE>> stream(dyn);
    Section<T> x = {}, ahead = {};
    int n;
    uint32_t j;
    float val, z;
    // (Places behind the message are read too and not used: waiting for the count first costs 0.15 us a call, rows that are held 2 %.)
    auto ask_message = [&](int64_t at) {
        n = at < p.N ? p.count[at] : 0;
        const bool mine = at < p.N && t < p.k;
        j = mine ? p.idx[at * p.k + t] : 0;
        val = mine ? p.val[at * p.k + t] : 0.0f;
    };
    auto begin_ahead = [&](int64_t at) {
        z = (unsigned)n <= (unsigned)p.k && t < n && j < (uint32_t)p.V ? load_logit<T>(p.logits, at, p.ld, (int)j) : -CUDART_INF_F;
        ahead = section_of<T, THREADS>(p.logits, at, p.ld, p.V, part, blocks);
    };
    auto ask_held = [&](int g) {  // trip g of the next row to place g
        if (n != 0 && g < ahead.trips) ask_trip<THREADS>(stream.source(ahead) + g * kTrip, stream.mine + g * kTrip);
        cp_async_commit();
    };
    ask_message(row);
    begin_ahead(row);
    if constexpr (HELD) {
        for (int g = 0; g < kPlaces<MODE>; ++g) ask_held(g);
    } else {
        stream.start(ahead, n != 0 ? ahead.trips : 0);
    }
    __syncthreads();
    for (int parity = 0; row < p.N; parity ^= 1) {
        x = ahead;
        char* grad = GRAD ? static_cast<char*>(p.grad) + row * p.ldg * (int64_t)sizeof(T) : nullptr;
        const RowSlots<T>& r = x.r;
        const bool aligned = GRAD && (reinterpret_cast<uintptr_t>(grad) & 15) == (uintptr_t)r.phase * sizeof(T);
        if (n == 0) {  // padding: its logits are not read
            if (part == 0) {
                if (t == 0) p.loss[row] = 0.0f;
                if (p.stat && t < 8) p.stat[row * 8 + t] = 0.0f;
            }
            if constexpr (GRAD) write_zeros<T, THREADS>(x, grad, aligned);
            if constexpr (HELD) {
                ask_message(next);
                begin_ahead(next);
                for (int g = 0; g < kPlaces<MODE>; ++g) ask_held(g);
                row = next;
                if (part == 0 && t == 0) tell(taken, parity);
                cluster.sync();
                next = sh.rows[parity];
                if (part == 0 && t == 0) taken = (int64_t)atomicAdd(p.counter, 1u);
                continue;
            } else {
                if constexpr (CLUSTER) cluster.barrier_wait();
                return;
            }
        }

        // the message: its bits in this section, both largest values
        int wrong = 0, here = n;
        if (here < 0 || here > p.k) {
            wrong = 1;
            here = 0;
        }
        float t_max = -CUDART_INF_F, z_max = -CUDART_INF_F;
        auto bit_of = [&](int e, int* word) {  // of index e, -1 in another section; the head's words are the first of the last batch
            const int s = (e + r.phase) / E, at = s - x.s0;
            const bool head = x.head && at < 0;
            *word = head ? (p.batches - 1) * THREADS + s : at / kTrip * THREADS + at % THREADS;
            return head ? (e + r.phase) % E : s >= x.s0 && s < x.s1 ? at / THREADS % U * E + (e + r.phase) % E : -1;
        };
        for (int i = t; i < here; i += THREADS) {
            if (i != t) {
                j = p.idx[row * p.k + i];
                val = p.val[row * p.k + i];
                z = j < (uint32_t)p.V ? load_logit<T>(p.logits, row, p.ld, (int)j) : -CUDART_INF_F;
            }
            if (!(fabsf(val) < CUDART_INF_F)) wrong |= 2;
            if (j < (uint32_t)p.V) {
                int word;
                const int bit = bit_of((int)j, &word);
                if (bit >= 0 && atomicOr(&bits[word], 1u << bit) >> bit & 1u) wrong |= 1;
            } else {
                wrong |= 1;
            }
            sent[i] = {(int)j, val, z};
            t_max = fmaxf(t_max, val);
            z_max = max_nan(z_max, z);
        }
        const float rest = p.use_rest ? p.rest[row] : -CUDART_INF_F;
        const float weight = GRAD && p.weight ? p.weight[row] : 1.0f;
        if constexpr (HELD) ask_message(next);
        t_max = warp_max(t_max);
        z_max = warp_max(z_max);
        if (lane == 0) {
            sh.tops[0][warp] = t_max;
            sh.tops[1][warp] = z_max;
        }
        __syncthreads();
        t_max = sh.tops[0][0];
        z_max = sh.tops[1][0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) {
            t_max = fmaxf(t_max, sh.tops[0][i]);
            z_max = max_nan(z_max, sh.tops[1][i]);
        }
        if (!(z_max < CUDART_INF_F)) wrong |= 2;
        // the sums over S; every block takes its share of them
        float u = 0.0f, y = 0.0f;
        if ((t - lane) * blocks + part < here) {  // the warp has some
            for (int i = t * blocks + part; i < here; i += THREADS * blocks) {
                const Sent e = sent[i];
                u += exp2_approx((e.t - t_max) * c);
                if (z_max > -CUDART_INF_F) y += exp2_approx((e.z - z_max) * c);
            }
#pragma unroll
            for (int i = 16; i; i >>= 1) {
                u += __shfl_xor_sync(0xFFFFFFFFu, u, i);
                y += __shfl_xor_sync(0xFFFFFFFFu, y, i);
            }
        }
        if (lane == 0) {
            sh.sums[0][warp] = u;
            sh.sums[1][warp] = y;
        }

        // the pass over the section
        ExpSum sum = {-CUDART_INF_F, 0.0f};
        auto add = [&](const uint4 (&q)[U]) {
            const float m = max_nan(sum.m, batch_max<T>(q)), ref = reference(m);
            sum.s = sum.s * exp2_approx((sum.m - ref) * c) + exp_sum<T, U>(q, ref, c);
            sum.m = m;
        };
        auto take = [&](int g, uint4* slots) {
            for (uint32_t b = bits[g * THREADS + t]; b; b &= b - 1u) {  // entries of S become -inf where they lie
                const int bit = __ffs((int)b) - 1;
                uint4* slot = slots + bit / E * THREADS;
                if constexpr (sizeof(T) == 4)
                    reinterpret_cast<uint32_t*>(slot)[bit % E] = 0xFF800000u;
                else
                    reinterpret_cast<uint16_t*>(slot)[bit % E] = 0xFF80u;
            }
            uint4 q[U];
            take_trip<THREADS>(slots, q);
            add(q);
        };
        if constexpr (HELD) {
#pragma unroll 1
            for (int g = 0; g < x.trips; ++g) {
                wait_groups(kPlaces<MODE> - 1 - g);
                take(g, stream.mine + g * kTrip);
            }
        } else {
            stream.run(x, take);
        }
        const bool head = x.head && warp == 0;
        if (x.rest > 0 || head) {
            uint4 q[U], one[1];
            load_rest<T, THREADS>(x, q);
            one[0] = load_head<T>(x);
            for (uint32_t b = x.rest > 0 ? bits[x.trips * THREADS + t] : 0u; b; b &= b - 1u) {
                const int bit = __ffs((int)b) - 1;
#pragma unroll
                for (int i = 0; i < U; ++i) drop_element<T>(q[i], bit - i * E);
            }
            add(q);
            if (head) {
                for (uint32_t b = bits[(p.batches - 1) * THREADS + t]; b; b &= b - 1u) drop_element<T>(one[0], __ffs((int)b) - 1);
                float v[E], m = sum.m;
                slot_values<T>(one[0], v);
#pragma unroll
                for (int e = 0; e < E; ++e) m = max_nan(m, v[e]);
                const float ref = reference(m);
                sum.s = sum.s * exp2_approx((sum.m - ref) * c) + exp_sum<T, 1>(one, ref, c);
                sum.m = m;
            }
        }
        if constexpr (HELD)
            begin_ahead(next);
        else if constexpr (GRAD)
            stream.start(x, x.trips);
        if (!(sum.m < CUDART_INF_F)) {
            wrong |= 2;
            sum = {-CUDART_INF_F, 0.0f};
        }
        sum = warp_exp_sum(sum, c);
        if (lane == 0) sh.warp_sum[warp] = sum;
        if (wrong) atomicOr(&sh.wrong, wrong);
        __syncthreads();
        for (int i = t; i < here; i += THREADS) {  // the bits are used
            int word;
            const int e = sent[i].j;
            if ((unsigned)e < (unsigned)p.V && bit_of(e, &word) >= 0) bits[word] = 0;
        }
        RowPart all = {};
        if (warp == 0) {
            const ExpSum joined = join_exp_sums(sh.warp_sum, WARPS, c);
            all.m = joined.m;
            all.s = joined.s;
            all.wrong = sh.wrong;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                all.u += sh.sums[0][i];
                all.p += sh.sums[1][i];
            }
        }
        if constexpr (CLUSTER) {  // (a block that is a row ahead writes to the other half)
            RowPart* parts = sh.part[parity];
            if constexpr (!HELD) cluster.barrier_wait();
            if (t < blocks) cluster.map_shared_rank(parts, t)[part] = all;
            if (HELD && part == 0 && t == 0) tell(taken, parity);
            cluster.sync();
            if (warp == 0) {
                const ExpSum joined = join_exp_sums(parts, blocks, c);
                all = {joined.m, 0, joined.s, 0.0f, 0.0f};
                for (int i = 0; i < blocks; ++i) {
                    all.wrong |= parts[i].wrong;
                    all.u += parts[i].u;
                    all.p += parts[i].p;
                }
            }
        }
        int64_t after = p.N;
        if constexpr (HELD) {
            after = sh.rows[parity];
            if (part == 0 && t == 0) taken = (int64_t)atomicAdd(p.counter, 1u);
        }
        float m = 0.0f, up = 0.0f, down = 0.0f, p_others = 0.0f, q_others = 0.0f, p_all = 0.0f, inv_q = 0.0f;
        if (warp == 0) {
            if (!(rest < CUDART_INF_F)) all.wrong |= 2;
            m = fmaxf(z_max, all.m);
            if (!(m > -CUDART_INF_F)) all.wrong |= 2;
            RowStat st = {};
            if (all.wrong) {
                st.m_r = st.others = st.m = st.inv_p = st.t_max = st.inv_q = CUDART_NAN_F;
            } else {
                // p is next to exp(m / T), q next to exp(t_max / T) times e^up
                const float far = exp2_approx((all.m - m) * c), near = exp2_approx((z_max - m) * c);
                up = fmaxf(rest, 0.0f);
                down = exp_of(-up);
                const float u_rest = exp_of(rest - up);
                p_all = all.p * near + all.s * far;
                st.m_r = all.m;
                st.m = m;
                st.inv_p = 1.0f / p_all;
                st.t_max = t_max;
                inv_q = 1.0f / (all.u * down + u_rest);
                st.inv_q = down * inv_q;
                p_others = all.s * far * st.inv_p;
                q_others = u_rest * inv_q;
                // p_r - q_r = p_r q_s - q_r p_s, s: all that is sent.  (Subtracted directly, two numbers next to 1 that are nearly equal leave few
                // digits, and what is lost is common to all of the row's gradient: a factor off by 1e-3 of itself where q_r / p_r is 1 - 6e-5.)
                Two left = Two{all.s, 0.0f}.times({all.u, 0.0f}).times({far, 0.0f}).times({down, 0.0f});
                const Two less = Two{all.p, 0.0f}.times({near, 0.0f}).times({u_rest, 0.0f});
                left.add(-less.hi);
                st.others = all.s > 0.0f ? (left.hi + (left.lo - less.lo)) * st.inv_p * inv_q / all.s : 0.0f;
            }
            if (lane == 0) {
                sh.stat = st;
                sh.broken = all.wrong & 1;
                sh.wrong = 0;
                if (p.stat && part == 0) *reinterpret_cast<RowStat*>(p.stat + row * 8) = st;
            }
        }
        if constexpr (GRAD) {
            __syncthreads();
            const RowStat st = sh.stat;
            const float w = weight * p.T, m_r = reference(st.m_r), factor = st.others * w;
            if constexpr (HELD) {
#pragma unroll 1
                for (int g = 0; g < kPlaces<MODE>; ++g) {
                    if (g < x.trips) write_trip<T, THREADS>(x, grad, aligned, g, stream.mine + g * kTrip, m_r, c, factor);
                    ask_held(g);
                }
            } else {
                stream.run(x, [&](int g, uint4* slots) { write_trip<T, THREADS>(x, grad, aligned, g, slots, m_r, c, factor); });
            }
            write_rest<T, THREADS>(x, grad, aligned, m_r, c, factor);
            __syncthreads();
            write_sent<T, THREADS>(x, grad, sh.broken ? 0 : here, st, w, c, sent);
        }
        if (warp == 0 && part == 0) {
            if (lane == 0 && all.wrong) set_status(p.status, all.wrong & 1 ? MLMC_ERR_ARG : MLMC_ERR_NONFINITE);
            Loss loss = {0.0f, 0.0f};
            if (!all.wrong) {
                const float inv_p = 1.0f / p_all, shift = (logf(p_all * inv_q) - up) * kPerUnit;
                for (int i = lane; i < here; i += 32) {
                    const Sent e = sent[i];
                    const Two x = Two::difference(e.t * kPerUnit, t_max * kPerUnit), y = Two::difference(e.z * kPerUnit, m * kPerUnit);
                    Two d = Two::difference(x.hi, y.hi);
                    d.lo += x.lo - y.lo;
                    d = d.times(p.by_T);
                    d.add(shift);
                    loss.add(exp2_approx((e.t - t_max) * c) * down * inv_q, exp2_approx((e.z - m) * c) * inv_p,
                             e.z > -CUDART_INF_F ? d.hi + d.lo : CUDART_INF_F);
                }
                if (lane == 31) {
                    const Two ln = log_of(all.s);
                    Two d = Two::difference(m * kPerUnit, all.m * kPerUnit).times(p.by_T);
                    d.add(rest * kPerUnit);
                    d.add(-ln.hi * kPerUnit);
                    d.add(shift);
                    loss.add(q_others, p_others, all.s > 0.0f ? d.hi + (d.lo - ln.lo * kPerUnit) : CUDART_INF_F);
                }
#pragma unroll
                for (int i = 16; i; i >>= 1) {
                    loss.near += __shfl_xor_sync(0xFFFFFFFFu, loss.near, i);
                    loss.far += __shfl_xor_sync(0xFFFFFFFFu, loss.far, i);
                }
            }
            if (lane == 0) p.loss[row] = all.wrong ? CUDART_NAN_F : loss.near * p.T2 + loss.far * p.T2 * kUnit;
        }
        if constexpr (!HELD) return;
        row = next;
        next = after;
        __syncthreads();  // the message's entries are used, the bits are 0
    }
}

// The gradient by itself: grid (rows, sections).
constexpr int kGradThreads = 128;

template <typename T>
__global__ void __launch_bounds__(kGradThreads, 7) distill_grad_kernel(const DistillPlan p) {
    extern __shared__ __align__(16) unsigned char dyn[];
    Sent* sent = reinterpret_cast<Sent*>(dyn + 3 * kPlaceBytes<kGradThreads>);
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    pdl_enter();
    int n = p.count[row];
    const RowStat st = *reinterpret_cast<const RowStat*>(p.stat + row * 8);
    const Section<T> x = section_of<T, kGradThreads>(p.logits, row, p.ld, p.V, (int)blockIdx.y, (int)gridDim.y);
    char* grad = static_cast<char*>(p.grad) + row * p.ldg * (int64_t)sizeof(T);
    const bool aligned = (reinterpret_cast<uintptr_t>(grad) & 15) == (uintptr_t)x.r.phase * sizeof(T);
    if (n == 0) {
        write_zeros<T, kGradThreads>(x, grad, aligned);
        return;
    }
    if (n < 0 || n > p.k) n = 0;  // stat is NaN
    TripStream<T, kGradThreads, 3> stream(dyn);
    stream.start(x, x.trips);
    for (int i = t; i < n; i += kGradThreads) {
        const int j = (int)p.idx[row * p.k + i];
        sent[i] = {j, p.val[row * p.k + i], j >= 0 && j < p.V ? load_logit<T>(p.logits, row, p.ld, j) : 0.0f};
    }
    __syncthreads();
    const float w = (p.weight ? p.weight[row] : 1.0f) * p.T, m_r = reference(st.m_r), factor = st.others * w, c = p.c;
    stream.run(x, [&](int g, uint4* slots) { write_trip<T, kGradThreads>(x, grad, aligned, g, slots, m_r, c, factor); });
    write_rest<T, kGradThreads>(x, grad, aligned, m_r, c, factor);
    __syncthreads();
    write_sent<T, kGradThreads>(x, grad, n, st, w, c, sent);
}

constexpr int kDistillSmemMost = 200 * 1024;
template <typename T, int MODE, int THREADS>
void launch_threads(Workspace& ws, DistillPlan& p, int blocks, cudaStream_t s) {
    p.batches = (int)(section_slots<T>(p.V, blocks) / (kSlots * THREADS)) + 2;
    const size_t smem = distill_smem<THREADS>(kPlaces<MODE>, p.batches, p.k);
    int64_t grid = p.N * blocks;
    if constexpr (MODE == kHeld) {
        const int64_t per_sm = std::min<int64_t>(kResident<MODE> / THREADS, (227 * 1024) / (int64_t)(smem + sizeof(DistillShared<THREADS>) + 1024));
        grid = std::min<int64_t>(grid, per_sm * ws.sm_count / blocks * blocks);
        cudaMemsetAsync(p.counter, 0, sizeof(uint32_t), s);  // (2 us of 200 and more; a counter that has to be left at 0 would stay wrong once it is)
        launch_kernel_cluster(ws, K_DISTILL, blocks, distill_kernel<T, MODE, true, THREADS>, dim3((unsigned)grid), THREADS, smem, s, p);
    } else if constexpr (THREADS > 64) {
        if (blocks > 1)
            launch_kernel_cluster(ws, K_DISTILL, blocks, distill_kernel<T, MODE, true, THREADS>, dim3((unsigned)grid), THREADS, smem, s, p);
        else
            launch_kernel(ws, K_DISTILL, distill_kernel<T, MODE, false, THREADS>, dim3((unsigned)grid), THREADS, smem, s, p);
    } else {
        launch_kernel(ws, K_DISTILL, distill_kernel<T, MODE, false, THREADS>, dim3((unsigned)grid), THREADS, smem, s, p);
    }
}

// Blocks per row: all resident at a time, each with a batch per thread; 64 KB of bits at most.
template <typename T, int MODE, int THREADS>
int blocks_of(const Workspace& ws, const DistillPlan& p) {
    const int64_t resident = kResident<MODE> / THREADS * ws.sm_count;
    const int64_t blocks = std::min<int64_t>({kRowClusterMost, resident / p.N, p.V / (THREADS * kBatch<T>)});
    return (int)std::max<int64_t>({1, blocks, (p.V + (1 << 18) - 1) >> 18});
}

// The loss.  Short rows take blocks of 64 threads, whose beginnings and ends overlap (4096 x 2000 bf16: 19 us, 35 us with 256 threads;
// 4096 x 32,000 bf16: 49 and 55 us); longer or fewer rows want more bytes on the way per row (1000 x 131,072 fp32: 100 and 87 us;
// 600 x 32,000 bf16: 21 and 15 us), and few enough that a row has clusters of smaller blocks (16 x 32,000 fp32: 4.7 us with 128 threads, 5.5
// with 256; 200 x 50,257 bf16: 10.9 and 12.0 us).
//
// With the gradient a row is read twice.  Up to 256 KB most second reads are L2 hits and the rule is like the loss's (4096 x 2000 bf16:
// 19, 27 and 56 us with 64, 128 and 256 threads; 4096 x 32,000 bf16: 130, 116 and 117 us; 511 x 50,257 bf16: 27 us with two blocks of 128
// threads each, 31 with one of 256; 64 x 131,072 bf16: 17 and 15 us with clusters of 128 and 256 threads).  Of many longer rows half of
// the second reads miss: clusters hold them in shared memory, where the sections fill it (1000 rows of fp32, read twice and held: 70,000
// logits 139 and 132 us, 131,072 252 and 206, 150,000 293 and 265; but 60,000 118 and 117, 82,000, whose sections are 2.5 trips, 160 and 200,
// 106,283 221 and 236).  Not bf16, of twice the exponentials per byte: 131,072 logits 125 and 128 us, 262,144 248 and 253.
template <typename T>
void launch_typed(Workspace& ws, DistillPlan& p, cudaStream_t s) {
    const int64_t bytes = p.V * (int64_t)sizeof(T);
    if (!p.grad) {
        if (bytes <= 16 * 1024 || (bytes <= 96 * 1024 && p.N > 8 * ws.sm_count))
            launch_threads<T, kLoss, 64>(ws, p, 1, s);
        else if (p.N < 2 * ws.sm_count)
            launch_threads<T, kLoss, 128>(ws, p, blocks_of<T, kLoss, 128>(ws, p), s);
        else
            launch_threads<T, kLoss, 256>(ws, p, blocks_of<T, kLoss, 256>(ws, p), s);
        return;
    }
    // blocks that hold a row, their trips in places, what is behind the trips read again; more than 8: too long
    constexpr int64_t kHeldSlots = (int64_t)(kPlaces<kHeld> + 1) * kSlots * kHeldThreads;
    constexpr int64_t kHeldLeast = (int64_t)kPlaces<kHeld> * kSlots * kHeldThreads * 15 / 16;
    int held = 2;
    while (held <= kRowClusterMost && section_slots<T>(p.V, held) >= kHeldSlots) held *= 2;
    if (bytes <= 16 * 1024)
        launch_threads<T, kReread, 64>(ws, p, 1, s);
    else if (bytes <= 64 * 1024 || (bytes <= 128 * 1024 && 2 * p.N <= kResident<kReread> / 128 * ws.sm_count))
        launch_threads<T, kReread, 128>(ws, p, blocks_of<T, kReread, 128>(ws, p), s);
    else if (sizeof(T) == 2 || bytes <= 256 * 1024 || p.N < 4 * ws.sm_count || held > kRowClusterMost || section_slots<T>(p.V, held) < kHeldLeast)
        launch_threads<T, kReread, 256>(ws, p, blocks_of<T, kReread, 256>(ws, p), s);
    else if constexpr (sizeof(T) == 4)
        launch_threads<T, kHeld, kHeldThreads>(ws, p, held, s);
}

template <typename T>
void launch_grad_typed(Workspace& ws, DistillPlan& p, cudaStream_t s) {
    const int64_t sections = std::max<int64_t>(1, std::min<int64_t>({64, 8 * ws.sm_count / p.N, p.V / (kGradThreads * kBatch<T>)}));
    launch_kernel(ws, K_DISTILL_GRAD, distill_grad_kernel<T>, dim3((unsigned)p.N, (unsigned)sections), kGradThreads,
                  3 * kPlaceBytes<kGradThreads> + (size_t)p.k * sizeof(Sent), s, p);
}

template <typename K>
bool allow_smem(K kernel) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDistillSmemMost) == cudaSuccess &&
           cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) == cudaSuccess;
}
template <typename T, int MODE, int THREADS>
bool allow_both() {
    return allow_smem(distill_kernel<T, MODE, false, THREADS>) && allow_smem(distill_kernel<T, MODE, true, THREADS>);
}
template <typename T>
bool allow_typed() {
    return allow_smem(distill_kernel<T, kLoss, false, 64>) && allow_both<T, kLoss, 128>() && allow_both<T, kLoss, 256>() &&
           allow_smem(distill_kernel<T, kReread, false, 64>) && allow_both<T, kReread, 128>() && allow_both<T, kReread, 256>() &&
           allow_smem(distill_grad_kernel<T>);
}

DistillPlan plan_of(Workspace& ws, const void* logits, int64_t V, int64_t N, int64_t ld, const mlmc_logit_msgs& msgs, double T, int rest,
                    const float* weight, void* grad, int64_t ldg) {
    DistillPlan p = {};
    p.logits = logits;
    p.V = (int)V;
    p.N = N;
    p.ld = ld;
    p.idx = msgs.idx;
    p.val = msgs.val;
    p.count = msgs.count;
    p.rest = msgs.rest;
    p.k = msgs.k;
    p.use_rest = rest != 0;
    p.T = (float)T;
    p.T2 = (float)(T * T);
    p.c = (float)(1.4426950408889634 / T);
    const double by_T = (double)p.c * 0.69314718055994531;
    p.by_T = {(float)by_T, (float)(by_T - (double)(float)by_T)};
    p.weight = weight;
    p.grad = grad;
    p.ldg = ldg;
    p.status = ws.status;
    p.counter = ws.row_counter;
    return p;
}

}  // namespace

int configure_distill() {
    return allow_typed<float>() && allow_typed<bf16_t>() && allow_smem(distill_kernel<float, kHeld, true, kHeldThreads>) ? MLMC_OK : MLMC_ERR_CUDA;
}

void launch_distill(Workspace& ws, const void* logits, int dtype, int64_t V, int64_t N, int64_t ld, const mlmc_logit_msgs& msgs, double T,
                    int rest, const float* weight, float* loss, float* stat, void* grad, int64_t ldg, cudaStream_t s) {
    DistillPlan p = plan_of(ws, logits, V, N, ld, msgs, T, rest, weight, grad, ldg);
    p.loss = loss;
    p.stat = stat;
    if (dtype == MLMC_BF16)
        launch_typed<bf16_t>(ws, p, s);
    else
        launch_typed<float>(ws, p, s);
}

void launch_distill_grad(Workspace& ws, const void* logits, int dtype, int64_t V, int64_t N, int64_t ld, const mlmc_logit_msgs& msgs,
                         double T, int rest, const float* weight, const float* stat, void* grad, int64_t ldg, cudaStream_t s) {
    DistillPlan p = plan_of(ws, logits, V, N, ld, msgs, T, rest, weight, grad, ldg);
    p.stat = const_cast<float*>(stat);
    if (dtype == MLMC_BF16)
        launch_grad_typed<bf16_t>(ws, p, s);
    else
        launch_grad_typed<float>(ws, p, s);
}

}  // namespace mlmc
