// Rows of logits: loads at any alignment, and sums of exponentials that carry their largest exponent.
#pragma once

#include <cfloat>

#include <cooperative_groups.h>
#include <math_constants.h>

#include "common.cuh"

namespace mlmc {

// A row is a sequence of 16-byte slots on 16-byte boundaries; the first may begin before the row, the last may end behind it.  A thread
// takes four slots at a time, a batch, a block's width (THREADS slots) apart.
constexpr int kSlots = 4;
template <typename T>
constexpr int kBatch = kSlots * ElemTraits<T>::kVec;  // logits
constexpr int kRowClusterMost = 8;

template <typename T>
struct RowSlots {
    const char* first;  // slot 0
    int phase;          // elements of slot 0 before the row
    int n;              // slots
    int V;
};

template <typename T>
__device__ __forceinline__ RowSlots<T> row_slots(const void* rows, int64_t row, int64_t ld, int V) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(rows) + (uintptr_t)(row * ld) * sizeof(T);
    RowSlots<T> r;
    r.phase = (int)(at & 15) / (int)sizeof(T);
    r.first = reinterpret_cast<const char*>(at & ~(uintptr_t)15);
    r.n = (V + r.phase + ElemTraits<T>::kVec - 1) / ElemTraits<T>::kVec;
    r.V = V;
    return r;
}

template <typename T>
__device__ __forceinline__ bool whole_slot(const RowSlots<T>& r, int s) {
    const int j = s * ElemTraits<T>::kVec - r.phase;
    return j >= 0 && j + ElemTraits<T>::kVec <= r.V;
}

// Slot s; what lies outside the row, or s outside the row, is -inf.  (Plain loads: the row may be overwritten by the same kernel.)
template <typename T>
__device__ __forceinline__ uint4 load_slot(const RowSlots<T>& r, int s) {
    constexpr int E = ElemTraits<T>::kVec;
    if (whole_slot<T>(r, s)) return *reinterpret_cast<const uint4*>(r.first + (int64_t)s * 16);
    constexpr uint32_t kNone = E == 4 ? 0xFF800000u : 0xFF80FF80u;
    if (s >= r.n) return make_uint4(kNone, kNone, kNone, kNone);
    uint32_t w[4];
    const int j = s * E - r.phase;
    const char* at = r.first + (int64_t)s * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (E == 4) {
            w[i] = j + i >= 0 && j + i < r.V ? reinterpret_cast<const uint32_t*>(at)[i] : 0xFF800000u;
        } else {
            const uint32_t lo = j + 2 * i >= 0 && j + 2 * i < r.V ? reinterpret_cast<const uint16_t*>(at)[2 * i] : 0xFF80u;
            const uint32_t hi = j + 2 * i + 1 >= 0 && j + 2 * i + 1 < r.V ? reinterpret_cast<const uint16_t*>(at)[2 * i + 1] : 0xFF80u;
            w[i] = lo | hi << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A block's section of a row: whole trips (a batch per thread), the slots behind them, of which the last may be partial, and for the first
// block the slots before the first trip, which begins on a boundary of LINE slots.
template <typename T>
struct Section {
    RowSlots<T> r;
    int s0, s1;        // slots, without the head
    int trips, rest;   // (s1 - s0) = trips kSlots THREADS + rest, rest <= kSlots THREADS
    bool head;         // this block has the slots [0, s0) too, LINE at most
};
template <typename T, int THREADS, int LINE = 1>
__device__ __forceinline__ Section<T> section_of(const void* rows, int64_t row, int64_t ld, int V, int part, int blocks) {
    Section<T> x;
    x.r = row_slots<T>(rows, row, ld, V);
    int first = -(int)(reinterpret_cast<uintptr_t>(x.r.first) >> 4) & (LINE - 1);
    if (x.r.phase && first == 0) first = LINE;
    first = min(first, x.r.n);
    const int n = x.r.n - first, per = ((n + blocks - 1) / blocks + LINE - 1) / LINE * LINE;
    x.s0 = first + min(n, part * per);
    x.s1 = min(x.s0 + per, first + n);
    const int end = (x.r.V + x.r.phase) / ElemTraits<T>::kVec;  // of the whole slots
    x.trips = max(min(x.s1, end) - x.s0, 0) / (kSlots * THREADS);
    x.rest = x.s1 - x.s0 - x.trips * kSlots * THREADS;
    x.head = first > 0 && part == 0;
    return x;
}
// Slots of the longest section, at most.
template <typename T, int LINE = 1>
int64_t section_slots(int64_t V, int blocks) {
    const int64_t slots = (V + 2 * ElemTraits<T>::kVec - 2) / ElemTraits<T>::kVec;
    return ((slots + blocks - 1) / blocks + LINE - 1) / LINE * LINE;
}
// A thread's slots behind the trips.
template <typename T, int THREADS>
__device__ __forceinline__ void load_rest(const Section<T>& x, uint4 (&q)[kSlots]) {
    const int at = x.s0 + x.trips * kSlots * THREADS + (int)threadIdx.x;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) q[u] = load_slot<T>(x.r, at + u * THREADS < x.s1 ? at + u * THREADS : x.r.n);
}
// Its slot of the head, if it has one (the first warp's).
template <typename T>
__device__ __forceinline__ uint4 load_head(const Section<T>& x) { return load_slot<T>(x.r, x.head && (int)threadIdx.x < x.s0 ? (int)threadIdx.x : x.r.n); }

// cp.async.wait_group takes a constant: waits until at most n <= 3 of this thread's groups are in flight.
__device__ __forceinline__ void wait_groups(int n) {
    switch (n) {
        case 0: cp_async_wait<0>(); break;
        case 1: cp_async_wait<1>(); break;
        case 2: cp_async_wait<2>(); break;
        default: cp_async_wait<3>(); break;
    }
}

// A thread's slots of a trip are THREADS apart, or (PACKED) next to each other: 64 bytes, which a second look at them wants.  The copies
// are the same, of 512 bytes in a row per warp; packed, a lane reads what others copied, and slot n of the warp's 128 lies at
// n ^ (n >> 3 & 3), so that neither side meets a bank twice.
template <int THREADS, bool PACKED>
__device__ __forceinline__ int slot_in_trip(int thread, int u) { return PACKED ? thread * kSlots + u : thread + u * THREADS; }

template <int THREADS>
__device__ __forceinline__ void ask_trip(const uint4* from, uint4* to) {
#pragma unroll
    for (int u = 0; u < kSlots; ++u) cp_async_16(to + u * THREADS, from + u * THREADS);
}
template <int THREADS>
__device__ __forceinline__ void take_trip(const uint4* from, uint4 (&q)[kSlots]) {
#pragma unroll
    for (int u = 0; u < kSlots; ++u) q[u] = from[u * THREADS];
}

// A section's trips on their way through PLACES places in shared memory, all but one asked for while that one is used.  A warp copies and
// reads its own slots only (not packed: a thread), so there is no barrier.  (512 MB of bf16 through sums of exponentials: 6.4 TB/s with
// three to six blocks of 128 threads per SM, 5.1 to 5.6 TB/s with eight of them and loads into registers, one batch ahead or none.)
template <int THREADS>
constexpr size_t kPlaceBytes = (size_t)kSlots * THREADS * sizeof(uint4);

template <typename T, int THREADS, int PLACES, bool PACKED = false>
struct TripStream {
    static constexpr int kTrip = kSlots * THREADS;
    uint4* mine;  // the thread's first slot; packed: the warp's
    __device__ __forceinline__ explicit TripStream(void* places)
        : mine(static_cast<uint4*>(places) + (PACKED ? (int)(threadIdx.x >> 5) * 32 * kSlots : (int)threadIdx.x)) {}
    __device__ __forceinline__ static const uint4* source(const Section<T>& x) {
        const int first = PACKED ? (int)(threadIdx.x >> 5) * 32 * kSlots + (int)(threadIdx.x & 31) : (int)threadIdx.x;
        return reinterpret_cast<const uint4*>(x.r.first) + x.s0 + first;
    }
    __device__ __forceinline__ static void ask(const uint4* from, uint4* to) {
        if constexpr (PACKED) {
            const int lane = threadIdx.x & 31;
#pragma unroll
            for (int u = 0; u < kSlots; ++u) cp_async_16(to + ((u * 32 + lane) ^ ((u * 32 + lane) >> 3 & 3)), from + u * 32);
        } else {
            ask_trip<THREADS>(from, to);
        }
    }
    // The thread's slots of a trip that f got.
    __device__ __forceinline__ static void take(const uint4* from, uint4 (&q)[kSlots]) {
        if constexpr (PACKED) {
            const int lane = threadIdx.x & 31;
#pragma unroll
            for (int u = 0; u < kSlots; ++u) q[u] = from[lane * kSlots + (u ^ (lane >> 1 & 3))];
        } else {
            take_trip<THREADS>(from, q);
        }
    }
    // Asks for the first trips.
    __device__ __forceinline__ void start(const Section<T>& x, int trips) {
        const uint4* from = source(x);
#pragma unroll
        for (int g = 0; g < PLACES - 1; ++g) {
            if (g < trips) ask(from + g * kTrip, mine + g * kTrip);
            cp_async_commit();
        }
    }
    // f(g, slots): trip g has arrived.
    template <typename F>
    __device__ __forceinline__ void run(const Section<T>& x, F&& f) {
        const uint4* from = source(x) + (PLACES - 1) * kTrip;
        int now = 0, free = (PLACES - 1) * kTrip;
#pragma unroll 1
        for (int g = 0; g < x.trips; ++g) {
            if (g + PLACES - 1 < x.trips) ask(from, mine + free);
            cp_async_commit();
            cp_async_wait<PLACES - 1>();
            if constexpr (PACKED) __syncwarp();  // the other lanes' copies
            f(g, mine + now);
            if constexpr (PACKED) __syncwarp();  // read by all, before it is written again
            from += kTrip;
            free = now;
            now = now + kTrip < PLACES * kTrip ? now + kTrip : 0;
        }
    }
};

template <typename T>
__device__ __forceinline__ float load_logit(const void* rows, int64_t row, int64_t ld, int j) {
    if constexpr (sizeof(T) == 4)
        return reinterpret_cast<const float*>(rows)[row * ld + j];
    else
        return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(rows)[row * ld + j] << 16);
}

// The values of a slot.
template <typename T>
__device__ __forceinline__ void slot_values(const uint4& q, float (&v)[ElemTraits<T>::kVec]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v[i] = __uint_as_float(w[i]);
        } else {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

// Sets element e of a slot to -inf.
template <typename T>
__device__ __forceinline__ void drop_element(uint4& q, int e) {
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            if (e == i) w[i] = 0xFF800000u;
        } else {
            if (e == 2 * i) w[i] = (w[i] & 0xFFFF0000u) | 0xFF80u;
            if (e == 2 * i + 1) w[i] = (w[i] & 0x0000FFFFu) | 0xFF800000u;
        }
    }
    q = make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_pair(uint32_t a, uint32_t b) {  // two bf16
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The largest logit of a batch; NaN where it holds one.
template <typename T>
__device__ __forceinline__ float batch_max(const uint4 (&q)[kSlots]) {
    if constexpr (sizeof(T) == 4) {
        float m = -CUDART_INF_F;
#pragma unroll
        for (int u = 0; u < kSlots; ++u)
            m = max_nan(m, max_nan(max_nan(__uint_as_float(q[u].x), __uint_as_float(q[u].y)),
                                   max_nan(__uint_as_float(q[u].z), __uint_as_float(q[u].w))));
        return m;
    } else {
        uint32_t m = 0xFF80FF80u;
#pragma unroll
        for (int u = 0; u < kSlots; ++u)
            m = max_nan_pair(m, max_nan_pair(max_nan_pair(q[u].x, q[u].y), max_nan_pair(q[u].z, q[u].w)));
        return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    }
}

// What an exponent is taken relative to: the lowest finite number instead of -inf, so that -inf - ref is -inf.
__device__ __forceinline__ float reference(float m) { return fmaxf(m, -FLT_MAX); }

// sum exp2((v - ref) c) over the logits of N slots.  The difference is rounded before it is scaled: (v c - ref c) would be off by half
// a last place of ref c in every term alike, up to 1e-6 of the sum.  (A quarter of
// the exponentials by polynomial, to spare the unit for them: no faster.)
template <typename T, int N>
__device__ __forceinline__ float exp_sum(const uint4 (&q)[N], float ref, float c) {
    const uint64_t minus = pair(-ref, -ref), scale = pair(c, c);
    uint64_t sum[2] = {pair(0.0f, 0.0f), pair(0.0f, 0.0f)};
#pragma unroll
    for (int u = 0; u < N; ++u) {
        float v[ElemTraits<T>::kVec];
        slot_values<T>(q[u], v);
#pragma unroll
        for (int i = 0; i < ElemTraits<T>::kVec; i += 2) {
            const uint64_t x = mul_pair(add_pair(pair(v[i], v[i + 1]), minus), scale);
            sum[i / 2 % 2] = add_pair(sum[i / 2 % 2], pair(exp2_approx(__uint_as_float((uint32_t)x)), exp2_approx(__uint_as_float((uint32_t)(x >> 32)))));
        }
    }
    const uint64_t all = add_pair(sum[0], sum[1]);
    return __uint_as_float((uint32_t)all) + __uint_as_float((uint32_t)(all >> 32));
}

// A sum of exponentials s exp(m / T), m the largest logit; nothing yet: m = -inf, s = 0.
struct ExpSum {
    float m, s;
    __device__ __forceinline__ void add(float m2, float s2, float c) {
        const float top = fmaxf(m, m2), ref = reference(top);
        s = s * exp2_approx((m - ref) * c) + s2 * exp2_approx((m2 - ref) * c);
        m = top;
    }
};
// The largest of a warp's numbers, NaN if one is.
__device__ __forceinline__ float warp_max(float m) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(m));
    return r;
}
__device__ __forceinline__ ExpSum warp_exp_sum(const ExpSum& mine, float c) {
    const float m = warp_max(mine.m);
    float s = mine.s * exp2_approx((mine.m - reference(m)) * c);
#pragma unroll
    for (int i = 16; i; i >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, i);
    return {m, s};
}
// The sum of a few sums.  (64-bit arithmetic is slow here: a logarithm and a division of 64 bits took 4,400 cycles of a loaded SM.)
template <typename S>
__device__ __forceinline__ ExpSum join_exp_sums(const S* sums, int n, float c) {
    ExpSum r = {-CUDART_INF_F, 0.0f};
    for (int i = 0; i < n; ++i) r.m = fmaxf(r.m, sums[i].m);
    for (int i = 0; i < n; ++i) r.s += sums[i].s * exp2_approx((sums[i].m - reference(r.m)) * c);
    return r;
}

// A number in two of 32 bits (Knuth's sum): chains of 64-bit additions wait 70 cycles for each on a loaded SM.
struct Two {
    float hi, lo;
    __device__ __forceinline__ void add(float x) {
        const float sum = hi + x, added = sum - hi;
        lo += (hi - (sum - added)) + (x - added);
        hi = sum;
    }
    // a - b
    __device__ __forceinline__ static Two difference(float a, float b) {
        Two r = {a, 0.0f};
        r.add(-b);
        return r;
    }
    __device__ __forceinline__ Two times(Two f) const {
        const float p = hi * f.hi;
        return {p, fmaf(hi, f.hi, -p) + fmaf(hi, f.lo, lo * f.hi)};
    }
};

// ln s, s a normal number: its exponent (ln 2 in two parts, the first of 16 bits) and 2 artanh((m - 1) / (m + 1)).  What is compared
// with it is to be as exact as the sum s is: rounded to fp32 it would be off by 3e-7, which is 1e-4 of a loss of 1e-3.
__device__ __forceinline__ Two log_of(float s) {
    const uint32_t bits = __float_as_uint(s), up = (bits & 0x7FFFFFu) > 0x3504F3u;  // m in (0.707, 1.415)
    const float e = (float)((int)(bits >> 23) - 127 + (int)up);
    const float m = __uint_as_float((bits & 0x7FFFFFu) | (up ? 0x3F000000u : 0x3F800000u));
    const Two below = Two::difference(m, -1.0f);
    const float r = 1.0f / below.hi, above = m - 1.0f, f = above * r;
    const float f_lo = (fmaf(-f, below.hi, above) - f * below.lo) * r, f2 = f * f;
    float g = 1.0f / 11.0f;
    g = g * f2 + 1.0f / 9.0f;
    g = g * f2 + 1.0f / 7.0f;
    g = g * f2 + 1.0f / 5.0f;
    g = g * f2 + 1.0f / 3.0f;
    Two ln = {e * 0.693145751953125f, 0.0f};
    ln.add(2.0f * f);
    ln.lo += e * 1.42860682e-6f + 2.0f * (f_lo + f * f2 * g);
    return ln;
}

// exp(x), x <= 0, of which -inf is one: x log2(e) is rounded nowhere (as one number it would be off by 2^-20 at x = -14, and so would
// everything that is multiplied by the result).
__device__ __forceinline__ float exp_of(float x) {
    constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596299e-8f;
    const float y = x * kLog2e, r = exp2_approx(y), low = fmaf(x, kLog2e, -y) + x * kLog2eLow;
    return r > 0.0f ? fmaf(r * low, 0.693147181f, r) : 0.0f;
}

// Numbers ordered like the logits: larger for larger ones, the same for -0 and 0.
__device__ __forceinline__ uint32_t logit_key(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return (int)u < 0 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((int)k < 0 ? k & 0x7FFFFFFFu : ~k); }
constexpr uint32_t kLowestKey = 0x00800000u;  // of the lowest finite logit; -inf lies below

// An entry of a row: larger for larger logits, among equal ones for lower indices.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int j) { return (uint64_t)key << 32 | (uint32_t)~j; }
__device__ __forceinline__ uint32_t entry_key(uint64_t e) { return (uint32_t)(e >> 32); }
__device__ __forceinline__ uint32_t entry_index(uint64_t e) { return ~(uint32_t)e; }

}  // namespace mlmc
