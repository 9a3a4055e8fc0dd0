// Beam search: the K best continuations of every sentence from the messages of its beams' logits, and the states that follow them.
#include <math_constants.h>

#include "common.cuh"

namespace mlmc {
namespace {

constexpr int kBeams = MLMC_MAX_BEAMS;
constexpr int kSelectThreads = 512;

struct SelectPlan {
    const uint32_t* idx;
    const float* val;
    const int32_t* count;
    const float* rest;
    int k;
    int W, K;
    double inv_T;
    const float* score;
    const uint8_t* done;
    int32_t eos;
    mlmc_beams out;
    int* status;
};

// A block per sentence.  Beam w's continuations are its message's entries, in order; their scores score_w + (val - val_0) / T - ln(sum)
// descend, so the rank of one among all is its place in its own list and, by bisection, how many of every other list come before it.
// Scores are summed and compared in 64 bits, so that a beam's own continuations, which differ by their logits alone, keep their order.
// Between beams they are as exact as the rests, whose rounding to fp32 is most of it: off by up to 6e-7 (rows of 2000 to 131,072 logits; the
// best continuations of two flat rows changed places up to 9e-7 apart).  Beams that are alike (score, message, rest to 2^-20) have the same
// scores even where their rows begin at different alignments and the rests' sums were rounded differently.
// Bound by its chain: a message's loads, one 64-bit exponential and logarithm, three barriers, the bisections; 4 us for W = K = 4, 7 us for
// 16 (13 us with a thread per continuation, and scores and counts read again for every pair of beams).
__global__ void __launch_bounds__(kSelectThreads) beam_select_kernel(const SelectPlan p) {
    extern __shared__ __align__(16) unsigned char dyn[];
    double* list = reinterpret_cast<double*>(dyn);  // [W][K]
    __shared__ int length[kBeams];
    __shared__ int count[kBeams];
    __shared__ float scores[kBeams];
    __shared__ uint8_t ended[kBeams];
    __shared__ double at_top[kBeams];   // score of the first continuation
    const int b = blockIdx.x, t = threadIdx.x, lane = t & 31, W = p.W, K = p.K;
    pdl_enter();
    for (int w = t >> 5; w < W; w += kSelectThreads / 32) {  // a warp per beam
        const int64_t row = (int64_t)b * W + w;
        const float score = p.score[row];
        const bool end = p.done && p.done[row];
        int n = 0, have = 0;
        if (!(score < CUDART_INF_F)) {
            if (lane == 0) set_status(p.status, MLMC_ERR_NONFINITE);
        } else if (score > -CUDART_INF_F) {
            if (end) {
                n = 1;
                if (lane == 0) list[w * K] = (double)score;
            } else {
                have = min(max(p.count[row], 0), p.k);
                const float* val = p.val + row * p.k;
                const double top = have ? (double)val[0] : 0.0;
                double sum = 0.0;  // the entries, and behind them the rest
                for (int i = lane; i < have + (have > 0); i += 32)
                    sum += exp(i < have ? ((double)val[i] - top) * p.inv_T : (double)p.rest[row]);
#pragma unroll
                for (int i = 16; i; i >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, i);
                if (lane == 0) at_top[w] = (double)score - log(sum);
                n = min(have, K);
            }
        }
        if (lane == 0) {
            length[w] = n;
            count[w] = have;
            scores[w] = score;
            ended[w] = end;
        }
    }
    __syncthreads();
    for (int w = t >> 5; w < W; w += kSelectThreads / 32) {
        const int64_t first = (int64_t)b * W, row = first + w;
        if (ended[w] || length[w] == 0) continue;
        const uint32_t* idx = p.idx + row * p.k;
        const float* val = p.val + row * p.k;
        const int have = count[w];
        int like = w;  // the first beam that is like this one
        for (int v = 0; v < like; ++v) {
            if (ended[v] || count[v] != have || scores[v] != scores[w]) continue;
            if (!(fabs(at_top[v] - at_top[w]) <= 0x1.0p-20)) continue;  // a rounding apart, not more
            bool same = true;
            for (int i = lane; i < have; i += 32) same = same && p.idx[(first + v) * p.k + i] == idx[i] && p.val[(first + v) * p.k + i] == val[i];
            if (__all_sync(0xFFFFFFFFu, same)) like = v;
        }
        for (int i = lane; i < length[w]; i += 32) list[w * K + i] = at_top[like] + ((double)val[i] - (double)val[0]) * p.inv_T;
    }
    __syncthreads();
    int total = 0;
    for (int w = 0; w < W; ++w) total += length[w];
    // as many neighbouring threads for one continuation as there are, each with its share of the lists
    int threads = 1;
    while (threads < 8 && 2 * threads * W * K <= kSelectThreads) threads *= 2;
    const int sub = t & (threads - 1);
    for (int at = 0; at < W * K; at += kSelectThreads / threads) {  // (whole warps)
        const int i = at + t / threads, w = i / K, r = i % K;
        const bool mine = i < W * K && r < length[w];
        const double x = mine ? list[i] : 0.0;
        int rank = 0;
        for (int v = sub; v < W && mine && r + rank < K; v += threads) {
            if (v == w) continue;
            int lo = 0, hi = length[v];  // entries of v before this one: larger, or equal in a lower beam
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                const double y = list[v * K + mid];
                if (y > x || (y == x && v < w))
                    lo = mid + 1;
                else
                    hi = mid;
            }
            rank += lo;
        }
        for (int step = threads / 2; step; step /= 2) rank += __shfl_xor_sync(0xFFFFFFFFu, rank, step);
        rank += r;
        if (!mine || sub != 0) continue;
        if (rank >= K) continue;
        const int64_t to = (int64_t)b * K + rank;
        const int32_t token = ended[w] ? p.eos : (int32_t)p.idx[((int64_t)b * W + w) * p.k + r];
        p.out.token[to] = token;
        p.out.parent[to] = w;
        p.out.score[to] = (float)x;
        if (p.out.done) p.out.done[to] = ended[w] || token == p.eos;
    }
    for (int i = total + t; i < K; i += kSelectThreads) {
        const int64_t to = (int64_t)b * K + i;
        p.out.token[to] = max(p.eos, 0);
        p.out.parent[to] = i % W;
        p.out.score[to] = -CUDART_INF_F;
        if (p.out.done) p.out.done[to] = 1;
    }
}

// ---- states ----
constexpr int kStatesPerLaunch = 48;
constexpr int kMoveThreads = 256;

struct StateMove {
    const char* src;
    char* dst;
    int64_t beam_stride, chunk_stride;
    int64_t columns;       // in all chunks
    uint32_t per_chunk;    // words of the access width per chunk, and with edges the single bytes around them
    uint32_t chunk_bytes;  // with edges
    uint32_t first_block;  // of the launch's blocks for one sentence
};
struct MovePlan {
    const int32_t* parent;
    int W, n;
    int* status;
    StateMove state[kStatesPerLaunch];
};

// A thread owns a column: one word at the same place of all the sentence's beams.  It loads the words of the parents of all beams that
// change, W independent loads, before it stores the first one, so a state can be reordered in place, whatever the permutation; a parent
// of several beams comes from L1 after the first time.  MOST: beams in registers, COLUMNS of them at a time for small W.
// EDGES: chunks may begin and end anywhere, but alike in all beams; their first and last bytes, less than a word each, are columns of one.
template <typename Word, int MOST, int COLUMNS, bool EDGES>
__global__ void __launch_bounds__(kMoveThreads) beam_reorder_kernel(const __grid_constant__ MovePlan p) {
    __shared__ int parents[MOST];
    __shared__ int wrong;
    const int t = threadIdx.x, W = p.W;
    pdl_enter();
    if (t == 0) wrong = 0;
    __syncthreads();
    if (t < W) {
        const int x = p.parent[(int64_t)blockIdx.y * W + t];
        parents[t] = x >= 0 && x < W ? x : -1;
        if (parents[t] < 0) wrong = 1;
    }
    __syncthreads();
    if (t == 0 && wrong && blockIdx.x == 0) set_status(p.status, MLMC_ERR_ARG);
    int i = 0;
    while (i + 1 < p.n && p.state[i + 1].first_block <= blockIdx.x) ++i;
    const StateMove& st = p.state[i];
    const bool in_place = st.src == st.dst;
    const int64_t base = (int64_t)blockIdx.y * W * st.beam_stride;
    const int64_t first = (int64_t)(blockIdx.x - st.first_block) * (kMoveThreads * COLUMNS) + t;
    Word x[COLUMNS][MOST];
    int64_t at[COLUMNS];
    bool live[COLUMNS], byte[COLUMNS];
#pragma unroll
    for (int c = 0; c < COLUMNS; ++c) {
        const int64_t column = first + c * kMoveThreads;
        live[c] = column < st.columns;
        byte[c] = false;
        const int64_t chunk = live[c] ? column / st.per_chunk : 0;
        at[c] = base + chunk * st.chunk_stride;
        uint32_t word = live[c] ? (uint32_t)(column - chunk * st.per_chunk) : 0u;
        if constexpr (EDGES) {
            constexpr uint32_t kSize = sizeof(Word);
            const uint32_t head = (uint32_t)(-(reinterpret_cast<uintptr_t>(st.src) + (uintptr_t)at[c])) & (kSize - 1);
            const uint32_t words = (st.chunk_bytes - head) / kSize, wide = st.chunk_bytes / kSize;  // in this chunk, at most
            if (word < wide) {
                live[c] = live[c] && word < words;
                at[c] += head;
            } else {
                word -= wide;
                live[c] = live[c] && word < st.chunk_bytes - words * kSize;
                at[c] += word < head ? word : words * kSize + word;
                word = 0;
                byte[c] = true;
            }
        }
        at[c] += (int64_t)word * (int64_t)sizeof(Word);
    }
    auto load = [](const char* from, bool one) {
        if (EDGES && one) {
            Word r = {};
            *reinterpret_cast<uint8_t*>(&r) = *reinterpret_cast<const uint8_t*>(from);
            return r;
        }
        return *reinterpret_cast<const Word*>(from);
    };
    auto store = [](char* to, const Word& x, bool one) {
        if (EDGES && one)
            *reinterpret_cast<uint8_t*>(to) = *reinterpret_cast<const uint8_t*>(&x);
        else
            *reinterpret_cast<Word*>(to) = x;
    };
#pragma unroll
    for (int w = 0; w < MOST; ++w) {
        const int from = w < W ? parents[w] : -1;
        const bool moves = from >= 0 && !(in_place && from == w);
#pragma unroll
        for (int c = 0; c < COLUMNS; ++c)
            if (moves && live[c]) x[c][w] = load(st.src + at[c] + from * st.beam_stride, byte[c]);
    }
#pragma unroll
    for (int w = 0; w < MOST; ++w) {
        const int from = w < W ? parents[w] : -1;
        const bool moves = from >= 0 && !(in_place && from == w);
#pragma unroll
        for (int c = 0; c < COLUMNS; ++c)
            if (moves && live[c]) store(st.dst + at[c] + w * st.beam_stride, x[c][w], byte[c]);
    }
}

template <typename Word, int MOST, int COLUMNS, bool EDGES>
void launch_moves(Workspace& ws, MovePlan& plan, int B, cudaStream_t s) {
    uint32_t blocks = 0;
    for (int i = 0; i < plan.n; ++i) {
        plan.state[i].first_block = blocks;
        blocks += (uint32_t)((plan.state[i].columns + kMoveThreads * COLUMNS - 1) / (kMoveThreads * COLUMNS));
    }
    launch_kernel(ws, K_BEAM_REORDER, beam_reorder_kernel<Word, MOST, COLUMNS, EDGES>, dim3(blocks, (unsigned)B), kMoveThreads, 0, s, plan);
}

template <typename Word, bool EDGES = false>
void launch_width(Workspace& ws, MovePlan& plan, int B, cudaStream_t s) {
    if (plan.W <= 4)
        launch_moves<Word, 4, 4, EDGES>(ws, plan, B, s);
    else if (plan.W <= 8)
        launch_moves<Word, 8, 2, EDGES>(ws, plan, B, s);
    else if (plan.W <= 16)
        launch_moves<Word, 16, 1, EDGES>(ws, plan, B, s);
    else
        launch_moves<Word, 32, 1, EDGES>(ws, plan, B, s);
}

}  // namespace

void launch_beam_select(Workspace& ws, const mlmc_logit_msgs& rows, int B, int W, double T, const float* score, const uint8_t* done,
                        int32_t eos, int K, const mlmc_beams& out, cudaStream_t s) {
    SelectPlan p = {rows.idx, rows.val, rows.count, rows.rest, rows.k, W, K, 1.0 / T, score, done, eos, out, ws.status};
    launch_kernel(ws, K_BEAM_SELECT, beam_select_kernel, dim3((unsigned)B), kSelectThreads, (size_t)W * K * sizeof(double), s, p);
}

void launch_beam_reorder(Workspace& ws, const int32_t* parent, int B, int W, const mlmc_beam_state* states, int n, cudaStream_t s) {
    // States in launches of one access width each: the widest that all their addresses and sizes are multiples of, or with edges the
    // widest that beams, source and destination are apart by multiples of, for chunks that have 32 words of it (192 beams, 12 chunks of
    // 1066 bytes, 1114 apart: 15.6 us by 2 bytes, 8.0 by 8 with edges; chunks of 250 bytes: 3.1 and 3.7).
    struct Kind {
        int width;
        bool edges;
    };
    for (const Kind kind : {Kind{16, true}, Kind{8, true}, Kind{16, false}, Kind{8, false}, Kind{4, false}, Kind{2, false}, Kind{1, false}}) {
        const int width = kind.width;
        MovePlan plan;
        plan.parent = parent;
        plan.W = W;
        plan.n = 0;
        plan.status = ws.status;
        int64_t blocks = 0;
        auto flush = [&] {
            if (!plan.n) return;
            switch (width) {
                case 16: kind.edges ? launch_width<uint4, true>(ws, plan, B, s) : launch_width<uint4>(ws, plan, B, s); break;
                case 8: kind.edges ? launch_width<uint2, true>(ws, plan, B, s) : launch_width<uint2>(ws, plan, B, s); break;
                case 4: launch_width<uint32_t>(ws, plan, B, s); break;
                case 2: launch_width<uint16_t>(ws, plan, B, s); break;
                default: launch_width<uint8_t>(ws, plan, B, s); break;
            }
            plan.n = 0;
            blocks = 0;
        };
        for (int i = 0; i < n; ++i) {
            const mlmc_beam_state& x = states[i];
            if (x.chunks == 0 || x.chunk_bytes == 0) continue;
            const uint64_t all = (uint64_t)reinterpret_cast<uintptr_t>(x.src) | reinterpret_cast<uintptr_t>(x.dst) |
                                 (B * W > 1 ? (uint64_t)x.beam_stride : 0) | (x.chunks > 1 ? (uint64_t)x.chunk_stride : 0) |
                                 (uint64_t)x.chunk_bytes | 16u;
            const uint64_t apart = (B * W > 1 ? (uint64_t)x.beam_stride : 0) | (uint64_t)(reinterpret_cast<uintptr_t>(x.src) - reinterpret_cast<uintptr_t>(x.dst)) | 16u;
            Kind own = {(int)(all & (~all + 1)), false};
            const int wide = (int)(apart & (~apart + 1));
            if (wide > own.width && wide >= 8 && x.chunk_bytes >= 32 * wide) own = {wide, true};
            if (own.width != width || own.edges != kind.edges) continue;
            StateMove m = {};
            m.src = static_cast<const char*>(x.src);
            m.dst = static_cast<char*>(x.dst);
            m.beam_stride = x.beam_stride;
            m.chunk_stride = x.chunk_stride;
            m.chunk_bytes = (uint32_t)x.chunk_bytes;
            m.per_chunk = (uint32_t)(x.chunk_bytes / width + (kind.edges ? 2 * (width - 1) : 0));
            m.columns = x.chunks * (int64_t)m.per_chunk;
            const int64_t more = m.columns / kMoveThreads + 1;  // at least as many blocks as it takes
            if (plan.n == kStatesPerLaunch || blocks + more > INT32_MAX) flush();
            blocks += more;
            plan.state[plan.n++] = m;
        }
        flush();
    }
}

}  // namespace mlmc
