// The balance loss of a router, with per-expert counts and what its gradient is taken from.
#include "router.hpp"

#include <algorithm>

namespace grouter {

namespace {

// ---- balance loss -------------------------------------------------------------------------------------------------------------
// Per sequence s of n tokens: f_e = count_e / (k n), P_e = mean of p_e, loss = alpha E sum_e f_e P_e, and what the gradient needs,
// coef_e = alpha E f_e / n.  The tokens are cut into chunks of equal length, one per workgroup; the part of a sequence inside a chunk
// leaves its sums in a slot of its own, chunk + sequence (both only grow along the tokens, so no two parts share one), and a second
// launch adds up each sequence's slots in order.  So work is even whatever the sequences' lengths, and no float is added atomically.
// 131072 x 256 in fp32 with the scores from memory: 34 us, 4.0 TB/s, what torch's sum over 4 GiB reads, and 6 for the join; over and over on one
// batch, most of which the last-level cache holds, the two take 28 to 33.  In bf16 24.8 us, 2.7 TB/s: neither reading nor the vector instructions
// (3891 per wave, 13 us by count, 16 with the exponentials' further cycles) fill it, but two waves per SIMD that load, sum across lanes
// and count in turn.  Where scores are few it is the chain of loads, barrier and second launch (30011 x 60 bf16 in 48 sequences: 7.3 us
// and 6.2 for the join).  The figures at the choices below are of passes over and over on one batch.
struct BalanceCell {
    float prob;
    int32_t count;
};
struct BalanceParts {
    BalanceCell* cells;  // [chunks + S][E]
    int32_t* tokens;     // [chunks + S], valid ones
    double* loss;        // [S][column blocks]
    uint32_t* done;      // workgroups that have left their loss
    int64_t rows;        // of a chunk
};

// 128, 256 and 512 threads: 131072 x 256 47.6, 33.3, 35.2 us (all of the call), 65536 x 128 in 256 sequences 29.4, 26.4, 30.9, 4096 x 64 in 64
// sequences 11.0, 11.7, 12.8.
constexpr int kPartThreads = 256;
// Rounds of tokens up to which one workgroup does it all.  In 4 rounds 6.1 to 6.8 us against 6.2 to 8.2 in two launches, and one launch less
// to enqueue (8 against 11 us where the host is what it waits for); in 8 rounds 9.6 to 10.8 against 6.2 to 8.1.
constexpr int kAloneRounds = 4;

struct BalanceOut {
    float alpha;
    int32_t* counts;
    float *prob, *coef, *loss;
    // results of one expert in a sequence with these sums; its part of the loss
    __device__ __forceinline__ double put(int64_t at, int E, int k, int tokens, double sum, int count) const {
        const double over = 1.0 / max(tokens, 1), mean = sum * over, scaled = (double)alpha * E / k * over * count;
        counts[at] = count;
        prob[at] = (float)mean;
        coef[at] = (float)(scaled * over);
        return scaled * mean;
    }
};

template <int STEP>
__device__ __forceinline__ float rotated(float v) { return __uint_as_float(dpp_move<0x120 + STEP>(__float_as_uint(v))); }   // row_ror

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int step = 32; step > 0; step /= 2) v += __shfl_xor(v, step);
    return v;
}

// A chunk is walked in tiles of as many tokens as the workgroup has groups of lanes.  While a tile lies within one sequence, its rows are
// added up in registers; where a sequence ends, the sums of the lanes are joined through LDS (flush).  Sequences that begin and end
// inside one tile are added up from a copy of the tile's rows in LDS, each by a wave of its own.
// ALONE: one workgroup takes all tokens of the only sequence and writes the results itself.
template <class Type, int L, int V, bool FULL, bool SIGMOID, bool ALONE>
__global__ __launch_bounds__(kPartThreads) void k_balance_parts(const typename Type::stored* __restrict__ scores, int64_t ld, int64_t T, int E, int k,
                                                                const uint8_t* __restrict__ token_mask,
                                                                const void* __restrict__ ids, int idx_dtype,
                                                                const int64_t* __restrict__ off, int64_t S, BalanceParts parts, BalanceOut out) {
    constexpr int kWaves = kPartThreads / 64, kTokens = kPartThreads / L, C = L * V, W = kPiece<Type>;
    constexpr int kAhead = L >= 8 ? 1 : L >= 4 ? 2 : 4;      // ids of a tile that a thread fetches ahead: 8 per token, shared by its lanes
    constexpr int kRows = L <= 16 ? 4 : 64 / L;      // partial sums that a wave leaves in LDS: one per 16 lanes, or per group
    constexpr int kSpan = 64 / kRows;
    __shared__ float s_rows[kTokens * C];            // a tile's rows, or the waves' partial sums, as the pieces that the lanes hold
    __shared__ int s_count[C], s_tokens[2];
    __shared__ int16_t s_ids[kAhead * kPartThreads];  // with a tile's rows, the ids of its first slots
    __shared__ uint32_t s_few[kWaves][C / 2];        // counts of a sequence inside one tile (at most 4096 slots), two in a word
    static_assert(kWaves * kRows <= kTokens, "partial sums fit where the rows do");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane % L;
    const int64_t row0 = blockIdx.x * parts.rows, row1 = min(T, row0 + parts.rows);
    if (!ALONE && blockIdx.x == 0 && threadIdx.x == 0) *parts.done = 0;
    for (int e = threadIdx.x; e < C; e += kPartThreads) s_count[e] = 0;
    if (threadIdx.x < 2) s_tokens[threadIdx.x] = 0;
    Row<Type, L, V, FULL> x, ahead;
    x.place(part, E);
    ahead = x;
    ahead.load(scores + min(row0 + threadIdx.x / L, row1 - 1) * ld, E);
    // the walk is in sequence s, whose tokens end before `next`; -1 and S: in none
    int64_t s = 0, next = T;
    if (off) s = offsets_up_to(off, S, row0, next) - 1;
    int64_t window = s + 1, ends = off ? off[min(window + 1 + lane, S)] : 0;     // lane i: the end of sequence window + i
    double loss = 0.0;
    bool empty = true, open = false;     // no sequence has been joined yet; the present one has tokens that are not joined
    float sum[V];
    int tokens = 0, turn = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.f;
    auto emit = [&](int64_t seq, int e, int n, float total, int count) {
        if (ALONE) loss += out.put(seq * E + e, E, k, n, total, count);
        else parts.cells[(blockIdx.x + seq) * E + e] = BalanceCell{total, count};
    };
    __syncthreads();
    for (int64_t t0 = row0; t0 < row1; t0 += kTokens) {
        const int64_t t = t0 + threadIdx.x / L, t1 = min(t0 + kTokens, row1);
        const bool live = t < row1 && !(token_mask && token_mask[t] == 0);
        x = ahead;
        if (t1 < row1) ahead.load(scores + min(t + kTokens, row1 - 1) * ld, E);
        // the tile's first ids while its probabilities are computed
        const uint32_t slots = (uint32_t)(t1 - t0) * (uint32_t)k;
        auto counted = [&](uint32_t i) {
            const int id = i < slots && !(token_mask && token_mask[t0 + i / (uint32_t)k] == 0) ? id_of(ids, idx_dtype, t0 * k + i) : -1;
            return (unsigned)id < (unsigned)E ? id : -1;
        };
        int id[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) id[i] = counted(threadIdx.x + i * kPartThreads);
        float p[V];
        if (!FULL) {     // compared in every tile: masks that wait for the next one would fill the scalar registers
#pragma unroll
            for (int i = 0; i < x.N; ++i) asm volatile("" : "+v"(x.skip[i]));
        }
        float scale = shares<SIGMOID>(x, p);
        if (__ballot(!live)) {     // (what a padding token holds may be NaN)
            scale = live ? scale : 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] = live ? p[v] : 0.f;
        }
        int64_t u = t0;      // the tile's tokens before u are done
        for (;;) {
            const int64_t w = min(next, t1);
            if (s >= 0 && s < S && u < w) {
                open = true;
                const bool in = live && t >= u && t < w;
                const float take = in ? scale : 0.f;
                if ((u == t0 && w == t1) || __ballot(in) == ~0ull) {
#pragma unroll
                    for (int v = 0; v < V; ++v) sum[v] = __builtin_fmaf(p[v], take, sum[v]);
                } else {     // another sequence's NaN stays its own
#pragma unroll
                    for (int v = 0; v < V; ++v) sum[v] += in ? p[v] * scale : 0.f;
                }
                tokens += in;
                const uint32_t lo = (uint32_t)(u - t0) * (uint32_t)k, hi = (uint32_t)(w - t0) * (uint32_t)k;
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const uint32_t at = threadIdx.x + i * kPartThreads;
                    if (id[i] >= 0 && at >= lo && at < hi) atomicAdd(&s_count[id[i]], 1);
                }
                for (uint32_t i = threadIdx.x + kAhead * kPartThreads; i < hi; i += kPartThreads) {
                    const int e = i >= lo ? counted(i) : -1;
                    if (e >= 0) atomicAdd(&s_count[e], 1);
                }
            }
            if (open && (next < t1 || t1 == row1)) {     // the sequence or the chunk ends
                open = empty = false;
                if (part == 0 && tokens) atomicAdd(&s_tokens[turn], tokens);
                // over the groups within 16 lanes in registers, over the rest in LDS
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if constexpr (L <= 1) sum[v] += rotated<1>(sum[v]);
                    if constexpr (L <= 2) sum[v] += rotated<2>(sum[v]);
                    if constexpr (L <= 4) sum[v] += rotated<4>(sum[v]);
                    if constexpr (L <= 8) sum[v] += rotated<8>(sum[v]);
                    if (lane % kSpan < L) s_rows[(wave * kRows + lane / kSpan) * C + (v / W * L + part) * W + v % W] = sum[v];
                    sum[v] = 0.f;
                }
                tokens = 0;
                __syncthreads();
                const int n = s_tokens[turn];
                for (int e = threadIdx.x; e < E; e += kPartThreads) {
                    float all = 0.f;
                    const float* rows = s_rows + x.place_of(e, E);
#pragma unroll 8
                    for (int w = 0; w < kWaves * kRows; ++w) all += rows[w * C];
                    emit(s, e, n, all, s_count[e]);
                    s_count[e] = 0;
                }
                if (!ALONE && threadIdx.x == 0) parts.tokens[blockIdx.x + s] = n;
                turn ^= 1;
                if (threadIdx.x == 0) s_tokens[turn] = 0;
                __syncthreads();
            }
            if (next >= t1) break;
            u = max(next, t0);
            bool copied = false;
            int whose = 0;
            for (++s; s < S; ++s) {
                if (s - window >= 64) {
                    window = s;
                    ends = off[min(window + 1 + lane, S)];
                }
                next = of_lane(ends, (int)(s - window));
                if (next >= t1) break;
                if (next > u) {
                    empty = false;
                    if (!copied) {
                        copied = true;
#pragma unroll
                        for (int v = 0; v < V; ++v)
                            s_rows[threadIdx.x / L * C + (v / W * L + part) * W + v % W] = p[v] * scale;
#pragma unroll
                        for (int i = 0; i < kAhead; ++i) s_ids[threadIdx.x + i * kPartThreads] = (int16_t)id[i];
                        __syncthreads();
                    }
                    if (whose == wave) {
                        uint32_t* few = s_few[wave];
                        for (int e = lane; e < C / 2; e += 64) few[e] = 0;
                        int n = 0;
                        const int a = (int)(u - t0), b = (int)(next - t0);
                        for (int i = a; i < b; i += 64) n += __popcll(__ballot(i + lane < b && !(token_mask && token_mask[t0 + min(i + lane, b - 1)] == 0)));
                        for (uint32_t i = (uint32_t)a * k + lane; i < (uint32_t)b * k; i += 64) {
                            const int e = i < kAhead * kPartThreads ? s_ids[i] : counted(i);
                            if (e >= 0) atomicAdd(&few[e >> 1], 1u << (16 * (e & 1)));
                        }
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        for (int e = lane; e < E; e += 64) {
                            float all = 0.f;
                            const float* rows = s_rows + x.place_of(e, E);
#pragma unroll 8
                            for (int i = a; i < b; ++i) all += rows[i * C];
                            emit(s, e, n, all, (int)(few[e >> 1] >> (16 * (e & 1)) & 0xffffu));
                        }
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        if (!ALONE && lane == 0) parts.tokens[blockIdx.x + s] = n;
                    }
                    whose = whose + 1 == kWaves ? 0 : whose + 1;
                    u = next;
                }
            }
            if (s >= S) next = INT64_MAX;
            if (copied) __syncthreads();
        }
    }
    if (ALONE) {
        __shared__ double s_loss[kWaves];
        if (empty)
            for (int e = threadIdx.x; e < E; e += kPartThreads) out.put(e, E, k, 0, 0.0, 0);
        loss = wave_sum(loss);
        if (lane == 0) s_loss[wave] = loss;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kWaves; ++w) loss += s_loss[w];
            *out.loss = (float)loss;
        }
    }
}

// Joins the slots of one sequence for COLUMNS experts; THREADS / COLUMNS threads share the slots of an expert.
template <int COLUMNS, int THREADS>
__global__ __launch_bounds__(THREADS) void k_balance_join(int64_t T, int E, int k, const uint8_t* __restrict__ token_mask,
                                                          const int64_t* __restrict__ off, int64_t S, BalanceParts parts, BalanceOut out) {
    constexpr int kWaves = THREADS / 64, kDeals = THREADS / COLUMNS;
    __shared__ double s_sum[kWaves][COLUMNS];
    __shared__ int s_count[kWaves][COLUMNS], s_tokens[kWaves];
    __shared__ bool s_last;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t s = blockIdx.x;
    const int64_t begin = off ? max((int64_t)0, off[s]) : 0, end = off ? min(T, off[s + 1]) : T;
    const uint32_t rows = (uint32_t)parts.rows;      // as all of begin, end: at most T
    const int64_t c0 = begin < end ? (uint32_t)begin / rows : 0, c1 = begin < end ? (uint32_t)(end - 1) / rows + 1 : 0;
    const int col = threadIdx.x % COLUMNS, e = blockIdx.y * COLUMNS + col;
    double sum = 0.0;
    int count = 0, tokens = 0;
    if (e < E)
#pragma unroll 8
        for (int64_t c = c0 + threadIdx.x / COLUMNS; c < c1; c += kDeals) {
            const BalanceCell cell = parts.cells[(c + s) * E + e];
            sum += (double)cell.prob;
            count += cell.count;
        }
    if (token_mask)
        for (int64_t c = c0 + threadIdx.x; c < c1; c += THREADS) tokens += parts.tokens[c + s];
#pragma unroll
    for (int step = COLUMNS; step < 64; step *= 2) {
        sum += __shfl_xor(sum, step);
        count += __shfl_xor(count, step);
    }
    if (token_mask)
#pragma unroll
        for (int step = 1; step < 64; step *= 2) tokens += __shfl_xor(tokens, step);
    if (lane < COLUMNS) {
        s_sum[wave][lane] = sum;
        s_count[wave][lane] = count;
    }
    if (lane == 0) s_tokens[wave] = tokens;
    __syncthreads();
    if (wave == 0) {
        double part = 0.0;
        if (lane < COLUMNS) {
            for (int w = 1; w < kWaves; ++w) {
                sum += s_sum[w][lane];
                count += s_count[w][lane];
            }
        }
        if (token_mask) {
            tokens = 0;
            for (int w = 0; w < kWaves; ++w) tokens += s_tokens[w];
        } else {
            tokens = (int)max((int64_t)0, end - begin);
        }
        if (lane < COLUMNS && e < E) part = out.put(s * E + e, E, k, tokens, sum, count);
        part = wave_sum(part);
        if (gridDim.x == 1 && gridDim.y == 1) {
            if (lane == 0) *out.loss = (float)part;
        } else if (lane == 0) {
            __hip_atomic_store(parts.loss + s * gridDim.y + blockIdx.y, part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = __hip_atomic_fetch_add(parts.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x * gridDim.y;
        }
    }
    if (gridDim.x == 1 && gridDim.y == 1) return;
    __syncthreads();
    if (!s_last) return;
    // the workgroup that finishes last adds up all losses, in their order whichever it is
    double all = 0.0;
    for (int64_t i = threadIdx.x; i < S * gridDim.y; i += THREADS) all += __hip_atomic_load(parts.loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all = wave_sum(all);
    __syncthreads();
    if (lane == 0) s_sum[wave][0] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) all += s_sum[w][0];
        *out.loss = (float)all;
    }
}

}  // namespace

// Tiles of a chunk, each of which adds one fp32 term to a lane's sums: 256 of them round by at most 256 2^-25 of the sum (equal terms come to
// half of that), and the join adds in 64 bits.  Without it 4 M equal rows of 534 scores, 2048 terms a lane, were off by 3e-5.  It takes effect from
// 131072 tokens per token of a tile on; 512 chunks and this, in us: 4 M x 534 bf16 3256 / 2514, 16 M x 256 bf16 2333 / 1797, 4 M x 1024 fp32 2929 /
// 2970, the same in bf16 in 64 sequences 2419 / 1996, 32 M x 64 bf16 1331 / 1074.
constexpr int64_t kMostTiles = 256;

// Chunks: otherwise two per CU at most, so that a sequence's slots are few, and not below the tokens that a workgroup takes at a time.  256, 512, 768,
// 1024 of them: 131072 x 256 47.9, 33.3, 33.2, 38.5 us, 131072 x 64 in bf16 17.0, 13.8, 14.3, 15.5.
BalanceLayout balance_layout(int64_t T, int E, int64_t S) {
    BalanceLayout l{};
    const int64_t at_once = kPartThreads / lanes_of(E), rows = std::min((T + 511) / 512, kMostTiles * at_once);
    l.rows = (rows + at_once - 1) / at_once * at_once;
    l.chunks = (T + l.rows - 1) / l.rows;
    const size_t slots = (size_t)(l.chunks + S);
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    l.done = take(256);
    l.loss = take(sizeof(double) * (size_t)S * ((size_t)(E + 15) / 16));
    l.tokens = take(sizeof(int32_t) * slots);
    l.cells = take(sizeof(BalanceCell) * slots * (size_t)E);
    l.total = o;
    return l;
}

hipError_t launch_balance(const void* scores, int dtype, int64_t ld, int64_t T, int E, int k, bool sigmoid, const uint8_t* token_mask, const void* ids,
                          int idx_dtype, const int64_t* off, int64_t S, float alpha, int32_t* counts, float* prob, float* coef,
                          float* loss, void* ws, hipStream_t s) {
    const BalanceLayout l = balance_layout(T, E, S);
    char* w = (char*)ws;
    const BalanceParts parts{(BalanceCell*)(w + l.cells), (int32_t*)(w + l.tokens), (double*)(w + l.loss), (uint32_t*)(w + l.done), l.rows};
    const BalanceOut out{alpha, counts, prob, coef, loss};
    // one workgroup and no second launch where it needs few rounds: see kAloneRounds
    const bool alone = S == 1 && T <= (int64_t)kAloneRounds * kPartThreads / lanes_of(E);
    BalanceParts whole = parts;
    if (alone) whole.rows = T;
    const hipError_t e = with_type(dtype, [&](auto type) {
        return with_lanes(E, [&](auto lanes, auto v, auto full) {
            return with_flag(sigmoid, [&](auto flag) {
                typedef decltype(type) Type;
                constexpr int L = decltype(lanes)::value, V = decltype(v)::value;
                constexpr bool FULL = decltype(full)::value, SIGMOID = decltype(flag)::value;
                const auto* x = (const typename Type::stored*)scores;
                if (alone)
                    hipLaunchKernelGGL((k_balance_parts<Type, L, V, FULL, SIGMOID, true>), dim3(1), dim3(kPartThreads), 0, s, x, ld, T, E, k, token_mask,
                                       ids, idx_dtype, off, S, whole, out);
                else
                    hipLaunchKernelGGL((k_balance_parts<Type, L, V, FULL, SIGMOID, false>), dim3((unsigned)l.chunks), dim3(kPartThreads), 0, s, x, ld, T, E,
                                       k, token_mask, ids, idx_dtype, off, S, parts, out);
                return hipGetLastError();
            });
        });
    });
    if (e != hipSuccess || alone) return e;
    // Many slots per sequence: 64 threads to an expert's and 16 experts to a workgroup; few: 4 and 64.  131072 x 256 in bf16, the former / the latter with
    // 1, 2, 4, 8, 16 sequences 27.3 / 31.5, 26.9 / 28.3, 27.0 / 26.5, 27.8 / 25.8, 30.5 / 25.9 us (all of the call); 16384 x 128 with 1, 2, 4
    // 10.3 / 14.3, 10.5 / 11.6, 9.9 / 10.0; 8192 x 64, where a sequence has 128 slots, with one 9.4 / 8.0.
    if (l.chunks > 128 * S)
        hipLaunchKernelGGL((k_balance_join<16, 1024>), dim3((unsigned)S, (unsigned)(E + 15) / 16), dim3(1024), 0, s, T, E, k, token_mask, off, S, parts, out);
    else
        hipLaunchKernelGGL((k_balance_join<64, 256>), dim3((unsigned)S, (unsigned)(E + 63) / 64), dim3(256), 0, s, T, E, k, token_mask, off, S, parts, out);
    return hipGetLastError();
}

}  // namespace grouter
