// The router of an expert layer: scores -> expert ids and gate weights (Eq. 2, r = g(TopK(s, k))), the way back, and the balance loss
// with per-expert counts.
//
// All three read a row of E scores per token.  A token belongs to a group of L neighbouring lanes, each of which holds V consecutive
// scores (V = 8 up to 512 experts, 16 beyond), so a wave works on 64 / L tokens at a time, a row is read with whole 16-byte loads,
// and every reduction over a row is one inside registers and log2(L) cross-lane moves.
#include "lanes.hpp"

namespace grouter {

namespace {

constexpr int kThreads = 256;

enum Gating { kSoftmaxSelected = 0, kSoftmaxAll = 1, kSigmoid = 2, kSigmoidNormalised = 3 };

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float shift_of(float top) { return top == -INFINITY ? 0.f : top; }   // a row of -inf shifts by nothing: all its terms are 0
// sigmoid(x) * e^-shift, without overflow or loss on either side of 0
__device__ __forceinline__ float sigmoid_of(float x, float shift = 0.f) {
    return exp_of(fminf(x, 0.f) - shift) * __builtin_amdgcn_rcpf(1.f + exp_of(-fabsf(x)));
}
__device__ __forceinline__ float reciprocal_or_zero(float z) { return z == 0.f ? 0.f : 1.f / z; }

// V consecutive scores of a row from column e0 on; what lies behind column E is not touched.
template <class Type, int V>
struct Scores {
    typename Type::stored raw[V];
    __device__ __forceinline__ void load(const typename Type::stored* __restrict__ row, int e0, int E, bool whole_pieces) {
        if (whole_pieces && e0 + V <= E) {
            typedef uint32_t Piece __attribute__((ext_vector_type(4)));
            constexpr int n = V * sizeof(typename Type::stored) / 16;
            Piece p[n];
#pragma unroll
            for (int i = 0; i < n; ++i) p[i] = reinterpret_cast<const Piece*>(row + e0)[i];
            __builtin_memcpy(raw, p, sizeof(raw));
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) raw[v] = e0 + v < E ? row[e0 + v] : typename Type::stored(0);
        }
    }
    __device__ __forceinline__ float operator[](int v) const { return Type::widen(raw[v]); }
};

// A whole number that orders like the score: NaN like -inf, -0 like +0; 0 is below all of them (a score taken already, or none).
template <class Type>
__device__ __forceinline__ uint32_t order_of(typename Type::stored raw) {
    uint32_t b = __float_as_uint(Type::widen(raw));
    b = (b & 0x7fffffffu) > 0x7f800000u ? 0xff800000u : b;
    b = b == 0x80000000u ? 0u : b;
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

template <class IdxT>
__device__ __forceinline__ int id_at(const void* ids, int64_t i) { return (int)((const IdxT*)ids)[i]; }
__device__ __forceinline__ int id_of(const void* ids, int idx_dtype, int64_t i) {
    return idx_dtype == 1 ? id_at<uint8_t>(ids, i) : id_at<int32_t>(ids, i);
}

// Ids and gates.  k rounds: the largest remaining order number of the group, the first lane that holds it (lanes hold ascending
// columns, so on ties the lowest expert), and there the first place.
template <class Type, int L, int V>
__global__ __launch_bounds__(kThreads) void k_route(const typename Type::stored* __restrict__ scores, int64_t ld, bool whole_pieces,
                                                    int64_t T, int E, int k, int gating, const uint8_t* __restrict__ token_mask,
                                                    void* __restrict__ ids, int idx_dtype, uint16_t* __restrict__ gates) {
    extern __shared__ uint16_t s_pick[];
    const int lane = threadIdx.x & 63, part = lane % L, e0 = part * V;
    const int local = threadIdx.x / L;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + local;
    const bool here = t < T;
    const auto* row = scores + (here ? t : T - 1) * ld;
    uint16_t* pick = s_pick + local * k;
    Scores<Type, V> x;
    x.load(row, e0, E, whole_pieces);
    uint32_t order[V];
#pragma unroll
    for (int v = 0; v < V; ++v) order[v] = e0 + v < E ? order_of<Type>(x.raw[v]) : 0u;
    float top = -INFINITY, z = 0.f;
    if (gating == kSoftmaxAll) {
#pragma unroll
        for (int v = 0; v < V; ++v) top = e0 + v < E ? fmaxf(top, x[v]) : top;
        top = shift_of(group_max<L>(top));
#pragma unroll
        for (int v = 0; v < V; ++v) z += e0 + v < E ? exp_of(x[v] - top) : 0.f;
        z = group_sum<L>(z);
    }
    const int first = lane - part;
    for (int j = 0; j < k; ++j) {
        uint32_t best = order[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = max(best, order[v]);
        const uint32_t most = group_max<L>(best);
        const uint64_t holders = __ballot(best == most) >> first;
        if (best == most && (holders & ((1ull << part) - 1)) == 0) {
            bool found = false;
            int at = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const bool hit = !found && order[v] == most;
                at = hit ? v : at;
                order[v] = hit ? 0u : order[v];
                found = found || hit;
            }
            pick[j] = (uint16_t)(e0 + at);
        }
    }
    __syncthreads();
    // the picked scores, one per lane and round, read again from the row that has just been fetched
    const bool masked = token_mask && here && token_mask[t] == 0;
    if (gating == kSoftmaxSelected) top = shift_of(Type::widen(row[pick[0]]));
    if (gating == kSigmoid) top = 0.f;
    if (gating == kSigmoidNormalised) top = shift_of(fminf(Type::widen(row[pick[0]]), 0.f));
    auto weight = [&](int j) {
        const float s = Type::widen(row[pick[j]]);
        return gating >= kSigmoid ? sigmoid_of(s, top) : exp_of(s - top);
    };
    if (gating == kSoftmaxSelected || gating == kSigmoidNormalised) {
        for (int j = part; j < k; j += L) z += weight(j);
        z = group_sum<L>(z);
    }
    const float scale = masked ? 0.f : gating == kSigmoid ? 1.f : reciprocal_or_zero(z);
    if (!here) return;
    for (int j = part; j < k; j += L) {
        const float g = masked ? 0.f : weight(j) * scale;
        gates[t * k + j] = Bf16::narrow(g);
        if (idx_dtype == 1) ((uint8_t*)ids)[t * k + j] = (uint8_t)pick[j];
        else ((int32_t*)ids)[t * k + j] = (int32_t)pick[j];
    }
}

// How many of the S + 1 ascending offsets are at most t; sequence s holds the tokens [off[s], off[s + 1]).
__device__ __forceinline__ int64_t offsets_up_to(const int64_t* __restrict__ off, int64_t S, int64_t t) {
    int64_t lo = 0, hi = S + 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (off[mid] <= t) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// Probabilities over all experts of a row, from what a lane holds: softmax, or sigmoids over their sum.  Zero behind column E.
template <class Type, int L, int V>
__device__ __forceinline__ void probabilities(const Scores<Type, V>& x, int e0, int E, bool sigmoid, float* p) {
    float top = -INFINITY, z = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) top = e0 + v < E ? fmaxf(top, x[v]) : top;
    top = group_max<L>(top);
    top = shift_of(sigmoid ? fminf(top, 0.f) : top);
    if (sigmoid) {
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] = e0 + v < E ? sigmoid_of(x[v], top) : 0.f;
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] = e0 + v < E ? exp_of(x[v] - top) : 0.f;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) z += p[v];
    const float scale = reciprocal_or_zero(group_sum<L>(z));
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] *= scale;
}

struct RouteGrad {
    const void* ids;             // k ids per token with the gradients by the logs of their gates, or null
    int idx_dtype, k;
    const float* dlog;
    const int64_t* off;          // sequences of the balance loss, null for one over all tokens
    int64_t S;
    const float* coef;           // [S][E], or null
    const uint8_t* token_mask;
    void* out;
    int out_dtype;
    int64_t out_ld;
};

__device__ __forceinline__ void store_as(void* out, int dtype, int64_t i, float v) {
    if (dtype == 0) ((float*)out)[i] = v;
    else ((uint16_t*)out)[i] = dtype == 1 ? Bf16::narrow(v) : Fp16::narrow(v);
}

// Gradient by the scores.  With p the probabilities over all experts, g the gates, q the gradients by the gates' logs and c the
// balance loss's coefficients: p_e (c_e - <c, p>) (times 1 - sigmoid(s_e) for sigmoids), plus at the picked experts q_j - g_j sum q
// (softmax over them), q_j and everywhere -p_e sum q (softmax over all), (1 - sigmoid) q_j or (1 - sigmoid) (q_j - g_j sum q).
// Nothing is divided by a gate, so a gate of 0 has a gradient of 0.  WHOLE: the row's scores are needed, not the picked ones alone.
template <class Type, int L, int V, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_route_bwd(const typename Type::stored* __restrict__ scores, int64_t ld, bool whole_pieces,
                                                        int64_t T, int E, int gating, RouteGrad a) {
    extern __shared__ float s_slot[];    // per token k contributions, then k expert numbers
    const int lane = threadIdx.x & 63, part = lane % L, e0 = part * V;
    const int local = threadIdx.x / L;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + local;
    const bool here = t < T, live = here && !(a.token_mask && a.token_mask[t] == 0);
    const auto* row = scores + (here ? t : T - 1) * ld;
    const bool sigmoid = gating >= kSigmoid;
    float ds[V], p[V];
    Scores<Type, V> x;
#pragma unroll
    for (int v = 0; v < V; ++v) ds[v] = 0.f;
    if (WHOLE) {
        x.load(row, e0, E, whole_pieces);
        probabilities<Type, L, V>(x, e0, E, sigmoid, p);
    }
    if (WHOLE && a.coef) {
        int64_t s = a.off ? offsets_up_to(a.off, a.S, t) - 1 : 0;
        if (s >= a.S) s = -1;     // behind the last sequence, as before the first: in none
        float c[V], dot = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            c[v] = s >= 0 && e0 + v < E ? a.coef[s * E + e0 + v] : 0.f;
            dot += c[v] * p[v];
        }
        dot = group_sum<L>(dot);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ds[v] = s >= 0 ? p[v] * (c[v] - dot) : 0.f;
            if (sigmoid) ds[v] *= s >= 0 ? sigmoid_of(-x[v]) : 0.f;
        }
    }
    if (a.dlog) {
        const int k = a.k;
        float* u = s_slot + local * 2 * k;
        int* e = (int*)(u + k);
        float sum = 0.f, top = -INFINITY, z = 0.f;
        for (int j = part; j < k; j += L) {
            const int id = here ? id_of(a.ids, a.idx_dtype, t * k + j) : -1;
            const bool ok = (unsigned)id < (unsigned)E;
            e[j] = ok ? id : -1;
            u[j] = ok ? a.dlog[t * k + j] : 0.f;
            sum += u[j];
            if (ok && (gating == kSoftmaxSelected || gating == kSigmoidNormalised)) top = fmaxf(top, Type::widen(row[id]));
        }
        sum = group_sum<L>(sum);
        if (gating == kSoftmaxSelected || gating == kSigmoidNormalised) {
            top = group_max<L>(top);
            top = shift_of(sigmoid ? fminf(top, 0.f) : top);
            for (int j = part; j < k; j += L)
                if (e[j] >= 0) z += sigmoid ? sigmoid_of(Type::widen(row[e[j]]), top) : exp_of(Type::widen(row[e[j]]) - top);
            const float scale = sum * reciprocal_or_zero(group_sum<L>(z));
            for (int j = part; j < k; j += L)
                if (e[j] >= 0) u[j] -= scale * (sigmoid ? sigmoid_of(Type::widen(row[e[j]]), top) : exp_of(Type::widen(row[e[j]]) - top));
        }
        if (sigmoid)
            for (int j = part; j < k; j += L)
                if (e[j] >= 0) u[j] *= sigmoid_of(-Type::widen(row[e[j]]));
        if (WHOLE && gating == kSoftmaxAll)
#pragma unroll
            for (int v = 0; v < V; ++v) ds[v] -= p[v] * sum;
        __syncthreads();
        for (int j = 0; j < k; ++j) {
            const int at = e[j] - e0;
            const float w = u[j];
#pragma unroll
            for (int v = 0; v < V; ++v) ds[v] += at == v ? w : 0.f;
        }
    }
    if (!here) return;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (e0 + v < E) store_as(a.out, a.out_dtype, t * a.out_ld + e0 + v, live ? ds[v] : 0.f);
}

// ---- balance loss -------------------------------------------------------------------------------------------------------------
// Per sequence s of n tokens: f_e = count_e / (k n), P_e = mean of p_e, loss = alpha E sum_e f_e P_e, and what the gradient needs,
// coef_e = alpha E f_e / n.  The tokens are cut into chunks of equal length, one per workgroup; the part of a sequence inside a chunk
// leaves its sums in a slot of its own, chunk + sequence (both only grow along the tokens, so no two parts share one), and a second
// launch adds up each sequence's slots in order.  So work is even whatever the sequences' lengths, and no float is added atomically.
struct BalanceParts {
    float* sum;       // [chunks + S][E]
    int32_t* count;   // [chunks + S][E]
    int32_t* tokens;  // [chunks + S]
    double* loss;     // [S]
    uint32_t* done;   // sequences finished
    int64_t rows;     // of a chunk
};

template <class Type, int L, int V>
__global__ __launch_bounds__(kThreads) void k_balance_parts(const typename Type::stored* __restrict__ scores, int64_t ld, bool whole_pieces,
                                                            int64_t T, int E, int k, bool sigmoid, const uint8_t* __restrict__ token_mask,
                                                            const void* __restrict__ ids, int idx_dtype,
                                                            const int64_t* __restrict__ off, int64_t S, BalanceParts parts) {
    __shared__ float s_sum[kThreads / 64][L * V];
    __shared__ int s_count[L * V];
    __shared__ int s_tokens;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = lane % L, e0 = part * V;
    const int64_t row0 = blockIdx.x * parts.rows, row1 = min(T, row0 + parts.rows);
    if (blockIdx.x == 0 && threadIdx.x == 0) *parts.done = 0;
    for (int64_t s = off ? max((int64_t)0, offsets_up_to(off, S, row0) - 1) : 0; s < S; ++s) {
        const int64_t begin = off ? off[s] : 0, end = off ? off[s + 1] : T;
        if (begin >= row1) break;
        const int64_t a = max(begin, row0), b = min(end, row1);
        if (a >= b) continue;
        for (int e = threadIdx.x; e < E; e += kThreads) s_count[e] = 0;
        if (threadIdx.x == 0) s_tokens = 0;
        __syncthreads();
        float sum[V];
        int tokens = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = 0.f;
        for (int64_t t0 = a; t0 < b; t0 += kThreads / L) {
            const int64_t t = t0 + threadIdx.x / L;
            const bool live = t < b && !(token_mask && token_mask[t] == 0);
            Scores<Type, V> x;
            x.load(scores + (t < b ? t : b - 1) * ld, e0, E, whole_pieces);
            float p[V];
            probabilities<Type, L, V>(x, e0, E, sigmoid, p);
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += live ? p[v] : 0.f;
            tokens += live;
        }
        for (int64_t i = a * k + threadIdx.x; i < b * k; i += kThreads) {
            const int id = id_of(ids, idx_dtype, i);
            if ((unsigned)id < (unsigned)E && !(token_mask && token_mask[i / k] == 0)) atomicAdd(&s_count[id], 1);
        }
        if (part == 0 && tokens) atomicAdd(&s_tokens, tokens);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            for (int step = L; step < 64; step *= 2) sum[v] += __shfl_xor(sum[v], step);
            if (lane < L) s_sum[wave][e0 + v] = sum[v];
        }
        __syncthreads();
        const int64_t slot = blockIdx.x + s;
        for (int e = threadIdx.x; e < E; e += kThreads) {
            float all = 0.f;
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) all += s_sum[w][e];
            parts.sum[slot * E + e] = all;
            parts.count[slot * E + e] = s_count[e];
        }
        if (threadIdx.x == 0) parts.tokens[slot] = s_tokens;
        __syncthreads();
    }
}

constexpr int kJoinThreads = 1024;

__global__ __launch_bounds__(kJoinThreads) void k_balance_join(int64_t T, int E, int k, const int64_t* __restrict__ off, int64_t S,
                                                               BalanceParts parts, float alpha, int32_t* __restrict__ counts,
                                                               float* __restrict__ prob, float* __restrict__ coef, float* __restrict__ loss) {
    __shared__ double s_sum[kJoinThreads];
    __shared__ int s_count[kJoinThreads], s_tokens;
    __shared__ bool s_last;
    const int64_t s = blockIdx.x;
    const int64_t begin = off ? max((int64_t)0, off[s]) : 0, end = off ? min(T, off[s + 1]) : T;
    const int64_t c0 = begin / parts.rows, c1 = begin < end ? (end - 1) / parts.rows + 1 : c0;
    if (threadIdx.x == 0) s_tokens = 0;
    __syncthreads();
    int mine = 0;
    for (int64_t c = c0 + threadIdx.x; c < c1; c += blockDim.x) mine += parts.tokens[c + s];
    if (mine) atomicAdd(&s_tokens, mine);
    // columns side by side, the slots dealt out over what threads are left
    int width = 64;
    while (width < E && width < (int)blockDim.x) width *= 2;
    const int col = threadIdx.x % width, deal = threadIdx.x / width, deals = blockDim.x / width;
    double total = 0.0;
    for (int e0 = 0; e0 < E; e0 += width) {
        const int e = e0 + col;
        double sum = 0.0;
        int count = 0;
        if (e < E)
#pragma unroll 4
            for (int64_t c = c0 + deal; c < c1; c += deals) {
                sum += (double)parts.sum[(c + s) * E + e];
                count += parts.count[(c + s) * E + e];
            }
        __syncthreads();
        s_sum[threadIdx.x] = sum;
        s_count[threadIdx.x] = count;
        __syncthreads();
        if (deal == 0 && e < E) {
            for (int d = 1; d < deals; ++d) {
                sum += s_sum[d * width + col];
                count += s_count[d * width + col];
            }
            const double n = s_tokens > 0 ? (double)s_tokens : 1.0;
            const double mean = sum / n, share = (double)count / (k * n);
            counts[s * E + e] = count;
            prob[s * E + e] = (float)mean;
            coef[s * E + e] = (float)((double)alpha * E * share / n);
            total += (double)alpha * E * share * mean;
        }
    }
    auto block_sum = [&](double v) {
        __syncthreads();
        s_sum[threadIdx.x] = v;
        __syncthreads();
        for (int step = blockDim.x / 2; step > 0; step /= 2) {
            if ((int)threadIdx.x < step) s_sum[threadIdx.x] += s_sum[threadIdx.x + step];
            __syncthreads();
        }
        return s_sum[0];
    };
    total = block_sum(total);
    if (S == 1) {
        if (threadIdx.x == 0) *loss = (float)total;
        return;
    }
    // the workgroup that finishes last adds up the sequences' losses, in their order whichever it is
    if (threadIdx.x == 0) {
        __hip_atomic_store(parts.loss + s, total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = __hip_atomic_fetch_add(parts.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == (uint32_t)S;
    }
    __syncthreads();
    if (!s_last) return;
    double all = 0.0;
    for (int64_t i = threadIdx.x; i < S; i += blockDim.x) all += __hip_atomic_load(parts.loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all = block_sum(all);
    if (threadIdx.x == 0) *loss = (float)all;
}

// Calls f with the lanes per token and the scores per lane that E experts take.
template <class F>
hipError_t with_lanes(int E, F f) {
#define GROUTER_LANES(L, V) return f(std::integral_constant<int, L>{}, std::integral_constant<int, V>{})
    if (E <= 8) GROUTER_LANES(1, 8);
    if (E <= 16) GROUTER_LANES(2, 8);
    if (E <= 32) GROUTER_LANES(4, 8);
    if (E <= 64) GROUTER_LANES(8, 8);
    if (E <= 128) GROUTER_LANES(16, 8);
    if (E <= 256) GROUTER_LANES(32, 8);
    if (E <= 512) GROUTER_LANES(64, 8);
    GROUTER_LANES(64, 16);
#undef GROUTER_LANES
}
template <class F>
hipError_t with_type(int dtype, F f) {
    if (dtype == 0) return f(Fp32{});
    if (dtype == 1) return f(Bf16{});
    return f(Fp16{});
}

bool whole_pieces(const void* p, int64_t ld, int dtype) { return (((uintptr_t)p | (uintptr_t)(ld * (dtype == 0 ? 4 : 2))) & 15u) == 0; }

}  // namespace

hipError_t launch_route(const void* scores, int dtype, int64_t ld, int64_t T, int E, int k, int gating, const uint8_t* token_mask, void* ids,
                        int idx_dtype, uint16_t* gates, hipStream_t s) {
    const bool whole = whole_pieces(scores, ld, dtype);
    return with_type(dtype, [&](auto type) {
        return with_lanes(E, [&](auto l, auto v) {
            typedef decltype(type) Type;
            constexpr int L = decltype(l)::value, V = decltype(v)::value, tokens = kThreads / L;
            hipLaunchKernelGGL((k_route<Type, L, V>), dim3((unsigned)((T + tokens - 1) / tokens)), dim3(kThreads), tokens * k * sizeof(uint16_t), s,
                               (const typename Type::stored*)scores, ld, whole, T, E, k, gating, token_mask, ids, idx_dtype, gates);
            return hipGetLastError();
        });
    });
}

hipError_t launch_route_bwd(const void* scores, int dtype, int64_t ld, int64_t T, int E, int gating, const uint8_t* token_mask, const void* ids,
                            int idx_dtype, int k, const float* dlog, const int64_t* off, int64_t S, const float* coef, void* out,
                            int out_dtype, int64_t out_ld, hipStream_t s) {
    const bool whole = whole_pieces(scores, ld, dtype);
    const RouteGrad a{ids, idx_dtype, k, dlog, off, S, coef, token_mask, out, out_dtype, out_ld};
    return with_type(dtype, [&](auto type) {
        return with_lanes(E, [&](auto l, auto v) {
            typedef decltype(type) Type;
            constexpr int L = decltype(l)::value, V = decltype(v)::value, tokens = kThreads / L;
            const dim3 grid((unsigned)((T + tokens - 1) / tokens));
            const size_t lds = dlog ? tokens * k * 2 * sizeof(float) : 0;
            if (coef || gating == kSoftmaxAll)
                hipLaunchKernelGGL((k_route_bwd<Type, L, V, true>), grid, dim3(kThreads), lds, s, (const typename Type::stored*)scores, ld, whole,
                                   T, E, gating, a);
            else
                hipLaunchKernelGGL((k_route_bwd<Type, L, V, false>), grid, dim3(kThreads), lds, s, (const typename Type::stored*)scores, ld, whole,
                                   T, E, gating, a);
            return hipGetLastError();
        });
    });
}

// Chunks: a few per CU at most, so that a sequence's slots are few, and not below the tokens that a workgroup takes at a time.
static int64_t balance_rows(int64_t T, int E) {
    int64_t at_once = kThreads;
    for (int e = 8; e < E && at_once > 4; e *= 2) at_once /= 2;
    const int64_t rows = (T + 511) / 512;
    return (rows + at_once - 1) / at_once * at_once;
}

BalanceLayout balance_layout(int64_t T, int E, int64_t S) {
    BalanceLayout l{};
    l.rows = balance_rows(T, E);
    l.chunks = (T + l.rows - 1) / l.rows;
    const size_t slots = (size_t)(l.chunks + S);
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    l.done = take(256);
    l.loss = take(sizeof(double) * (size_t)S);
    l.tokens = take(sizeof(int32_t) * slots);
    l.sum = take(sizeof(float) * slots * (size_t)E);
    l.count = take(sizeof(int32_t) * slots * (size_t)E);
    l.total = o;
    return l;
}

hipError_t launch_balance(const void* scores, int dtype, int64_t ld, int64_t T, int E, int k, bool sigmoid, const uint8_t* token_mask, const void* ids,
                          int idx_dtype, const int64_t* off, int64_t S, float alpha, int32_t* counts, float* prob, float* coef,
                          float* loss, void* ws, hipStream_t s) {
    const bool whole = whole_pieces(scores, ld, dtype);
    const BalanceLayout l = balance_layout(T, E, S);
    char* w = (char*)ws;
    const BalanceParts parts{(float*)(w + l.sum), (int32_t*)(w + l.count), (int32_t*)(w + l.tokens), (double*)(w + l.loss), (uint32_t*)(w + l.done), l.rows};
    const hipError_t e = with_type(dtype, [&](auto type) {
        return with_lanes(E, [&](auto lanes, auto v) {
            typedef decltype(type) Type;
            hipLaunchKernelGGL((k_balance_parts<Type, decltype(lanes)::value, decltype(v)::value>), dim3((unsigned)l.chunks), dim3(kThreads), 0, s,
                               (const typename Type::stored*)scores, ld, whole, T, E, k, sigmoid, token_mask, ids, idx_dtype, off, S, parts);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_balance_join, dim3((unsigned)S), dim3(S == 1 ? kJoinThreads : 256), 0, s, T, E, k, off, S, parts, alpha, counts, prob, coef, loss);
    return hipGetLastError();
}

}  // namespace grouter
