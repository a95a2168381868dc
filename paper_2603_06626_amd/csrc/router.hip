// The router of an expert layer: scores -> expert ids and gate weights (Eq. 2, r = g(TopK(s, k))), and the way back.
#include "router.hpp"

namespace grouter {

namespace {

constexpr int kThreads = 256;

// ---- keys: whole numbers, all different within a row, that order like the scores and among equal scores by the lower column -------
// A score's bits become a two's complement number (-0 and +0 both 0), moved up by the distance of the largest positive NaN from the
// largest number, so that positive NaNs wrap round to the far end and a maximum with -inf's number sends all NaNs to -inf.  The
// column, inverted, stands below it: 16-bit scores fill a 32-bit key, 32-bit scores the upper bits of a positive double, for which
// the hardware has a maximum and a minimum in one instruction each.
template <class Type>
struct Keys16 {
    typedef int32_t Key;
    static constexpr uint16_t kInf = Type::kInf, kMove = 0x7fff - kInf;
    static __device__ __forceinline__ Key none() { return INT32_MIN; }
    static __device__ __forceinline__ void make(const uint16_t* raw, int column, Key* out) {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        typedef int16_t s16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            u16x2 u;
            __builtin_memcpy(&u, raw + i, 4);
            const s16x2 sign = __builtin_bit_cast(s16x2, u) >> 15;
            const u16x2 s = __builtin_bit_cast(u16x2, sign);
            const u16x2 t = ((u & (uint16_t)0x7fff) ^ s) + ((u16x2)(kMove) - s);
            const s16x2 k = __builtin_elementwise_max(__builtin_bit_cast(s16x2, t), (s16x2)((int16_t)(kMove - kInf)));
            const uint32_t word = __builtin_bit_cast(uint32_t, k);
            out[i] = (int32_t)(word << 16 | (uint32_t)(0xffff - column - i));
            out[i + 1] = (int32_t)((word & 0xffff0000u) | (uint32_t)(0xffff - column - i - 1));
        }
    }
    static __device__ __forceinline__ int column(Key k) { return 0xffff - (k & 0xffff); }
    // the score; -inf also where it was NaN
    static __device__ __forceinline__ float score(Key k) {
        const int v = (k >> 16) - kMove;
        return Type::widen((uint16_t)((v < 0 ? -v : v) | (v < 0 ? 0x8000 : 0)));
    }
    static __device__ __forceinline__ Key larger(Key a, Key b) { return max(a, b); }
    static __device__ __forceinline__ Key smaller(Key a, Key b) { return min(a, b); }
    template <int STEP>
    static __device__ __forceinline__ Key from_partner(Key k) { return (Key)partner<STEP>((uint32_t)k); }
};
struct Keys32 {
    typedef double Key;
    static constexpr uint32_t kInf = 0x7f800000u, kMove = 0x7fffffffu - kInf;
    static __device__ __forceinline__ Key none() { return 0.0; }
    static __device__ __forceinline__ void make(const float* raw, int column, Key* out) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t b = __float_as_uint(raw[i]), s = (uint32_t)((int32_t)b >> 31);
            const int32_t k = max((int32_t)(((b & 0x7fffffffu) ^ s) + (kMove - s)), (int32_t)(kMove - kInf));
            const uint32_t u = (uint32_t)k ^ 0x80000000u;
            out[i] = __builtin_bit_cast(double, (uint64_t)u << 30 | (uint32_t)(0x3ff - column - i));
        }
    }
    static __device__ __forceinline__ int column(Key k) { return 0x3ff - (int)(__builtin_bit_cast(uint64_t, k) & 0x3ffu); }
    static __device__ __forceinline__ float score(Key k) {
        const int32_t v = (int32_t)((uint32_t)(__builtin_bit_cast(uint64_t, k) >> 30) ^ 0x80000000u) - (int32_t)kMove;
        return __uint_as_float((uint32_t)(v < 0 ? -v : v) | (v < 0 ? 0x80000000u : 0u));
    }
    static __device__ __forceinline__ Key larger(Key a, Key b) { return __builtin_fmax(a, b); }
    static __device__ __forceinline__ Key smaller(Key a, Key b) { return __builtin_fmin(a, b); }
    template <int STEP>
    static __device__ __forceinline__ Key from_partner(Key k) {
        const uint64_t b = __builtin_bit_cast(uint64_t, k);
        return __builtin_bit_cast(double, (uint64_t)partner<STEP>((uint32_t)(b >> 32)) << 32 | partner<STEP>((uint32_t)b));
    }
};
template <class Type> struct KeysOf { typedef Keys16<Type> type; };
template <> struct KeysOf<Fp32> { typedef Keys32 type; };

template <class K, int A, int B, int N>
__device__ __forceinline__ void exchange(typename K::Key (&x)[N]) {
    const auto a = x[A], b = x[B];
    x[A] = K::larger(a, b);
    x[B] = K::smaller(a, b);
}
template <class K>
__device__ __forceinline__ void sort_list(typename K::Key (&x)[4]) {   // largest first
    exchange<K, 0, 2>(x); exchange<K, 1, 3>(x);
    exchange<K, 0, 1>(x); exchange<K, 2, 3>(x);
    exchange<K, 1, 2>(x);
}
template <class K>
__device__ __forceinline__ void sort_list(typename K::Key (&x)[8]) {
    exchange<K, 0, 2>(x); exchange<K, 1, 3>(x); exchange<K, 4, 6>(x); exchange<K, 5, 7>(x);
    exchange<K, 0, 4>(x); exchange<K, 1, 5>(x); exchange<K, 2, 6>(x); exchange<K, 3, 7>(x);
    exchange<K, 0, 1>(x); exchange<K, 2, 3>(x); exchange<K, 4, 5>(x); exchange<K, 6, 7>(x);
    exchange<K, 2, 4>(x); exchange<K, 3, 5>(x);
    exchange<K, 1, 4>(x); exchange<K, 3, 6>(x);
    exchange<K, 1, 2>(x); exchange<K, 3, 4>(x); exchange<K, 5, 6>(x);
}
// sorts N keys that rise and fall once
template <class K, int N>
__device__ __forceinline__ void sort_bitonic(typename K::Key* x) {
#pragma unroll
    for (int step = N / 2; step > 0; step /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(i & step)) {
                const auto a = x[i], b = x[i + step];
                x[i] = K::larger(a, b);
                x[i + step] = K::smaller(a, b);
            }
}
template <class K>
__device__ __forceinline__ void sort_list(typename K::Key (&x)[16]) {
    typename K::Key a[8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        a[i] = x[i];
        b[i] = x[8 + i];
    }
    sort_list<K>(a);
    sort_list<K>(b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = K::larger(a[i], b[7 - i]);
        x[8 + i] = K::smaller(a[i], b[7 - i]);
    }
    sort_bitonic<K, 8>(x);
    sort_bitonic<K, 8>(x + 8);
}
// x becomes the largest of two lists, each sorted: the larger of x[i] and y[last - i] are they, and rise and fall once
template <class K, int M>
__device__ __forceinline__ void merge_list(typename K::Key (&x)[M], const typename K::Key (&y)[M]) {
#pragma unroll
    for (int i = 0; i < M; ++i) x[i] = K::larger(x[i], y[M - 1 - i]);
    sort_bitonic<K, M>(x);
}
template <class K, int L, int M, int STEP = 1>
__device__ __forceinline__ void merge_group(typename K::Key (&x)[M]) {
    if constexpr (STEP < L) {
        typename K::Key y[M];
#pragma unroll
        for (int i = 0; i < M; ++i) y[i] = K::template from_partner<STEP>(x[i]);
        merge_list<K>(x, y);
        merge_group<K, L, M, 2 * STEP>(x);
    }
}
template <class K, int L, int STEP = 1>
__device__ __forceinline__ typename K::Key largest_of_group(typename K::Key k) {
    if constexpr (STEP >= L) return k;
    else return largest_of_group<K, L, 2 * STEP>(K::larger(k, K::template from_partner<STEP>(k)));
}

struct RouteOut {
    void* ids;
    int idx_dtype;
    uint16_t* gates;
    __device__ __forceinline__ void put(int64_t i, int id, float gate) const {
        gates[i] = Bf16::narrow(gate);
        if (idx_dtype == 1) ((uint8_t*)ids)[i] = (uint8_t)id;
        else ((int32_t*)ids)[i] = id;
    }
};

template <class Type, int L, int V, bool FULL>
__device__ __forceinline__ float exp_sum(const Row<Type, L, V, FULL>& x, float top) {
    float z = 0.f;
#pragma unroll
    for (int p = 0; p < x.N; ++p)
#pragma unroll
        for (int w = 0; w < x.W; ++w) z += x.has(p, w) ? exp_of(x.at(p, w) - top) : 0.f;
    return group_sum<L>(z);
}

// The weight of a picked score before it is divided by the sum over what its gate is a share of.
__device__ __forceinline__ float gate_weight(int gating, float s, float top) { return gating >= kSigmoid ? sigmoid_of(s, top) : exp_of(s - top); }
__device__ __forceinline__ float gate_shift(int gating, float largest) {
    return gating == kSigmoid ? 0.f : shift_of(gating == kSigmoidNormalised ? fminf(largest, 0.f) : largest);
}

// Ids and gates, k <= M.  A lane sorts its keys in lists of M, merges them to their M largest, and log2(L) more merges with its partners'
// lists leave every lane of the group with the row's, without a branch or memory in between.  262144 tokens, E = 128, k = 8: 21.0 us a
// pass with bf16 scores, 23.2 in a kernel trace (the copy rate would allow 15.3), 36 with fp32 ones in a trace (4.0 TB/s); k rounds of a maximum
// over the group took 51.6 us with bf16.  Bound by vector instructions with 16-bit scores: 383 per wave, 4 cycles each, 32 waves per SIMD are
// 20.4 us at 2.4 GHz (E = 256 44.4 of 48.3 us, 65536 tokens of E = 1024 51 of 57, k = 16 among them 91 of 101).
template <class Type, int L, int V, bool FULL, int M>
__global__ __launch_bounds__(kThreads) void k_route_lists(const typename Type::stored* __restrict__ scores, int64_t ld, int64_t T, int E, int k,
                                                          int gating, const uint8_t* __restrict__ token_mask, RouteOut out) {
    typedef typename KeysOf<Type>::type K;
    typedef typename K::Key Key;
    const int part = threadIdx.x % L;
    const int64_t t = group_of_grid() * (kThreads / L) + threadIdx.x / L;
    const bool here = t < T;
    const auto* row = scores + (here ? t : T - 1) * ld;
    Row<Type, L, V, FULL> x;
    x.place(part, E);
    x.load(row, E);
    const bool masked = token_mask && here && token_mask[t] == 0;
    Key keys[V];
#pragma unroll
    for (int p = 0; p < x.N; ++p) {
        K::make(x.raw[p], x.from[p], keys + p * x.W);
#pragma unroll
        for (int w = 0; w < x.W; ++w) keys[p * x.W + w] = x.has(p, w) ? keys[p * x.W + w] : K::none();
    }
    Key list[M];
#pragma unroll
    for (int a = 0; a < V; a += M) {
        Key next[M];
#pragma unroll
        for (int i = 0; i < M; ++i) next[i] = keys[a + i];
        sort_list<K>(next);
        if (a == 0) {
#pragma unroll
            for (int i = 0; i < M; ++i) list[i] = next[i];
        } else {
            merge_list<K>(list, next);
        }
    }
    merge_group<K, L, M>(list);
    // slot j of the row to lane j % L
    constexpr int S = (M + L - 1) / L;
    const float top = gate_shift(gating, K::score(list[0]));
    float weight[S], z = 0.f;
    int column[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        Key mine = list[i * L];
#pragma unroll
        for (int j = 1; j < L && i * L + j < M; ++j) mine = part == j ? list[i * L + j] : mine;
        const int j = i * L + part;
        column[i] = j < k ? K::column(mine) : 0;
        float s = K::score(mine);
        if (j < k && s == -INFINITY) s = Type::widen(row[column[i]]);     // or NaN, which ranks with it
        weight[i] = j < k ? gate_weight(gating, s, top) : 0.f;
        z += weight[i];
    }
    z = gating == kSoftmaxAll ? exp_sum(x, top) : group_sum<L>(z);
    const float scale = gating == kSigmoid ? 1.f : reciprocal_or_zero(z);
    if (!here) return;
#pragma unroll
    for (int i = 0; i < S; ++i)
        if (i * L + part < k) out.put(t * k + i * L + part, column[i], masked ? 0.f : weight[i] * scale);
}

// Ids and gates for any k: k rounds, each of which takes the largest key left in the group.
template <class Type, int L, int V, bool FULL>
__global__ __launch_bounds__(kThreads) void k_route_rounds(const typename Type::stored* __restrict__ scores, int64_t ld, int64_t T, int E, int k,
                                                           int gating, const uint8_t* __restrict__ token_mask, RouteOut out) {
    typedef typename KeysOf<Type>::type K;
    typedef typename K::Key Key;
    extern __shared__ uint16_t s_pick[];
    const int part = threadIdx.x % L, local = threadIdx.x / L;
    const int64_t t = group_of_grid() * (kThreads / L) + local;
    const bool here = t < T;
    const auto* row = scores + (here ? t : T - 1) * ld;
    uint16_t* pick = s_pick + local * k;
    Row<Type, L, V, FULL> x;
    x.place(part, E);
    x.load(row, E);
    const bool masked = token_mask && here && token_mask[t] == 0;
    Key keys[V];
#pragma unroll
    for (int p = 0; p < x.N; ++p) {
        K::make(x.raw[p], x.from[p], keys + p * x.W);
#pragma unroll
        for (int w = 0; w < x.W; ++w) keys[p * x.W + w] = x.has(p, w) ? keys[p * x.W + w] : K::none();
    }
    float top = 0.f;
    for (int j = 0; j < k; ++j) {
        Key best = keys[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = K::larger(best, keys[v]);
        best = largest_of_group<K, L>(best);
#pragma unroll
        for (int v = 0; v < V; ++v) keys[v] = keys[v] == best ? K::none() : keys[v];
        if (j == 0) top = gate_shift(gating, K::score(best));
        if (part == j % L) pick[j] = (uint16_t)K::column(best);     // read again by this lane alone
    }
    float z = 0.f;
    if (gating == kSoftmaxAll) {
        z = exp_sum(x, top);
    } else {
        for (int j = part; j < k; j += L) z += gate_weight(gating, Type::widen(row[pick[j]]), top);
        z = group_sum<L>(z);
    }
    const float scale = gating == kSigmoid ? 1.f : reciprocal_or_zero(z);
    if (!here) return;
    for (int j = part; j < k; j += L) out.put(t * k + j, pick[j], masked ? 0.f : gate_weight(gating, Type::widen(row[pick[j]]), top) * scale);
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

template <class Out, int W>
__device__ __forceinline__ void store_piece(void* out, int64_t at, int end, const float* v) {
    auto* o = (typename Out::stored*)out + at;
    typename Out::stored q[W];
#pragma unroll
    for (int w = 0; w < W; ++w) q[w] = Out::narrow(v[w]);
    if (end == W) {
        __builtin_memcpy(o, q, sizeof(q));
    } else {
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < end) o[w] = q[w];
    }
}

// Gradient by the scores.  With p the probabilities over all experts, g the gates, q the gradients by the gates' logs and c the
// balance loss's coefficients: p_e (c_e - <c, p>) (times 1 - sigmoid(s_e) for sigmoids), plus at the picked experts q_j - g_j sum q
// (softmax over them), q_j and everywhere -p_e sum q (softmax over all), (1 - sigmoid) q_j or (1 - sigmoid) (q_j - g_j sum q).
// Nothing is divided by a gate, so a gate of 0 has a gradient of 0.  WHOLE: the row's scores are needed, not the picked ones alone.
// One pass: 131072 x 256 fp32 scores to bf16 gradients of the balance loss 31 us (201 MB, 6.5 TB/s, part of the scores from the last-level cache that
// the loss left them in); of picked gates alone, 16384 x 128 bf16, 8 us, most of it the chain ids -> scores -> sums -> stores.
template <class Type, int L, int V, bool FULL, bool WHOLE, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void k_route_bwd(const typename Type::stored* __restrict__ scores, int64_t ld, int64_t T, int E, int gating,
                                                        RouteGrad a) {
    extern __shared__ float s_slot[];    // per token k contributions, then k expert numbers
    constexpr int W = kPiece<Type>, N = V / W;
    const int part = threadIdx.x % L, local = threadIdx.x / L;
    const int64_t t = group_of_grid() * (kThreads / L) + local;
    const bool here = t < T, live = here && !(a.token_mask && a.token_mask[t] == 0);
    const auto* row = scores + (here ? t : T - 1) * ld;
    constexpr bool sigmoid = SIGMOID;
    float ds[V], prob[V];
    Row<Type, L, V, FULL> x;
    x.place(part, E);
#pragma unroll
    for (int v = 0; v < V; ++v) ds[v] = 0.f;
    if (WHOLE) x.load(row, E);
    int64_t s = 0;
    if (WHOLE && a.off) {
        // the sequence of the wave's first token is most often that of all its tokens
        const int64_t first = group_of_grid() * (kThreads / L) + (threadIdx.x & ~63) / L;
        int64_t next;
        s = offsets_up_to(a.off, a.S, first, next);
        if (next < first + 64 / L) {
            int64_t hi = a.S + 1;
            while (s < hi) {
                const int64_t mid = (s + hi) >> 1;
                if (a.off[mid] <= t) s = mid + 1;
                else hi = mid;
            }
        }
        s = s > a.S ? -1 : s - 1;     // behind the last sequence, as before the first: in none
    }
    float scale = 0.f;
    if (WHOLE) scale = shares<SIGMOID>(x, prob);
    if (WHOLE && a.coef) {
        float c[V], dot = 0.f;
        const float* coef = a.coef + (s >= 0 ? s : 0) * E;
#pragma unroll
        for (int p = 0; p < N; ++p) {
            x.fetch(p, coef, E, c + p * W);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) dot += x.has(v / W, v % W) ? c[v] * prob[v] : 0.f;
        dot = group_sum<L>(dot) * scale;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ds[v] = prob[v] * scale * (c[v] - dot);
            if (sigmoid) ds[v] *= sigmoid_of(-x.at(v / W, v % W));
        }
        if (__ballot(s < 0)) {
#pragma unroll
            for (int v = 0; v < V; ++v) ds[v] = s >= 0 ? ds[v] : 0.f;
        }
    }
    if (a.dlog) {
        const int k = a.k;
        const bool shared = gating == kSoftmaxSelected || gating == kSigmoidNormalised;
        float* u = s_slot + local * 2 * k;
        int* e = (int*)(u + k);
        float sum = 0.f, top = -INFINITY, z = 0.f;
        for (int j = part; j < k; j += L) {
            const int id = here ? id_of(a.ids, a.idx_dtype, t * k + j) : -1;
            const bool ok = (unsigned)id < (unsigned)E;
            e[j] = ok ? id : -1;
            u[j] = ok ? a.dlog[t * k + j] : 0.f;
            sum += u[j];
            if (ok && shared) top = fmaxf(top, Type::widen(row[id]));
        }
        sum = group_sum<L>(sum);
        if (shared) {
            top = gate_shift(gating, group_max<L>(top));
            for (int j = part; j < k; j += L)
                if (e[j] >= 0) z += gate_weight(gating, Type::widen(row[e[j]]), top);
            z = group_sum<L>(z);
            // a quotient, not a product with 1 / z: the only one selected has a gate of exactly 1 and a gradient of exactly 0
            for (int j = part; j < k; j += L)
                if (e[j] >= 0 && z != 0.f) u[j] -= sum * (gate_weight(gating, Type::widen(row[e[j]]), top) / z);
        }
        if (sigmoid)
            for (int j = part; j < k; j += L)
                if (e[j] >= 0) u[j] *= sigmoid_of(-Type::widen(row[e[j]]));
        if (WHOLE && gating == kSoftmaxAll) {
#pragma unroll
            for (int v = 0; v < V; ++v) ds[v] -= prob[v] * (scale * sum);
        }
        __syncthreads();
        for (int j = 0; j < k; ++j) {
            const int id = e[j];
            const float w = u[j];
#pragma unroll
            for (int v = 0; v < V; ++v) ds[v] += id == x.from[v / W] + v % W ? w : 0.f;
        }
    }
    if (!here) return;
    if (__ballot(!live)) {
#pragma unroll
        for (int v = 0; v < V; ++v) ds[v] = live ? ds[v] : 0.f;
    }
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const int64_t at = t * a.out_ld + x.from[p];
        if (!FULL && x.skip[p] >= W) continue;     // no element of its own; others are written by both lanes that have them, alike
        const int end = x.kShort ? x.end : W;
        if (a.out_dtype == 0) store_piece<Fp32, W>(a.out, at, end, ds + p * W);
        else if (a.out_dtype == 1) store_piece<Bf16, W>(a.out, at, end, ds + p * W);
        else store_piece<Fp16, W>(a.out, at, end, ds + p * W);
    }
}

}  // namespace

hipError_t launch_route(const void* scores, int dtype, int64_t ld, int64_t T, int E, int k, int gating, const uint8_t* token_mask, void* ids,
                        int idx_dtype, uint16_t* gates, hipStream_t s) {
    const RouteOut out{ids, idx_dtype, gates};
    return with_type(dtype, [&](auto type) {
        return with_lanes(E, [&](auto l, auto v, auto full) {
            typedef decltype(type) Type;
            constexpr int L = decltype(l)::value, V = decltype(v)::value, tokens = kThreads / L;
            constexpr bool FULL = decltype(full)::value;
            const dim3 grid = grid_of((T + tokens - 1) / tokens), threads(kThreads);
            const auto* x = (const typename Type::stored*)scores;
            if (k <= 4) {
                hipLaunchKernelGGL((k_route_lists<Type, L, V, FULL, 4>), grid, threads, 0, s, x, ld, T, E, k, gating, token_mask, out);
            } else if (k <= 8) {
                hipLaunchKernelGGL((k_route_lists<Type, L, V, FULL, 8>), grid, threads, 0, s, x, ld, T, E, k, gating, token_mask, out);
            } else if constexpr (V == 16) {     // (more than 8 experts)
                // Lists of 16 cost the same for 9 and for 16 experts, rounds grow with k (262144 tokens; rounds / lists in us): E = 128, k = 10
                // 38 / 35 with bf16 and 71 / 49 with fp32 scores, k = 16 52 / 35 and 98 / 49; bf16, E = 256 73 / 76 and 98 / 75; a quarter of
                // the tokens with E = 512 37 / 43 and 52 / 43, with E = 1024 74 / 92 and 100 / 91; fp32, E = 1024 138 / 131 and 200 / 127.
                if (k <= 16 && (dtype == 0 || E <= 256 || k > 12))
                    hipLaunchKernelGGL((k_route_lists<Type, L, V, FULL, 16>), grid, threads, 0, s, x, ld, T, E, k, gating, token_mask, out);
                else if constexpr (L > 1)     // (up to 16 experts always have lists)
                    hipLaunchKernelGGL((k_route_rounds<Type, L, V, FULL>), grid, threads, tokens * k * sizeof(uint16_t), s, x, ld, T, E, k, gating,
                                       token_mask, out);
            }
            return hipGetLastError();
        });
    });
}

hipError_t launch_route_bwd(const void* scores, int dtype, int64_t ld, int64_t T, int E, int gating, const uint8_t* token_mask, const void* ids,
                            int idx_dtype, int k, const float* dlog, const int64_t* off, int64_t S, const float* coef, void* out,
                            int out_dtype, int64_t out_ld, hipStream_t s) {
    const RouteGrad a{ids, idx_dtype, k, dlog, off, S, coef, token_mask, out, out_dtype, out_ld};
    return with_type(dtype, [&](auto type) {
        return with_lanes(E, [&](auto l, auto v, auto full) {
            typedef decltype(type) Type;
            constexpr int L = decltype(l)::value, V = decltype(v)::value, tokens = kThreads / L;
            constexpr bool FULL = decltype(full)::value;
            const dim3 grid = grid_of((T + tokens - 1) / tokens);
            const size_t lds = dlog ? tokens * k * 2 * sizeof(float) : 0;
            const auto* x = (const typename Type::stored*)scores;
            return with_flag(gating >= kSigmoid, [&](auto sigmoid) {
                constexpr bool SIGMOID = decltype(sigmoid)::value;
                if (coef || gating == kSoftmaxAll)
                    hipLaunchKernelGGL((k_route_bwd<Type, L, V, FULL, true, SIGMOID>), grid, dim3(kThreads), lds, s, x, ld, T, E, gating, a);
                else
                    hipLaunchKernelGGL((k_route_bwd<Type, L, V, FULL, false, SIGMOID>), grid, dim3(kThreads), lds, s, x, ld, T, E, gating, a);
                return hipGetLastError();
            });
        });
    });
}

}  // namespace grouter
