// The router of an expert layer: scores -> expert ids and gate weights (Eq. 2, r = g(TopK(s, k))), the way back, and the balance loss
// with per-expert counts.
//
// All of them read a row of E scores per token.  A token belongs to a group of L neighbouring lanes, each of which holds V scores as
// pieces of 16 bytes, piece p of lane i being number p L + i of the row: every load instruction of a group covers whole lines, and
// every reduction over a row is one inside registers and log2(L) cross-lane moves.  V is 16 beyond 8 experts: few cross-lane steps
// (each costs as much as one over all registers), and 64 / L tokens of a wave share the instructions of what follows.
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

template <class Type>
constexpr int kPiece = 16 / sizeof(typename Type::stored);

// What a lane holds of a row: N pieces of W columns.  A piece that would reach behind column E is fetched from earlier columns, so that
// only the row's own elements are read, and its first `skip` elements count as absent (they belong to the piece before).  Rows
// shorter than a piece are fetched one by one.  Addresses need no more than the elements' own alignment.  FULL: E = L V, nothing is
// absent and nothing has to be compared for it.
template <class Type, int L, int V, bool FULL>
struct Row {
    static constexpr int W = kPiece<Type>, N = V / W;
    static constexpr bool kShort = L == 1 && V == 8 && !FULL;     // E may be less than a piece
    typename Type::stored raw[N][W];
    int from[N], skip[N], end;     // columns from .. from + W - 1, elements skip .. end - 1 present
    __device__ __forceinline__ void place(int part, int E) {
        end = kShort ? min(E, W) : W;
#pragma unroll
        for (int p = 0; p < N; ++p) {
            const int start = (p * L + part) * W;
            from[p] = FULL ? start : max(0, min(start, E - W));
            skip[p] = FULL ? 0 : min(start - from[p], W);
        }
    }
    // W elements of a row of anything, where the lane's piece p is
    template <class T>
    __device__ __forceinline__ void fetch(int p, const T* __restrict__ row, int E, T* out) const {
        if (kShort && E < W) {
#pragma unroll
            for (int w = 0; w < W; ++w) out[w] = w < E ? row[w] : T(0);
        } else {
            __builtin_memcpy(out, row + from[p], W * sizeof(T));
        }
    }
    __device__ __forceinline__ void load(const typename Type::stored* __restrict__ row, int E) {
#pragma unroll
        for (int p = 0; p < N; ++p) fetch(p, row, E, raw[p]);
    }
    __device__ __forceinline__ bool has(int p, int w) const { return FULL || (w >= skip[p] && (!kShort || w < end)); }
    // where column e stands when all lanes' pieces are put side by side: in the last piece that is not whole, behind the absent ones
    static __device__ __forceinline__ int place_of(int e, int E) {
        const int whole = E / W * W;
        return FULL || E < W || e < whole ? e : e + W - E % W;
    }
    __device__ __forceinline__ float at(int p, int w) const { return Type::widen(raw[p][w]); }
};

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
// x becomes the largest of two lists, each sorted: the larger of x[i] and y[last - i] are they, and rise and fall once
template <class K>
__device__ __forceinline__ void merge_list(typename K::Key (&x)[4], const typename K::Key (&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = K::larger(x[i], y[3 - i]);
    exchange<K, 0, 2>(x); exchange<K, 1, 3>(x);
    exchange<K, 0, 1>(x); exchange<K, 2, 3>(x);
}
template <class K>
__device__ __forceinline__ void merge_list(typename K::Key (&x)[8], const typename K::Key (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = K::larger(x[i], y[7 - i]);
    exchange<K, 0, 4>(x); exchange<K, 1, 5>(x); exchange<K, 2, 6>(x); exchange<K, 3, 7>(x);
    exchange<K, 0, 2>(x); exchange<K, 1, 3>(x); exchange<K, 4, 6>(x); exchange<K, 5, 7>(x);
    exchange<K, 0, 1>(x); exchange<K, 2, 3>(x); exchange<K, 4, 5>(x); exchange<K, 6, 7>(x);
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
// lists leave every lane of the group with the row's.  No branch, no memory in between: for 128 experts, k = 8 and 16-bit scores about
// 25 of the 60 instructions per token; k rounds of a maximum over the group take twice as many.
template <class Type, int L, int V, bool FULL, int M>
__global__ __launch_bounds__(kThreads) void k_route_lists(const typename Type::stored* __restrict__ scores, int64_t ld, int64_t T, int E, int k,
                                                          int gating, const uint8_t* __restrict__ token_mask, RouteOut out) {
    typedef typename KeysOf<Type>::type K;
    typedef typename K::Key Key;
    const int part = threadIdx.x % L;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
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
    const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + local;
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

__device__ __forceinline__ int id_of(const void* ids, int idx_dtype, int64_t i) {
    return idx_dtype == 1 ? (int)((const uint8_t*)ids)[i] : (int)((const int32_t*)ids)[i];
}

// v of one lane, the same for all: a scalar
__device__ __forceinline__ int64_t of_lane(int64_t v, int lane) {
    const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane), high = (uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane);
    return (int64_t)((uint64_t)high << 32 | low);
}

// How many of the S + 1 ascending offsets are at most t, t the same in all lanes, and the offset after them (INT64_MAX behind the last):
// 64 probes at a time, so up to 63 sequences take a single load.  Sequence s holds the tokens [off[s], off[s + 1]).
__device__ __forceinline__ int64_t offsets_up_to(const int64_t* __restrict__ off, int64_t S, int64_t t, int64_t& next) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = S + 1;
    next = INT64_MAX;
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, probe = lo + (lane + 1) * step - 1;
        const int64_t value = probe < hi ? off[probe] : INT64_MAX;
        const int passed = __popcll(__ballot(value <= t));
        if (passed < 64) {
            const int64_t above = of_lane(value, passed);
            if (above != INT64_MAX) next = above;     // else the one that an earlier round of probes found
        }
        lo += passed * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

// What the probabilities over all experts of a row are shares of, softmax or sigmoids, for all that a lane fetched (an absent element has
// the value that it has where it is present, and is left out of the sum).  Returns what they are to be multiplied with.  The shift goes into the product with log2 e as a fused sum: its rounding is
// the same for all of a row, so no share depends on it.
template <bool SIGMOID, class Type, int L, int V, bool FULL>
__device__ __forceinline__ float shares(const Row<Type, L, V, FULL>& x, float (&share)[V]) {
    float top = -INFINITY, z = 0.f;
#pragma unroll
    for (int p = 0; p < x.N; ++p)
#pragma unroll
        for (int w = 0; w < x.W; ++w) {
            share[p * x.W + w] = !x.kShort || w < x.end ? x.at(p, w) : -INFINITY;     // (nothing was fetched behind a short row)
            top = fmaxf(top, share[p * x.W + w]);
        }
    top = group_max<L>(top);
    if (SIGMOID) {
        top = shift_of(fminf(top, 0.f));
#pragma unroll
        for (int v = 0; v < V; ++v) share[v] = sigmoid_of(share[v], top);
    } else {
        top = shift_of(top) * 1.44269504f;
#pragma unroll
        for (int v = 0; v < V; ++v) share[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(share[v], 1.44269504f, -top));
    }
#pragma unroll
    for (int v = 0; v < V; ++v) z += x.has(v / x.W, v % x.W) ? share[v] : 0.f;
    return reciprocal_or_zero(group_sum<L>(z));
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
template <class Type, int L, int V, bool FULL, bool WHOLE, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void k_route_bwd(const typename Type::stored* __restrict__ scores, int64_t ld, int64_t T, int E, int gating,
                                                        RouteGrad a) {
    extern __shared__ float s_slot[];    // per token k contributions, then k expert numbers
    constexpr int W = kPiece<Type>, N = V / W;
    const int part = threadIdx.x % L, local = threadIdx.x / L;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + local;
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
        const int64_t first = (int64_t)blockIdx.x * (kThreads / L) + (threadIdx.x & ~63) / L;
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

// ---- balance loss -------------------------------------------------------------------------------------------------------------
// Per sequence s of n tokens: f_e = count_e / (k n), P_e = mean of p_e, loss = alpha E sum_e f_e P_e, and what the gradient needs,
// coef_e = alpha E f_e / n.  The tokens are cut into chunks of equal length, one per workgroup; the part of a sequence inside a chunk
// leaves its sums in a slot of its own, chunk + sequence (both only grow along the tokens, so no two parts share one), and a second
// launch adds up each sequence's slots in order.  So work is even whatever the sequences' lengths, and no float is added atomically.
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

constexpr int kPartThreads = 256;
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
    const int64_t c0 = begin / parts.rows, c1 = begin < end ? (end - 1) / parts.rows + 1 : c0;
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

template <bool B>
struct Flag {
    static constexpr bool value = B;
};
// Calls f with the lanes per token and the scores per lane that E experts take, and whether E fills them.
template <class F>
hipError_t with_lanes(int E, F f) {
#define GROUTER_LANES(L, V)                                                                                         \
    if (E == L * V) return f(std::integral_constant<int, L>{}, std::integral_constant<int, V>{}, Flag<true>{});     \
    if (E < L * V) return f(std::integral_constant<int, L>{}, std::integral_constant<int, V>{}, Flag<false>{})
    GROUTER_LANES(1, 8);
    GROUTER_LANES(1, 16);
    GROUTER_LANES(2, 16);
    GROUTER_LANES(4, 16);
    GROUTER_LANES(8, 16);
    GROUTER_LANES(16, 16);
    GROUTER_LANES(32, 16);
    GROUTER_LANES(64, 16);
#undef GROUTER_LANES
    return hipErrorInvalidValue;
}
template <class F>
hipError_t with_flag(bool b, F f) { return b ? f(Flag<true>{}) : f(Flag<false>{}); }
int lanes_of(int E) {
    int l = 1;
    while (l * 16 < E) l *= 2;
    return l;
}
template <class F>
hipError_t with_type(int dtype, F f) {
    if (dtype == 0) return f(Fp32{});
    if (dtype == 1) return f(Bf16{});
    return f(Fp16{});
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
            const dim3 grid((unsigned)((T + tokens - 1) / tokens)), threads(kThreads);
            const auto* x = (const typename Type::stored*)scores;
            if (k <= 4) hipLaunchKernelGGL((k_route_lists<Type, L, V, FULL, 4>), grid, threads, 0, s, x, ld, T, E, k, gating, token_mask, out);
            else if (k <= 8) hipLaunchKernelGGL((k_route_lists<Type, L, V, FULL, 8>), grid, threads, 0, s, x, ld, T, E, k, gating, token_mask, out);
            else hipLaunchKernelGGL((k_route_rounds<Type, L, V, FULL>), grid, threads, tokens * k * sizeof(uint16_t), s, x, ld, T, E, k, gating, token_mask, out);
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
            const dim3 grid((unsigned)((T + tokens - 1) / tokens));
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

// Chunks: a few per CU at most, so that a sequence's slots are few, and not below the tokens that a workgroup takes at a time.
BalanceLayout balance_layout(int64_t T, int E, int64_t S) {
    BalanceLayout l{};
    const int64_t at_once = kPartThreads / lanes_of(E), rows = (T + 511) / 512;
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
    // many slots per sequence: 64 threads to an expert's; few: 4
    if (S < 8)
        hipLaunchKernelGGL((k_balance_join<16, 1024>), dim3((unsigned)S, (unsigned)(E + 15) / 16), dim3(1024), 0, s, T, E, k, token_mask, off, S, parts, out);
    else
        hipLaunchKernelGGL((k_balance_join<64, 256>), dim3((unsigned)S, (unsigned)(E + 63) / 64), dim3(256), 0, s, T, E, k, token_mask, off, S, parts, out);
    return hipGetLastError();
}

}  // namespace grouter
