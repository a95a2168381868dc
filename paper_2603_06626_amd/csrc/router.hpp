// Rows of scores in registers: what the router and the balance loss share.
//
// All of them read a row of E scores per token.  A token belongs to a group of L neighbouring lanes, each of which holds V scores as
// pieces of 16 bytes, piece p of lane i being number p L + i of the row: every load instruction of a group covers whole lines, and
// every reduction over a row is one inside registers and log2(L) cross-lane moves.  V is 16 beyond 8 experts: few cross-lane steps
// (each costs as much as one over all registers), and 64 / L tokens of a wave share the instructions of what follows.
#pragma once
#include "lanes.hpp"

namespace grouter {

namespace {

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
// the value that it has where it is present, and is left out of the sum).  Returns what they are to be multiplied with.  The row's largest
// is subtracted before the product with log2 e: a product of its own would round by up to 2^-24 of a score that may be anything (an expert closed
// by the type's lowest value, in a row of nothing else), and that error would be an exponent.
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
        top = shift_of(top);
#pragma unroll
        for (int v = 0; v < V; ++v) share[v] = exp_of(share[v] - top);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) z += x.has(v / x.W, v % x.W) ? share[v] : 0.f;
    return reciprocal_or_zero(group_sum<L>(z));
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

}  // namespace grouter
