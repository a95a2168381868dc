// One AdamW step over many tensors: with g the scaled gradient,
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  w = w - (lr wd w + lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)).
//
// A pass over memory and little else: 22 to 30 bytes per element with 32-bit moments, 10 to 18 with 8-bit ones.  554 M elements with fp32
// masters and moments and bf16 gradients 2.88 ms (5.4 TB/s; a large copy reaches 4.8), in bf16 with 8-bit moments 1.04 to 1.06 ms (5.3 to
// 5.4 TB/s; 1.07 to 1.12 ms in a kernel trace), where 606 vector instructions per wave take as long by count: 4 cycles each, 1056 waves per
// SIMD, 1.07 ms at 2.4 GHz.  A launch takes the
// addresses of up to kAdamwPerLaunch tensors in its arguments (nothing to copy to the device first, and a graph holds them by value);
// its workgroups are dealt to the tensors by size.
//
// 8-bit moments.  m and r = sqrt(v) are e4m3 numbers (4 exponent bits, 3 mantissa bits, largest 448) times a power of two per 32
// neighbours, the smallest under which the largest is at most 448.  A root spans in 8 bits what v would need 16 binades more for.
// Both are rounded up or down with the probability of the remainder: v changes by a thousandth per step at b2 = 0.999, which rounding to
// nearest would throw away every time.  A root above zero never becomes zero (a step divided by eps alone would follow), a block with an
// infinity or NaN becomes NaN as a whole.  The random bits are a function of the element's number and the seed: of a word's 32, m takes the
// upper 20 (all that a remainder has), the root the lower 12 and what kFineBelow says, a bf16 parameter the upper 16, which are m's too.
//
// The moments are computed with separately rounded products and sums (no fused multiply-add), so that their codes follow from the
// formulas alone.
#include "lanes.hpp"

#include <type_traits>

#pragma clang fp contract(off)

namespace grouter {

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;                            // elements under one exponent

enum ParamKind { kFp32Param = 0, kMasterParam = 1, kBf16Param = 2 };

// Elements of a thread: 4, which are 16 bytes of every fp32 stream, so that a wave's loads are whole lines one after the other; 8 where no
// stream is that wide.  Measured on 12 bf16 tensors of 262144 with fp32 masters and moments, 75 fp32 ones of up to 300001 with 8-bit
// moments, 554 M elements of the former kind and as many in bf16 with 8-bit moments: 4 elements 15.2, 41.2, 2880, 1230 us, 8 elements
// 16.6, 45.4, 2977, 1150, 16 elements 22.1, 59.0, 3477, 1138.  One such piece per thread and no loop: two to eight in a row took 1.1 times
// as long.
constexpr int each_of(int kind, bool grad_bf16, bool eight) { return kind == kBf16Param && grad_bf16 && eight ? 8 : 4; }

struct Batch {
    AdamwTensor tensor[kAdamwPerLaunch];
    uint32_t first_group[kAdamwPerLaunch + 1];        // workgroups before each tensor
    uint64_t first_place[kAdamwPerLaunch];            // elements before each tensor, every tensor rounded up to whole blocks
    int count;
    AdamwHyper hyper;
    const AdamwHyper* hyper_device;
    const float* grad_scale;
};
static_assert(sizeof(Batch) <= 4000, "a launch's arguments are limited to 4 KB");

// 32 random bits of an element, from its place in the list and the seed: noise_of(first_noise(place, seed) + j) for the j-th behind one
// whose place is a multiple of 4 or 8, j below that
__device__ __forceinline__ uint32_t first_noise(uint64_t place, uint32_t seed) {
    return (uint32_t)place + (uint32_t)(place >> 32) * 0x632BE5ABu + seed * 0x9E3779B1u;
}
__device__ __forceinline__ uint32_t noise_of(uint32_t h) {
    h ^= h >> 16;
    h *= 0xA3D95FA9u;
    h ^= h >> 15;
    h *= 0x7B1D4E65u;
    return h ^ (h >> 16);
}

// A root without gradients decays by (1 - beta2)/2 of itself per step, 8 to 16 times that of a code: at beta2 = 1 - 2^-10 16 of 4096 at
// least, so that the word's lower 12 bits and a half of one keep the rate to 1/32 of it.  Closer to 1 the remainder is below that
// resolution (0.9999: rates up to a fifth off, 0.99999: codes never move); there the word's product with an odd number gives 8 bits in the
// half's place, which for every value of the 12 take all values equally often.  554 M elements in bf16 with 8-bit moments 1044 us,
// 1038 without the choice, 1060 where the bits are taken.
constexpr float kFineBelow = 0x1p-10f;

// sqrt(v) to 1 unit; the hardware's takes what is below 2^-126 for 0, so where a wave holds such numbers (zeros mostly) all go the longer way
template <int N>
__device__ __forceinline__ void roots_of(const float (&v)[N], float (&root)[N]) {
    float least = v[0];
#pragma unroll
    for (int j = 1; j < N; ++j) least = fminf(least, v[j]);
    if (__ballot(least < 0x1p-96f)) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const bool small = v[j] < 0x1p-96f;
            root[j] = __builtin_amdgcn_sqrtf(small ? v[j] * 0x1p64f : v[j]) * (small ? 0x1p-32f : 1.f);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) root[j] = __builtin_amdgcn_sqrtf(v[j]);
    }
}
__device__ __forceinline__ float power_of_two(int biased) {   // 2^(biased - 127); 255 is NaN
    return __uint_as_float(biased == 255 ? 0x7fc00000u : biased == 0 ? 0x00400000u : (uint32_t)biased << 23);
}
// e4m3 codes of x >= 0 times 2^(127 - exp); up: 20 random bits each.  Numbers below 2^-6 (less than a 28000th of the block's largest) have
// codes in equal steps, and blocks that are not finite one code for all: both are looked at only where a wave has some.  ROOT: x is the
// hardware's root of v, off by up to one unit; where that could make another code (two of 2^20 random numbers), the root is taken
// again, rounded to nearest, so that the code is that of the formula on every machine.
template <bool ROOT, int N>
__device__ __forceinline__ void codes_of(const float (&x)[N], const float (&v)[N], int exp, const uint32_t (&up)[N], uint32_t (&code)[N]) {
    const float scale = power_of_two(254 - exp);
    float y[N], least = INFINITY;
    uint32_t nearest = 2;     // how near a sum's low bits come to the next code, from either side
#pragma unroll
    for (int j = 0; j < N; ++j) {
        y[j] = x[j] * scale;
        least = fminf(least, y[j]);
        const uint32_t sum = __float_as_uint(y[j]) + up[j];
        if (ROOT) nearest = min(nearest, (sum + 1) & 0xfffffu);
        code[j] = min((sum >> 20) - 960u, 126u);
    }
    if (__ballot(least < 0x1p-6f || exp == 255 || (ROOT && nearest < 2))) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (ROOT) y[j] = (float)__builtin_sqrt((double)v[j]) * scale;
            const uint32_t normal = min(((__float_as_uint(y[j]) + up[j]) >> 20) - 960u, 126u);
            const uint32_t small = (uint32_t)(y[j] * 512.f + (float)up[j] * 0x1p-20f);
            code[j] = exp == 255 ? 127u : y[j] < 0x1p-6f ? small : normal;
        }
    }
}
__device__ __forceinline__ void decode4(uint32_t codes, float scale, float* out) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    out[0] = a.x * scale;
    out[1] = a.y * scale;
    out[2] = b.x * scale;
    out[3] = b.y * scale;
}

constexpr int min_of(int a, int b) { return a < b ? a : b; }

// kEach elements from place `at` on; not WHOLE: n of them there, the others 0
template <class Type, int kEach, bool WHOLE>
__device__ __forceinline__ void fetch(const void* p, int64_t at, int n, typename Type::stored* out) {
    const auto* q = (const typename Type::stored*)p + at;
    if (WHOLE) {
        __builtin_memcpy(out, __builtin_assume_aligned(q, min_of(16, kEach * (int)sizeof(*q))), kEach * sizeof(*q));
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) out[i] = i < n ? q[i] : typename Type::stored(0);
    }
}
template <int kEach, bool WHOLE, class T>
__device__ __forceinline__ void put(T* p, int64_t at, int n, const T* v) {
    if (WHOLE) {
        __builtin_memcpy(__builtin_assume_aligned(p + at, min_of(16, kEach * (int)sizeof(T))), v, sizeof(T) * kEach);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i < n) p[at + i] = v[i];
    }
}
struct Byte {
    typedef uint8_t stored;
};

// The step of kEach elements.  WHOLE: the workgroup's elements all exist, so that every stream is one or two loads without a branch,
// all on their way before the first is waited for (a choice per stream between whole and single loads had the compiler wait after each).
template <int KIND, class Grad, bool EIGHT, bool WHOLE>
__device__ __forceinline__ void step(const AdamwTensor& t, const AdamwHyper& h, float scale, uint64_t place, int64_t at, int n) {
    constexpr int kEach = each_of(KIND, std::is_same_v<Grad, Bf16>, EIGHT);
    typedef std::conditional_t<KIND == kBf16Param, Bf16, Fp32> Weight;
    typedef std::conditional_t<EIGHT, Byte, Fp32> Moment;
    typename Grad::stored raw_g[kEach];
    typename Weight::stored raw_w[kEach];
    typename Moment::stored raw_m[kEach], raw_v[kEach];
    const int64_t from = WHOLE || n > 0 ? at : 0;
    fetch<Grad, kEach, WHOLE>(t.grad, from, n, raw_g);
    fetch<Weight, kEach, WHOLE>(KIND == kMasterParam ? t.master : t.param, from, n, raw_w);
    fetch<Moment, kEach, WHOLE>(t.m, from, n, raw_m);
    fetch<Moment, kEach, WHOLE>(t.v, from, n, raw_v);
    float m[kEach], v[kEach], w[kEach], root[kEach];
    if constexpr (EIGHT) {
        const float sm = power_of_two(t.m_exp[from / kBlock]), sv = power_of_two(t.v_exp[from / kBlock]);
#pragma unroll
        for (int j = 0; j < kEach; j += 4) {
            uint32_t a, b;
            __builtin_memcpy(&a, raw_m + j, 4);
            __builtin_memcpy(&b, raw_v + j, 4);
            decode4(a, sm, m + j);
            decode4(b, sv, v + j);
        }
        if (!WHOLE) {     // zero times a block that is NaN
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                m[j] = j < n ? m[j] : 0.f;
                v[j] = j < n ? v[j] : 0.f;
            }
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] = v[j] * v[j];
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            m[j] = raw_m[j];
            v[j] = raw_v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const float s = Grad::widen(raw_g[j]) * scale;
        w[j] = Weight::widen(raw_w[j]);
        m[j] = m[j] * h.beta1 + s * h.one_minus_beta1;
        v[j] = v[j] * h.beta2 + s * s * h.one_minus_beta2;
    }
    roots_of(v, root);
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        w[j] = w[j] - (w[j] * h.decay + m[j] * __builtin_amdgcn_rcpf(root[j] * h.inv_root_correction + h.eps) * h.step_size);
    uint32_t noise[kEach];
    if (EIGHT || KIND == kBf16Param) {
        const uint32_t first = first_noise(place + at, h.seed);
#pragma unroll
        for (int j = 0; j < kEach; ++j) noise[j] = noise_of(first + j);
    }
    if (KIND == kFp32Param) put<kEach, WHOLE>((float*)t.param, at, n, w);
    if (KIND == kMasterParam) put<kEach, WHOLE>(t.master, at, n, w);
    if (KIND != kFp32Param) {
        uint16_t b[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            b[j] = Bf16::narrow(w[j]);
            if (KIND == kBf16Param) {   // a step is often less than half a unit of bf16: up or down with the probability of the remainder
                const uint32_t u = __float_as_uint(w[j]);
                b[j] = (u & 0x7fffffffu) < 0x7f800000u ? (uint16_t)((u + (noise[j] >> 16)) >> 16) : b[j];
            }
        }
        put<kEach, WHOLE>((uint16_t*)t.param, at, n, b);
    }
    if (!EIGHT) {
        put<kEach, WHOLE>((float*)t.m, at, n, m);
        put<kEach, WHOLE>((float*)t.v, at, n, v);
    } else {
        uint32_t pm = 0, pv = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (!WHOLE && j >= n) m[j] = v[j] = root[j] = 0.f;     // (a scale that is not finite makes NaN of no gradient, too)
            pm = max(pm, __float_as_uint(m[j]) & 0x7fffffffu);
            pv = max(pv, __float_as_uint(v[j]));
        }
        pm = group_max<kBlock / kEach>(pm);
        pv = group_max<kBlock / kEach>(pv);
        // the least power of two under which the largest is at most 448 = 1.75 * 2^8; for the root of v, 1.75^2 = 3.0625 per 4^k
        const int em = pm >= 0x7f800000u ? 255 : max((int)((pm + 0x1fffffu) >> 23) - 8, 0);
        // (numbers below 2^-126 have no leading bit to go by: 56 fits them all)
        const int ev = pv >= 0x7f800000u ? 255 : pv - 1u < 0x7fffffu ? 56 : (((int)pv - (127 << 23) + 0x3bffff) >> 24) + 119;
        uint32_t up[kEach], code[kEach];
        float size[kEach];
        uint8_t cm[kEach], cv[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            size[j] = fabsf(m[j]);
            up[j] = noise[j] >> 12;
        }
        codes_of<false>(size, size, em, up, code);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            cm[j] = (uint8_t)(code[j] | (__float_as_uint(m[j]) >> 31 << 7));
            up[j] = (noise[j] & 0xfffu) << 8 | 128u;
        }
        if (h.one_minus_beta2 < kFineBelow) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) up[j] = (up[j] & ~0xffu) | noise[j] * 0x85EBCA6Du >> 24;
        }
        codes_of<true>(root, v, ev, up, code);
#pragma unroll
        for (int j = 0; j < kEach; ++j) cv[j] = (uint8_t)(v[j] > 0.f ? max(code[j], 1u) : code[j]);
        put<kEach, WHOLE>((uint8_t*)t.m, at, n, cm);
        put<kEach, WHOLE>((uint8_t*)t.v, at, n, cv);
        if ((WHOLE || n > 0) && at % kBlock == 0) {
            t.m_exp[at / kBlock] = (uint8_t)em;
            t.v_exp[at / kBlock] = (uint8_t)ev;
        }
    }
}

template <int KIND, class Grad, bool EIGHT>
__global__ __launch_bounds__(kThreads) void k_adamw(const Batch batch) {
    const uint32_t group = (uint32_t)group_of_grid();
    if (group >= batch.first_group[batch.count]) return;
    int i = 0;
    for (int step = 32; step > 0; step /= 2)
        if (i + step < batch.count && batch.first_group[i + step] <= group) i += step;
    const AdamwTensor t = batch.tensor[i];
    const AdamwHyper h = batch.hyper_device ? *batch.hyper_device : batch.hyper;
    const float scale = batch.grad_scale ? h.grad_scale * *batch.grad_scale : h.grad_scale;
    constexpr int kEach = each_of(KIND, std::is_same_v<Grad, Bf16>, EIGHT);
    constexpr int64_t kPerGroup = kThreads * kEach;
    const int64_t begin = (int64_t)(group - batch.first_group[i]) * kPerGroup, at = begin + (int64_t)threadIdx.x * kEach;
    if (begin + kPerGroup <= t.n) step<KIND, Grad, EIGHT, true>(t, h, scale, batch.first_place[i], at, kEach);
    else step<KIND, Grad, EIGHT, false>(t, h, scale, batch.first_place[i], at, (int)max((int64_t)0, min((int64_t)kEach, t.n - at)));
}

template <int KIND, class Grad, bool EIGHT>
hipError_t launch(const Batch& b, unsigned groups, hipStream_t s) {
    hipLaunchKernelGGL((k_adamw<KIND, Grad, EIGHT>), grid_of(groups), dim3(kThreads), 0, s, b);
    return hipGetLastError();
}

hipError_t launch_batch(const Batch& b, unsigned groups, int kind, int grad_dtype, int bits, hipStream_t s) {
    if (groups == 0) return hipSuccess;
#define GROUTER_CASE(KIND)                                                                                      \
    if (kind == KIND) {                                                                                         \
        if (grad_dtype == 0) return bits == 8 ? launch<KIND, Fp32, true>(b, groups, s) : launch<KIND, Fp32, false>(b, groups, s); \
        return bits == 8 ? launch<KIND, Bf16, true>(b, groups, s) : launch<KIND, Bf16, false>(b, groups, s);   \
    }
    GROUTER_CASE(kFp32Param)
    GROUTER_CASE(kMasterParam)
    GROUTER_CASE(kBf16Param)
#undef GROUTER_CASE
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_adamw(const AdamwTensor* tensors, int count, int param_kind, int grad_dtype, int state_bits, const AdamwHyper* host,
                        const AdamwHyper* device, const float* grad_scale, hipStream_t s) {
    Batch b{};
    if (host) b.hyper = *host;
    b.hyper_device = device;
    b.grad_scale = grad_scale;
    const uint64_t per_group = (uint64_t)kThreads * each_of(param_kind, grad_dtype == 1, state_bits == 8);
    uint64_t place = 0;
    uint64_t groups = 0;
    auto flush = [&]() {
        b.first_group[b.count] = (uint32_t)groups;
        const hipError_t e = launch_batch(b, (unsigned)groups, param_kind, grad_dtype, state_bits, s);
        b.count = 0;
        groups = 0;
        return e;
    };
    for (int i = 0; i < count; ++i) {
        const uint64_t need = ((uint64_t)tensors[i].n + per_group - 1) / per_group;
        if (tensors[i].n > 0) {
            if (b.count == kAdamwPerLaunch || groups + need > 0x7fffffffu) {
                const hipError_t e = flush();
                if (e != hipSuccess) return e;
            }
            b.tensor[b.count] = tensors[i];
            b.first_group[b.count] = (uint32_t)groups;
            b.first_place[b.count] = place;
            ++b.count;
            groups += need;
        }
        place += ((uint64_t)tensors[i].n + kBlock - 1) / kBlock * kBlock;
    }
    return flush();
}

}  // namespace grouter
