// One AdamW step over a ragged tensor set:
//     g' = c g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//     w = w (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// with the moments in 32 bits, or in 8: m and the root of v as e4m3 codes, one 32-bit scale for each block of 256.
//
// Weights, gradients and moments are read once, weights and moments written once: 22 bytes an element with 16-bit weights and gradients, 10
// with 8-bit moments.  The moments of all tensors lie in one array, every tensor at a multiple of a block; a warp takes a run of
// blocks, finds a block's tensor by searching the tensors' places, and needs nobody else: a block's largest moments are a reduction
// over half a warp.  With 32-bit moments memory is the bound: on one B200 the 1.31e9 bf16 weights of a 24-layer file take 4.65 ms,
// 6.2 TB/s (4.9 with three CTAs per SM, whose 80 registers are too few); 200 packed tensors with 32-bit copies 290 us, 5.8 TB/s.  With 8-bit
// moments it is the instructions, some 54 an element: the same file takes 3.14 ms, 4.2 TB/s, 200 packed tensors with float32 gradients
// 213 us.  Seven small tensors take 5 to 7 us on the device.
//
// The moments' averages change by a part in a thousand a step, far less than an 8-bit code's step, so rounding to nearest would
// hold them where they are.  They are rounded up with the probability that the lost bits give instead, by
// random words that are a hash of (seed, step, element): the same call gives the same bits.
#pragma once
#include "element_dev.cuh"
#include "iv_internal.h"
#include "row_dev.cuh"

namespace ivk {

namespace {

using elem::Pair;
using elem::unpack8;

constexpr uint32_t kBlock = IV_ADAMW_BLOCK;
constexpr uint32_t kWarps = 8;
constexpr uint32_t kGolden = 0x9E3779B9u;      // the golden ratio's fraction

// A hash of 32-bit words; the factors are the fractions of the roots of 2 and 3.
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

struct Coefficients {
    float beta1, rest1, beta2, rest2;          // rest = 1 - beta
    float factor;                              // of the gradients
    float step, root, eps, keep;               // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), eps, 1 - lr decay
    float nothing;                             // -0: a product plus this is the product rounded, which no later addition takes in
    uint32_t key0, key1;
    bool skip;
};

// By one thread, from the number of steps taken and the norm's record as they are on the device.
__device__ __forceinline__ void make_coefficients(const AdamwArgs &a, Coefficients &c) {
    c.skip = false;
    c.factor = 1.f;
    if (a.d_norm) {
        const volatile iv_norm_result *r = a.d_norm;
        c.skip = r->n_nonfinite != 0u;
        const double norm = sqrt(r->sum_squares);
        c.factor = norm <= (double)a.max_norm ? 1.f : (float)((double)a.max_norm / norm);
    }
    const uint64_t t = *reinterpret_cast<const volatile uint64_t *>(a.d_step) + 1u;
    const double lr = a.d_lr ? (double)*reinterpret_cast<const volatile float *>(a.d_lr) : a.lr;
    c.beta1 = a.beta1;
    c.rest1 = a.rest1;
    c.beta2 = a.beta2;
    c.rest2 = a.rest2;
    c.step = (float)(lr / -expm1((double)t * a.log_beta1));
    c.root = (float)(1.0 / sqrt(-expm1((double)t * a.log_beta2)));
    c.eps = a.eps;
    c.nothing = -0.f;
    c.keep = (float)(1.0 - lr * a.weight_decay);
    c.key0 = mix(mix(mix((uint32_t)a.seed + kGolden) + (uint32_t)(a.seed >> 32)) + (uint32_t)t);
    c.key1 = mix(c.key0 + (uint32_t)(t >> 32) + kGolden);
}

// The random words of a group of eight elements: word k is b + (k + 1) a.
struct Words {
    uint32_t b, a;
    __device__ __forceinline__ Words(uint32_t group, const Coefficients &c) {
        b = mix(group ^ c.key0);
        a = mix(b + c.key1);
    }
    __device__ __forceinline__ uint32_t word(uint32_t k) const { return b + (k + 1u) * a; }
};

__device__ __forceinline__ Pair negative(Pair x) {
    float lo, hi;
    x.get(lo, hi);
    return Pair(-lo, -hi);
}
// `better` where it is a number.
__device__ __forceinline__ Pair unless_nan(Pair better, Pair x) {
    float a[2], b[2];
    better.get(a[0], a[1]);
    x.get(b[0], b[1]);
    return Pair(a[0] == a[0] ? a[0] : b[0], a[1] == a[1] ? a[1] : b[1]);
}
// The root by one step of Heron's method: with y near 1 / sqrt(v), s = v y misses the root by (v - s^2) y / 2 but for the square of y's
// error, 2^-45 of it.  So it is the root rounded, to 2^-24, or within 2^-23 where v is below 2^-100 and the difference a small one; NaN
// where 1 / sqrt(v) is none or v is below 2^-126.  With sqrt.approx alone, 2^-23, one code in some 6e6 of the second moments' is not the one that
// elementary operations give.  268M weights, sqrt.approx, this, an IEEE root: 540, 576, 617 us with 8-bit moments, 930, 930, 935 with 32-bit ones.
__device__ __forceinline__ Pair root_of(Pair v) {
    float lo, hi;
    v.get(lo, hi);
    asm("rsqrt.approx.ftz.f32 %0, %0;" : "+f"(lo));
    asm("rsqrt.approx.ftz.f32 %0, %0;" : "+f"(hi));
    const Pair y(lo, hi), s = v * y;
    return fma2(fma2(negative(s), s, v), y * Pair(0.5f), s);
}
// To 2^-23, of any number.
__device__ __forceinline__ Pair root_approx(Pair x) {
    float lo, hi;
    x.get(lo, hi);
    asm("sqrt.approx.f32 %0, %0;" : "+f"(lo));
    asm("sqrt.approx.f32 %0, %0;" : "+f"(hi));
    return Pair(lo, hi);
}
// n / d, d below 2^-126 being taken for 0.  EXACT: what the approximate reciprocal's quotient, within 2^-22, leaves of n gives the rest, to
// 2^-24.  That costs the step with 32-bit moments, which waits for memory, nothing (930 us either way, IEEE divisions 935 to 973); that
// with 8-bit moments has no instructions to spare (IEEE divisions 617 -> 730 us), and 2^-22 of an update is below the
// last place of a weight that the update changes by less than a quarter.
template <bool EXACT>
__device__ __forceinline__ Pair quotient(Pair n, Pair d) {
    float lo, hi;
    d.get(lo, hi);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(lo));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(hi));
    const Pair inverse(lo, hi), q = n * inverse;
    if constexpr (!EXACT) return q;
    else return unless_nan(fma2(fma2(negative(q), d, n), inverse, q), q);
}

// Two 32-bit values as 16-bit ones, with random bits added in the place of those that go; infinities stay, NaN too.
template <typename T> __device__ __forceinline__ uint32_t round_random2(float lo, float hi, uint32_t word_lo, uint32_t word_hi);
template <> __device__ __forceinline__ uint32_t round_random2<__nv_bfloat16>(float lo, float hi, uint32_t word_lo, uint32_t word_hi) {
    // the bits of a NaN that an operation gives, 0x7fffffff, would carry into the sign
    auto sum = [](float x, uint32_t word) { return (uint32_t)min((int32_t)__float_as_uint(x), 0x7fff0000) + (word >> 16); };
    return __byte_perm(sum(lo, word_lo), sum(hi, word_hi), 0x7632);
}
template <> __device__ __forceinline__ uint32_t round_random2<__half>(float lo, float hi, uint32_t word_lo, uint32_t word_hi) {
    auto code = [](float x, uint32_t word) -> uint32_t {
        if (!(fabsf(x) < 65536.f)) return __half_as_ushort(__float2half_rn(x));
        // times 2^-112 a half's exponent and digits, small ones too, are the upper bits of the float's
        return (__float_as_uint(fabsf(x) * 0x1p-112f) + (word >> 19)) >> 13 | __float_as_uint(x) >> 31 << 15;
    };
    return __byte_perm(code(lo, word_lo), code(hi, word_hi), 0x5410);
}

// Eight codes as 32-bit values times a scale.
__device__ __forceinline__ void decode8(uint2 codes, float scale, Pair (&out)[4]) {
    const Pair by(scale);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t lo, hi;
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
            : "=r"(lo), "=r"(hi) : "r"(i ? codes.y : codes.x));
        float a, b;
        elem::unpack2<__half>(lo, a, b);
        out[2 * i] = Pair(a, b) * by;
        elem::unpack2<__half>(hi, a, b);
        out[2 * i + 1] = Pair(a, b) * by;
    }
}

// What a block's values are multiplied by on their way to codes, and its scale.  kTop lies just below the largest code, 448, so
// that no rounding reaches the code behind it, which is NaN; the largest value is taken as 2^-110 at least, so that neither
// factor leaves the range of 32 bits.
constexpr float kTop = 447.9995f;

// Largest magnitude of eight values and `top`; NaN if there is one.
__device__ __forceinline__ float largest(const Pair (&x)[4], float top) {
    float lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i].get(lo, hi);
        asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(lo), "f"(hi));
    }
    return top;
}
// The same over what is finite.
__device__ __forceinline__ float largest_finite(const Pair (&x)[4], float top) {
    float lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i].get(lo, hi);
        if (isfinite(lo)) top = fmaxf(top, fabsf(lo));
        if (isfinite(hi)) top = fmaxf(top, fabsf(hi));
    }
    return top;
}

// A block's factors and scales, from its lanes' largest magnitudes m and v.  WIDTH lanes hold a block: half of them work out the
// first moments', half the roots'.
struct Tops {
    float m_inverse, v_inverse, scale;                   // scale: of the first moments in the block's lower lanes, of the roots in the upper ones
    bool bad;                                            // an infinity or a NaN in a block of the warp
};
template <uint32_t WIDTH, typename F>
__device__ __forceinline__ Tops block_tops(float m, float v, F finite) {
    const bool second = threadIdx.x & (WIDTH / 2u);
    auto reduce = [&](float a, float b) {
        float x = second ? b : a, y = __shfl_xor_sync(0xffffffffu, second ? a : b, WIDTH / 2u);
#pragma unroll
        for (uint32_t d = WIDTH / 4u;; d /= 2u) {
            asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(y));
            if (d == 0u) return x;
            y = __shfl_xor_sync(0xffffffffu, x, d);
        }
    };
    Tops t;
    float top = reduce(m, v);
    t.bad = __any_sync(0xffffffffu, !(top < __uint_as_float(0x7f800000u)));
    if (t.bad) {
        finite(m, v);
        top = reduce(m, v);
    }
    const float root = __fsqrt_rn(top), x = second ? root : top, safe = fmaxf(x, 0x1p-110f);
    const float inverse = x > 0.f ? __fmul_rn(__frcp_rn(safe), kTop) : 0.f;
    t.scale = x > 0.f ? safe * (float)(1.0 / 447.9995) : 0.f;
    t.m_inverse = __shfl_sync(0xffffffffu, inverse, 0, WIDTH);
    t.v_inverse = __shfl_sync(0xffffffffu, inverse, WIDTH / 2u, WIDTH);
    return t;
}

// Codes.  Times 2^-120 a value's exponent and digits, small ones too, are the upper bits of the float's, and 20 random bits are
// added to the 20 that go; four bits further up the code is the upper byte.
__device__ __forceinline__ uint32_t upper_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
__device__ __forceinline__ uint2 upper_bytes(const uint32_t (&x)[8]) {
    return make_uint2(upper_bytes(x[0], x[1], x[2], x[3]), upper_bytes(x[4], x[5], x[6], x[7]));
}
__device__ __forceinline__ bool has_zero_byte(uint32_t w) { return ((w - 0x01010101u) & ~w & 0x80808080u) != 0u; }
constexpr uint32_t kNanCode = 0x7f000000u;

__device__ __forceinline__ uint2 encode_first(const Pair (&m)[4], const Tops &s, const Words &words) {
    uint32_t code[8];
    const Pair inverse(s.m_inverse), shift(0x1p-120f);
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
        float y[2];
        (m[i] * inverse * shift).get(y[0], y[1]);
#pragma unroll
        for (uint32_t k = 0; k < 2u; ++k) {
            const uint32_t sum = __float_as_uint(y[k]) + (words.word(2u * i + k) >> 12);       // the sign stays where it is
            code[2 * i + k] = sum * 16u | (sum & 0x80000000u);
        }
    }
    if (s.bad) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            float x[2];
            m[i / 2].get(x[0], x[1]);
            if (!isfinite(x[i & 1])) code[i] = kNanCode;
        }
    }
    return upper_bytes(code);
}
// Of the roots r of v; one that is not 0 keeps a code that is not 0.
__device__ __forceinline__ uint2 encode_second(const Pair (&v)[4], const Pair (&r)[4], const Tops &s, const Words &words) {
    uint32_t code[8];
    const Pair inverse(s.v_inverse), shift(0x1p-120f);
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
        float y[2];
        (r[i] * inverse * shift).get(y[0], y[1]);
#pragma unroll
        for (uint32_t k = 0; k < 2u; ++k) code[2 * i + k] = (__float_as_uint(y[k]) + (words.word(8u + 2u * i + k) >> 12)) * 16u;
    }
    if (s.bad) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            float x[2];
            v[i / 2].get(x[0], x[1]);
            if (!isfinite(x[i & 1])) code[i] = kNanCode;
        }
    }
    uint2 out = upper_bytes(code);
    if (has_zero_byte(out.x) || has_zero_byte(out.y)) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            float x[2];
            v[i / 2].get(x[0], x[1]);
            if (x[i & 1] > 0.f) code[i] = max(code[i], 1u << 24);
        }
        out = upper_bytes(code);
    }
    return out;
}

// A lane's eight elements.
template <int BITS>
struct Lane {
    Pair w[4], g[4], m[4], v[4], r[4];         // before update(), 8 bits: v holds the roots

    // New moments, roots r and weights.  The moments' products and sums are rounded one by one, so that elementary operations
    // give the same bits.
    __device__ __forceinline__ void update(const Coefficients &c) {
        const Pair factor(c.factor), beta1(c.beta1), rest1(c.rest1), beta2(c.beta2), rest2(c.rest2), root(c.root), eps(c.eps), step(-c.step), keep(c.keep),
            nothing(c.nothing);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Pair g1 = g[i] * factor, square = BITS == 32 ? v[i] : v[i] * v[i];
            m[i] = fma2(m[i], beta1, nothing) + fma2(g1, rest1, nothing);
            v[i] = fma2(square, beta2, nothing) + fma2(g1 * g1, rest2, nothing);
            r[i] = root_of(v[i]);
        }
        float some = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            r[i].get(lo, hi);
            asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(some) : "f"(lo), "f"(hi));
        }
        if (some != some) {                              // 0, a subnormal, infinity or NaN
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = unless_nan(r[i], root_approx(v[i]));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = fma2(w[i], keep, quotient<BITS == 32>(m[i] * step, fma2(r[i], root, eps)));
    }
    // The weights as elements of type T.
    template <typename T>
    __device__ __forceinline__ elem::Packed<T, 8> rounded(bool stochastic, const Words &words) const {
        elem::Packed<T, 8> out;
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i].get(x[2 * i], x[2 * i + 1]);
        if constexpr (sizeof(T) == 2) {
            if (stochastic) {
#pragma unroll
                for (uint32_t i = 0; i < 8u; i += 2u)
                    out.w[i / 2] = round_random2<T>(x[i], x[i + 1], words.word(16u + i), words.word(17u + i));
                return out;
            }
        }
        out.pack(x);
        return out;
    }
};

__device__ __forceinline__ void load8(const float *p, Pair (&x)[4]) {
    asm volatile("ld.global.v4.b64 {%0, %1, %2, %3}, [%4];" : "=l"(x[0].bits), "=l"(x[1].bits), "=l"(x[2].bits), "=l"(x[3].bits) : "l"(p));
}
__device__ __forceinline__ void store8(float *p, const Pair (&x)[4]) {
    asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(x[0].bits), "l"(x[1].bits), "l"(x[2].bits), "l"(x[3].bits) : "memory");
}
// Vectors of consecutive lanes, `width` lanes to a run of elements.  WALIGN: 16 or 8 where they start at such a boundary.  `count` is 8, or 0 to
// store nothing.
template <typename T, int WALIGN>
__device__ __forceinline__ void store_lanes(T *p, const elem::Packed<T, 8> &own, uint32_t count, uint32_t width) {
    constexpr int kStep = WALIGN == 8 ? 2 : 4;
    if (WALIGN > 0 || elem::misalignment(p) == 0u) {
        if (count) {
#pragma unroll
            for (int i = 0; i < elem::Packed<T, 8>::kWords; i += kStep) elem::store_aligned<kStep>(reinterpret_cast<uint32_t *>(p) + i, own.w + i);
        }
    } else {
        rows::store_pieces<T>(p, own, count, width);
    }
}

// A lane's share of a block with 32-bit moments as it lies in memory.
template <typename Tw, typename Tg, bool MASTER, int WALIGN, int GALIGN>
struct Raw {
    elem::Vector<Tg, 8, GALIGN> g;
    elem::Vector<Tw, 8, MASTER ? 16 : WALIGN> w;         // not with MASTER
    Pair master[4], m[4], v[4];
    __device__ __forceinline__ void load(const AdamwArgs &a, uint64_t at, const Tw *pw, const Tg *pg) {
        g.load(pg, elem::misalignment(pg));
        if constexpr (MASTER) load8(a.d_master + at, master);
        else w.load(pw, elem::misalignment(pw));
        load8(static_cast<const float *>(a.d_m) + at, m);
        load8(static_cast<const float *>(a.d_v) + at, v);
    }
    __device__ __forceinline__ void get(const Tw *pw, const Tg *pg, Lane<32> &e) const {
        unpack8(g.get(elem::misalignment(pg)), e.g);
        if constexpr (!MASTER) unpack8(w.get(elem::misalignment(pw)), e.w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (MASTER) e.w[i] = master[i];
            e.m[i] = m[i];
            e.v[i] = v[i];
        }
    }
};

// `count` whole blocks from state element s on, of the tensor whose weights and gradients are at w and g: a block by the warp.
template <typename Tw, typename Tg, bool MASTER, int WALIGN, int GALIGN>
__device__ __forceinline__ void whole_blocks32(const AdamwArgs &a, const Coefficients &c, uint64_t s, uint32_t count, Tw *w, const Tg *g) {
    const uint32_t lane = threadIdx.x & 31u;
    uint64_t at = s + lane * 8u;
    w += lane * 8u;
    g += lane * 8u;
#pragma unroll 1
    for (uint32_t b = 0; b < count; ++b, at += kBlock, w += kBlock, g += kBlock) {
        Raw<Tw, Tg, MASTER, WALIGN, GALIGN> raw;
        Lane<32> e;
        raw.load(a, at, w, g);
        raw.get(w, g, e);
        e.update(c);
        store_lanes<Tw, WALIGN>(w, e.template rounded<Tw>(a.stochastic, Words((uint32_t)(at / 8u), c)), 8u, 32u);
        if constexpr (MASTER) store8(a.d_master + at, e.w);
        store8(static_cast<float *>(a.d_m) + at, e.m);
        store8(static_cast<float *>(a.d_v) + at, e.v);
    }
}
// With 8-bit moments half a warp takes a block, sixteen elements a lane in two vectors half a block apart: what a block costs
// beside its elements (tops, scales, addresses) is shared by twice as many.  Two blocks of a warp come through a ring in shared
// memory that the warp fills with asynchronous copies, two steps ahead (268M bf16 weights: 560 us where a block per warp and
// the next one in registers took 617).
template <typename Tw, typename Tg, bool MASTER>
struct Ring {
    // 16-byte pieces of half a block, at any alignment: weights, gradients, the 32-bit weights, the two moments' codes
    static constexpr uint32_t kW = MASTER ? 0u : 8u * sizeof(Tw) + 1u, kG = 8u * sizeof(Tg) + 1u, kMaster = MASTER ? 32u : 0u;
    static constexpr uint32_t kAtG = kW, kAtMaster = kAtG + kG, kAtM = kAtMaster + kMaster, kAtV = kAtM + 8u, kHalf = kAtV + 8u;
    static constexpr uint32_t kStep = 4u * kHalf + 1u;   // two halves of two blocks, and their four scales
    static constexpr int kStages = 3u * 16u * kStep * kWarps <= (108u << 10) ? 3 : 2;
    static constexpr uint32_t kBytes = 16u * kStep * kStages * kWarps;
    static_assert(2u * kBytes <= 220u << 10, "two CTAs per SM");
};
template <int BYTES>
__device__ __forceinline__ void copy_async_small(void *shared, const void *global) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(global), "n"(BYTES) : "memory");
}

template <typename Tw, typename Tg, bool MASTER, int WALIGN, int GALIGN>
__device__ __forceinline__ void whole_blocks8(const AdamwArgs &a, const Coefficients &c, uint4 *ring, uint64_t s, uint32_t count, Tw *w, const Tg *g) {
    using R = Ring<Tw, Tg, MASTER>;
    using W = rows::Segment<Tw, 16, (WALIGN > 0) ? rows::kExactRows : rows::kShiftedRows>;
    using G = rows::Segment<Tg, 16, GALIGN == 16 ? rows::kExactRows : rows::kShiftedRows>;
    using M = rows::Segment<float, 16, rows::kExactRows>;
    constexpr uint32_t kHalf = kBlock / 2u;
    constexpr int kStages = R::kStages;
    const uint32_t lane = threadIdx.x & 15u, half = threadIdx.x >> 4 & 1u;
    // this half warp's block in step i; where there is none the other half's, of which it stores nothing
    auto block_of = [&](uint32_t i) { return 2u * i + half < count ? 2u * i + half : 2u * i; };
    auto fetch = [&](uint32_t i, uint4 *to) {
        const uint32_t first = block_of(i) * kBlock;
        const uint64_t at = s + first;
#pragma unroll
        for (uint32_t j = 0; j < 2u; ++j) {
            uint4 *const here = to + (half * 2u + j) * R::kHalf;
            const uint32_t e = first + j * kHalf;
            if constexpr (MASTER) {
                M::fetch(here + R::kAtMaster, a.d_master + s + e, lane, lane, kHalf);
            } else if constexpr (WALIGN == 8) {            // pieces of 8 bytes bring them to 16-byte boundaries
#pragma unroll
                for (uint32_t i = 0; i < sizeof(Tw); ++i)
                    copy_async_small<8>(reinterpret_cast<uint2 *>(here) + i * 16u + lane, reinterpret_cast<const uint8_t *>(w + e) + (i * 16u + lane) * 8u);
            } else {
                W::fetch(here, w + e, lane, lane, kHalf);
            }
            G::fetch(here + R::kAtG, g + e, lane, lane, kHalf);
            copy_async_small<8>(reinterpret_cast<uint2 *>(here + R::kAtM) + lane, static_cast<const uint8_t *>(a.d_m) + s + e + lane * 8u);
            copy_async_small<8>(reinterpret_cast<uint2 *>(here + R::kAtV) + lane, static_cast<const uint8_t *>(a.d_v) + s + e + lane * 8u);
        }
        if ((lane & 7u) == 0u)
            copy_async_small<4>(reinterpret_cast<float *>(to + 4u * R::kHalf) + half * 2u + lane / 8u, (lane ? a.d_v_scales : a.d_m_scales) + at / kBlock);
    };
    const uint32_t steps = (count + 1u) / 2u;
    __syncwarp();                                        // the warp has read what the run of blocks before left in the ring
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
        if ((uint32_t)i < steps) fetch(i, ring + i * R::kStep);
        rows::commit_copies();
    }
    uint32_t now = 0, last = (kStages - 1) * R::kStep;
#pragma unroll 1
    for (uint32_t i = 0; i < steps; ++i) {
        __syncwarp();                                    // and what it is filled with again now
        if (i + kStages - 1u < steps) fetch(i + kStages - 1u, ring + last);
        rows::commit_copies();
        rows::wait_copies<kStages - 1>();
        __syncwarp();
        const uint4 *const from = ring + now;
        const bool live = 2u * i + half < count;
        const uint32_t first = block_of(i) * kBlock + lane * 8u;
        const uint64_t at = s + first;
        const float2 scales = *(reinterpret_cast<const float2 *>(from + 4u * R::kHalf) + half);
        Lane<8> e[2];
        float m_top = 0.f, v_top = 0.f;
#pragma unroll
        for (uint32_t j = 0; j < 2u; ++j) {
            const uint4 *const here = from + (half * 2u + j) * R::kHalf;
            Tw *const pw = w + first + j * kHalf;
            const Tg *const pg = g + first + j * kHalf;
            if constexpr (MASTER) unpack8(M::get(here + R::kAtMaster, 0u, lane, lane, kHalf, true), e[j].w);
            else unpack8(W::get(here, elem::misalignment(pw), lane, lane, kHalf, true), e[j].w);
            unpack8(G::get(here + R::kAtG, elem::misalignment(pg), lane, lane, kHalf, true), e[j].g);
            decode8(reinterpret_cast<const uint2 *>(here + R::kAtM)[lane], scales.x, e[j].m);
            decode8(reinterpret_cast<const uint2 *>(here + R::kAtV)[lane], scales.y, e[j].v);
            e[j].update(c);
            m_top = largest(e[j].m, m_top);
            v_top = largest(e[j].v, v_top);
            store_lanes<Tw, WALIGN>(pw, e[j].template rounded<Tw>(a.stochastic, Words((uint32_t)(at / 8u) + j * (kHalf / 8u), c)), live ? 8u : 0u, 16u);
            if constexpr (MASTER)
                if (live) store8(a.d_master + at + j * kHalf, e[j].w);
        }
        const Tops tops = block_tops<16>(m_top, v_top, [&](float &m, float &v) {
            m = largest_finite(e[1].m, largest_finite(e[0].m, 0.f));
            v = largest_finite(e[1].v, largest_finite(e[0].v, 0.f));
        });
#pragma unroll
        for (uint32_t j = 0; j < 2u; ++j) {
            const Words words((uint32_t)(at / 8u) + j * (kHalf / 8u), c);
            const uint2 m = encode_first(e[j].m, tops, words), v = encode_second(e[j].v, e[j].r, tops, words);
            if (live) {
                *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.d_m) + at + j * kHalf) = m;
                *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.d_v) + at + j * kHalf) = v;
            }
        }
        if (live && (lane & 7u) == 0u) (lane ? a.d_v_scales : a.d_m_scales)[at / kBlock] = tops.scale;
        last = now;
        now = now + R::kStep == kStages * R::kStep ? 0u : now + R::kStep;
    }
}
template <typename Tw, typename Tg, int BITS, bool MASTER, int WALIGN, int GALIGN>
__device__ __forceinline__ void whole_blocks(const AdamwArgs &a, const Coefficients &c, uint4 *ring, uint64_t s, uint32_t count, Tw *w, const Tg *g) {
    if constexpr (BITS == 32) whole_blocks32<Tw, Tg, MASTER, WALIGN, GALIGN>(a, c, s, count, w, g);
    else whole_blocks8<Tw, Tg, MASTER, WALIGN, GALIGN>(a, c, ring, s, count, w, g);
}

// A tensor's last block: one element at a time; what lies behind the tensor stays as it is.
template <typename Tw, typename Tg, int BITS, bool MASTER>
__device__ __noinline__ void part_block(const AdamwArgs &a, const Coefficients &c, uint64_t s, uint32_t left, Tw *w, const Tg *g) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t at = s + lane * 8u;
    const uint32_t count = left > lane * 8u ? (left - lane * 8u < 8u ? left - lane * 8u : 8u) : 0u;
    Lane<BITS> e;
    w += lane * 8u;
    g += lane * 8u;
    float x[4][8];                                       // weights, gradients, moments
    if constexpr (BITS == 8) {
        decode8(*reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.d_m) + at), a.d_m_scales[s / kBlock], e.m);
        decode8(*reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.d_v) + at), a.d_v_scales[s / kBlock], e.v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e.m[i].get(x[2][2 * i], x[2][2 * i + 1]);
            e.v[i].get(x[3][2 * i], x[3][2 * i + 1]);
        }
        __syncwarp();                                    // every lane has the scales
    }
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        const bool there = i < count;
        if constexpr (MASTER) x[0][i] = there ? a.d_master[at + i] : 0.f;
        else x[0][i] = there ? elem::to_float(w[i]) : 0.f;
        x[1][i] = there ? elem::to_float(g[i]) : 0.f;
        if constexpr (BITS == 32) {
            x[2][i] = there ? static_cast<const float *>(a.d_m)[at + i] : 0.f;
            x[3][i] = there ? static_cast<const float *>(a.d_v)[at + i] : 0.f;
        } else {
            x[2][i] = there ? x[2][i] : 0.f;
            x[3][i] = there ? x[3][i] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e.w[i] = Pair(x[0][2 * i], x[0][2 * i + 1]);
        e.g[i] = Pair(x[1][2 * i], x[1][2 * i + 1]);
        e.m[i] = Pair(x[2][2 * i], x[2][2 * i + 1]);
        e.v[i] = Pair(x[3][2 * i], x[3][2 * i + 1]);
    }
    e.update(c);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        float y[2];
        e.m[i / 2].get(y[0], y[1]);
        x[2][i] = i < count ? y[i & 1] : 0.f;            // 0 * infinity, if the gradients' factor is that
        e.v[i / 2].get(y[0], y[1]);
        x[3][i] = i < count ? y[i & 1] : 0.f;
        e.w[i / 2].get(y[0], y[1]);
        x[0][i] = y[i & 1];
    }
    const Words words((uint32_t)(at / 8u), c);
    uint2 m_codes, v_codes;
    if constexpr (BITS == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e.m[i] = Pair(x[2][2 * i], x[2][2 * i + 1]);
            e.v[i] = Pair(x[3][2 * i], x[3][2 * i + 1]);
        }
        const Tops tops = block_tops<32>(largest(e.m, 0.f), largest(e.v, 0.f), [&](float &m, float &v) {
            m = largest_finite(e.m, 0.f);
            v = largest_finite(e.v, 0.f);
        });
        m_codes = encode_first(e.m, tops, words);
        v_codes = encode_second(e.v, e.r, tops, words);
        if ((lane & 15u) == 0u) (lane ? a.d_v_scales : a.d_m_scales)[s / kBlock] = tops.scale;
    }
    const elem::Packed<Tw, 8> out = e.template rounded<Tw>(a.stochastic, words);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        if (i >= count) continue;
        if constexpr (sizeof(Tw) == 4) reinterpret_cast<uint32_t *>(w)[i] = out.w[i];
        else reinterpret_cast<uint16_t *>(w)[i] = (uint16_t)(out.w[i / 2] >> (16u * (i & 1u)));
        if constexpr (MASTER) a.d_master[at + i] = x[0][i];
        if constexpr (BITS == 32) {
            static_cast<float *>(a.d_m)[at + i] = x[2][i];
            static_cast<float *>(a.d_v)[at + i] = x[3][i];
        } else {
            static_cast<uint8_t *>(a.d_m)[at + i] = (uint8_t)((i < 4u ? m_codes.x : m_codes.y) >> (8u * (i & 3u)));
            static_cast<uint8_t *>(a.d_v)[at + i] = (uint8_t)((i < 4u ? v_codes.x : v_codes.y) >> (8u * (i & 3u)));
        }
    }
}

// The last tensor whose place is at or before s; by the whole warp, 32 places at a time (0 if there is none).
__device__ __forceinline__ uint64_t tensor_at(const uint64_t *places, uint64_t n, uint64_t s) {
    const uint32_t lane = threadIdx.x & 31u;
    uint64_t lo = 0, count = n;
    while (count > 1) {
        const uint64_t step = (count + 31u) / 32u, at = lane * step;
        const uint32_t found = __popc(__ballot_sync(0xffffffffu, at < count && places[lo + at] <= s));
        const uint64_t part = found ? found - 1u : 0u;
        lo += part * step;
        count = count - part * step < step ? count - part * step : step;
    }
    return lo;
}

// Tensor k of the set; elements is 0 for one that is ill-formed: a length, an address or a place that is not a multiple of its
// unit, or no room up to the next tensor's place (or the state's end).
template <typename Tw, typename Tg>
struct Tensor {
    uint64_t place, elements;
    Tw *w;
    const Tg *g;
    bool good;
    __device__ __forceinline__ Tensor(const AdamwArgs &a, uint64_t k) {
        place = a.d_state_offsets[k];
        const uint64_t bytes = a.set.d_lengths[k];
        const uint64_t end = k + 1u < a.set.n ? a.d_state_offsets[k + 1u] : a.size;
        w = reinterpret_cast<Tw *>(a.set.d_base + a.set.d_offsets[k]);
        g = reinterpret_cast<const Tg *>(a.d_grads + a.d_grad_offsets[k]);
        elements = bytes / sizeof(Tw);
        good = bytes % sizeof(Tw) == 0u && reinterpret_cast<uintptr_t>(w) % sizeof(Tw) == 0u && reinterpret_cast<uintptr_t>(g) % sizeof(Tg) == 0u &&
               place % kBlock == 0u && place <= end && end <= a.size && elements <= end - place;
        if (!good) elements = 0u;
    }
};

template <typename Tw, typename Tg, int BITS, bool MASTER>
__global__ void __launch_bounds__(kWarps * 32, 2)
adamw_kernel(const __grid_constant__ AdamwArgs a, uint32_t run, uint32_t *arrived, uint32_t *status) {
    __shared__ Coefficients shared;
    extern __shared__ uint4 rings[];                     // 8 bits only
    uint4 *ring = nullptr;
    if constexpr (BITS == 8) ring = rings + (threadIdx.x >> 5) * (Ring<Tw, Tg, MASTER>::kStep * Ring<Tw, Tg, MASTER>::kStages);
    allow_next_kernel();
    wait_for_previous_kernel();
    if (threadIdx.x == 0) make_coefficients(a, shared);
    __syncthreads();
    for (uint64_t k = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; k < a.set.n; k += (uint64_t)gridDim.x * blockDim.x)
        if (!Tensor<Tw, Tg>(a, k).good) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
    if (shared.skip) return;
    const uint64_t blocks = a.set.n ? a.size / kBlock : 0u, warps = (uint64_t)gridDim.x * kWarps;
    uint64_t from = 1, to = 0;                           // the blocks' elements of the tensor at hand
    Tw *w = nullptr;
    const Tg *g = nullptr;
    uint64_t elements_end = 0;
    for (uint64_t first = ((uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * run; first < blocks; first += warps * run) {
        const uint64_t last = first + run < blocks ? first + run : blocks;
        for (uint64_t b = first; b < last;) {
            const uint64_t s = b * kBlock;
            if (s < from || s >= to) {
                const uint64_t k = tensor_at(a.d_state_offsets, a.set.n, s);
                const Tensor<Tw, Tg> tensor(a, k);
                from = tensor.place;
                to = k + 1u < a.set.n ? a.d_state_offsets[k + 1u] : a.size;
                elements_end = from + tensor.elements;
                w = tensor.w;
                g = tensor.g;
            }
            if (s < from || s >= elements_end) {
                ++b;
                continue;
            }
            Tw *wb = w + (s - from);
            const Tg *gb = g + (s - from);
            const uint64_t whole = (elements_end - s) / kBlock;
            if (whole == 0u) {
                part_block<Tw, Tg, BITS, MASTER>(a, shared, s, (uint32_t)(elements_end - s), wb, gb);
                ++b;
                continue;
            }
            const uint32_t count = (uint32_t)(whole < last - b ? whole : last - b), w_off = elem::misalignment(wb), g_off = elem::misalignment(gb);
            if (g_off == 0u && w_off == 0u) whole_blocks<Tw, Tg, BITS, MASTER, 16, 16>(a, shared, ring, s, count, wb, gb);
            else if (g_off == 0u && w_off == 8u) whole_blocks<Tw, Tg, BITS, MASTER, 8, 16>(a, shared, ring, s, count, wb, gb);
            else whole_blocks<Tw, Tg, BITS, MASTER, elem::kAny, elem::kAny>(a, shared, ring, s, count, wb, gb);
            b += count;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && arrive_add(arrived, 1u) + 1u == gridDim.x) {
        *arrived = 0u;                                   // every CTA has read the number of steps
        *a.d_step += 1u;
    }
}

template <typename Tw, typename Tg, int BITS, bool MASTER>
cudaError_t launch_instance(const AdamwArgs &a, uint32_t *arrived, uint32_t *d_status, int sm_count, cudaStream_t stream) {
    const uint64_t blocks = a.size / kBlock, ctas = (blocks + kWarps - 1) / kWarps, most = (uint64_t)sm_count * 2u;
    const uint32_t grid = (uint32_t)(ctas < most ? (ctas ? ctas : 1u) : most);
    const uint64_t share = blocks / ((uint64_t)grid * kWarps);
    constexpr uint64_t kRun = BITS == 8 ? 32 : 16;
    const uint32_t run = (uint32_t)(share < 1u ? 1u : share < kRun ? share : kRun);
    auto kernel = adamw_kernel<Tw, Tg, BITS, MASTER>;
    uint32_t bytes = 0;
    if constexpr (BITS == 8) {
        bytes = Ring<Tw, Tg, MASTER>::kBytes;
        static bool done[kMaxDevices] = {};
        cudaError_t e = ensure_dynamic_smem(kernel, bytes, done);
        if (e != cudaSuccess) return e;
    }
    return launch_overlapping(kernel, dim3(grid), dim3(kWarps * 32), bytes, stream, a, run, arrived, d_status);
}

}  // namespace

template <typename Tw, typename Tg>
cudaError_t adamw_typed(const AdamwArgs &a, uint32_t *arrived, uint32_t *d_status, int sm_count, cudaStream_t stream) {
    if constexpr (sizeof(Tw) == 2)
        if (a.d_master)
            return a.bits == 8 ? launch_instance<Tw, Tg, 8, true>(a, arrived, d_status, sm_count, stream)
                               : launch_instance<Tw, Tg, 32, true>(a, arrived, d_status, sm_count, stream);
    return a.bits == 8 ? launch_instance<Tw, Tg, 8, false>(a, arrived, d_status, sm_count, stream)
                       : launch_instance<Tw, Tg, 32, false>(a, arrived, d_status, sm_count, stream);
}

}  // namespace ivk
