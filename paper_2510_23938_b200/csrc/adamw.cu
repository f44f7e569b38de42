// One AdamW step over a ragged tensor set:
//     g' = c g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//     w = w (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// with the moments in 32 bits, or in 8: m and the root of v as e4m3 codes, one 32-bit scale for each block of 256.
//
// Bound by memory: weights, gradients and moments are read once, weights and moments written once (22 bytes an element with
// 16-bit weights and gradients, 10 with 8-bit moments).  The moments of all tensors lie in one array, every tensor at a multiple of
// a block; a warp takes a block at a time, eight elements a lane, finds its tensor by searching the tensors' places,
// and needs nobody else: a block's largest moments are a warp's reduction.
//
// The moments' averages change by a part in a thousand a step, far less than an 8-bit code's step, so rounding to nearest would
// hold them where they are.  They are rounded up with the probability that the lost bits give instead, by
// random words that are a hash of (seed, step, element): the same call gives the same bits.
#include "element_dev.cuh"
#include "iv_internal.h"

namespace ivk {

namespace {

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

__device__ __forceinline__ float root_approx(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A 32-bit value rounded to a 16-bit type by random bits in the place of those that go; infinities and NaN as they are.
template <typename T> __device__ __forceinline__ T round_random(float x, uint32_t word);
template <> __device__ __forceinline__ float round_random<float>(float x, uint32_t) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 round_random<__nv_bfloat16>(float x, uint32_t word) {
    const uint32_t bits = __float_as_uint(x);
    if ((bits & 0x7f800000u) == 0x7f800000u) return __float2bfloat16_rn(x);
    return __ushort_as_bfloat16((uint16_t)((bits + (word >> 16)) >> 16));
}
template <> __device__ __forceinline__ __half round_random<__half>(float x, uint32_t word) {
    if (!(fabsf(x) < 65536.f)) return __float2half_rn(x);
    // times 2^-112 a half's exponent and digits, small ones too, are the upper bits of the float's
    const uint32_t code = (__float_as_uint(fabsf(x) * 0x1p-112f) + (word >> 19)) >> 13;
    return __ushort_as_half((uint16_t)(code | (__float_as_uint(x) >> 31 << 15)));
}

// Four codes of a word as 32-bit values.
__device__ __forceinline__ void decode4(uint32_t w, float *out) {
    uint32_t lo, hi;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    elem::unpack2<__half>(lo, out[0], out[1]);
    elem::unpack2<__half>(hi, out[2], out[3]);
}

// What a block's values are multiplied by on their way to codes, and its scale.  kTop lies just below the largest code, 448, so
// that no rounding reaches the code behind it, which is NaN; the largest value is taken as 2^-110 at least, so that neither
// factor leaves the range of 32 bits.
constexpr float kTop = 447.9995f;
struct BlockScale {
    float inverse, scale;
    bool bad;                                  // an infinity or a NaN in the block; the scale is the others'
};
__device__ __forceinline__ BlockScale block_scale(float top, bool bad) {
    const float safe = fmaxf(top, 0x1p-110f);
    return {top > 0.f ? __fmul_rn(__frcp_rn(safe), kTop) : 0.f, top > 0.f ? safe * (float)(1.0 / 447.9995) : 0.f, bad};
}

// The largest of a warp's values, which are not negative or are looked at without their sign; infinities and NaN left out.
__device__ __forceinline__ float block_top(const float (&x)[8], bool &bad) {
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    bad = top >= 0x7f800000u;
    if (bad) {
        top = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = __float_as_uint(x[i]) & 0x7fffffffu;
            top = max(top, bits < 0x7f800000u ? bits : 0u);
        }
        top = __reduce_max_sync(0xffffffffu, top);
    }
    return __uint_as_float(top);
}

// A lane's eight elements of a block.
template <typename Tw, typename Tg, int BITS, bool MASTER>
struct Lane {
    float w[8], g[8], m[8], r[8];              // r: second moments (32 bits) or their roots (8 bits)

    // New moments and weights; r becomes the roots.  The moments' products and sums are rounded one by one, so that elementary
    // operations give the same bits; the root and the quotient are approximate to 2^-22 of an update, which is small against the
    // weight that it changes.
    __device__ __forceinline__ void update(const Coefficients &c, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float g1 = __fmul_rn(g[i], c.factor), square = BITS == 32 ? r[i] : __fmul_rn(r[i], r[i]);
            m[i] = __fadd_rn(__fmul_rn(m[i], c.beta1), __fmul_rn(g1, c.rest1));
            v[i] = __fadd_rn(__fmul_rn(square, c.beta2), __fmul_rn(__fmul_rn(g1, g1), c.rest2));
            r[i] = root_approx(v[i]);
            w[i] = fmaf(w[i], c.keep, -__fdividef(m[i] * c.step, fmaf(r[i], c.root, c.eps)));
        }
    }
};

__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
    uint32_t b[8];
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3]), "=r"(b[4]),
                 "=r"(b[5]), "=r"(b[6]), "=r"(b[7]) : "l"(p));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(b[i]);
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(x[i]);
    elem::store_32_bytes(p, b);
}

// A warp's 256 consecutive elements at any element alignment: every lane but the last stores the aligned pieces that begin in its
// elements, with its neighbour's first bytes behind its own; what lies before the first and behind the last goes one by one.
template <typename T>
__device__ __forceinline__ void store_warp(T *p, const elem::Packed<T, 8> &own) {
    constexpr int W = elem::Packed<T, 8>::kWords;
    const uint32_t lane = threadIdx.x & 31u, off = elem::misalignment(p);
    if (off == 0u) {
#pragma unroll
        for (int i = 0; i < W; i += 4) elem::store_aligned<4>(reinterpret_cast<uint32_t *>(p) + i, own.w + i);
        return;
    }
    if (off == 8u) {
#pragma unroll
        for (int i = 0; i < W; i += 2) elem::store_aligned<2>(reinterpret_cast<uint32_t *>(p) + i, own.w + i);
        return;
    }
    uint32_t x[W + 4];
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = own.w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[W + i] = __shfl_down_sync(0xffffffffu, own.w[i], 1);
    const uint32_t skip = 16u - off;                     // bytes of this lane before its first piece
    if (skip & 8u) {
#pragma unroll
        for (int i = 0; i < W + 2; ++i) x[i] = x[i + 2];
    }
    if (skip & 4u) {
#pragma unroll
        for (int i = 0; i < W + 1; ++i) x[i] = x[i + 1];
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = __funnelshift_r(x[i], x[i + 1], (skip & 2u) * 8u);
    }
    uint32_t *pieces = reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(p) + skip);
#pragma unroll
    for (int i = 0; i < W; i += 4)
        if (lane < 31u || i + 4 < W) elem::store_aligned<4>(pieces + i, x + i);
    // the first lane's elements before its first piece, the last one's behind its last whole piece
    const uint32_t head = skip / (uint32_t)sizeof(T), tail = (uint32_t)(sizeof(T) * 8u - off) / (uint32_t)sizeof(T);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i)
        if ((lane == 0u && i < head) || (lane == 31u && i >= tail)) {
            if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(p)[i] = own.w[i];
            else reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(own.w[i / 2] >> (16u * (i & 1u)));
        }
}

// Codes of eight values into two words.  Times 2^-120 a value's exponent and digits, small ones too, are the upper bits of the
// float's, and 20 random bits are added to the 20 that go.  Infinities and NaN give 0x7f, NaN.
__device__ __forceinline__ uint32_t pack_codes(const uint32_t *c) { return c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24; }
__device__ __forceinline__ uint32_t code_of(uint32_t bits, uint32_t word) { return (bits + (word >> 12)) >> 20; }
__device__ __forceinline__ uint2 encode_first(const float (&m)[8], const BlockScale &s, const Words &words) {
    uint32_t code[8];
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        code[i] = code_of(__float_as_uint(fabsf(m[i]) * s.inverse * 0x1p-120f), words.word(i));
        if (s.bad && !isfinite(m[i])) code[i] = 0x7fu;
        code[i] |= __float_as_uint(m[i]) >> 24 & 0x80u;
    }
    return make_uint2(pack_codes(code), pack_codes(code + 4));
}
// Of the roots, which stay above zero once they are.  `top` is the exact root of the block's largest finite v: the element that has it
// gets the code that the exact root has (the approximate ones are taken 2^-21 larger and no larger than it).
__device__ __forceinline__ uint2 encode_second(const float (&r)[8], float top, const BlockScale &s, const Words &words) {
    uint32_t code[8];
    const float inverse = s.inverse * (1.f + 0x1p-21f);
    const uint32_t cap = __float_as_uint(top * s.inverse * 0x1p-120f);
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        code[i] = code_of(min(__float_as_uint(r[i] * inverse * 0x1p-120f), cap), words.word(8u + i));
        code[i] = max(code[i], min(__float_as_uint(r[i]), 1u));
        if (s.bad && !isfinite(r[i])) code[i] = 0x7fu;
    }
    return make_uint2(pack_codes(code), pack_codes(code + 4));
}

// The new moments' codes and scales; r: the approximate roots of v.
__device__ __forceinline__ void encode_block(const float (&m)[8], const float (&v)[8], const float (&r)[8], const Words &words, uint2 &m_codes,
                                             uint2 &v_codes, float &m_scale, float &v_scale) {
    bool bad;
    const float m_top = block_top(m, bad);
    const BlockScale first = block_scale(m_top, bad);
    const float v_top = __fsqrt_rn(block_top(v, bad));
    const BlockScale second = block_scale(v_top, bad);
    m_codes = encode_first(m, first, words);
    v_codes = encode_second(r, v_top, second, words);
    m_scale = first.scale;
    v_scale = second.scale;
}

// One block: state elements s .. s + 255, of which `left` belong to the tensor whose weights and gradients are at w and g.
template <typename Tw, typename Tg, int BITS, bool MASTER, int WALIGN, int GALIGN>
__device__ __forceinline__ void whole_block(const AdamwArgs &a, const Coefficients &c, uint64_t s, Tw *w, const Tg *g) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t at = s + lane * 8u;
    Lane<Tw, Tg, BITS, MASTER> e;
    w += lane * 8u;
    g += lane * 8u;
    elem::Vector<Tw, 8, WALIGN> raw_w;
    elem::Vector<Tg, 8, GALIGN> raw_g;
    const uint32_t w_off = elem::misalignment(w), g_off = elem::misalignment(g);
    uint2 m8, v8;
    float m_scale = 1.f, v_scale = 1.f;
    raw_g.load(g, g_off);
    if constexpr (BITS == 32) {
        load8(static_cast<const float *>(a.d_m) + at, e.m);
        load8(static_cast<const float *>(a.d_v) + at, e.r);
    } else {
        m8 = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.d_m) + at);
        v8 = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.d_v) + at);
        m_scale = a.d_m_scales[s / kBlock];
        v_scale = a.d_v_scales[s / kBlock];
    }
    if constexpr (MASTER) load8(a.d_master + at, e.w);
    else {
        raw_w.load(w, w_off);
        raw_w.get(w_off).unpack(e.w);
    }
    raw_g.get(g_off).unpack(e.g);
    if constexpr (BITS == 8) {
        decode4(m8.x, e.m);
        decode4(m8.y, e.m + 4);
        decode4(v8.x, e.r);
        decode4(v8.y, e.r + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e.m[i] *= m_scale;
            e.r[i] *= v_scale;
        }
    }
    float v[8];
    e.update(c, v);
    const Words words((uint32_t)(at / 8u), c);
    if constexpr (MASTER) store8(a.d_master + at, e.w);
    elem::Packed<Tw, 8> out;
    if (sizeof(Tw) == 2 && a.stochastic) {
        if constexpr (sizeof(Tw) == 2) {
#pragma unroll
            for (uint32_t i = 0; i < 8u; i += 2u) {
                const Tw lo = round_random<Tw>(e.w[i], words.word(16u + i)), hi = round_random<Tw>(e.w[i + 1], words.word(17u + i));
                out.w[i / 2] = (uint32_t)*reinterpret_cast<const uint16_t *>(&lo) | (uint32_t)*reinterpret_cast<const uint16_t *>(&hi) << 16;
            }
        }
    } else {
        out.pack(e.w);
    }
    store_warp<Tw>(w, out);
    if constexpr (BITS == 32) {
        store8(static_cast<float *>(a.d_m) + at, e.m);
        store8(static_cast<float *>(a.d_v) + at, v);
    } else {
        uint2 m_codes, v_codes;
        float new_m, new_v;
        encode_block(e.m, v, e.r, words, m_codes, v_codes, new_m, new_v);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.d_m) + at) = m_codes;
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.d_v) + at) = v_codes;
        if (lane == 0u) {
            a.d_m_scales[s / kBlock] = new_m;
            a.d_v_scales[s / kBlock] = new_v;
        }
    }
}

// A tensor's last block: one element at a time; what lies behind the tensor stays as it is.
template <typename Tw, typename Tg, int BITS, bool MASTER>
__device__ __noinline__ void part_block(const AdamwArgs &a, const Coefficients &c, uint64_t s, uint32_t left, Tw *w, const Tg *g) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t at = s + lane * 8u;
    const uint32_t count = left > lane * 8u ? (left - lane * 8u < 8u ? left - lane * 8u : 8u) : 0u;
    Lane<Tw, Tg, BITS, MASTER> e;
    w += lane * 8u;
    g += lane * 8u;
    uint2 m8 = make_uint2(0u, 0u), v8 = m8;
    float m_scale = 1.f, v_scale = 1.f;
    if constexpr (BITS == 8) {
        m8 = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.d_m) + at);
        v8 = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.d_v) + at);
        m_scale = a.d_m_scales[s / kBlock];
        v_scale = a.d_v_scales[s / kBlock];
        decode4(m8.x, e.m);
        decode4(m8.y, e.m + 4);
        decode4(v8.x, e.r);
        decode4(v8.y, e.r + 4);
        __syncwarp();                                    // every lane has the scales
    }
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        const bool there = i < count;
        e.g[i] = there ? elem::to_float(g[i]) : 0.f;
        if constexpr (MASTER) e.w[i] = there ? a.d_master[at + i] : 0.f;
        else e.w[i] = there ? elem::to_float(w[i]) : 0.f;
        if constexpr (BITS == 32) {
            e.m[i] = there ? static_cast<const float *>(a.d_m)[at + i] : 0.f;
            e.r[i] = there ? static_cast<const float *>(a.d_v)[at + i] : 0.f;
        } else {
            e.m[i] = there ? e.m[i] * m_scale : 0.f;
            e.r[i] = there ? e.r[i] * v_scale : 0.f;
        }
    }
    float v[8];
    e.update(c, v);
    const Words words((uint32_t)(at / 8u), c);
    uint2 m_codes, v_codes;
    if constexpr (BITS == 8) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i)
            if (i >= count) e.m[i] = e.r[i] = v[i] = 0.f;       // 0 * infinity, if the gradients' factor is that
        float new_m, new_v;
        encode_block(e.m, v, e.r, words, m_codes, v_codes, new_m, new_v);
        if (lane == 0u) {
            a.d_m_scales[s / kBlock] = new_m;
            a.d_v_scales[s / kBlock] = new_v;
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        if (i >= count) continue;
        w[i] = a.stochastic ? round_random<Tw>(e.w[i], words.word(16u + i)) : elem::from_float<Tw>(e.w[i]);
        if constexpr (MASTER) a.d_master[at + i] = e.w[i];
        if constexpr (BITS == 32) {
            static_cast<float *>(a.d_m)[at + i] = e.m[i];
            static_cast<float *>(a.d_v)[at + i] = v[i];
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
__global__ void __launch_bounds__(kWarps * 32, 3)
adamw_kernel(const __grid_constant__ AdamwArgs a, uint32_t run, uint32_t *arrived, uint32_t *status) {
    __shared__ Coefficients shared;
    if (threadIdx.x == 0) make_coefficients(a, shared);
    __syncthreads();
    const Coefficients c = shared;
    for (uint64_t k = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; k < a.set.n; k += (uint64_t)gridDim.x * blockDim.x)
        if (!Tensor<Tw, Tg>(a, k).good) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
    if (c.skip) return;
    const uint64_t blocks = a.set.n ? a.size / kBlock : 0u, warps = (uint64_t)gridDim.x * kWarps;
    uint64_t from = 1, to = 0;                           // the blocks' elements of the tensor at hand
    Tw *w = nullptr;
    const Tg *g = nullptr;
    uint64_t elements_end = 0;
    for (uint64_t first = ((uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * run; first < blocks; first += warps * run) {
        const uint64_t last = first + run < blocks ? first + run : blocks;
        for (uint64_t b = first; b < last; ++b) {
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
            if (s < from || s >= elements_end) continue;
            Tw *wb = w + (s - from);
            const Tg *gb = g + (s - from);
            if (elements_end - s < kBlock) {
                part_block<Tw, Tg, BITS, MASTER>(a, shared, s, (uint32_t)(elements_end - s), wb, gb);
                continue;
            }
            const uint32_t w_off = elem::misalignment(wb), g_off = elem::misalignment(gb);
            if (g_off == 0u && w_off == 0u) whole_block<Tw, Tg, BITS, MASTER, 16, 16>(a, c, s, wb, gb);
            else if (g_off == 0u && w_off == 8u) whole_block<Tw, Tg, BITS, MASTER, 8, 16>(a, c, s, wb, gb);
            else whole_block<Tw, Tg, BITS, MASTER, elem::kAny, elem::kAny>(a, c, s, wb, gb);
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
    const uint64_t blocks = a.size / kBlock, ctas = (blocks + kWarps - 1) / kWarps, most = (uint64_t)sm_count * 3u;
    const uint32_t grid = (uint32_t)(ctas < most ? (ctas ? ctas : 1u) : most);
    const uint64_t share = blocks / ((uint64_t)grid * kWarps);
    const uint32_t run = (uint32_t)(share < 1u ? 1u : share < 16u ? share : 16u);
    adamw_kernel<Tw, Tg, BITS, MASTER><<<grid, kWarps * 32, 0, stream>>>(a, run, arrived, d_status);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_adamw(const AdamwArgs &a, uint32_t *d_arrived, uint32_t *d_status, int sm_count, cudaStream_t stream, uint64_t *launches) {
    ++*launches;
    return by_types(a.set.type, a.grad_type, [&](auto weight, auto grad) {
        using Tw = typename decltype(weight)::type;
        using Tg = typename decltype(grad)::type;
        if constexpr (sizeof(Tw) == 2)
            if (a.d_master)
                return a.bits == 8 ? launch_instance<Tw, Tg, 8, true>(a, d_arrived, d_status, sm_count, stream)
                                   : launch_instance<Tw, Tg, 32, true>(a, d_arrived, d_status, sm_count, stream);
        return a.bits == 8 ? launch_instance<Tw, Tg, 8, false>(a, d_arrived, d_status, sm_count, stream)
                           : launch_instance<Tw, Tg, 32, false>(a, d_arrived, d_status, sm_count, stream);
    });
}

}  // namespace ivk
