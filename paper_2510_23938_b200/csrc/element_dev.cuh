// Elements of the training-step operators: 32-bit floats and the two 16-bit types, read and written as vectors at any
// element alignment.  Tensors inside a weight file or a packed gradient buffer start at any multiple of their element
// size, so a vector may straddle two aligned pieces of memory: both are loaded (the second is the neighbouring lane's
// first, an L1 hit) and the wanted bytes are shifted out.  Every aligned piece that is touched holds at least one
// byte that was asked for, so nothing outside the 16-byte granules of the tensor is read.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cstdint>

#include "iv_internal.h"

namespace ivk {
namespace elem {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two 16-bit values in a word.
template <typename T> __device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi);
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float &lo, float &hi) {
    lo = __uint_as_float(w << 16);                    // bf16 is the upper half of a 32-bit float
    hi = __uint_as_float(w & 0xffff0000u);
}
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float &lo, float &hi) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    lo = f.x;
    hi = f.y;
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&x);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&x);
}

// V elements of type T as 32-bit words.
template <typename T, int V>
struct Packed {
    static constexpr int kBytes = V * (int)sizeof(T);
    static constexpr int kWords = kBytes / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void unpack(float (&v)[V]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) unpack2<T>(w[i], v[2 * i], v[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void pack(const float (&v)[V]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) w[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
        }
    }
};

// Aligned vector access of 8 or 16 bytes.
template <int WORDS>
__device__ __forceinline__ void load_aligned(const void *p, uint32_t *w) {
    if constexpr (WORDS == 4) {
        const uint4 q = *static_cast<const uint4 *>(p);
        w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    } else {
        static_assert(WORDS == 2, "8 or 16 bytes");
        const uint2 q = *static_cast<const uint2 *>(p);
        w[0] = q.x; w[1] = q.y;
    }
}
template <int WORDS>
__device__ __forceinline__ void store_aligned(void *p, const uint32_t *w) {
    if constexpr (WORDS == 4) *static_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else {
        static_assert(WORDS == 2, "8 or 16 bytes");
        *static_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    }
}

__device__ __forceinline__ void store_32_bytes(void *p, const uint32_t *w) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// V consecutive elements (a multiple of 16 bytes) with the aligned pieces of memory they lie in; load() only loads,
// get() shifts the wanted bytes out, so that several loads can be in flight.  ALIGN: 16 or 8 bytes (tables of weight
// files: their header is a multiple of 8), which need no shifting; 0 for any other element alignment; kAny for all of
// them (nothing of the last piece is wanted, and it is not touched, when the vector starts at a piece).
constexpr int kAny = -1;
template <typename T, int V, int ALIGN>
struct Vector {
    static constexpr int W = Packed<T, V>::kWords;
    static constexpr int P = W % 4 == 0 ? 4 : 2;                          // words of an aligned piece: 16 bytes, or 8 of a vector of 8
    static constexpr int kLoaded = ALIGN > 0 ? W : W + P;
    uint32_t w[kLoaded];
    __device__ __forceinline__ void load(const T *p, uint32_t off) {
        const uint8_t *q = reinterpret_cast<const uint8_t *>(p) - (ALIGN > 0 ? 0u : off & (4u * P - 1u));
        constexpr int kStep = ALIGN == 8 ? 2 : P;
#pragma unroll
        for (int i = 0; i < kLoaded; i += kStep)
            if (i < W || ALIGN == 0 || (off & (4u * P - 1u))) load_aligned<kStep>(q + 4 * i, w + i);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kLoaded; ++i) w[i] = 0u;
    }
    // `off`: bytes from the 16-byte boundary, the same for all lanes that walk one tensor with a stride of whole vectors
    __device__ __forceinline__ Packed<T, V> get(uint32_t off) const {
        Packed<T, V> out;
        if constexpr (ALIGN > 0) {
#pragma unroll
            for (int i = 0; i < W; ++i) out.w[i] = w[i];
        } else {
            uint32_t x[W + 4];
#pragma unroll
            for (int i = 0; i < W + 4; ++i) x[i] = i < kLoaded ? w[i] : 0u;
            if (P == 4 && (off & 8u)) {
#pragma unroll
                for (int i = 0; i < W + 2; ++i) x[i] = x[i + 2];
            }
            if (off & 4u) {
#pragma unroll
                for (int i = 0; i < W + 1; ++i) x[i] = x[i + 1];
            }
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int i = 0; i < W; ++i) out.w[i] = x[i];
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i) out.w[i] = __funnelshift_r(x[i], x[i + 1], (off & 2u) * 8u);
            }
        }
        return out;
    }
};

// Two 32-bit floats that one instruction works on, each rounded by itself (but a product that is added may become one multiply-add).
struct Pair {
    uint64_t bits;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(bits) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit Pair(float both) : Pair(both, both) {}
    __device__ __forceinline__ float sum() const {
        float lo, hi;
        get(lo, hi);
        return lo + hi;
    }
    __device__ __forceinline__ void get(float &lo, float &hi) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(bits)); }
};
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}

template <typename T>
__device__ __forceinline__ void unpack8(const Packed<T, 8> &packed, Pair (&x)[4]) {
    float e[8];
    packed.unpack(e);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = Pair(e[2 * i], e[2 * i + 1]);
}

__device__ __forceinline__ void unpair(const Pair (&x)[4], float (&e)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i].get(e[2 * i], e[2 * i + 1]);
}

// (a0, a1) += (x0^2, x1^2), each rounded as a multiply-add of its own.
__device__ __forceinline__ void add_squares2(float &a0, float &a1, float x0, float x1) {
    asm("{\n\t.reg .b64 a, x;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 x, {%2, %3};\n\tfma.rn.f32x2 a, x, x, a;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "+f"(a0), "+f"(a1) : "f"(x0), "f"(x1));
}

__device__ __forceinline__ uint32_t misalignment(const void *p) { return (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u; }

// V consecutive elements at any element alignment, at once.
template <typename T, int V>
__device__ __forceinline__ void load_any(const T *p, Packed<T, V> &out) {
    const uint32_t off = misalignment(p);
    if (off == 0u) {
        Vector<T, V, 16> x;
        x.load(p, 0u);
        out = x.get(0u);
    } else {
        Vector<T, V, 0> x;
        x.load(p, off);
        out = x.get(off);
    }
}

// Elements per vector of a map.  Widening: 8 bytes in, 16 out, so that a warp's stores are contiguous (two 16-byte stores
// 32 bytes apart from lane to lane write half sectors: 284 against 207 us for 65,536 rows of 4096); narrowing: 32 in, 16 out (loads that
// share sectors meet in L1).
template <typename Tin, typename Tout>
struct MapShape {
    static constexpr int V = sizeof(Tout) == 4 ? 4 : 8;
};

template <typename Tin, typename Tout, int ALIGN, typename F>
__device__ __forceinline__ void map_vectors(const Tin *in, Tout *out, uint32_t vecs, uint32_t lane, uint32_t lanes, F f) {
    constexpr int V = MapShape<Tin, Tout>::V;
    // bytes in flight per thread: 64, or 32 and their neighbours; one vector in the form for all alignments, where more
    // warps serve better than more registers (65,536 rows of 4095 16-bit columns: 150 us with 32 registers, 215 with 64)
    constexpr int kBytes = V * (int)sizeof(Tin), kFlight = ALIGN > 0 ? 64 : ALIGN == 0 ? 32 : 16;
    constexpr int UNROLL = kBytes < kFlight ? kFlight / kBytes : 1;
    const uint32_t off = misalignment(in);
    for (uint32_t v0 = lane; v0 < vecs; v0 += lanes * UNROLL) {
        Vector<Tin, V, ALIGN> raw[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint32_t v = v0 + u * lanes;
            if (v < vecs) raw[u].load(in + (uint64_t)v * V, off);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint32_t v = v0 + u * lanes;
            if (v < vecs) {
                float x[V];
                raw[u].get(off).unpack(x);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = f(x[i]);
                Packed<Tout, V> y;
                y.pack(x);
#pragma unroll
                for (int i = 0; i < Packed<Tout, V>::kWords; i += 4)
                    store_aligned<4>(reinterpret_cast<uint32_t *>(out + (uint64_t)v * V) + i, y.w + i);
            }
        }
    }
}

// out[i] = f(in[i]) for i < n by the `lanes` threads (at least 8) of which this is number `lane`, in vectors.
// The input starts at a multiple of ALIGN bytes (0: of an element), the output of 16.
template <typename Tin, typename Tout, int ALIGN, typename F>
__device__ __forceinline__ void map_aligned(const Tin *in, Tout *out, uint32_t n, uint32_t lane, uint32_t lanes, F f) {
    constexpr int V = MapShape<Tin, Tout>::V;
    const uint32_t vecs = n / V, done = vecs * V;
    map_vectors<Tin, Tout, ALIGN>(in, out, vecs, lane, lanes, f);
    if (lane < n - done) out[done + lane] = from_float<Tout>(f(to_float(in[done + lane])));
}
// Both at any element alignment: single elements up to the first 16-byte boundary of the output.  BY_CLASS: one loop for
// each class of alignment (few spans with their own alignment), else one for all.
template <typename Tin, typename Tout, bool BY_CLASS, typename F>
__device__ __forceinline__ void map_any(const Tin *in, Tout *out, uint32_t n, uint32_t lane, uint32_t lanes, F f) {
    uint32_t head = ((16u - misalignment(out)) & 15u) / (uint32_t)sizeof(Tout);
    if (head > n) head = n;
    if (lane < head) out[lane] = from_float<Tout>(f(to_float(in[lane])));
    in += head;
    out += head;
    n -= head;
    if constexpr (BY_CLASS) {
        const uint32_t off = misalignment(in);
        if (off == 0u) map_aligned<Tin, Tout, 16>(in, out, n, lane, lanes, f);
        else if (off == 8u) map_aligned<Tin, Tout, 8>(in, out, n, lane, lanes, f);
        else map_aligned<Tin, Tout, 0>(in, out, n, lane, lanes, f);
    } else {
        map_aligned<Tin, Tout, kAny>(in, out, n, lane, lanes, f);
    }
}

}  // namespace elem

// Calls f(tag of the input type, tag of the output type) for the pairs of element types the operators support: equal
// ones, and a 16-bit type with 32 bits on the other side.
template <typename T> struct TypeTag { using type = T; };
template <typename F>
inline cudaError_t by_types(int in, int out, F f) {
    using f32 = TypeTag<float>;
    using f16 = TypeTag<__half>;
    using bf16 = TypeTag<__nv_bfloat16>;
    switch (in * 3 + out) {
        case IV_F32 * 3 + IV_F32: return f(f32{}, f32{});
        case IV_F32 * 3 + IV_F16: return f(f32{}, f16{});
        case IV_F32 * 3 + IV_BF16: return f(f32{}, bf16{});
        case IV_F16 * 3 + IV_F32: return f(f16{}, f32{});
        case IV_F16 * 3 + IV_F16: return f(f16{}, f16{});
        case IV_BF16 * 3 + IV_F32: return f(bf16{}, f32{});
        case IV_BF16 * 3 + IV_BF16: return f(bf16{}, bf16{});
        default: return cudaErrorInvalidValue;     // checked at the entry points
    }
}
}  // namespace ivk
