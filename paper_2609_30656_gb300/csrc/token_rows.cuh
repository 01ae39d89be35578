// token_rows.cuh -- pieces of rows of any storage type and alignment, and positions of
// tokens in sequences, for the token lookup and its gradient.
#pragma once

#include "tbe_internal.cuh"

namespace cbtbe {

// V consecutive values of type DT at `p`, which is aligned to their size (V = 1, 2, 4, 8, or
// 16 of 16 bits: 2 to 32 bytes).
template <int DT, int V>
struct Piece {
    static constexpr int kBytes = V * (DT == CB_F32 ? 4 : 2);
    uint32_t w[kBytes < 4 ? 1 : kBytes / 4];
};
template <bool READ_ONLY, class T>
__device__ __forceinline__ T load_as(const void* p) {
    if constexpr (READ_ONLY) return __ldg(static_cast<const T*>(p));
    else return *static_cast<const T*>(p);
}
// READ_ONLY: memory that this kernel does not write.
template <int DT, int V, bool READ_ONLY = true>
__device__ __forceinline__ Piece<DT, V> load_piece(const void* p) {
    Piece<DT, V> x;
    constexpr int B = Piece<DT, V>::kBytes;
    if constexpr (B == 2) {
        x.w[0] = load_as<READ_ONLY, unsigned short>(p);
    } else if constexpr (B == 4) {
        x.w[0] = load_as<READ_ONLY, unsigned int>(p);
    } else if constexpr (B == 8) {
        const uint2 v = load_as<READ_ONLY, uint2>(p);
        x.w[0] = v.x;
        x.w[1] = v.y;
    } else if constexpr (B == 32 && READ_ONLY) {
        asm("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
            : "=r"(x.w[0]), "=r"(x.w[1]), "=r"(x.w[2]), "=r"(x.w[3]), "=r"(x.w[4]), "=r"(x.w[5]), "=r"(x.w[6]),
              "=r"(x.w[7])
            : "l"(p));
    } else {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) {
            const uint4 v = load_as<READ_ONLY, uint4>(static_cast<const uint4*>(p) + i);
            x.w[4 * i] = v.x;
            x.w[4 * i + 1] = v.y;
            x.w[4 * i + 2] = v.z;
            x.w[4 * i + 3] = v.w;
        }
    }
    return x;
}
template <int DT, int V>
__device__ __forceinline__ Piece<DT, V> zero_piece() {
    Piece<DT, V> x;
#pragma unroll
    for (uint32_t& w : x.w) w = 0u;
    return x;
}
template <int DT>
__device__ __forceinline__ float widen(uint32_t half) {
    if constexpr (DT == CB_BF16) return __uint_as_float(half << 16);
    const uint16_t b = static_cast<uint16_t>(half);
    __half h;
    memcpy(&h, &b, 2);
    return __half2float(h);
}
template <int DT, int V>
__device__ __forceinline__ void widen(const Piece<DT, V>& x, float (&f)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (DT == CB_F32) f[i] = __uint_as_float(x.w[i]);
        else f[i] = widen<DT>(i & 1 ? x.w[i / 2] >> 16 : x.w[i / 2] & 0xffffu);
    }
}
template <int DT>
__device__ __forceinline__ uint32_t narrow(float v) {
    static_assert(DT != CB_F32, "16-bit types");
    uint16_t b;
    if constexpr (DT == CB_BF16) {
        const __nv_bfloat16 h = __float2bfloat16_rn(v);
        memcpy(&b, &h, 2);
    } else {
        const __half h = __float2half_rn(v);
        memcpy(&b, &h, 2);
    }
    return b;
}
// Rounds to nearest even, once, and stores past the caches' reuse (outputs are written once).
template <int DT, int V>
__device__ __forceinline__ void store_piece(void* p, const float (&f)[V]) {
    constexpr int B = Piece<DT, V>::kBytes;
    if constexpr (B == 2) {
        *static_cast<uint16_t*>(p) = static_cast<uint16_t>(narrow<DT>(f[0]));
    } else {
        uint32_t w[B / 4];
#pragma unroll
        for (int i = 0; i < B / 4; ++i) {
            if constexpr (DT == CB_F32) w[i] = __float_as_uint(f[i]);
            else w[i] = narrow<DT>(f[2 * i]) | narrow<DT>(f[2 * i + 1]) << 16;
        }
        if constexpr (B == 4) *static_cast<uint32_t*>(p) = w[0];
        else if constexpr (B == 8) __stcs(static_cast<uint2*>(p), make_uint2(w[0], w[1]));
        else if constexpr (B == 32) {
            asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]),
                         "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p)
                         : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < B / 16; ++i)
                __stcs(static_cast<uint4*>(p) + i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
        }
    }
}

// Elements named by position i: sequence i / length, place i % length, strides in values.
// Equally spaced ones have length 0 and are at i * place.
struct Positions {
    uint32_t length;
    int64_t sequence, place;
    __device__ __forceinline__ int64_t at(uint32_t i) const {
        if (length == 0) return static_cast<int64_t>(i) * place;
        const uint32_t s = i / length;
        return s * sequence + static_cast<int64_t>(i - s * length) * place;
    }
};
inline Positions positions(int64_t sequences, int64_t length, int64_t sequence_stride, int64_t place_stride) {
    if (length == 1) return {0, 0, sequence_stride};
    if (sequences <= 1 || sequence_stride == length * place_stride) return {0, 0, place_stride};
    return {static_cast<uint32_t>(length), sequence_stride, place_stride};
}

struct Tokens {
    const void* data;
    Positions at;
    uint32_t n;
    int32_t is32;
    int64_t rows;  // valid tokens are 0 .. rows - 1
    __device__ __forceinline__ int64_t load(uint32_t i) const { return load_index(data, at.at(i), is32); }
};

}  // namespace cbtbe
