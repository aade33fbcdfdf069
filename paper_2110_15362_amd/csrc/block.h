// What the kernels of a feed-forward sublayer share (block.hip, gated.hip): elements and their 16-byte vectors, reductions, launches.
#ifndef BT_BLOCK_H
#define BT_BLOCK_H

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "bittrain.h"

namespace btb {

constexpr int kWave = 64;
constexpr int kVec = 16;                  // bytes of a vector load

typedef uint32_t raw16 __attribute__((ext_vector_type(4)));      // a vector's bits
typedef float float2v __attribute__((ext_vector_type(2)));

struct bf16 { uint16_t bits; };
struct f16 { _Float16 v; };

// A vector at any address that its elements may have: the hardware takes such accesses, at full speed where they happen to be aligned.
template <class T> struct __attribute__((packed, aligned(sizeof(T)))) Unaligned { raw16 v; };

template <class T> constexpr int kPer = kVec / (int)sizeof(T);     // elements of a vector

__device__ inline float widen(float x) { return x; }
__device__ inline float widen(f16 x) { return (float)x.v; }
__device__ inline float widen(bf16 x) { return __builtin_bit_cast(float, (uint32_t)x.bits << 16); }

// The one rounding of a result, to nearest even.
template <class T> __device__ inline T narrow(float x);
template <> __device__ inline float narrow<float>(float x) { return x; }
template <> __device__ inline f16 narrow<f16>(float x) { return f16{(_Float16)x}; }
template <> __device__ inline bf16 narrow<bf16>(float x) { return bf16{__builtin_bit_cast(uint16_t, (__bf16)x)}; }

// The elements of a vector as floats, and back.
template <class T> __device__ inline void unpack(const raw16 v, float (&x)[kPer<T>]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(float, (uint32_t)v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same_v<T, bf16>) {
                x[2 * i] = __builtin_bit_cast(float, v[i] << 16);
                x[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
            } else {
                x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)v[i]);
                x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(v[i] >> 16));
            }
        }
    }
}

template <class T> __device__ inline uint32_t pack2(const float a, const float b) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    if constexpr (std::is_same_v<T, bf16>) return __builtin_bit_cast(uint32_t, bf2{(__bf16)a, (__bf16)b});
    else return __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
}

template <class T> __device__ inline raw16 pack(const float (&x)[kPer<T>]) {
    raw16 v;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
    }
    return v;
}

// Elements [0, left) of the vector at p, zeros behind them.  A vector that ends beyond its row is read from further in front, where the row has
// `before` elements, and moved: one load instead of up to seven.
template <class T> __device__ inline raw16 load_vec(const T *p, const int left, const int before) {
    if (left >= kPer<T>) return reinterpret_cast<const Unaligned<T> *>(p)->v;
    raw16 v = {0, 0, 0, 0};
    if (left <= 0) return v;
    if (sizeof(T) == 2 && left + before >= kPer<T>) {
        typedef uint64_t two __attribute__((ext_vector_type(2)));
        raw16 bits = reinterpret_cast<const Unaligned<T> *>(p + left - kPer<T>)->v;
        // (Or the compiler makes one load of this and the one above, and waves without such a vector wait for theirs to be moved by nothing.)
        asm volatile("" : "+v"(bits));
        const two x = __builtin_bit_cast(two, bits);
        const uint32_t shift = (uint32_t)(kPer<T> - left) * (8 * sizeof(T));      // 0 < shift < 128
        const uint64_t low = x[0], high = x[1];
        return __builtin_bit_cast(raw16, shift >= 64 ? two{high >> (shift - 64), 0} : two{low >> shift | high << (64 - shift), high >> shift});
    }
#pragma unroll
    for (int i = 0; i < kPer<T>; ++i)
        if (i < left) {
            if constexpr (sizeof(T) == 4) v[i] = __builtin_bit_cast(uint32_t, p[i]);
            else v[i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[i]) << (16 * (i & 1));
        }
    return v;
}

// Elements [0, left) of v; of a part of a vector its halves, quarters and single elements.
template <class T> __device__ inline void store_vec(T *p, const int left, const raw16 v) {
    struct __attribute__((packed, aligned(sizeof(T)))) Eight { uint64_t v; };
    struct __attribute__((packed, aligned(sizeof(T)))) Four { uint32_t v; };
    if (left >= kPer<T>) {
        reinterpret_cast<Unaligned<T> *>(p)->v = v;
        return;
    }
    if (left <= 0) return;
    uint64_t x = (uint64_t)v[1] << 32 | v[0];
    if (left & (8 / sizeof(T))) {
        reinterpret_cast<Eight *>(p)->v = x;
        p += 8 / sizeof(T);
        x = (uint64_t)v[3] << 32 | v[2];
    }
    if (left & (4 / sizeof(T))) {
        reinterpret_cast<Four *>(p)->v = (uint32_t)x;
        p += 4 / sizeof(T);
        x >>= 32;
    }
    if constexpr (sizeof(T) == 2)
        if (left & 1) *p = __builtin_bit_cast(T, (uint16_t)x);
}

template <class T> static __global__ __launch_bounds__(256) void zero_kernel(T *p, const uint64_t n) {
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) p[i] = narrow<T>(0.0f);
}

// ---- host ------------------------------------------------------------------------------------------------------

inline int width_of(const bt_dtype dt) { return dt == BT_F32 ? 4 : dt == BT_F16 || dt == BT_BF16 ? 2 : 0; }

inline bool misaligned(const void *p, const size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// hipLaunchKernel's status is this launch's own.
template <class... P>
bt_status launch(void (*kernel)(P...), const dim3 grid, const int block, hipStream_t hs, const std::common_type_t<P> &...args) {
    void *where[] = {const_cast<void *>(static_cast<const void *>(&args))...};
    if (hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3((unsigned)block), where, 0, hs) == hipSuccess) return BT_OK;
    (void)hipGetLastError();
    return BT_ERR_HIP;
}

template <class Go> bt_status with_type(const bt_dtype dt, Go go) {
    if (dt == BT_F32) return go(float{});
    if (dt == BT_F16) return go(f16{});
    return go(bf16{});
}

template <class T> bt_status zeros(void *p, const uint64_t n, hipStream_t hs) {
    const uint64_t blocks = (n + 255) / 256;
    return n == 0 ? BT_OK : launch(zero_kernel<T>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), 256, hs, (T *)p, n);
}

}  // namespace btb
#endif  // BT_BLOCK_H
