// What the operators over a paged cache share on the device: where a slot's row is, and rows of eight elements a lane.
#pragma once

#include "common.hpp"

namespace ann {

// A paged cache as the kernels see it; strides in bytes.
struct Paged {
    char *k, *v;
    int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
    int pages, heads, slots_log, d;
};

// Eight consecutive elements of a row, in 32 bits.  (fp32: two chunks of 16 bytes; d is a multiple of 8.)
template <class T>
struct Eight;

template <>
struct Eight<F16> {
    u4 raw;
    __device__ __forceinline__ void load(const char *p) { raw = load_chunk(p); }
    __device__ __forceinline__ void store(char *p) const { *reinterpret_cast<u4 *>(p) = raw; }
    __device__ __forceinline__ void zero() { raw = zero_chunk(); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const h8 a = __builtin_bit_cast(h8, raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        h8 a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = (_Float16)x[i];
        raw = __builtin_bit_cast(u4, a);
    }
};
template <>
struct Eight<BF16> {
    u4 raw;
    __device__ __forceinline__ void load(const char *p) { raw = load_chunk(p); }
    __device__ __forceinline__ void store(char *p) const { *reinterpret_cast<u4 *>(p) = raw; }
    __device__ __forceinline__ void zero() { raw = zero_chunk(); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(raw[i] << 16);
            x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        b8 a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
        raw = __builtin_bit_cast(u4, a);
    }
};
template <>
struct Eight<F32> {
    u4 raw[2];
    __device__ __forceinline__ void load(const char *p) { raw[0] = load_chunk(p); raw[1] = load_chunk(p + 16); }
    __device__ __forceinline__ void store(char *p) const {
        reinterpret_cast<u4 *>(p)[0] = raw[0];
        reinterpret_cast<u4 *>(p)[1] = raw[1];
    }
    __device__ __forceinline__ void zero() { raw[0] = raw[1] = zero_chunk(); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(raw[i / 4][i % 4]);
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i / 4][i % 4] = __float_as_uint(x[i]);
    }
};

}  // namespace ann
