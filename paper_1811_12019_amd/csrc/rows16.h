// Rows of any alignment in 16-byte vectors, and their elements as floats.  KIND 0: bf16, 1: fp16, 2: fp32.
#pragma once

#include "common.h"

namespace kfac {

template <int KIND> constexpr int elem_bytes = KIND == 2 ? 4 : 2;
template <int KIND> constexpr int elems16 = 16 / elem_bytes<KIND>;

typedef unsigned u4 __attribute__((ext_vector_type(4)));
// (gfx950 loads and stores 16 bytes a lane at any address; the declared alignment is the elements')
typedef u4 u4_a2 __attribute__((aligned(2)));
typedef u4 u4_a4 __attribute__((aligned(4)));
template <int ES> struct Unaligned { typedef u4_a4 type; };
template <> struct Unaligned<2> { typedef u4_a2 type; };
template <int ES> struct Word { typedef unsigned type; };
template <> struct Word<2> { typedef uint16_t type; };

typedef KFAC_AS1 char gchar;

// `count` elements at p, at most a vector's; the others of the vector are zeros.
template <int ES, bool STREAM = false>
__device__ __forceinline__ u4 load_row16(const gchar* p, int count) {
    typedef typename Unaligned<ES>::type vec;
    typedef typename Word<ES>::type word;
    constexpr int V = 16 / ES;
    if (count >= V) {
        if constexpr (STREAM) return __builtin_nontemporal_load((const KFAC_AS1 vec*)p);
        else return *(const KFAC_AS1 vec*)p;
    }
    u4 r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < V - 1; ++i)
        if (i < count) r[i * ES / 4] |= (unsigned)((const KFAC_AS1 word*)p)[i] << (i * ES % 4 * 8);
    return r;
}
template <int ES, bool STREAM = false>
__device__ __forceinline__ void store_row16(gchar* p, const u4& r, int count) {
    typedef typename Unaligned<ES>::type vec;
    typedef typename Word<ES>::type word;
    constexpr int V = 16 / ES;
    if (count >= V) {
        if constexpr (STREAM) __builtin_nontemporal_store(r, (KFAC_AS1 vec*)p);
        else *(KFAC_AS1 vec*)p = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < V - 1; ++i)
        if (i < count) ((KFAC_AS1 word*)p)[i] = (word)(r[i * ES / 4] >> (i * ES % 4 * 8));
}

template <int KIND>
__device__ __forceinline__ void unpack16(const u4& r, float (&f)[elems16<KIND>]) {
#pragma unroll
    for (int i = 0; i < elems16<KIND>; ++i) {
        if constexpr (KIND == 2) f[i] = __uint_as_float(r[i]);
        else if constexpr (KIND == 0) f[i] = i & 1 ? __uint_as_float(r[i / 2] & 0xFFFF0000u) : __uint_as_float(r[i / 2] << 16);
        else f[i] = half_bits_to_float((uint16_t)(r[i / 2] >> (i & 1) * 16));
    }
}
template <int KIND>
__device__ __forceinline__ u4 pack16(const float (&f)[elems16<KIND>]) {
    u4 r;
    if constexpr (KIND == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(f[i]);
    } else if constexpr (KIND == 0) {
        v8bf v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];
        __builtin_memcpy(&r, &v, 16);
    } else {
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        h8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (_Float16)f[i];
        __builtin_memcpy(&r, &v, 16);
    }
    return r;
}

}  // namespace kfac
