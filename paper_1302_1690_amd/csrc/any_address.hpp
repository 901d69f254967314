// Eight consecutive numbers at any address that is a multiple of an element's size, as one or two 128-bit words
// (global memory takes them unaligned).
#pragma once
#include "storage.hpp"

namespace mpcnn {

typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 b8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef float v8f __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v8f load8(const float* p)
{
    const f4_any a = *reinterpret_cast<const f4_any*>(p), b = *reinterpret_cast<const f4_any*>(p + 4);
    return v8f{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ v8f load8(const bf16* p)
{
    return __builtin_convertvector(*reinterpret_cast<const b8_any*>(p), v8f);
}
__device__ __forceinline__ void store8(float* p, v8f v)
{
    *reinterpret_cast<f4_any*>(p) = f4_any{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f4_any*>(p + 4) = f4_any{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(bf16* p, v8f v)
{
    *reinterpret_cast<b8_any*>(p) = __builtin_convertvector(v, b8_any);
}

// E (4 or 8) numbers as they lie in memory (half the registers for bf16): raw_any fetches, widen converts
typedef __bf16 b4_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename T, int E> struct Raw;
template <> struct Raw<float, 8> { f4_any a, b; };
template <> struct Raw<float, 4> { f4_any a; };
template <> struct Raw<bf16, 8> { b8_any a; };
template <> struct Raw<bf16, 4> { b4_any a; };
template <typename T> using Raw8 = Raw<T, 8>;
template <int E, typename T>
__device__ __forceinline__ Raw<T, E> raw_any(const T* p)
{
    Raw<T, E> r;
    if constexpr (sizeof(T) == 4 && E == 8) {
        r.a = *reinterpret_cast<const f4_any*>(p);
        r.b = *reinterpret_cast<const f4_any*>(p + 4);
    } else {
        r.a = *reinterpret_cast<const decltype(r.a)*>(p);
    }
    return r;
}
template <typename T> __device__ __forceinline__ Raw8<T> raw8(const T* p) { return raw_any<8>(p); }
__device__ __forceinline__ v8f widen(const Raw<float, 8>& r) { return v8f{r.a[0], r.a[1], r.a[2], r.a[3], r.b[0], r.b[1], r.b[2], r.b[3]}; }
__device__ __forceinline__ v4f widen(const Raw<float, 4>& r) { return r.a; }
__device__ __forceinline__ v8f widen(const Raw<bf16, 8>& r) { return __builtin_convertvector(r.a, v8f); }
__device__ __forceinline__ v4f widen(const Raw<bf16, 4>& r) { return __builtin_convertvector(r.a, v4f); }
__device__ __forceinline__ void set_raw(Raw<float, 8>& r, int z, float v) { if (z < 4) r.a[z] = v; else r.b[z - 4] = v; }
template <typename T, int E> __device__ __forceinline__ void set_raw(Raw<T, E>& r, int z, T v) { r.a[z] = v; }
__device__ __forceinline__ void store_any(float* p, v8f v) { store8(p, v); }
__device__ __forceinline__ void store_any(bf16* p, v8f v) { store8(p, v); }
__device__ __forceinline__ void store_any(float* p, v4f v) { *reinterpret_cast<f4_any*>(p) = v; }
__device__ __forceinline__ void store_any(bf16* p, v4f v) { *reinterpret_cast<b4_any*>(p) = __builtin_convertvector(v, b4_any); }

// Numbers row[at .. at + E - 1] of a row of n, zeros beyond its end (at may be beyond it too).  The loads of a row's end are not conditional,
// only their addresses and results are chosen: branches with a load in each would wait for memory one after the other.
template <int E, typename T>
__device__ __forceinline__ Raw<T, E> raw_of(const T* row, int at, int n)
{
    if (at + E <= n) return raw_any<E>(row + at);
    T u[E];
    Raw<T, E> r;
#pragma unroll
    for (int z = 0; z < E; ++z) u[z] = row[at + z < n ? at + z : n - 1];
#pragma unroll
    for (int z = 0; z < E; ++z) set_raw(r, z, at + z < n ? u[z] : (T)0.f);
    return r;
}
template <typename T> __device__ __forceinline__ Raw8<T> raw8_of(const T* row, int at, int n) { return raw_of<8>(row, at, n); }
template <typename T> __device__ __forceinline__ v8f load8_of(const T* row, int at, int n) { return widen(raw8_of(row, at, n)); }

// Eight bf16 numbers at addresses of which some are no multiple of four, as the words that they lie in (each holds one of them at least), and turned
// by 16 bits where they begin in the middle of one.  The memory pipeline takes 128-bit fetches at such addresses apart.
struct Odd8 {
    typedef unsigned u4_any __attribute__((ext_vector_type(4), aligned(4)));
    u4_any a;
    unsigned b;
};
__device__ __forceinline__ Odd8 odd8(const bf16* p)
{
    const unsigned* const q = reinterpret_cast<const unsigned*>((uintptr_t)p & ~(uintptr_t)3);
    return Odd8{*reinterpret_cast<const Odd8::u4_any*>(q), q[(uintptr_t)p & 2 ? 4 : 0]};
}
__device__ __forceinline__ Odd8 odd8_of(const bf16* row, int at, int n)
{
    const Odd8::u4_any r = __builtin_bit_cast(Odd8::u4_any, raw8_of(row, at, n).a);
    if (!((uintptr_t)(row + at) & 2)) return Odd8{r, 0};
    return Odd8{Odd8::u4_any{r[0] << 16, r[0] >> 16 | r[1] << 16, r[1] >> 16 | r[2] << 16, r[2] >> 16 | r[3] << 16}, r[3] >> 16};
}
__device__ __forceinline__ v8f widen(const Odd8& o, const bf16* p)       // p: where they were fetched, or anything as far from a multiple of four
{
    const unsigned by = 8 * ((unsigned)(uintptr_t)p & 2);
    Raw8<bf16> r;
    r.a = __builtin_bit_cast(b8_any, Odd8::u4_any{__builtin_amdgcn_alignbit(o.a[1], o.a[0], by), __builtin_amdgcn_alignbit(o.a[2], o.a[1], by),
                                                  __builtin_amdgcn_alignbit(o.a[3], o.a[2], by), __builtin_amdgcn_alignbit(o.b, o.a[3], by)});
    return widen(r);
}

}  // namespace mpcnn
