// Rows of fp32 or bf16 values read and written 16 bytes at a time.
#pragma once
#include "owt_common.hpp"

namespace owt {

// A piece of a row, 16 bytes of storage type: 4 fp32 or 8 bf16 values.  Rows of any number of values start at any multiple of the type's
// size, so the accesses claim no more alignment than that (one instruction all the same: global memory takes them unaligned).  ONCE: for
// what is not read again while caches could hold it; it leaves their places to others.
template <class T> struct Piece;
template <> struct Piece<float> {
    static constexpr int V = 4;
    typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(4)));
    template <bool ONCE = false> static __device__ __forceinline__ void load(const float *p, float (&v)[4])
    {
        const Raw r = ONCE ? __builtin_nontemporal_load((const Raw *)p) : *(const Raw *)p;
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = __uint_as_float(r[i]);
    }
    template <bool ONCE = false> static __device__ __forceinline__ void store(float *p, const float (&v)[4])
    {
        Raw r;
#pragma unroll
        for (int i = 0; i < 4; i++) r[i] = __float_as_uint(v[i]);
        if (ONCE) __builtin_nontemporal_store(r, (Raw *)p);
        else *(Raw *)p = r;
    }
};
template <> struct Piece<bf16_t> {
    static constexpr int V = 8;
    typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(2)));
    template <bool ONCE = false> static __device__ __forceinline__ void load(const bf16_t *p, float (&v)[8])
    {
        const Raw r = ONCE ? __builtin_nontemporal_load((const Raw *)p) : *(const Raw *)p;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t w = r[i];
            v[2 * i] = __uint_as_float(w << 16);
            v[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
    template <bool ONCE = false> static __device__ __forceinline__ void store(bf16_t *p, const float (&v)[8])
    {
        Raw r;
#pragma unroll
        for (int i = 0; i < 4; i++) r[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
        if (ONCE) __builtin_nontemporal_store(r, (Raw *)p);
        else *(Raw *)p = r;
    }
};

// Piece j of a row of `cols` values: what lies past them reads as zero and is not written.
template <class T, bool ONCE = false> __device__ __forceinline__ void load_piece(const T *row, int j, int cols, float (&v)[Piece<T>::V])
{
    constexpr int V = Piece<T>::V;
    const int c = j * V;
    if (c + V <= cols) Piece<T>::template load<ONCE>(row + c, v);
    else {
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = c + i < cols ? load1(row, c + i) : 0.f;
    }
}
// The same where a row's last values would wait for each other behind their branches (for more registers).
template <class T> __device__ __forceinline__ void load_piece_at_once(const T *row, int j, int cols, float (&v)[Piece<T>::V])
{
    constexpr int V = Piece<T>::V;
    const int c = j * V;
    if (c + V <= cols) Piece<T>::load(row + c, v);
    else {
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = load1(row, min(c + i, cols - 1));
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = c + i < cols ? v[i] : 0.f;
    }
}
template <class T, bool ONCE = false> __device__ __forceinline__ void store_piece(T *row, int j, int cols, const float (&v)[Piece<T>::V])
{
    constexpr int V = Piece<T>::V;
    const int c = j * V;
    if (c + V <= cols) Piece<T>::template store<ONCE>(row + c, v);
    else {
#pragma unroll
        for (int i = 0; i < V; i++)
            if (c + i < cols) store1(row, (size_t)(c + i), v[i]);
    }
}

}  // namespace owt
