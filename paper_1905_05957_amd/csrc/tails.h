// What a decoding pass over the server's message does with the elements it has decoded.  A pass calls, for four
// consecutive elements e..e+3 of its row (e a multiple of 4, e < d),
//   wants(e, d)      the flags of the elements that take part; none: the pass may leave at once
//   put(q, e, d, f)  the decoded elements and those flags
// after ask() at its top, and takes the 2048-element tile that `tiles` lists for its workgroup: those with an element that
// takes part (nullptr: all).
// Matrices of a plan are marked in a plane of bits (bit j & 63 of word j >> 6) that covers ceil(d / 64) words: a quad costs one
// byte of it, and the matrices may lie anywhere, column blocks of a wider array among them.
#pragma once
#include "ds_device.h"

namespace ds {

// Kernel arguments, read together at the top.  They lie in host memory: the first read of one of their lines by a compute unit
// takes microseconds, and arguments that are read one branch after the other take that again and again (AdamW of 500,000
// elements 16.8 us, 3.7 us so; 50 M elements 212 and 191 us).
template <class T>
__device__ __forceinline__ void ask_for_one(T v)
{
    asm volatile("" : : "s"(v));
}

template <class... T>
__device__ __forceinline__ void ask_for(T... v)
{
    (ask_for_one(v), ...);
}

struct TailTiles {
    const int32_t *tiles;
    int32_t n;                                       // workgroups

    __device__ __forceinline__ int64_t first() const { return static_cast<int64_t>(tiles ? tiles[blockIdx.x] : static_cast<int32_t>(blockIdx.x)) * kTile; }
};

__device__ __forceinline__ uint32_t quad_flags(int64_t e, int64_t d)
{
    return (e + 4 <= d) ? 15u : (1u << (d - e)) - 1u;
}

// Elements of p whose flag is set; the others read as 0 and are not touched.
__device__ __forceinline__ f32x4 ld4_flags(const float *__restrict__ p, int64_t e, uint32_t f)
{
    if (f == 15u) return __builtin_nontemporal_load(reinterpret_cast<const f32x4_any *>(p + e));
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (f & 1u) r.x = p[e];
    if (f & 2u) r.y = p[e + 1];
    if (f & 4u) r.z = p[e + 2];
    if (f & 8u) r.w = p[e + 3];
    return r;
}

__device__ __forceinline__ void st4_flags(float *__restrict__ p, int64_t e, uint32_t f, f32x4 v)
{
    if (f == 15u) {
        __builtin_nontemporal_store(static_cast<f32x4_any>(v), reinterpret_cast<f32x4_any *>(p + e));
        return;
    }
    if (f & 1u) p[e] = v.x;
    if (f & 2u) p[e + 1] = v.y;
    if (f & 4u) p[e + 2] = v.z;
    if (f & 8u) p[e + 3] = v.w;
}

// Elements of matrices: m <- fma(beta, m, q), and what is to be orthogonalised into u: fma(beta, m, q) once more
// (Nesterov), or without a momentum buffer q itself; u == nullptr: that is m.
struct TailMomentum : TailTiles {
    const uint64_t *inside;
    float *m, *u;
    float beta;

    __device__ __forceinline__ void ask() const { ask_for(tiles, inside, m, u, beta); }
    __device__ __forceinline__ uint32_t wants(int64_t e, int64_t d) const
    {
        return load_sign_nibble(inside, e) & quad_flags(e, d);
    }
    __device__ __forceinline__ void put(f32x4 q, int64_t e, int64_t, uint32_t f) const
    {
        f32x4 v = q;
        if (m) {
            v = fma4(beta, ld4_flags(m, e, f), q);
            st4_flags(m, e, f, v);
            if (u) v = fma4(beta, v, q);
        }
        if (u) st4_flags(u, e, f, v);
    }
};

// AdamW on every element outside the matrices (inside == nullptr: on all of them):
//   m <- fma(beta1, m, (1 - beta1) q) ; v <- fma(beta2, v, (1 - beta2) q q)
//   x <- fma(-rate, m / (sqrt(v) * root + eps), keep * x)
// with rate = gamma / (1 - beta1^(t+1)), root = 1 / sqrt(1 - beta2^(t+1)), keep = 1 - gamma * decay from the host, in 64 bits.
// Bound by memory: 24 bytes an element and the message, 124 M elements in 0.515 ms, 5.8 TB/s.  Past the caches at every size: a
// training step in between leaves nothing of x, m and v in them (11.2 M elements 56 us on buffers that were not touched
// since, 61 us with ordinary accesses; called again on the same buffers 57 and 48).
struct TailAdamW : TailTiles {
    const uint64_t *inside;
    float *x, *m, *v;
    float beta1, rest1, beta2, rest2, rate, root, eps, keep;

    __device__ __forceinline__ void ask() const { ask_for(tiles, inside, x, m, v, beta1, rest1, beta2, rest2, rate, root, eps, keep); }
    __device__ __forceinline__ uint32_t wants(int64_t e, int64_t d) const
    {
        const uint32_t f = quad_flags(e, d);
        return inside ? f & ~load_sign_nibble(inside, e) : f;
    }
    __device__ __forceinline__ float step(float xv, float mv, float vv) const
    {
        return __fmaf_rn(-rate, mv / __fmaf_rn(__fsqrt_rn(vv), root, eps), keep * xv);
    }
    __device__ __forceinline__ void put(f32x4 q, int64_t e, int64_t, uint32_t f) const
    {
        const f32x4 xv = ld4_flags(x, e, f), mo = ld4_flags(m, e, f), vo = ld4_flags(v, e, f);
        const f32x4 mv = fma4(beta1, mo, rest1 * q), vv = fma4(beta2, vo, (rest2 * q) * q);
        st4_flags(m, e, f, mv);
        st4_flags(v, e, f, vv);
        st4_flags(x, e, f, f32x4{step(xv.x, mv.x, vv.x), step(xv.y, mv.y, vv.y), step(xv.z, mv.z, vv.z), step(xv.w, mv.w, vv.w)});
    }
};

}  // namespace ds
