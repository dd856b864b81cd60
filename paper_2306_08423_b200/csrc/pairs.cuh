// Eight neighbouring values of a row as pairs of floats.
#pragma once

#include "vectors.cuh"

namespace distsim {

// Eight neighbouring values as four pairs.
struct Oct {
    Pair v[4];
};

// Eight values as they lie in memory.
template <class T>
struct Eight {
    uint4 w[sizeof(T) * 8 / 16];
};
template <class T>
__device__ __forceinline__ Oct widen(const Eight<T> &r)
{
    Oct o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (sizeof(T) == 4) {
            const uint4 &w = r.w[i / 2];
            o.v[i] = i & 1 ? make_pair2(__uint_as_float(w.z), __uint_as_float(w.w)) : make_pair2(__uint_as_float(w.x), __uint_as_float(w.y));
        } else {
            const uint32_t w = i == 0 ? r.w[0].x : i == 1 ? r.w[0].y : i == 2 ? r.w[0].z : r.w[0].w;
            const float2 f = unpack_pair<typename std::conditional<sizeof(T) == 4, __half, T>::type>(w);
            o.v[i] = make_pair2(f.x, f.y);
        }
    }
    return o;
}
// Puts `other` in place of the values from the valid-th on.
__device__ __forceinline__ void cut8(Oct &o, int valid, float other = 0.f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = halves(o.v[i]);
        o.v[i] = make_pair2(2 * i < valid ? t.x : other, 2 * i + 1 < valid ? t.y : other);
    }
}
// One by one; values beyond the row read as zero.
template <class T>
__device__ __forceinline__ Eight<T> fetch8(const T *p, int valid)
{
    Eight<T> r;
    T *e = reinterpret_cast<T *>(r.w);
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = i < valid ? p[i] : from_float<T>(0.f);
    return r;
}
// Eight 2-byte values at any address of a matrix that starts at `begin` and ends before `end`: the two
// aligned pieces that hold them are requested, if both lie in the matrix, and shifted once they are
// here (without a branch between requests, several are under way together).
template <bool EXACT>
struct Request {
    uint4 v, w;
    bool wide;
};
template <>
struct Request<true> {
    uint4 v;
};
template <class T>
__device__ __forceinline__ void request8(Request<true> &q, const T *p, const T *, const T *) { q.v = *reinterpret_cast<const uint4 *>(p); }
template <class T>
__device__ __forceinline__ void request8(Request<false> &q, const T *p, const T *begin, const T *end)
{
    static_assert(sizeof(T) == 2, "");
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), a = at & ~(uintptr_t)15;
    const bool second = at & 15;
    q.wide = a >= reinterpret_cast<uintptr_t>(begin) && a + (second ? 32 : 16) <= reinterpret_cast<uintptr_t>(end);
    q.v = q.w = make_uint4(0, 0, 0, 0);
    if (q.wide) q.v = *reinterpret_cast<const uint4 *>(a);
    if (q.wide && second) q.w = *(reinterpret_cast<const uint4 *>(a) + 1);
}
template <class T>
__device__ __forceinline__ Oct receive8(const Request<true> &q, const T *, int) { return widen(Eight<T>{{q.v}}); }
// Values beyond the row are zero.
template <class T>
__device__ __forceinline__ Oct receive8(const Request<false> &q, const T *p, int valid)
{
    if (!q.wide) return widen(fetch8(p, valid));
    uint32_t c[8] = {q.v.x, q.v.y, q.v.z, q.v.w, q.w.x, q.w.y, q.w.z, q.w.w};
    shift_words(c, (uint32_t)reinterpret_cast<uintptr_t>(p) & 15);
    Oct o = widen(Eight<T>{{make_uint4(c[0], c[1], c[2], c[3])}});
    if (valid < 8) cut8(o, valid);
    return o;
}
template <class T, bool EXACT>
__device__ __forceinline__ void write8(T *p, int valid, bool vec, const Oct &o)
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = halves(o.v[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
    store8<T>(p, EXACT ? 8 : valid, EXACT || vec, f);
}
__device__ __forceinline__ void cut_front8(Oct &o, int lead, float other)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = halves(o.v[i]);
        o.v[i] = make_pair2(2 * i < lead ? other : t.x, 2 * i + 1 < lead ? other : t.y);
    }
}

}  // namespace distsim
