// Element types of tensors that come from a model: 32-bit floats, bfloat16 and half, 16 bytes at a time, all arithmetic in 32 bits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace ef21 {

template <typename T> struct Elem;

template <> struct Elem<float> {
    static constexpr int VEC = 4;                            // elements in 16 bytes
    static constexpr unsigned NEG_INF = 0xff800000u;         // a 32-bit word of elements that are -inf
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
    static __device__ __forceinline__ void unpack(uint4 u, float (&f)[4]) {
        f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float top(uint4 u) {   // largest element; NaN only where all are
        return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
    }
};

template <> struct Elem<__nv_bfloat16> {
    static constexpr int VEC = 8;
    static constexpr unsigned NEG_INF = 0xff80ff80u;
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
    static __device__ __forceinline__ void two(unsigned u, float& a, float& b) { a = __uint_as_float(u << 16); b = __uint_as_float(u & 0xffff0000u); }
    static __device__ __forceinline__ unsigned both(float a, float b) {
        __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<unsigned*>(&v);
    }
    static __device__ __forceinline__ void unpack(uint4 u, float (&f)[8]) {
        two(u.x, f[0], f[1]); two(u.y, f[2], f[3]); two(u.z, f[4], f[5]); two(u.w, f[6], f[7]);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        return make_uint4(both(f[0], f[1]), both(f[2], f[3]), both(f[4], f[5]), both(f[6], f[7]));
    }
    static __device__ __forceinline__ float top(uint4 u) {
        const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&u);
        const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
};

template <> struct Elem<__half> {
    static constexpr int VEC = 8;
    static constexpr unsigned NEG_INF = 0xfc00fc00u;
    static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
    static __device__ __forceinline__ void two(unsigned u, float& a, float& b) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
        a = f.x; b = f.y;
    }
    static __device__ __forceinline__ unsigned both(float a, float b) {
        __half2 v = __floats2half2_rn(a, b);
        return *reinterpret_cast<unsigned*>(&v);
    }
    static __device__ __forceinline__ void unpack(uint4 u, float (&f)[8]) {
        two(u.x, f[0], f[1]); two(u.y, f[2], f[3]); two(u.z, f[4], f[5]); two(u.w, f[6], f[7]);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        return make_uint4(both(f[0], f[1]), both(f[2], f[3]), both(f[4], f[5]), both(f[6], f[7]));
    }
    static __device__ __forceinline__ float top(uint4 u) {
        const __half2* p = reinterpret_cast<const __half2*>(&u);
        const __half2 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
};

// 16 bytes that are read once: past the L1.  (volatile: stays behind the wait of the dependent launch)
__device__ __forceinline__ uint4 load_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store_vec(void* p, uint4 v) { *reinterpret_cast<uint4*>(p) = v; }

// N times 16 bytes from any address: the lanes of a warp, all of them, take consecutive 16 bytes (in: this lane does; last: nobody behind it does), N * 32 of these
// `step` bytes apart.  Two aligned loads would do for each, of which the second is the next lane's first.  What is read beside the bytes wanted lies in the same
// aligned 16 bytes as one of them.
template <int N>
__device__ __forceinline__ void load_unaligned(const void* const (&p)[N], const bool (&in)[N], const bool (&last)[N], uint4 (&out)[N]) {
    const int lane = threadIdx.x & 31;
    uint4 own[N], more[N];
    bool extra[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p[k]);
        own[k] = more[k] = make_uint4(0u, 0u, 0u, 0u);
        extra[k] = in[k] && (last[k] || lane == 31) && (at & 15u) != 0;
        if (in[k]) own[k] = load_once(reinterpret_cast<const void*>(at & ~(uintptr_t)15));
        if (extra[k]) more[k] = load_once(reinterpret_cast<const void*>((at & ~(uintptr_t)15) + 16));
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        unsigned w[8] = {own[k].x, own[k].y, own[k].z, own[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 + i] = __shfl_down_sync(0xffffffffu, w[i], 1);
        if (extra[k]) { w[4] = more[k].x; w[5] = more[k].y; w[6] = more[k].z; w[7] = more[k].w; }
        const unsigned by = (unsigned)(reinterpret_cast<uintptr_t>(p[k]) & 15u);
        if (by & 8u) {
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
        }
        if (by & 4u) {
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
        }
        const unsigned bits = (by & 3u) * 8u;
        out[k] = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
    }
}

// Indices are 32 or 64 bits wide.
__device__ __forceinline__ i64 index_at(const void* p, int wide, i64 i) {
    return wide ? static_cast<const long long*>(p)[i] : (i64)static_cast<const int*>(p)[i];
}

// 2^x: an instruction (2 units in the last place); results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// e^x to a few units in the last place: what the product with log2 e loses is put back to first order.  (Below 2^-126: 0.)  Where 2^t is 0, infinite or NaN there is nothing to put
// back to: infinity less a little is NaN.
__device__ __forceinline__ float exp_fast(float x) {
    const float t = x * LOG2E, y = exp2_fast(t), lost = fmaf(x, LOG2E, -t);
    return fabsf(t) < 128.f ? fmaf(y, lost * LN2, y) : y;
}

// Two fp32 values, and one instruction for both.
typedef unsigned long long Two;
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ Two two(float a) { return two(a, a); }
__device__ __forceinline__ void split(Two v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Elements in front of the first 16-byte boundary of a row.
template <typename T>
__device__ __forceinline__ int row_head(const T* row) {
    return (int)(((16u - (unsigned)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / sizeof(T));
}


}  // namespace ef21
