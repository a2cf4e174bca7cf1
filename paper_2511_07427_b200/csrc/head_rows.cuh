// Rows of single heads as the calls on plain rows see them: eight consecutive elements per lane, head_dim / 8 lanes per
// row, loaded from strided fp32 / bf16 arrays and stored as fp32, bf16 or e4m3 with the row's power-of-two scale.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "fp8_rows.cuh"

namespace dkv {

// Eight elements as they lie in memory, and as floats.
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T* p, bool vec) {
    Raw8<T> r;
    if (vec) {
        r.w[0] = *reinterpret_cast<const uint4*>(p);
        if constexpr (sizeof(T) == 4) r.w[1] = *reinterpret_cast<const uint4*>(p + 4);
    } else if constexpr (sizeof(T) == 4) {
        const unsigned* u = reinterpret_cast<const unsigned*>(p);
        r.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
        r.w[1] = make_uint4(u[4], u[5], u[6], u[7]);
    } else {
        const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
        r.w[0] = make_uint4(u[0] | (unsigned)u[1] << 16, u[2] | (unsigned)u[3] << 16, u[4] | (unsigned)u[5] << 16, u[6] | (unsigned)u[7] << 16);
    }
    return r;
}
template <typename T>
__device__ __forceinline__ Raw8<T> zero_raw8() {
    Raw8<T> r;
    r.w[0] = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (sizeof(T) == 4) r.w[1] = r.w[0];
    return r;
}
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float (&x)[8]) {
    const unsigned w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
    if constexpr (sizeof(T) == 4) {
        const unsigned v[4] = {r.w[1].x, r.w[1].y, r.w[1].z, r.w[1].w};
#pragma unroll
        for (int i = 0; i < 4; i++) { x[i] = __uint_as_float(w[i]); x[4 + i] = __uint_as_float(v[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
}

// Two fp32 products and sums in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
        " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// Eight consecutive floats.  vec: p is 16-byte aligned; else the elements are loaded one by one.
__device__ __forceinline__ void load8(const float* p, bool vec, float (&x)[8]) {
    if (vec) {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = p[i];
    }
}

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// fp8_row_exp for any largest magnitude, an infinite one included (which gives 120): from the bits of amax, whose NaNs
// the maximum has dropped.  amax = 1.m * 2^(field - 127); 448 = 1.75 * 2^8.  Subnormals land below the clamp.
__device__ __forceinline__ int row_exp_any(float amax) {
    if (!(amax > 0.f)) return 0;
    const unsigned b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(-120, min(120, e));
}

// This lane's elements into a cache row (`row`: its index in the whole pool): NC runs of eight, run c at l * 8 + c * HD / NC
// of the row, HD / 8 / NC lanes per row.  All lanes of the row's group call it together; the maximum of an FP8 row is
// exchanged inside the group.
template <int HD, int NC>
__device__ __forceinline__ void store_cache(const dynakv_row_cache& c, bool is_v, long long row, bool live, int l, const float (&x)[NC][8]) {
    constexpr int LG = HD / 8 / NC;
    void* pool = is_v ? c.v : c.k;
    const size_t at = (size_t)row * HD + l * 8;
    if (c.kv_dtype == DYNAKV_F32) {
        if (live) {
#pragma unroll
            for (int y = 0; y < NC; y++) store8(reinterpret_cast<float*>(pool) + at + y * (HD / NC), x[y]);
        }
    } else if (c.kv_dtype == DYNAKV_BF16) {
        if (live) {
#pragma unroll
            for (int y = 0; y < NC; y++) store8(reinterpret_cast<__nv_bfloat16*>(pool) + at + y * (HD / NC), x[y]);
        }
    } else {
        float m = 0.f;
#pragma unroll
        for (int y = 0; y < NC; y++)
#pragma unroll
            for (int i = 0; i < 8; i++) m = fmaxf(m, fabsf(x[y][i]));
        m = group_max(m, LG);
        const int e = row_exp_any(m);
        const float inv = pow2f(-e);
#pragma unroll
        for (int y = 0; y < NC; y++) {
            uint2 b;
            b.x = fp8_pack2(x[y][0], x[y][1], inv) | ((unsigned)fp8_pack2(x[y][2], x[y][3], inv) << 16);
            b.y = fp8_pack2(x[y][4], x[y][5], inv) | ((unsigned)fp8_pack2(x[y][6], x[y][7], inv) << 16);
            if (live) *reinterpret_cast<uint2*>(reinterpret_cast<unsigned char*>(pool) + at + y * (HD / NC)) = b;
        }
        if (live && l == 0) (is_v ? c.v_exp : c.k_exp)[row] = (int8_t)e;
    }
}

// Element e of a row of the pool, as a number.
template <int DT>
__device__ __forceinline__ float cache_elem(const unsigned char* pool, const signed char* exps, long long row, int hd, int e) {
    if constexpr (DT == DYNAKV_F32) return reinterpret_cast<const float*>(pool)[row * hd + e];
    else if constexpr (DT == DYNAKV_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(pool)[row * hd + e]);
    else return fp8_unpack2((unsigned short)pool[row * hd + e], pow2f(exps[row])).x;
}

// Host side: what every call on a cache checks.
static inline bool row_cache_ok(const dynakv_row_cache* c) {
    if (!c || !c->k || !c->v || c->n_pages < 1 || c->n_kv_heads < 1 || (c->head_dim != 64 && c->head_dim != 128)) return false;
    if (c->kv_dtype != DYNAKV_F32 && c->kv_dtype != DYNAKV_BF16 && c->kv_dtype != DYNAKV_FP8) return false;
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return false;
    if (c->kv_dtype == DYNAKV_FP8 && (!c->k_exp || !c->v_exp || (((uintptr_t)c->k_exp | (uintptr_t)c->v_exp) & 15))) return false;
    return c->n_pages < (1ll << 31) && c->n_pages * c->n_kv_heads < (1ll << 26);      // rows of 32-row pages fit 31 bits
}

}  // namespace dkv
