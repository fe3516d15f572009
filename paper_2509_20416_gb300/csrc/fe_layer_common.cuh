// Device helpers shared by the dense operators: activations and the products' epilogue.
#pragma once

#include "fe_layer_kernels.h"
#include "fe_target_common.cuh"

namespace fe {

__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ float load_one(const bf16_t* p) { return bf16_to_f32(p->bits); }

// 1 / (1 + e^-x); 0 and 1 at the ends. FAST: by the hardware's approximations, off by some 2^-21, for
// results that are rounded to bfloat16 (a tile of 128 x 256 is finished while the next is summed only with them)
template <bool FAST>
__device__ __forceinline__ float sigmoid(float x) {
    if (FAST) return __fdividef(1.0f, 1.0f + ex2_approx(-kLog2e * x));
    return 1.0f / (1.0f + expf(-x));
}

constexpr float kGeluA = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.07135481627260025f;  // kGeluA * 0.044715

// (1 + tanh(u)) / 2 = sigmoid(2 u). Past |z| = 12 the cube adds nothing to a sigmoid that is 0 or 1
// in float32, and a square that overflows would make the gradient's 0 times it NaN.
template <bool FAST>
__device__ __forceinline__ float act_value(int act, float z) {
    switch (act) {
        case FE_ACT_RELU: return z < 0.f ? 0.f : z;
        case FE_ACT_SILU: return z * sigmoid<FAST>(z);
        case FE_ACT_GELU: {
            const float c = fminf(fmaxf(z, -12.f), 12.f);
            const float s = sigmoid<FAST>(c * (kGeluA + kGeluB * c * c));
            return (z < -12.f && z > -INFINITY) ? 0.f : z * s;
        }
        default: return z;
    }
}

// act(z) and act'(z)
template <bool FAST>
__device__ __forceinline__ void act_both(int act, float z, float& v, float& dv) {
    switch (act) {
        case FE_ACT_RELU:
            v = z < 0.f ? 0.f : z;
            dv = z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
            return;
        case FE_ACT_SILU: {
            const float s = sigmoid<FAST>(z);
            v = z * s;
            dv = s * (1.f + z * (1.f - s));
            return;
        }
        case FE_ACT_GELU: {
            const float c = fminf(fmaxf(z, -12.f), 12.f);
            const float s = sigmoid<FAST>(c * (kGeluA + kGeluB * c * c));
            v = (z < -12.f && z > -INFINITY) ? 0.f : z * s;
            dv = s + c * s * (1.f - s) * (kGeluA + 3.f * kGeluB * c * c);
            if (z != z) dv = z;
            return;
        }
        default:
            v = z;
            dv = 1.f;
    }
}

// a template parameter for the type whose results are rounded coarsely
template <typename T> constexpr bool kCoarse = sizeof(T) == 2;

// N consecutive elements of a row (N a multiple of 16 bytes where vec, else any) from and to floats;
// elements from `have` on are left out
template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, int have, bool vec, float* f) {
    constexpr int V = Vec16<T>::kN;
    if (N % V == 0 && vec && have >= N) {
#pragma unroll
        for (int i = 0; i < N / V; ++i) Vec16<T>::widen(reinterpret_cast<const uint4*>(p)[i], f + i * V);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = i < have ? load_one(p + i) : 0.f;
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, int have, bool vec, const float* f) {
    constexpr int V = Vec16<T>::kN;
    if (N % V == 0 && vec && have >= N) {
#pragma unroll
        for (int i = 0; i < N / V; ++i) reinterpret_cast<uint4*>(p)[i] = pack16<T>(f + i * V);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) store_one(p + i, f[i]);
    }
}

// What becomes of a float32 product: NV columns of row m from column n on, of a plain product z (overwritten)
template <int NV>
__device__ __forceinline__ void epilogue_plain(const Finish& e, int64_t m, int n, int N, float* z) {
    const int have = N - n;
    if (have <= 0) return;
    float t[NV];
    if (e.bias) {
        load_row<float, NV>((const float*)e.bias + n, have, e.vec, t);
#pragma unroll
        for (int i = 0; i < NV; ++i) z[i] += t[i];
    }
    if (e.pre) store_row<float, NV>(e.pre + m * e.pre_row + n, have, e.vec, z);
    if (e.act != FE_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < NV; ++i) z[i] = act_value<false>(e.act, z[i]);
    }
    if (e.res) {
        load_row<float, NV>((const float*)e.res + m * e.res_row + n, have, e.vec, t);
#pragma unroll
        for (int i = 0; i < NV; ++i) z[i] += t[i];
    }
    store_row<float, NV>((float*)e.out + m * e.out_row + n, have, e.vec, z);
}

// the same of a gated pair of products g and u (g is overwritten)
template <int NV>
__device__ __forceinline__ void epilogue_gated(const Finish& e, int64_t m, int n, int N, float* g, const float* u) {
    const int have = N - n;
    if (have <= 0) return;
    if (e.pre) {
        store_row<float, NV>(e.pre + m * e.pre_row + n, have, e.vec, g);
        store_row<float, NV>(e.pre2 + m * e.pre2_row + n, have, e.vec, u);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) g[i] = act_value<false>(e.act, g[i]) * u[i];
    store_row<float, NV>((float*)e.out + m * e.out_row + n, have, e.vec, g);
}

// the gradients of a gated pair for the product z = dh, and the pair's own result
template <int NV>
__device__ __forceinline__ void epilogue_gated_grad(const Finish& e, int64_t m, int n, int N, float* z) {
    const int have = N - n;
    if (have <= 0) return;
    float g[NV], u[NV];
    load_row<float, NV>(e.pre + m * e.pre_row + n, have, e.vec, g);
    load_row<float, NV>(e.pre2 + m * e.pre2_row + n, have, e.vec, u);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float v, dv;
        act_both<false>(e.act, g[i], v, dv);
        g[i] = z[i] * v;
        dv *= z[i] * u[i];
        u[i] *= v;
        z[i] = dv;
    }
    store_row<float, NV>((float*)e.out + m * e.out_row + n, have, e.vec, z);
    store_row<float, NV>((float*)e.out2 + m * e.out2_row + n, have, e.vec, g);
    store_row<float, NV>((float*)e.out3 + m * e.out3_row + n, have, e.vec, u);
}

template <int NV>
__device__ __forceinline__ void epilogue_one(const Finish& e, int64_t m, int n, int N, float* z) {
    if (e.kind == FINISH_GATED_GRAD) epilogue_gated_grad<NV>(e, m, n, N, z);
    else epilogue_plain<NV>(e, m, n, N, z);
}

}  // namespace fe
