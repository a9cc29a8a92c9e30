// What the forward and the backward kernels of norm, gate and residual share: how rows are laid over a
// workgroup, sums over a row, the launch by width.
//
// A row is taken by a team of W wavefronts, a lane C vectors of eight features.  Up to 1,024 features a team is
// one wavefront, which needs no barrier (four teams a workgroup); wider rows take a workgroup.
#pragma once

#include "device.hip.h"

namespace deto {
namespace model {

constexpr int64_t kMaxNormWidth = 16384;

template <int W, int C>
struct Team {
    static constexpr int kWavesWg = W == 1 ? 4 : W;
    static constexpr int kThreadsWg = kWavesWg * kLanes;
    static constexpr int kTeamsWg = kWavesWg / W;
    static constexpr int kSlots = 2 * kWavesWg * 4;    // floats of LDS for sums

    float* lds;
    int parity = 0;

    __device__ __forceinline__ explicit Team(float* l) : lds(l) {}
    static __device__ __forceinline__ int wave() { return threadIdx.x / kLanes % W; }
    static __device__ __forceinline__ int64_t index() {     // of the team in the launch
        return static_cast<int64_t>(blockIdx.x) * kTeamsWg + threadIdx.x / kLanes / W;
    }
    // first feature of vector c: lanes of a wavefront side by side
    static __device__ __forceinline__ int feature(int c) {
        return 8 * ((c * W + wave()) * kLanes + static_cast<int>(threadIdx.x % kLanes));
    }
    static __device__ __forceinline__ int count(int c, int D) {
        const int left = D - feature(c);
        return left >= 8 ? 8 : left > 0 ? left : 0;
    }
    // N sums over the row, in every lane.  Two sets of slots in turn: one barrier a sum, since a wavefront that
    // writes a set again has passed the barrier of the set between, which all reach after reading this one.
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N]) {
        static_assert(N <= 4, "slots");
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
        if constexpr (W > 1) {
            float* at = lds + parity * kWavesWg * 4;
            if (threadIdx.x % kLanes == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) at[wave() * 4 + i] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = at[i];
#pragma unroll
                for (int w = 1; w < W; ++w) v[i] += at[w * 4 + i];
            }
            parity ^= 1;
        }
    }
};

// Teams by width, for a generic lambda that takes Team's arguments as types.
template <class F>
inline void by_width(int64_t D, F f) {
    if (D <= 512) f(Type<1>{}, Type<1>{});
    else if (D <= 1024) f(Type<1>{}, Type<2>{});
    else if (D <= 2048) f(Type<4>{}, Type<1>{});
    else if (D <= 4096) f(Type<8>{}, Type<1>{});
    else if (D <= 8192) f(Type<16>{}, Type<1>{});
    else f(Type<16>{}, Type<2>{});
}

inline bool valid_kind(int k) { return k >= DETO_NORM_NONE && k <= DETO_NORM_LAYER; }

// deto_status of a configuration for T rows of D
inline int check_norm(const deto_norm_residual* c, int64_t T, int64_t D) {
    if (!c) return DETO_ERR_NULL;
    if (!valid_kind(c->pre) || !valid_kind(c->post) || !valid_type(c->param_dtype))
        return DETO_ERR_BAD_CONFIG;
    if (!(c->eps_pre >= 0.f) || !(c->eps_post >= 0.f) || !std::isfinite(c->eps_pre) ||
        !std::isfinite(c->eps_post) || !std::isfinite(c->scale))
        return DETO_ERR_BAD_CONFIG;
    if (T < 0 || D < 1 || c->rows_per_gate < 0) return DETO_ERR_BAD_CONFIG;
    if (D > kMaxNormWidth) return DETO_ERR_UNSUPPORTED;
    if (c->gate && c->rows_per_gate && T > c->rows_per_gate && c->ld_gate < D)
        return DETO_ERR_BAD_CONFIG;
    const size_t a = type_size(c->param_dtype);
    return is_aligned(c->w_pre, a) && is_aligned(c->b_pre, a) && is_aligned(c->w_post, a) &&
                   is_aligned(c->b_post, a) && is_aligned(c->gate, a)
               ? DETO_OK
               : DETO_ERR_ALIGN;
}

// f(Type<x's type>, Type<f's type>): x is fp32 or of f's type
template <class F>
inline int by_types(int xt, int ft, F f) {
    return by_type(ft, [&](auto t) {
        return xt == t.value ? f(t, t) : f(Type<DETO_F32>{}, t);
    });
}

}  // namespace model
}  // namespace deto
