// What the forward and the backward kernels of norm, gate and residual share: how rows are laid over a
// workgroup, sums over a row, the launch by width.
//
// A row is taken by a team of W wavefronts, a lane C vectors of eight features.  Up to 512 features a team is
// one wavefront or a part of L lanes of one, which needs no barrier (several teams a workgroup); wider rows take a
// workgroup.
#pragma once

#include <type_traits>

#include "device.hip.h"

namespace deto {
namespace model {

constexpr int64_t kMaxNormWidth = 16384;

// WHOLE: rows of a multiple of eight features, a lane's vectors are whole or empty.
// HALVES (of WHOLE rows): a lane's eight features of a vector are two times four, half the vector's width apart.  An fp32
// access of all lanes is then one run of memory instead of every other 16 bytes of two (forward, 16,384 x 2,048, fp32 and
// bf16, us: 71 / 60), a 16-bit one two runs instead of one.
template <int W, int C, int L, bool WHOLE, bool HALVES = false>
struct Team {
    static_assert(WHOLE || !HALVES, "halves are whole");
    static_assert(W == 1 || L == kLanes, "a part of a wavefront is a team by itself");
    static constexpr int kWavesWg = W == 1 ? 4 : W;
    static constexpr int kThreadsWg = kWavesWg * kLanes;
    static constexpr int kTeamsWg = kThreadsWg / (W * L);
    // A lane of a workgroup of 1,024 has 128 registers: not enough to hold the parameters and the next row too.  (Backward,
    // and forward above 8,192 features or with a layer norm, they spill all the same: RMS backward at 8,192 x 5,120, fp32 and
    // bf16, 4.0 TB/s where 4,096 features have 4.7, two layer norms 0.9.)
    static constexpr bool kLean = W >= 16;
    static constexpr int kSlots = 2 * kWavesWg * 4;    // floats of LDS for sums

    float* lds;
    int parity = 0;

    __device__ __forceinline__ explicit Team(float* l) : lds(l) {}
    static __device__ __forceinline__ int wave() { return threadIdx.x / kLanes % W; }
    static __device__ __forceinline__ int64_t index() {     // of the team in the launch
        return static_cast<int64_t>(blockIdx.x) * kTeamsWg + threadIdx.x / (W * L);
    }
    // first feature of vector c: lanes of a wavefront side by side
    static __device__ __forceinline__ int feature(int c) {
        return 8 * ((c * W + wave()) * L + static_cast<int>(threadIdx.x % L));
    }
    // first feature of half h of vector c
    static __device__ __forceinline__ int half(int c, int h) {
        return 8 * (c * W + wave()) * L + 4 * (h * L + static_cast<int>(threadIdx.x % L));
    }
    // whether value j of vector c is there
    static __device__ __forceinline__ bool has(int c, int j, int D) {
        if constexpr (HALVES) return half(c, j / 4) < D;
        return j < count(c, D);
    }
    template <int DT>
    static __device__ __forceinline__ void store4(char* p, const float (&v)[4], bool once) {
        using Vec = std::conditional_t<DT == DETO_F32, u32x4_any4, u32x2_any2>;
        Vec a;
        if constexpr (DT == DETO_F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = f32_bits(v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j)
                a[j] = DT == DETO_BF16 ? pack_bf16(v[2 * j], v[2 * j + 1]) : pack_f16(v[2 * j], v[2 * j + 1]);
        }
        if (once) {
            asm volatile("");            // (or the two stores become one, without the hint)
            __builtin_nontemporal_store(a, reinterpret_cast<Vec*>(p));
            asm volatile("");
        } else {
            *reinterpret_cast<Vec*>(p) = a;
        }
    }
    // a row of y in 8 bits
    static __device__ __forceinline__ void put8(const deto_act8& m, int64_t t, int c, int D, const float (&v)[8]) {
        if constexpr (!HALVES) {
            act8_put(m, t, feature(c), v, count(c, D));
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float four[4] = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                const int d = half(c, h);
                uint32_t e;
                const uint32_t codes = act8_encode4(four, e);
                if (d < D) {
                    *reinterpret_cast<u32_any1*>(m.codes + t * m.ld_codes + d) = codes;
                    if (d % DETO_ACT8_GROUP == 0) m.exps[t * m.ld_exps + d / DETO_ACT8_GROUP] = static_cast<uint8_t>(e);
                }
            }
        }
    }
    static __device__ __forceinline__ int count(int c, int D) {
        const int left = D - feature(c);
        if constexpr (WHOLE) return left > 0 ? 8 : 0;
        return left >= 8 ? 8 : left > 0 ? left : 0;
    }
    template <int DT>
    static __device__ __forceinline__ Raw8<DT> load(const void* base, int64_t row, int c, int D) {
        if constexpr (!WHOLE) {
            // Past the row's end: its last eight features, put right by unpack().  (A branch here would make each of
            // a row's loads wait for the one before: 16,384 x 2,047 bf16, backward, 170 us instead of 116.)
            if (D < 8) return load8<DT>(base, row, feature(c), count(c, D));
            const int d = feature(c) < D - 8 ? feature(c) : D - 8;
            return load8_whole<DT>(static_cast<const char*>(base) + (row + d) * kSize<DT>);
        }
        Raw8<DT> r = {};
        if constexpr (HALVES) {
            const char* p = static_cast<const char*>(base) + row * kSize<DT>;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (half(c, h) < D) {
                    const char* q = p + half(c, h) * kSize<DT>;
                    if constexpr (DT == DETO_F32) {
                        (h ? r.b : r.a) = *reinterpret_cast<const u32x4_any4*>(q);
                    } else {
                        const u32x2 v = *reinterpret_cast<const u32x2_any2*>(q);
                        r.a[2 * h] = v[0];
                        r.a[2 * h + 1] = v[1];
                    }
                }
            return r;
        }
        if (feature(c) < D) r = load8<DT>(base, row, feature(c), 8);
        return r;
    }
    // the values of what load() gave, zeros past the row's end
    template <int DT>
    static __device__ __forceinline__ void unpack(Raw8<DT> r, int c, int D, float (&v)[8]) {
        if constexpr (!WHOLE) {
            const int by = feature(c) - (D - 8);
            if (D >= 8 && by > 0) {
                if (by < 8) move_down<DT>(r, by);
                else r = {};
            }
        }
        unpack8<DT>(r, v);
    }
    static __device__ __forceinline__ void load_any(const void* base, int dtype, int64_t row, int c, int D,
                                                    float (&v)[8]) {
        if (dtype == DETO_F32) unpack<DETO_F32>(load<DETO_F32>(base, row, c, D), c, D, v);
        else if (dtype == DETO_BF16) unpack<DETO_BF16>(load<DETO_BF16>(base, row, c, D), c, D, v);
        else unpack<DETO_F16>(load<DETO_F16>(base, row, c, D), c, D, v);
    }
    // (once: past the caches)
    template <int DT>
    static __device__ __forceinline__ void store(void* base, int64_t row, int c, int D, const float (&v)[8],
                                                 bool once = false) {
        if constexpr (!WHOLE) store8<DT>(base, row + feature(c), v, count(c, D));
        else if constexpr (HALVES) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (half(c, h) < D) {
                    const float four[4] = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                    store4<DT>(static_cast<char*>(base) + (row + half(c, h)) * kSize<DT>, four, once);
                }
        } else if (feature(c) < D) {
            if (once) {
                asm volatile("");        // (or the two stores become one, without the hint)
                store8<DT, true>(base, row + feature(c), v, 8);
                asm volatile("");
            } else {
                store8<DT>(base, row + feature(c), v, 8);
            }
        }
    }
    // N sums over the row, in every lane.  Two sets of slots in turn: one barrier a sum, since a wavefront that
    // writes a set again has passed the barrier of the set between, which all reach after reading this one.
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N]) {
        static_assert(N <= 4, "slots");
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_sum<L>(v[i]);
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
    auto g = [&](auto w, auto c, auto l) {
        if (D % 8 == 0) f(w, c, l, std::true_type{});
        else f(w, c, l, std::false_type{});
    };
    if (D <= 128) g(Type<1>{}, Type<1>{}, Type<16>{});
    else if (D <= 256) g(Type<1>{}, Type<1>{}, Type<32>{});
    else if (D <= 512) g(Type<1>{}, Type<1>{}, Type<64>{});
    else if (D <= 1024) g(Type<2>{}, Type<1>{}, Type<64>{});
    else if (D <= 2048) g(Type<4>{}, Type<1>{}, Type<64>{});
    else if (D <= 4096) g(Type<8>{}, Type<1>{}, Type<64>{});
    else if (D <= 8192) g(Type<16>{}, Type<1>{}, Type<64>{});
    else g(Type<16>{}, Type<2>{}, Type<64>{});
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
