// Activations in 8 bits: the codec, and act(a) (.) b with its gradient out of the saved bytes.
//
// All four are streams: a lane takes eight consecutive features of a row (16 bytes of a 16-bit type), four
// lanes in a row are a group of 32, so a group's largest magnitude is two moves between neighbouring lanes
// and no element is read twice.  Items (a lane's eight features) are numbered through the matrix, each row
// padded to whole groups: one launch whatever the shape, no wavefront half empty because a row is short.
//
// Measured (8,192 x 8,192 bf16, gated SiLU): forward 89 us, backward 89 us, 6.1 TB/s each: memory.  16,384 x 768 bf16:
// encode 9 us, decode 7 us (4.2 and 5.2 TB/s: a launch's start and end).
#include "device.hip.h"

namespace deto {
namespace model {
namespace {

constexpr int kThreads = kItemThreads;

int check_shape(int64_t T, int64_t D) {
    return T < 0 || D < 1 || D > (int64_t{1} << 30) ? DETO_ERR_BAD_CONFIG : DETO_OK;
}

template <int DT, bool ONCE>
__global__ __launch_bounds__(kThreads) void encode_kernel(Items items, deto_rows x, deto_act8 x8) {
    const auto at = items.at(blockIdx.x * kThreads + threadIdx.x);
    float v[8];
    unpack8<DT>(load8<DT, ONCE>(x.data, at.t * x.ld, at.d, at.count), v);
    act8_put<ONCE>(x8, at.t, at.d, v, at.count);
}

template <int DT, bool ONCE>
__global__ __launch_bounds__(kThreads) void decode_kernel(Items items, deto_act8 x8, deto_rows x) {
    const auto at = items.at(blockIdx.x * kThreads + threadIdx.x);
    float v[8];
    act8_get<ONCE>(x8, at.t, at.d, v, at.count);
    store8<DT, ONCE>(x.data, at.t * x.ld + at.d, v, at.count);
}

// e^x for results of type DT.  The fast form rounds x / log 2 first, which is up to |x| 2^-24 of its value: 2^-19 of SiLU(-20),
// nothing in a 16-bit result (or in one of 8 bits made beside it), but more than fp32's rounding.  (8,192 x 8,192 bf16, SiLU
// without a gate, forward and backward, us: 117, with expf 139; gated 183 and 203.  4,096 x 8,192 fp32: 173 and 174.)
template <int DT>
__device__ __forceinline__ float exponential(float x) {
    if constexpr (DT == DETO_F32) return expf(x);
    else return __expf(x);
}

// act(x), and its slope where that is asked for
template <int DT, int ACT>
__device__ __forceinline__ float act_value(float x) {
    if constexpr (ACT == DETO_ACT_RELU) return x > 0.f ? x : (x != x ? x : 0.f);
    else if constexpr (ACT == DETO_ACT_SILU) return x / (1.f + exponential<DT>(-x));
    else if constexpr (ACT == DETO_ACT_GELU) return 0.5f * x * (1.f + erff(x * 0.70710678118654752f));
    else return 0.5f * x * (1.f + tanhf(0.79788456080286536f * (x + 0.044715f * x * x * x)));
}

template <int DT, int ACT>
__device__ __forceinline__ void act_both(float x, float& value, float& slope) {
    if constexpr (ACT == DETO_ACT_RELU) {
        value = act_value<DT, ACT>(x);
        slope = x > 0.f ? 1.f : (x != x ? x : 0.f);
    } else if constexpr (ACT == DETO_ACT_SILU) {
        const float g = 1.f / (1.f + exponential<DT>(-x));
        value = x * g;
        slope = g * (1.f + x * (1.f - g));
    } else if constexpr (ACT == DETO_ACT_GELU) {
        const float p = 0.5f * (1.f + erff(x * 0.70710678118654752f));
        value = x * p;
        slope = p + x * 0.39894228040143268f * exponential<DT>(-0.5f * x * x);
    } else {
        const float t = tanhf(0.79788456080286536f * (x + 0.044715f * x * x * x));
        value = 0.5f * x * (1.f + t);
        const float square = fminf(x * x, 256.f);       // (from there on 1 - t t is 0, and has to meet a number)
        slope = 0.5f * (1.f + t) +
                0.5f * x * (1.f - t * t) * 0.79788456080286536f * (1.f + 3.f * 0.044715f * square);
    }
}

template <int DT, int ACT, bool GATED, bool ONCE>
__global__ __launch_bounds__(kThreads) void glu_forward_kernel(Items items, deto_rows a, deto_rows b,
                                                               deto_rows h, deto_act8 a8,
                                                               deto_act8 b8) {
    const auto at = items.at(blockIdx.x * kThreads + threadIdx.x);
    const Raw8<DT> ra = load8<DT, ONCE>(a.data, at.t * a.ld, at.d, at.count);
    Raw8<DT> rb = {};
    if constexpr (GATED) rb = load8<DT, ONCE>(b.data, at.t * b.ld, at.d, at.count);
    float va[8], vb[8], vh[8];
    unpack8<DT>(ra, va);
    unpack8<DT>(rb, vb);
#pragma unroll
    for (int j = 0; j < 8; ++j) vh[j] = act_value<DT, ACT>(va[j]) * (GATED ? vb[j] : 1.f);
    if (a8.codes) act8_put<ONCE>(a8, at.t, at.d, va, at.count);
    if (GATED && b8.codes) act8_put<ONCE>(b8, at.t, at.d, vb, at.count);
    store8<DT, ONCE>(h.data, at.t * h.ld + at.d, vh, at.count);
}

template <int DT, int ACT, bool GATED, bool ONCE>
__global__ __launch_bounds__(kThreads) void glu_backward_kernel(Items items, deto_rows dh,
                                                                deto_act8 a8, deto_act8 b8,
                                                                deto_rows da, deto_rows db,
                                                                deto_act8 h8) {
    const auto at = items.at(blockIdx.x * kThreads + threadIdx.x);
    const Raw8<DT> rd = load8<DT, ONCE>(dh.data, at.t * dh.ld, at.d, at.count);
    float va[8], vb[8], vd[8], vh[8];
    act8_get<ONCE>(a8, at.t, at.d, va, at.count);
    if constexpr (GATED) act8_get<ONCE>(b8, at.t, at.d, vb, at.count);
    unpack8<DT>(rd, vd);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float value, slope;
        act_both<DT, ACT>(va[j], value, slope);
        va[j] = GATED ? vd[j] * vb[j] * slope : vd[j] * slope;
        vh[j] = GATED ? value * vb[j] : value;
        if constexpr (GATED) vb[j] = vd[j] * value;
    }
    if (h8.codes) act8_put<ONCE>(h8, at.t, at.d, vh, at.count);
    store8<DT, ONCE>(da.data, at.t * da.ld + at.d, va, at.count);
    if constexpr (GATED) store8<DT, ONCE>(db.data, at.t * db.ld + at.d, vb, at.count);
}

// Matrices that the caches do not hold until the next kernel takes them are loaded and stored without a trace there.  (8,192 x
// 8,192 bf16, gated SiLU forward and backward, us: 182, with the outputs left there 190; forward with the product that reads h
// next 285 and 278.)
template <class F>
int by_size(int64_t T, int64_t D, int dtype, F f) {
    return T * D * type_size(dtype) >= kCacheBytes / 4 ? f(std::true_type{}) : f(std::false_type{});
}

template <class F>
int by_act(int act, bool gated, F f) {
    auto g = [&](auto a) { return gated ? f(a, std::true_type{}) : f(a, std::false_type{}); };
    switch (act) {
        case DETO_ACT_SILU: return g(Type<DETO_ACT_SILU>{});
        case DETO_ACT_GELU: return g(Type<DETO_ACT_GELU>{});
        case DETO_ACT_GELU_TANH: return g(Type<DETO_ACT_GELU_TANH>{});
        default: return g(Type<DETO_ACT_RELU>{});
    }
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int detonation_act8_encode(int64_t T, int64_t D, const deto_rows* x, const deto_act8* x8,
                           void* stream) {
    int rc = check_shape(T, D);
    if (rc || T == 0) return rc;
    if (!here(x) || !here(x8)) return DETO_ERR_NULL;
    rc = first_error(check_rows(x, T, D), check_act8(x8, T, D));
    if (rc) return rc;
    return for_items(T, D, [&](const Items& it, unsigned grid) {
        by_type(x->dtype, [&](auto dt) {
            return by_size(T, D, x->dtype, [&](auto once) {
                encode_kernel<dt.value, once.value>
                    <<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(it, *x, *x8);
                return 0;
            });
        });
    });
}

int detonation_act8_decode(int64_t T, int64_t D, const deto_act8* x8, const deto_rows* x,
                           void* stream) {
    int rc = check_shape(T, D);
    if (rc || T == 0) return rc;
    if (!here(x) || !here(x8)) return DETO_ERR_NULL;
    rc = first_error(check_rows(x, T, D), check_act8(x8, T, D));
    if (rc) return rc;
    return for_items(T, D, [&](const Items& it, unsigned grid) {
        by_type(x->dtype, [&](auto dt) {
            return by_size(T, D, x->dtype, [&](auto once) {
                decode_kernel<dt.value, once.value>
                    <<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(it, *x8, *x);
                return 0;
            });
        });
    });
}

int detonation_glu_forward(int act, int64_t T, int64_t D, const deto_rows* a, const deto_rows* b,
                           const deto_rows* h, const deto_act8* a8, const deto_act8* b8,
                           void* stream) {
    int rc = check_shape(T, D);
    if (rc) return rc;
    if (act < DETO_ACT_SILU || act > DETO_ACT_RELU) return DETO_ERR_BAD_CONFIG;
    if (T == 0) return DETO_OK;
    const bool gated = here(b);
    if (!here(a) || !here(h)) return DETO_ERR_NULL;
    if (here(b8) && !gated) return DETO_ERR_BAD_CONFIG;
    rc = first_error(check_rows(a, T, D), gated ? check_rows(b, T, D) : 0, check_rows(h, T, D),
                     here(a8) ? check_act8(a8, T, D) : 0, here(b8) ? check_act8(b8, T, D) : 0);
    if (rc) return rc;
    if (h->dtype != a->dtype || (gated && b->dtype != a->dtype)) return DETO_ERR_BAD_CONFIG;
    const deto_rows none = {};
    const deto_act8 none8 = {};
    return for_items(T, D, [&](const Items& it, unsigned grid) {
        by_type(a->dtype, [&](auto dt) {
            return by_act(act, gated, [&](auto k, auto g) {
                return by_size(T, D, a->dtype, [&](auto once) {
                    glu_forward_kernel<dt.value, k.value, g.value, once.value>
                        <<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                            it, *a, gated ? *b : none, *h, here(a8) ? *a8 : none8, here(b8) ? *b8 : none8);
                    return 0;
                });
            });
        });
    });
}

int detonation_glu_backward(int act, int64_t T, int64_t D, const deto_rows* dh, const deto_act8* a8,
                            const deto_act8* b8, const deto_rows* da, const deto_rows* db,
                            const deto_act8* h8, void* stream) {
    int rc = check_shape(T, D);
    if (rc) return rc;
    if (act < DETO_ACT_SILU || act > DETO_ACT_RELU) return DETO_ERR_BAD_CONFIG;
    if (T == 0) return DETO_OK;
    const bool gated = here(b8);
    if (!here(dh) || !here(a8) || !here(da) || (gated && !here(db))) return DETO_ERR_NULL;
    if (!gated && here(db)) return DETO_ERR_BAD_CONFIG;
    rc = first_error(check_rows(dh, T, D), check_rows(da, T, D), gated ? check_rows(db, T, D) : 0,
                     check_act8(a8, T, D), gated ? check_act8(b8, T, D) : 0,
                     here(h8) ? check_act8(h8, T, D) : 0);
    if (rc) return rc;
    if (da->dtype != dh->dtype || (gated && db->dtype != dh->dtype)) return DETO_ERR_BAD_CONFIG;
    const deto_rows none = {};
    const deto_act8 none8 = {};
    return for_items(T, D, [&](const Items& it, unsigned grid) {
        by_type(dh->dtype, [&](auto dt) {
            return by_act(act, gated, [&](auto k, auto g) {
                return by_size(T, D, dh->dtype, [&](auto once) {
                    glu_backward_kernel<dt.value, k.value, g.value, once.value>
                        <<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                            it, *dh, *a8, gated ? *b8 : none8, *da, gated ? *db : none,
                            here(h8) ? *h8 : none8);
                    return 0;
                });
            });
        });
    });
}

}  // extern "C"
