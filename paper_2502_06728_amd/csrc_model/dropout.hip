// Dropout from a counter-based generator: out = residual + kept x / (1 - rate), the mask never stored.
//
// A stream: a lane takes eight consecutive features of a row, and one Philox counter gives them 16 bits each.  So the
// same call drops the same elements wherever it runs, forward and backward, whatever the types and strides.
//
// Philox 4x32 (Salmon, Moraes, Dror and Shaw, 2011): ten rounds of two 32 x 32 -> 64 bit products, which the vector
// units do at a quarter of their rate.  32 bits an element would take two counters and make the products the bound for
// 16-bit matrices.  Bound by memory: 16,384 x 2,048, bf16 onto an fp32 residual 61 us (5.5 TB/s), its gradient 28 (7.2: part
// of it stays in the caches); 197 x 771 fp16 2.8 (a launch).
#include "device.hip.h"

namespace deto {
namespace model {
namespace {

constexpr int kThreads = kItemThreads;

struct Draw {
    uint64_t seed, offset;
    const uint64_t* more;
    uint32_t dropped;      // of 65536
    float scale;           // of what is kept
};

__device__ __forceinline__ u32x4 philox(u32x4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = uint64_t{0xD2511F53u} * c[0], r = uint64_t{0xCD9E8D57u} * c[2];
        c = {static_cast<uint32_t>(r >> 32) ^ c[1] ^ k0, static_cast<uint32_t>(r),
             static_cast<uint32_t>(p >> 32) ^ c[3] ^ k1, static_cast<uint32_t>(p)};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

template <int IN, int OUT, bool ADD, bool ONCE>
__global__ __launch_bounds__(kThreads) void dropout_kernel(Items items, Draw draw, deto_rows x, deto_rows residual,
                                                           deto_rows out) {
    const auto at = items.at(blockIdx.x * kThreads + threadIdx.x);
    const Raw8<IN> rx = load8<IN, ONCE>(x.data, at.t * x.ld, at.d, at.count);
    Raw8<OUT> rr = {};
    if constexpr (ADD) rr = load8<OUT, ONCE>(residual.data, at.t * residual.ld, at.d, at.count);
    const uint64_t offset = draw.offset + (draw.more ? *draw.more : 0);
    const u32x4 bits = philox(u32x4{static_cast<uint32_t>(at.d / 8), static_cast<uint32_t>(at.t),
                                    static_cast<uint32_t>(offset), static_cast<uint32_t>(offset >> 32)},
                              static_cast<uint32_t>(draw.seed), static_cast<uint32_t>(draw.seed >> 32));
    float v[8], r[8];
    unpack8<IN>(rx, v);
    unpack8<OUT>(rr, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t word = bits[j / 2], own = j % 2 ? word >> 16 : word & 0xFFFFu;
        const float kept = own >= draw.dropped ? v[j] * draw.scale : 0.f;     // (what is dropped may be a NaN)
        v[j] = ADD ? r[j] + kept : kept;
    }
    store8<OUT, ONCE>(out.data, at.t * out.ld + at.d, v, at.count);
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int detonation_dropout(const deto_dropout* cfg, int64_t T, int64_t D, const deto_rows* x,
                       const deto_rows* residual, const deto_rows* out, void* stream) {
    if (!cfg) return DETO_ERR_NULL;
    if (T < 0 || T > (int64_t{1} << 32) || D < 1 || D > (int64_t{1} << 30)) return DETO_ERR_BAD_CONFIG;
    if (!(cfg->rate >= 0.f && cfg->rate < 1.f) || cfg->reserved != 0) return DETO_ERR_BAD_CONFIG;
    if (cfg->device_offset && !is_aligned(cfg->device_offset, 8)) return DETO_ERR_ALIGN;
    if (T == 0) return DETO_OK;
    if (!here(x) || !here(out)) return DETO_ERR_NULL;
    const bool add = here(residual);
    const int rc = first_error(check_rows(x, T, D), check_rows(out, T, D), add ? check_rows(residual, T, D) : 0);
    if (rc) return rc;
    if (add && residual->dtype != out->dtype) return DETO_ERR_BAD_CONFIG;
    if (x->dtype != out->dtype && x->dtype != DETO_F32 && out->dtype != DETO_F32) return DETO_ERR_BAD_CONFIG;

    const double wanted = nearbyint(static_cast<double>(cfg->rate) * 65536.0);
    const uint32_t dropped = wanted > 65535.0 ? 65535u : static_cast<uint32_t>(wanted);
    const Draw draw = {cfg->seed, cfg->offset, cfg->device_offset, dropped,
                       static_cast<float>(65536.0 / (65536.0 - dropped))};
    const deto_rows none = {};
    const bool once = T * D * type_size(out->dtype) > kCacheBytes / 4;
    return for_items(T, D, [&](const Items& it, unsigned grid) {
        const auto launch = [&](auto in, auto to, auto adds, auto streams) {
            dropout_kernel<in.value, to.value, adds.value != 0, streams.value != 0>
                <<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(it, draw, *x, add ? *residual : none, *out);
            return 0;
        };
        const auto by_size = [&](auto in, auto to, auto adds) {
            return once ? launch(in, to, adds, Type<1>{}) : launch(in, to, adds, Type<0>{});
        };
        const auto by_kind = [&](auto in, auto to) {
            return add ? by_size(in, to, Type<1>{}) : by_size(in, to, Type<0>{});
        };
        by_type(x->dtype, [&](auto in) {
            if (x->dtype == out->dtype) return by_kind(in, in);
            if constexpr (in.value == DETO_F32)
                return out->dtype == DETO_BF16 ? by_kind(in, Type<DETO_BF16>{}) : by_kind(in, Type<DETO_F16>{});
            else return by_kind(in, Type<DETO_F32>{});
        });
    });
}

}  // extern "C"
