// Rotary positions: pairs of features turned by their row's position times the pair's frequency.
//
// A stream of rows: a lane takes eight pairs of a head (16 bytes of each half of a 16-bit head, or 32 bytes in a run where
// pairs lie side by side) and the same eight of some of the row's other heads, so that the angles, which depend on
// the position and the pair alone, are worked out once for all of these.
//
// The angle in turns is a 64-bit product; only its part of a quarter turn, exact to 2^-24 of itself, goes to 32 bits.
// Sine and cosine of at most an eighth of a turn are their Taylor series, to within an fp32 rounding.
//
// Bound by memory: 16,384 rows of 32 heads of 128 in bf16, two thirds of the rows they lie in, take 46 us (5.8 TB/s);
// 4,095 x 12 x 80 fp16 in pairs, from odd addresses, 8 (2.0 TB/s, short rows); one row 2.7 (a launch).
#include "device.hip.h"

namespace deto {
namespace model {
namespace {

constexpr int kThreads = 256;
constexpr int kPairs = 8;              // of a lane

struct Plan {
    int64_t T;
    int32_t heads, head_dim, half;     // half: pairs of a head
    int32_t each;                      // heads of a lane
    FastDiv units, slices;             // lanes of a head; lanes along the heads
    uint32_t turning;                  // units that turn; those behind copy 16 features that are not turned
    const double* freqs;
    const void* positions;
    int32_t wide, inverse;             // wide: 64-bit positions
    int64_t first, period;
    float magnitude;
    uint32_t count;                    // lanes of this launch
    int64_t row0;
};

// sine and cosine of a quarter turn times r, |r| <= 1/2, r off by its own rounding
__device__ __forceinline__ void sincos_quarter(float r, float& s, float& c) {
    const float x = r * 1.57079632679489662f, y = x * x;
    s = 2.75573192e-6f;                                   // 1 / 9!, -1 / 7!, ...: the next term is below 2^-28
    s = fmaf(s, y, -1.98412698e-4f);
    s = fmaf(s, y, 8.33333333e-3f);
    s = fmaf(s, y, -1.66666667e-1f);
    s = fmaf(s * y, x, x);
    c = -2.75573192e-7f;                                  // -1 / 10!, 1 / 8!, ...
    c = fmaf(c, y, 2.48015873e-5f);
    c = fmaf(c, y, -1.38888889e-3f);
    c = fmaf(c, y, 4.16666667e-2f);
    c = fmaf(c, y, -0.5f);
    c = fmaf(c, y, 1.f);
}

// elements d ... d + count - 1 of a row, d any: load8, which goes back before d for a short vector, where the row has
// that many in front
template <int DT>
__device__ __forceinline__ void load_any(const void* base, int64_t row, int64_t d, int count, float (&v)[8]) {
    if (count >= 8 || d + count >= 8) {
        unpack8<DT>(load8<DT>(base, row, d, count), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < count ? load1<DT>(base, row + d + j) : 0.f;
    }
}

__device__ __forceinline__ int count_of(int64_t left) { return left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0; }

template <int DT, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Plan p, deto_rows x, deto_rows out) {
    const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
    if (id >= p.count) return;
    const uint32_t by_unit = p.units.div(id), unit = id - by_unit * p.units.d;
    const uint32_t row = p.slices.div(by_unit), slice = by_unit - row * p.slices.d;
    const int64_t t = p.row0 + row, from = t * x.ld, to = t * out.ld;
    // heads slice, slice + slices, ...: neighbouring lanes stay in neighbouring heads
    if (unit >= p.turning) {
        const int32_t at = 2 * p.half + 16 * static_cast<int32_t>(unit - p.turning);
        for (int h = slice; h < p.heads; h += p.slices.d) {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const int64_t d = int64_t{h} * p.head_dim + at + 8 * part;
                const int n = count_of(p.head_dim - at - 8 * part);
                float v[8];
                load_any<DT>(x.data, from, d, n, v);
                store8<DT>(out.data, to + d, v, n);
            }
        }
        return;
    }
    const int32_t pair = kPairs * static_cast<int32_t>(unit);
    int64_t position;
    if (p.positions)
        position = p.wide ? static_cast<const int64_t*>(p.positions)[t] : static_cast<const int32_t*>(p.positions)[t];
    else position = p.first + (p.period ? t % p.period : t);
    const double turns = static_cast<double>(position) * 0.15915494309189534;    // 1 / (2 pi)
    float s[kPairs], c[kPairs];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        const double w = turns * p.freqs[pair + j < p.half ? pair + j : p.half - 1];
        const double quarters = 4.0 * (w - rint(w)), whole = rint(quarters);
        const int q = static_cast<int>(whole);                  // -2 ... 2
        float sine, cosine;
        sincos_quarter(static_cast<float>(quarters - whole), sine, cosine);
        const float a = q & 1 ? cosine : sine, b = q & 1 ? sine : cosine;
        s[j] = (q & 2 ? -a : a) * p.magnitude;
        c[j] = ((q + 1) & 2 ? -b : b) * p.magnitude;
        if (p.inverse) s[j] = -s[j];
    }
    const int left = p.half - pair;                             // pairs of this lane, 1 or more
    const int n0 = count_of(PAIRS ? 2 * left : left), n1 = count_of(PAIRS ? 2 * left - 8 : left);
    const int32_t d0 = PAIRS ? 2 * pair : pair, d1 = PAIRS ? d0 + 8 : d0 + p.half;
    const auto turn = [&](float (&a)[8], float (&b)[8]) {
        if constexpr (PAIRS) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a0 = a[2 * j], a1 = a[2 * j + 1], b0 = b[2 * j], b1 = b[2 * j + 1];
                a[2 * j] = a0 * c[j] - a1 * s[j];
                a[2 * j + 1] = a0 * s[j] + a1 * c[j];
                b[2 * j] = b0 * c[j + 4] - b1 * s[j + 4];
                b[2 * j + 1] = b0 * s[j + 4] + b1 * c[j + 4];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float u = a[j], v = b[j];
                a[j] = u * c[j] - v * s[j];
                b[j] = u * s[j] + v * c[j];
            }
        }
    };
    int h = slice;
    const int step = p.slices.d;
    if (n0 == 8 && n1 == 8) {
        // four heads' loads in flight (one after the other: 16,384 x 32 x 128 bf16 57 us, so 46)
        for (; h + 3 * step < p.heads; h += 4 * step) {
            Raw8<DT> r[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const char* const head = static_cast<const char*>(x.data) + (from + int64_t{h + i * step} * p.head_dim) * kSize<DT>;
                r[i][0] = load8_whole<DT>(head + d0 * kSize<DT>);
                r[i][1] = load8_whole<DT>(head + d1 * kSize<DT>);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float a[8], b[8];
                unpack8<DT>(r[i][0], a);
                unpack8<DT>(r[i][1], b);
                turn(a, b);
                const int64_t head = to + int64_t{h + i * step} * p.head_dim;
                store8<DT>(out.data, head + d0, a, 8);
                store8<DT>(out.data, head + d1, b, 8);
            }
        }
    }
    for (; h < p.heads; h += step) {
        const int64_t head = int64_t{h} * p.head_dim;
        float a[8], b[8];
        load_any<DT>(x.data, from, head + d0, n0, a);
        load_any<DT>(x.data, from, head + d1, n1, b);
        turn(a, b);
        store8<DT>(out.data, to + head + d0, a, n0);
        store8<DT>(out.data, to + head + d1, b, n1);
    }
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int detonation_rotary(const deto_rotary* cfg, int64_t T, const deto_rows* x, const double* freqs,
                      const void* positions, int position_bytes, const deto_rows* out, void* stream) {
    if (!cfg) return DETO_ERR_NULL;
    if (T < 0 || cfg->heads < 1 || cfg->head_dim < 2 || int64_t{cfg->heads} * cfg->head_dim > (int64_t{1} << 30))
        return DETO_ERR_BAD_CONFIG;
    if (cfg->layout != DETO_ROTARY_HALVES && cfg->layout != DETO_ROTARY_PAIRS) return DETO_ERR_BAD_CONFIG;
    if (cfg->rotary_dim < 2 || cfg->rotary_dim > cfg->head_dim || cfg->rotary_dim % 2) return DETO_ERR_BAD_CONFIG;
    if ((cfg->inverse != 0 && cfg->inverse != 1) || !isfinite(cfg->magnitude)) return DETO_ERR_BAD_CONFIG;
    if (cfg->first < 0 || cfg->first > (int64_t{1} << 52) || cfg->period < 0 || cfg->period > (int64_t{1} << 52))
        return DETO_ERR_BAD_CONFIG;
    if (positions && position_bytes != 4 && position_bytes != 8) return DETO_ERR_BAD_CONFIG;
    if (T == 0) return DETO_OK;
    if (!here(x) || !here(out) || !freqs) return DETO_ERR_NULL;
    const int64_t D = int64_t{cfg->heads} * cfg->head_dim;
    const int rc = first_error(check_rows(x, T, D), check_rows(out, T, D));
    if (rc) return rc;
    if (x->dtype != out->dtype) return DETO_ERR_BAD_CONFIG;
    if (!is_aligned(freqs, 8) || (positions && !is_aligned(positions, position_bytes))) return DETO_ERR_ALIGN;

    const int half = cfg->rotary_dim / 2, rest = cfg->head_dim - cfg->rotary_dim;
    const bool in_place = x->data == out->data && (x->ld == out->ld || T == 1);
    const uint32_t turning = (half + kPairs - 1) / kPairs, copying = in_place ? 0 : (rest + 15) / 16;
    const uint32_t units = turning + copying;
    // Angles are worked out once for `each` heads, as long as that leaves the chip's lanes busy.
    int64_t each = T * units * cfg->heads / (int64_t{1} << 19);
    each = each < 1 ? 1 : each > 8 ? 8 : each;
    each = each < cfg->heads ? each : cfg->heads;
    const uint32_t slices = static_cast<uint32_t>((cfg->heads + each - 1) / each);
    const int64_t per_row = int64_t{units} * slices, rows = (int64_t{1} << 31) / per_row;    // of a launch
    fresh();
    for (int64_t t = 0; t < T; t += rows) {
        const int64_t n = (T - t < rows ? T - t : rows) * per_row;
        const Plan p = {T, cfg->heads, cfg->head_dim, half, static_cast<int32_t>(each), FastDiv(units), FastDiv(slices),
                        turning, freqs, positions, position_bytes == 8, cfg->inverse, cfg->first, cfg->period,
                        cfg->magnitude, static_cast<uint32_t>(n), t};
        const unsigned grid = static_cast<unsigned>((n + kThreads - 1) / kThreads);
        by_type(x->dtype, [&](auto dt) {
            if (cfg->layout == DETO_ROTARY_PAIRS)
                rotary_kernel<dt.value, true><<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(p, *x, *out);
            else rotary_kernel<dt.value, false><<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(p, *x, *out);
            return 0;
        });
    }
    return enqueued();
}

}  // extern "C"
