// Device- and host-side helpers shared by the operators of include/detonation_model.h: rows of any of the
// three types eight elements at a time, the 8-bit form, reductions, argument checks.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/detonation_model.h"

namespace deto {
namespace model {

constexpr int kLanes = 64;
constexpr int64_t kCacheBytes = int64_t{1} << 28;     // the cache that all of the chip shares

// ---- Eight consecutive elements of a row.  Rows start at any multiple of the element's size: the
// vectors below say so, and the compiler still makes 16-byte accesses of them (global memory on gfx950
// takes them at any address; they cost more lines only where they straddle one).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any2 __attribute__((aligned(2)));
typedef u32x4 u32x4_any4 __attribute__((aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any1 __attribute__((aligned(1)));
typedef u32x2 u32x2_any2 __attribute__((aligned(2)));
typedef uint32_t u32_any1 __attribute__((aligned(1)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int DT> struct Raw8;          // eight elements as loaded
template <> struct Raw8<DETO_F32> { u32x4 a, b; };
template <> struct Raw8<DETO_BF16> { u32x4 a; };
template <> struct Raw8<DETO_F16> { u32x4 a; };

template <int DT> constexpr int kSize = DT == DETO_F32 ? 4 : 2;

__device__ __forceinline__ float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t f32_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {     // round to nearest even
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

template <int DT>
__device__ __forceinline__ float load1(const void* base, int64_t at) {
    if constexpr (DT == DETO_F32) return static_cast<const float*>(base)[at];
    else if constexpr (DT == DETO_BF16)
        return bits_f32(static_cast<uint32_t>(static_cast<const uint16_t*>(base)[at]) << 16);
    else return static_cast<float>(static_cast<const _Float16*>(base)[at]);
}
template <int DT>
__device__ __forceinline__ void store1(void* base, int64_t at, float v) {
    if constexpr (DT == DETO_F32) static_cast<float*>(base)[at] = v;
    else if constexpr (DT == DETO_BF16)
        static_cast<uint16_t*>(base)[at] = static_cast<uint16_t>(pack_bf16(v, 0.f));
    else static_cast<_Float16*>(base)[at] = static_cast<_Float16>(v);
}

// ONCE: data that nothing reads again soon (large streams): it need not stay in the caches
template <int DT, bool ONCE = false>
__device__ __forceinline__ Raw8<DT> load8_whole(const char* p) {
    using Vec = std::conditional_t<DT == DETO_F32, u32x4_any4, u32x4_any2>;
    const Vec* v = reinterpret_cast<const Vec*>(p);
    Raw8<DT> r;
    if constexpr (ONCE) r.a = __builtin_nontemporal_load(v);
    else r.a = *v;
    if constexpr (DT == DETO_F32) {
        if constexpr (ONCE) r.b = __builtin_nontemporal_load(v + 1);
        else r.b = v[1];
    }
    return r;
}

// element j <- element j + by (0 ... 7), zeros from above
template <int DT>
__device__ __forceinline__ void move_down(Raw8<DT>& r, int by) {
    if constexpr (DT == DETO_F32) {
        uint32_t w[8] = {r.a[0], r.a[1], r.a[2], r.a[3], r.b[0], r.b[1], r.b[2], r.b[3]};
#pragma unroll
        for (int s = 4; s; s >>= 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (by & s) w[j] = j + s < 8 ? w[j + s < 8 ? j + s : 0] : 0u;
        }
        r.a = {w[0], w[1], w[2], w[3]};
        r.b = {w[4], w[5], w[6], w[7]};
    } else {
        uint32_t w[4] = {r.a[0], r.a[1], r.a[2], r.a[3]};
#pragma unroll
        for (int s = 2; s; s >>= 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (by & (2 * s)) w[j] = j + s < 4 ? w[j + s < 4 ? j + s : 0] : 0u;
        }
        if (by & 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = w[j] >> 16 | (j < 3 ? w[j < 3 ? j + 1 : 0] << 16 : 0u);
        }
        r.a = {w[0], w[1], w[2], w[3]};
    }
}

// elements d .. d + 7 (d a multiple of 8) of a row that starts at element `row`, of which `count` (0 ... 8) are there;
// the others read as zeros.  A row's partial last vector is read as the eight elements that end with the row and
// moved down: one access, where element by element takes seven and a register each.  (Only rows of fewer than
// eight elements have to be.)
template <int DT, bool ONCE = false>
__device__ __forceinline__ Raw8<DT> load8(const void* base, int64_t row, int64_t d, int count) {
    Raw8<DT> r = {};
    const bool whole = count >= 8;
    if (whole || (count > 0 && d > 0)) {
        const int short_by = whole ? 0 : 8 - count;
        const char* p = static_cast<const char*>(base) + (row + d - short_by) * kSize<DT>;
        r = load8_whole<DT, ONCE>(p);
        if (!whole) move_down<DT>(r, short_by);
    } else if (count > 0) {
        const char* p = static_cast<const char*>(base) + row * kSize<DT>;
#pragma unroll 1
        for (int j = count - 1; j >= 0; --j) {      // each in front of what is there
            if constexpr (DT == DETO_F32) {
                r.b = {r.a[3], r.b[0], r.b[1], r.b[2]};
                r.a = {reinterpret_cast<const uint32_t*>(p)[j], r.a[0], r.a[1], r.a[2]};
            } else {
                r.a = {r.a[0] << 16 | reinterpret_cast<const uint16_t*>(p)[j], r.a[1] << 16 | r.a[0] >> 16,
                       r.a[2] << 16 | r.a[1] >> 16, r.a[3] << 16 | r.a[2] >> 16};
            }
        }
    }
    return r;
}

template <int DT>
__device__ __forceinline__ void unpack8(const Raw8<DT>& r, float (&v)[8]) {
    if constexpr (DT == DETO_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = bits_f32(r.a[j]);
            v[j + 4] = bits_f32(r.b[j]);
        }
    } else if constexpr (DT == DETO_BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bits_f32(r.a[j] << 16);
            v[2 * j + 1] = bits_f32(r.a[j] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t word = r.a[j];    // (a cast of the element itself reads the first one for all j)
            const f16x2 h = __builtin_bit_cast(f16x2, word);
            v[2 * j] = static_cast<float>(h.x);
            v[2 * j + 1] = static_cast<float>(h.y);
        }
    }
}

template <int DT, bool ONCE = false>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&v)[8], int count) {
    char* p = static_cast<char*>(base) + at * kSize<DT>;
    if (count >= 8) {
        if constexpr (DT == DETO_F32) {
            u32x4 a, b;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = f32_bits(v[j]);
                b[j] = f32_bits(v[j + 4]);
            }
            u32x4_any4* at = reinterpret_cast<u32x4_any4*>(p);
            if constexpr (ONCE) {
                __builtin_nontemporal_store(u32x4_any4(a), at);
                __builtin_nontemporal_store(u32x4_any4(b), at + 1);
            } else {
                at[0] = a;
                at[1] = b;
            }
        } else {
            u32x4 a;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                a[j] = DT == DETO_BF16 ? pack_bf16(v[2 * j], v[2 * j + 1])
                                       : pack_f16(v[2 * j], v[2 * j + 1]);
            u32x4_any2* at = reinterpret_cast<u32x4_any2*>(p);
            if constexpr (ONCE) __builtin_nontemporal_store(u32x4_any2(a), at);
            else *at = a;
        }
    } else if (count > 0) {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < count) store1<DT>(p, j, v[j]);
    }
}

// ---- The 8-bit form.  Four lanes in a row hold a group of 32 features, eight each.

// maximum over the four lanes of an aligned group of four
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, bits_f32(__builtin_amdgcn_mov_dpp(f32_bits(v), 0xB1, 0xF, 0xF, true)));   // lanes 1 0 3 2
    return fmaxf(v, bits_f32(__builtin_amdgcn_mov_dpp(f32_bits(v), 0x4E, 0xF, 0xF, true)));  // 2 3 0 1
}

// The exponent byte of a group whose largest magnitude is `top`: with top = 1.m * 2^E, 127 * 2^(E-6) holds it
// as long as 64 * 1.m rounds to 127 or less, which is 1.m < 127.5 / 64 (mantissa below 0x7F0000).
__device__ __forceinline__ uint32_t act8_exponent(float top) {
    const uint32_t b = f32_bits(top);
    const int e = static_cast<int>(b >> 23) - 6 + ((b & 0x7FFFFFu) >= 0x7F0000u ? 1 : 0);
    return e < 1 ? 1u : static_cast<uint32_t>(e);
}

// Eight values of a lane into codes (two words) and the group's exponent byte.  Lanes without elements bring
// zeros.  An infinity or a NaN among the group's values: exponent byte 255, codes 0.
__device__ __forceinline__ u32x2 act8_encode8(const float (&v)[8], uint32_t& exponent) {
    float top = 0.f;
    bool odd = false;                   // (a maximum would drop a NaN)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        top = fmaxf(top, fabsf(v[j]));
        odd |= v[j] != v[j];
    }
    top = quad_max(odd ? __builtin_inff() : top);
    const bool finite = top < __builtin_inff();
    exponent = finite ? act8_exponent(top) : 255u;
    const float inv = finite ? bits_f32((254u - exponent) << 23) : 0.f;
    u32x2 q;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = finite ? rintf(v[4 * w + j] * inv) : 0.f;
            word |= (static_cast<uint32_t>(static_cast<int>(x)) & 0xFFu) << (8 * j);
        }
        q[w] = word;
    }
    return q;
}

// The same for four values of each of eight lanes in a row.
__device__ __forceinline__ uint32_t act8_encode4(const float (&v)[4], uint32_t& exponent) {
    float top = 0.f;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        top = fmaxf(top, fabsf(v[j]));
        odd |= v[j] != v[j];
    }
    top = quad_max(odd ? __builtin_inff() : top);
    top = fmaxf(top, bits_f32(__builtin_amdgcn_mov_dpp(f32_bits(top), 0x141, 0xF, 0xF, true)));  // the other four
    const bool finite = top < __builtin_inff();
    exponent = finite ? act8_exponent(top) : 255u;
    const float inv = finite ? bits_f32((254u - exponent) << 23) : 0.f;
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float x = finite ? rintf(v[j] * inv) : 0.f;
        word |= (static_cast<uint32_t>(static_cast<int>(x)) & 0xFFu) << (8 * j);
    }
    return word;
}

__device__ __forceinline__ float act8_scale(uint32_t exponent) {
    return bits_f32(exponent == 255u ? 0x7FC00000u : exponent << 23);
}

__device__ __forceinline__ void act8_decode8(const u32x2& q, uint32_t exponent, float (&v)[8]) {
    const float s = act8_scale(exponent);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        v[j] = static_cast<float>(static_cast<int8_t>((q[j / 4] >> (8 * (j % 4))) & 0xFFu)) * s;
}

// codes d ... d + 7 of a row, as load8
template <bool ONCE = false>
__device__ __forceinline__ u32x2 load_codes(const int8_t* row, int64_t d, int count) {
    u32x2 q = {0u, 0u};
    if (count >= 8) {
        const u32x2_any1* at = reinterpret_cast<const u32x2_any1*>(row + d);
        if constexpr (ONCE) q = __builtin_nontemporal_load(at);
        else q = *at;
    } else if (count > 0 && d > 0) {
        q = *reinterpret_cast<const u32x2_any1*>(row + d - (8 - count));
        q = __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, q) >> (8 * (8 - count)));
    } else {
        uint64_t bits = 0;
#pragma unroll 1
        for (int j = count - 1; j >= 0; --j) bits = bits << 8 | static_cast<uint8_t>(row[j]);
        q = __builtin_bit_cast(u32x2, bits);
    }
    return q;
}

template <bool ONCE = false>
__device__ __forceinline__ void store_codes(int8_t* p, const u32x2& q, int count) {
    if (count >= 8) {
        u32x2_any1* at = reinterpret_cast<u32x2_any1*>(p);
        if constexpr (ONCE) __builtin_nontemporal_store(u32x2_any1(q), at);
        else *at = q;
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < count) p[j] = static_cast<int8_t>((q[j / 4] >> (8 * (j % 4))) & 0xFFu);
    }
}

// Eight values at feature d (a multiple of 8) of row t: codes, and the exponent from the group's first lane.
// Every lane of a group of four takes part, whatever its count.
template <bool ONCE = false>
__device__ __forceinline__ void act8_put(const deto_act8& m, int64_t t, int64_t d, const float (&v)[8],
                                         int count) {
    uint32_t e;
    const u32x2 q = act8_encode8(v, e);
    if (count > 0) {
        store_codes<ONCE>(m.codes + t * m.ld_codes + d, q, count);
        if (d % DETO_ACT8_GROUP == 0) m.exps[t * m.ld_exps + d / DETO_ACT8_GROUP] = static_cast<uint8_t>(e);
    }
}

template <bool ONCE = false>
__device__ __forceinline__ void act8_get(const deto_act8& m, int64_t t, int64_t d, float (&v)[8],
                                         int count) {
    if (count > 0)
        act8_decode8(load_codes<ONCE>(m.codes + t * m.ld_codes, d, count),
                     m.exps[t * m.ld_exps + d / DETO_ACT8_GROUP], v);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
}

// ---- n / d for 32-bit n and a d known on the host: floor(n * (2^(32 + s) / d rounded up) / 2^(32 + s))
// with s = ceil(log2 d); the factor's 33rd bit is the added n (Granlund and Montgomery, 1994).
struct FastDiv {
    uint32_t d, mul, shift;
    explicit FastDiv(uint32_t by) : d(by), mul(0), shift(0) {
        while (shift < 32 && (uint64_t{1} << shift) < by) ++shift;
        mul = static_cast<uint32_t>(((uint64_t{1} << 32) * ((uint64_t{1} << shift) - by)) / by + 1);
    }
    __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const {
        const uint64_t hi = (static_cast<uint64_t>(n) * mul) >> 32;
        return static_cast<uint32_t>((hi + n) >> shift);
    }
};

// ---- sums over a wavefront, the same in every lane: within rows of 16 lanes by moves between neighbours (no
// LDS), then the four rows
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
    return bits_f32(__builtin_amdgcn_update_dpp(0, f32_bits(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return bits_f32(__builtin_amdgcn_readlane(f32_bits(v), lane));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0xB1>(v);     // lanes 1 0 3 2
    v += moved<0x4E>(v);     // lanes 2 3 0 1
    v += moved<0x141>(v);    // the other half of eight
    v += moved<0x140>(v);    // the other half of sixteen
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
// sums over each L lanes in a row (16, 32 or all), the same in all of them
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (L == kLanes) return wave_sum(v);
    v += moved<0xB1>(v);
    v += moved<0x4E>(v);
    v += moved<0x141>(v);
    v += moved<0x140>(v);
    if constexpr (L == 32) v += __shfl_xor(v, 16);
    return v;
}

// ---- host side
inline bool valid_type(int d) { return d == DETO_F32 || d == DETO_BF16 || d == DETO_F16; }
inline int type_size(int d) { return d == DETO_F32 ? 4 : 2; }
inline bool here(const deto_rows* m) { return m && m->data; }
inline bool here(const deto_act8* m) { return m && m->codes; }
inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// deto_status of rows that are there
inline int check_rows(const deto_rows* m, int64_t T, int64_t D) {
    if (!valid_type(m->dtype) || m->reserved != 0) return DETO_ERR_BAD_CONFIG;
    if (T > 1 && m->ld < D) return DETO_ERR_BAD_CONFIG;
    return is_aligned(m->data, type_size(m->dtype)) ? DETO_OK : DETO_ERR_ALIGN;
}
inline int check_act8(const deto_act8* m, int64_t T, int64_t D) {
    if (!m->exps) return DETO_ERR_NULL;
    if (T > 1 && (m->ld_codes < D || m->ld_exps < (D + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP))
        return DETO_ERR_BAD_CONFIG;
    return DETO_OK;
}
inline int first_error() { return DETO_OK; }
template <class... R>
inline int first_error(int a, R... rest) { return a != DETO_OK ? a : first_error(rest...); }

inline void fresh() { (void)hipGetLastError(); }
inline int enqueued() { return hipGetLastError() == hipSuccess ? DETO_OK : DETO_ERR_HIP; }

template <int V> struct Type { static constexpr int value = V; };

// f(Type<dtype>)
template <class F>
inline int by_type(int dtype, F f) {
    return dtype == DETO_F32 ? f(Type<DETO_F32>{}) : dtype == DETO_BF16 ? f(Type<DETO_BF16>{})
                                                                        : f(Type<DETO_F16>{});
}

// ---- Items: eight consecutive features of a row, numbered through a matrix whose rows are padded to whole groups of
// 32 (four items).
constexpr int kItemThreads = 256;

struct Items {
    FastDiv per_row;    // lane-items of a row, a multiple of 4
    uint32_t count;     // lane-items of this launch
    int64_t D;
    int64_t row0;       // of this launch
    struct At { int64_t t, d; int count; };
    // Lanes past the end get count 0 (they still take part in their group's maximum).
    __device__ __forceinline__ At at(uint32_t item) const {
        const uint32_t row = per_row.div(item);
        const int64_t d = int64_t{8} * (item - row * per_row.d);
        const int64_t left = item < count ? D - d : 0;
        return {row0 + row, d, left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0};
    }
};

// One launch for each run of rows whose items can be numbered in 31 bits.
template <class F>
inline int for_items(int64_t T, int64_t D, F launch) {
    if (T == 0) return DETO_OK;
    const int64_t per_row = (D + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP * (DETO_ACT8_GROUP / 8);
    const int64_t rows = (int64_t{1} << 31) / per_row - 1;
    fresh();
    for (int64_t t = 0; t < T; t += rows) {
        const int64_t n = (T - t < rows ? T - t : rows) * per_row;
        launch(Items{FastDiv(static_cast<uint32_t>(per_row)), static_cast<uint32_t>(n), D, t},
               static_cast<unsigned>((n + kItemThreads - 1) / kItemThreads));
    }
    return enqueued();
}

}  // namespace model
}  // namespace deto
