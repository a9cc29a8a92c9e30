// dw[n][k] = sum_t dy[t][n] x[t][k] with x in 8 bits: a linear layer's weight gradient on the matrix cores.
//
// Codes times a power of two are exact in bf16, so x enters the bf16 matrix instructions without a rounding.
// dy does too: bf16 as it is, fp16 as the sum of two bf16 numbers, fp32 as the sum of three (each takes the
// leading 8 bits of what is left).  Products are exact, sums fp32.
//
// Both operands have the sum's index t as their slow one, and a matrix instruction wants eight consecutive t of
// one n (or k) in a lane.  The turn happens on the way into LDS: a thread takes four rows of eight columns,
// packs pairs of rows (a byte permute for dy; for x the conversion from fp32 packs any two) and writes four t
// of each column.  LDS holds [column][64 t]; the 16-byte pieces of a column's 128 bytes are rotated by
// (column / 8) ^ column, so that neither the writes (columns eight apart) nor the reads (columns side by side)
// meet in a bank.
//
// Bound by the matrix cores for large products; few tiles are cut along t and joined by a second launch, always
// in the same order.
#include "device.hip.h"

namespace deto {
namespace model {
namespace {

constexpr int kDepth = 64;              // rows t of a step
constexpr int kRowBytes = kDepth * 2;   // of an LDS column

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int BM_, int BN_, int WM_, int WN_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;   // of a workgroup, of a wavefront: n, k
    static constexpr int kThreads = (BM / WM) * (BN / WN) * kLanes;
    static_assert((kDepth / 4) * (BM / 8) % kThreads == 0 && (kDepth / 4) * (BN / 8) % kThreads == 0, "");
    static constexpr int kUnitsA = (kDepth / 4) * (BM / 8) / kThreads;
    static constexpr int kUnitsB = (kDepth / 4) * (BN / 8) / kThreads;
    static constexpr int lds(int terms) { return 2 * (BM * terms + BN) * kRowBytes; }
};
using Large = Tile<256, 256, 128, 64>;
using Small = Tile<128, 128, 64, 64>;

struct Args {
    int64_t T, N, K;
    deto_rows dy, dw;
    deto_act8 x;
    int accumulate;
    int tiles_k;         // tiles along k
    int splits;
    int64_t span;        // rows t of a split, a multiple of kDepth
    float* parts;        // [split][N][K], if splits > 1
};

__device__ __forceinline__ uint32_t lds_at(int column, int t8) {     // byte offset of rows 8 t8 ... + 7
    return column * kRowBytes + (((t8 ^ (column >> 3) ^ column) & 7) << 4);
}

__device__ __forceinline__ uint32_t low_halves(uint32_t first, uint32_t second) {
    return __builtin_amdgcn_perm(second, first, 0x05040100u);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t first, uint32_t second) {
    return __builtin_amdgcn_perm(second, first, 0x07060302u);
}

template <int DT> constexpr int kTerms = DT == DETO_BF16 ? 1 : DT == DETO_F16 ? 2 : 3;

// What is left of v above its leading 8 bits.  (An infinity is one term, a NaN stays one.)
__device__ __forceinline__ float rest(float v) {
    const float r = v - bits_f32(f32_bits(v) & 0xFFFF0000u);
    return fabsf(v) == __builtin_inff() ? 0.f : r;
}

template <int DT> struct UnitA { Raw8<DT> row[4]; };
struct UnitB { u32x2 codes[4]; uint32_t exps[4]; };

// ---- Loads of a step.  NEAR: through buffer resources that end where the matrix does: rows past its end read as
// zeros without a comparison, a lane needs one 32-bit offset, and columns past a row's end read whatever comes
// next (they add to columns of dw that are not written).  Otherwise (rows far apart, or not at multiples of four
// bytes) element by element where a row ends.
typedef __amdgpu_buffer_rsrc_t Rsrc;

// (The words that hold the last bytes count whole: a buffer gives no part of a word.  They are aligned.)
__device__ __forceinline__ Rsrc resource(const void* base, int64_t bytes) {
    const int n = bytes > 0x7FFFFFF0 ? 0x7FFFFFF0 : bytes > 0 ? (static_cast<int>(bytes) + 3) & ~3 : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, n, 0x00020000);
}

__device__ __forceinline__ int exps_left(int64_t bytes) {      // bytes, read one by one
    return bytes > 0x7FFFFFF0 ? 0x7FFFFFF0 : bytes > 0 ? static_cast<int>(bytes) : 0;
}

template <int DT, class TL, bool NEAR>
struct Loader {
    const Args& a;
    int64_t n0, k0, end;
    __device__ __forceinline__ Loader(const Args& args, int64_t n, int64_t k, int64_t e)
        : a(args), n0(n), k0(k), end(e) {}

    __device__ __forceinline__ void load(int64_t t, UnitA<DT> (&ua)[TL::kUnitsA],
                                         UnitB (&ub)[TL::kUnitsB]) const {
        if constexpr (NEAR) {
            constexpr int kElem = kSize<DT>;
            const int ld = static_cast<int>(a.dy.ld) * kElem, ldc = static_cast<int>(a.x.ld_codes),
                      lde = static_cast<int>(a.x.ld_exps);
            const int64_t at_a = (t * a.dy.ld + n0) * kElem, at_c = t * a.x.ld_codes + k0,
                          at_e = t * a.x.ld_exps + k0 / DETO_ACT8_GROUP;
            const Rsrc ra = resource(static_cast<const char*>(a.dy.data) + at_a,
                                     ((end - 1) * a.dy.ld + a.N) * kElem - at_a);
            const Rsrc rc = resource(a.x.codes + at_c, (end - 1) * a.x.ld_codes + a.K - at_c);
            const Rsrc re = __builtin_amdgcn_make_buffer_rsrc(
                a.x.exps + at_e, 0, exps_left((end - 1) * a.x.ld_exps +
                                              (a.K + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP - at_e),
                0x00020000);
#pragma unroll
            for (int i = 0; i < TL::kUnitsA; ++i) {
                const int u = threadIdx.x + i * TL::kThreads;
                const int off = u / (TL::BM / 8) * 4 * ld + u % (TL::BM / 8) * 8 * kElem;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    ua[i].row[r].a = __builtin_amdgcn_raw_buffer_load_b128(ra, off, r * ld, 0);
                    if constexpr (DT == DETO_F32)
                        ua[i].row[r].b = __builtin_amdgcn_raw_buffer_load_b128(ra, off + 16, r * ld, 0);
                }
            }
#pragma unroll
            for (int i = 0; i < TL::kUnitsB; ++i) {
                const int u = threadIdx.x + i * TL::kThreads;
                const int t4 = u / (TL::BN / 8) * 4, c8 = u % (TL::BN / 8);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    ub[i].codes[r] = __builtin_amdgcn_raw_buffer_load_b64(rc, t4 * ldc + c8 * 8, r * ldc, 0);
                    ub[i].exps[r] = __builtin_amdgcn_raw_buffer_load_b8(re, t4 * lde + c8 / 4, r * lde, 0);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < TL::kUnitsA; ++i) {
                const int u = threadIdx.x + i * TL::kThreads;
                const int64_t n = n0 + u % (TL::BM / 8) * 8, left = a.N - n, row = t + u / (TL::BM / 8) * 4;
                const int count = left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    ua[i].row[r] = load8<DT>(a.dy.data, (row + r) * a.dy.ld + n, row + r < end ? count : 0);
            }
#pragma unroll
            for (int i = 0; i < TL::kUnitsB; ++i) {
                const int u = threadIdx.x + i * TL::kThreads;
                const int64_t k = k0 + u % (TL::BN / 8) * 8, left = a.K - k, row = t + u / (TL::BN / 8) * 4;
                const int count = left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool on = row + r < end && count > 0;
                    ub[i].codes[r] = load_codes(a.x.codes + (row + r) * a.x.ld_codes + k, on ? count : 0);
                    ub[i].exps[r] = on ? a.x.exps[(row + r) * a.x.ld_exps + k / DETO_ACT8_GROUP] : 0u;
                }
            }
        }
    }
};

// four rows (quarter tq of the step) of column `column`: 8 bytes
__device__ __forceinline__ void put4(char* lds, int column, int tq, uint32_t first, uint32_t second) {
    const u32x2 v = {first, second};
    *reinterpret_cast<u32x2*>(lds + lds_at(column, tq >> 1) + (tq & 1) * 8) = v;
}

template <int DT, class TL>
__device__ __forceinline__ void store_a(const UnitA<DT>& u, char* lds, int column, int tq) {
    if constexpr (DT == DETO_BF16) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            put4(lds, column + 2 * p, tq, low_halves(u.row[0].a[p], u.row[1].a[p]),
                 low_halves(u.row[2].a[p], u.row[3].a[p]));
            put4(lds, column + 2 * p + 1, tq, high_halves(u.row[0].a[p], u.row[1].a[p]),
                 high_halves(u.row[2].a[p], u.row[3].a[p]));
        }
    } else {
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack8<DT>(u.row[i], v[i]);
#pragma unroll
        for (int term = 0; term < kTerms<DT>; ++term) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                put4(lds + term * TL::BM * kRowBytes, column + j, tq,
                     high_halves(f32_bits(v[0][j]), f32_bits(v[1][j])),
                     high_halves(f32_bits(v[2][j]), f32_bits(v[3][j])));
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i][j] = rest(v[i][j]);
            }
        }
    }
}

__device__ __forceinline__ void store_b(const UnitB& u, char* lds, int column, int tq) {
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) act8_decode8(u.codes[i], u.exps[i], v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j)         // (the lower halves are zeros: bf16 holds the value)
        put4(lds, column + j, tq, high_halves(f32_bits(v[0][j]), f32_bits(v[1][j])),
             high_halves(f32_bits(v[2][j]), f32_bits(v[3][j])));
}

template <int DT>
__device__ __forceinline__ void write_dw(const deto_rows& dw, int64_t n, int64_t k, float v, int accumulate) {
    const int64_t at = n * dw.ld + k;
    if (accumulate) v += load1<DT>(dw.data, at);
    store1<DT>(dw.data, at, v);
}
__device__ __forceinline__ void write_any(const deto_rows& dw, int64_t n, int64_t k, float v, int accumulate) {
    if (dw.dtype == DETO_F32) write_dw<DETO_F32>(dw, n, k, v, accumulate);
    else if (dw.dtype == DETO_BF16) write_dw<DETO_BF16>(dw, n, k, v, accumulate);
    else write_dw<DETO_F16>(dw, n, k, v, accumulate);
}

template <int DT, class TL, bool NEAR>
__global__ __launch_bounds__(TL::kThreads) void weight_grad_kernel(Args a) {
    extern __shared__ __align__(16) char lds[];
    constexpr int kTermsA = kTerms<DT>;
    constexpr int kBytesA = TL::BM * kRowBytes, kBuffer = (TL::BM * kTermsA + TL::BN) * kRowBytes;
    const int tile = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int64_t n0 = static_cast<int64_t>(tile / a.tiles_k) * TL::BM;
    const int64_t k0 = static_cast<int64_t>(tile % a.tiles_k) * TL::BN;
    const int64_t t0 = split * a.span;
    const int64_t end = t0 + a.span < a.T ? t0 + a.span : a.T;
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const int wm = wave / (TL::BN / TL::WN) * TL::WM, wn = wave % (TL::BN / TL::WN) * TL::WN;

    f32x16 acc[TL::WM / 32][TL::WN / 32];
#pragma unroll
    for (int i = 0; i < TL::WM / 32; ++i)
#pragma unroll
        for (int j = 0; j < TL::WN / 32; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    UnitA<DT> ua[TL::kUnitsA];
    UnitB ub[TL::kUnitsB];
    const Loader<DT, TL, NEAR> loader(a, n0, k0, end);
    auto store = [&](char* at) {
#pragma unroll
        for (int i = 0; i < TL::kUnitsA; ++i) {
            const int u = threadIdx.x + i * TL::kThreads;
            store_a<DT, TL>(ua[i], at, u % (TL::BM / 8) * 8, u / (TL::BM / 8));
        }
#pragma unroll
        for (int i = 0; i < TL::kUnitsB; ++i) {
            const int u = threadIdx.x + i * TL::kThreads;
            store_b(ub[i], at + kTermsA * kBytesA, u % (TL::BN / 8) * 8, u / (TL::BN / 8));
        }
    };
    // Where a lane's operands of 16 rows t are, from the first of a wavefront's 32-column blocks.  (A block further
    // flips the third bit of column / 8, which is that of rows 32 further.)
    uint32_t at_a[kDepth / 16], at_b[kDepth / 16];
#pragma unroll
    for (int s = 0; s < kDepth / 16; ++s) {
        at_a[s] = lds_at(wm + lane % 32, 2 * s + lane / 32);
        at_b[s] = lds_at(wn + lane % 32, 2 * s + lane / 32);
    }
    int buffer = 0;
    if (t0 < end) {
        loader.load(t0, ua, ub);
        store(lds);
    }
    __syncthreads();
    for (int64_t t = t0; t < end; t += kDepth) {
        const bool more = t + kDepth < end;
        if (more) loader.load(t + kDepth, ua, ub);
        const char* la = lds + buffer * kBuffer;
        const char* lb = la + kTermsA * kBytesA;
#pragma unroll
        for (int s = 0; s < kDepth / 16; ++s) {
            bf16x8 fb[TL::WN / 32];
#pragma unroll
            for (int j = 0; j < TL::WN / 32; ++j)
                fb[j] = *reinterpret_cast<const bf16x8*>(lb + at_b[s ^ 2 * (j % 2)] + j * 32 * kRowBytes);
#pragma unroll
            for (int term = 0; term < kTermsA; ++term) {
                bf16x8 fa[TL::WM / 32];
#pragma unroll
                for (int i = 0; i < TL::WM / 32; ++i)
                    fa[i] = *reinterpret_cast<const bf16x8*>(la + term * kBytesA + at_a[s ^ 2 * (i % 2)] +
                                                             i * 32 * kRowBytes);
#pragma unroll
                for (int i = 0; i < TL::WM / 32; ++i)
#pragma unroll
                    for (int j = 0; j < TL::WN / 32; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
            }
        }
        buffer ^= 1;
        if (more) store(lds + buffer * kBuffer);
        __syncthreads();
    }
    // lane l holds column l % 32, rows 8 (r / 4) + 4 (l / 32) + r % 4 of a 32 x 32 block
#pragma unroll
    for (int i = 0; i < TL::WM / 32; ++i)
#pragma unroll
        for (int j = 0; j < TL::WN / 32; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t n = n0 + wm + i * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
                const int64_t k = k0 + wn + j * 32 + lane % 32;
                if (n < a.N && k < a.K) {
                    if (a.splits > 1) a.parts[(split * a.N + n) * a.K + k] = acc[i][j][r];
                    else write_any(a.dw, n, k, acc[i][j][r], a.accumulate);
                }
            }
}

__global__ __launch_bounds__(256) void weight_grad_join_kernel(Args a) {
    const int64_t all = a.N * a.K;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (at >= all) return;
    float s = 0.f;
    for (int i = 0; i < a.splits; ++i) s += a.parts[i * all + at];
    write_any(a.dw, at / a.K, at % a.K, s, a.accumulate);
}

bool bad_shape(int64_t T, int64_t N, int64_t K) {
    constexpr int64_t kMost = int64_t{1} << 30;
    return T < 0 || T > kMost || N < 1 || N > kMost || K < 1 || K > kMost;
}

struct Plan {
    bool large;
    int64_t tiles, tiles_k, splits, span;
};

Plan plan_with(int64_t T, int64_t N, int64_t K, bool large) {
    const int64_t b = large ? Large::BM : Small::BM;
    Plan p = {};
    p.large = large;
    p.tiles_k = (K + b - 1) / b;
    p.tiles = (N + b - 1) / b * p.tiles_k;
    const int64_t steps = T ? (T + kDepth - 1) / kDepth : 1;
    const int64_t slots = large ? 256 : 512;      // workgroups that run side by side
    int64_t splits = slots / p.tiles;
    if (splits > steps / 4) splits = steps / 4;   // four steps at least
    if (splits > 32) splits = 32;
    if (splits < 1) splits = 1;
    p.span = (steps + splits - 1) / splits * kDepth;
    p.splits = T ? (T + p.span - 1) / p.span : 1;
    return p;
}

// Whether a step's rows lie within 2^31 bytes and at multiples of four: the loader's buffers.
bool reaches(const Args& a) {
    const int64_t e = type_size(a.dy.dtype), most = (int64_t{1} << 31) / (2 * kDepth);
    return a.dy.ld * e < most && a.x.ld_codes < most && a.x.ld_exps < most && a.dy.ld * e % 4 == 0 &&
           a.x.ld_codes % 4 == 0 && is_aligned(a.dy.data, 4) && is_aligned(a.x.codes, 4);
}

// Large tiles where they fill the chip by themselves, and dy is one term.
Plan plan_of(int64_t T, int64_t N, int64_t K, bool may_be_large) {
    const Plan p = plan_with(T, N, K, true);
    return may_be_large && p.tiles >= 192 ? p : plan_with(T, N, K, false);
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int64_t detonation_act8_weight_grad_workspace(int64_t T, int64_t N, int64_t K) {
    if (bad_shape(T, N, K)) return -1;
    int64_t most = 0;
    for (bool large : {true, false}) {
        const Plan p = plan_of(T, N, K, large);
        if (p.splits > 1 && p.splits > most) most = p.splits;
    }
    return most * N * K * static_cast<int64_t>(sizeof(float));
}

int detonation_act8_weight_grad(int64_t T, int64_t N, int64_t K, const deto_rows* dy,
                                const deto_act8* x8, const deto_rows* dw, int accumulate,
                                void* workspace, void* stream) {
    if (bad_shape(T, N, K)) return DETO_ERR_BAD_CONFIG;
    if (!here(dw) || (T && (!here(dy) || !here(x8)))) return DETO_ERR_NULL;
    const int rc = first_error(check_rows(dw, N, K), T ? check_rows(dy, T, N) : 0,
                               T ? check_act8(x8, T, K) : 0);
    if (rc) return rc;
    const int dtype = T ? dy->dtype : static_cast<int>(DETO_BF16);
    const deto_rows none = {};
    const deto_act8 none8 = {};
    Args a = {T, N, K, T ? *dy : none, *dw, T ? *x8 : none8, accumulate != 0, 0, 0, 0,
              static_cast<float*>(workspace)};
    if (T <= 1) {           // (a single row's distance to the next one says nothing)
        a.dy.ld = (N + 1) / 2 * 2;
        a.x.ld_codes = (K + 3) / 4 * 4;
        a.x.ld_exps = (K + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP;
    }
    const bool near = T > 0 && reaches(a);
    const Plan p = plan_of(T, N, K, near && dtype == DETO_BF16);
    if (p.splits > 1 && !workspace) return DETO_ERR_NULL;
    if (p.splits > 1 && !is_aligned(workspace, 16)) return DETO_ERR_ALIGN;
    const int64_t blocks = (N * K + 255) / 256;
    if (p.tiles * p.splits > 0x7FFFFFFF || (p.splits > 1 && blocks > 0x7FFFFFFF))
        return DETO_ERR_UNSUPPORTED;
    a.tiles_k = static_cast<int>(p.tiles_k);
    a.splits = static_cast<int>(p.splits);
    a.span = p.span;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned grid = static_cast<unsigned>(p.tiles * p.splits);
    fresh();
    if (p.large)
        weight_grad_kernel<DETO_BF16, Large, true><<<grid, Large::kThreads, Large::lds(1), st>>>(a);
    else
        by_type(dtype, [&](auto dt) {
            constexpr int kLds = Small::lds(kTerms<dt.value>);
            if (near) weight_grad_kernel<dt.value, Small, true><<<grid, Small::kThreads, kLds, st>>>(a);
            else weight_grad_kernel<dt.value, Small, false><<<grid, Small::kThreads, kLds, st>>>(a);
            return 0;
        });
    if (p.splits > 1)
        weight_grad_join_kernel<<<static_cast<unsigned>(blocks), 256, 0, st>>>(a);
    return enqueued();
}

}  // extern "C"
