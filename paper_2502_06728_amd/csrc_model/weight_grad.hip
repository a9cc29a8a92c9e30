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

constexpr int kBand = 4;                // tiles along n that share their part of x
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

template <int DT>
__device__ __forceinline__ float element(const Raw8<DT>& r, int j) {
    if constexpr (DT == DETO_F32) return bits_f32(j < 4 ? r.a[j & 3] : r.b[j & 3]);
    else {
        const uint32_t word = r.a[j / 2];
        const f16x2 h = __builtin_bit_cast(f16x2, word);
        return static_cast<float>(j % 2 ? h.y : h.x);
    }
}

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

    __device__ __forceinline__ void load_a(int64_t t, UnitA<DT> (&ua)[TL::kUnitsA]) const {
        if constexpr (NEAR) {
            constexpr int kElem = kSize<DT>;
            const int ld = static_cast<int>(a.dy.ld) * kElem;
            const int64_t at_a = (t * a.dy.ld + n0) * kElem;
            const Rsrc ra = resource(static_cast<const char*>(a.dy.data) + at_a,
                                     ((end - 1) * a.dy.ld + a.N) * kElem - at_a);
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
        } else {
#pragma unroll
            for (int i = 0; i < TL::kUnitsA; ++i) {
                const int u = threadIdx.x + i * TL::kThreads;
                const int64_t n = n0 + u % (TL::BM / 8) * 8, left = a.N - n, row = t + u / (TL::BM / 8) * 4;
                const int count = left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    ua[i].row[r] = load8<DT>(a.dy.data, (row + r) * a.dy.ld, n, row + r < end ? count : 0);
            }
        }
    }

    __device__ __forceinline__ void load_b(int64_t t, UnitB (&ub)[TL::kUnitsB]) const {
        if constexpr (NEAR) {
            const int ldc = static_cast<int>(a.x.ld_codes), lde = static_cast<int>(a.x.ld_exps);
            const int64_t at_c = t * a.x.ld_codes + k0, at_e = t * a.x.ld_exps + k0 / DETO_ACT8_GROUP;
            const Rsrc rc = resource(a.x.codes + at_c, (end - 1) * a.x.ld_codes + a.K - at_c);
            const Rsrc re = __builtin_amdgcn_make_buffer_rsrc(
                a.x.exps + at_e, 0, exps_left((end - 1) * a.x.ld_exps +
                                              (a.K + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP - at_e),
                0x00020000);
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
            for (int i = 0; i < TL::kUnitsB; ++i) {
                const int u = threadIdx.x + i * TL::kThreads;
                const int64_t k = k0 + u % (TL::BN / 8) * 8, left = a.K - k, row = t + u / (TL::BN / 8) * 4;
                const int count = left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool on = row + r < end && count > 0;
                    ub[i].codes[r] = load_codes(a.x.codes + (row + r) * a.x.ld_codes, k, on ? count : 0);
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

// Quarter Q (two columns) of a unit of dy, in all its terms.
template <int DT, class TL, int Q>
__device__ __forceinline__ void store_a(const UnitA<DT>& u, char* lds, int column, int tq) {
    if constexpr (DT == DETO_BF16) {
        put4(lds, column + 2 * Q, tq, low_halves(u.row[0].a[Q], u.row[1].a[Q]),
             low_halves(u.row[2].a[Q], u.row[3].a[Q]));
        put4(lds, column + 2 * Q + 1, tq, high_halves(u.row[0].a[Q], u.row[1].a[Q]),
             high_halves(u.row[2].a[Q], u.row[3].a[Q]));
    } else {
#pragma unroll
        for (int j = 2 * Q; j < 2 * Q + 2; ++j) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = element<DT>(u.row[i], j);
#pragma unroll
            for (int term = 0; term < kTerms<DT>; ++term) {
                put4(lds + term * TL::BM * kRowBytes, column + j, tq,
                     high_halves(f32_bits(v[0]), f32_bits(v[1])), high_halves(f32_bits(v[2]), f32_bits(v[3])));
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = rest(v[i]);
            }
        }
    }
}

// Byte J of a word of codes as fp32.
template <int J>
__device__ __forceinline__ float code_value(uint32_t word) {
    float f;
    if constexpr (J == 0)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(word));
    else if constexpr (J == 1)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(word));
    else if constexpr (J == 2)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(word));
    else
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(word));
    return f;
}

// Column J of a unit of x.  (The lower halves of the values are zeros: bf16 holds them.)
template <int J>
__device__ __forceinline__ void store_b(const UnitB& u, const float (&scale)[4], char* lds, int column, int tq) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t word = u.codes[i][J / 4];
        v[i] = code_value<J % 4>(word) * scale[i];
    }
    put4(lds, column + J, tq, high_halves(f32_bits(v[0]), f32_bits(v[1])),
         high_halves(f32_bits(v[2]), f32_bits(v[3])));
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

// f(Type<0>) ... f(Type<N - 1>)
template <int N, class F>
__device__ __forceinline__ void each_of(F f) {
    if constexpr (N > 0) {
        each_of<N - 1>(f);
        f(Type<N - 1>{});
    }
}

template <int DT, class TL, bool NEAR>
__global__ __launch_bounds__(TL::kThreads) void weight_grad_kernel(Args a) {
    extern __shared__ __align__(16) char lds[];
    constexpr int kTermsA = kTerms<DT>;
    constexpr int kBytesA = TL::BM * kRowBytes, kBuffer = (TL::BM * kTermsA + TL::BN) * kRowBytes;
    // Workgroups go to the chip's eight parts in turn: a part takes a run of tiles, four high, whose operands
    // its own cache then holds for all of them.
    const unsigned all = gridDim.x, part = blockIdx.x % 8, each = all / 8, more_parts = all % 8;
    const unsigned id = part * each + (part < more_parts ? part : more_parts) + blockIdx.x / 8;
    const int tiles = all / a.splits, split = id / tiles;
    const int tile = id % tiles, tiles_n = tiles / a.tiles_k;
    const int band = tile / (kBand * a.tiles_k), within = tile % (kBand * a.tiles_k);
    const int high = tiles_n - band * kBand < kBand ? tiles_n - band * kBand : kBand;
    const int64_t n0 = static_cast<int64_t>(band * kBand + within % high) * TL::BM;
    const int64_t k0 = static_cast<int64_t>(within / high) * TL::BN;
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
    // (A's and B's units lie alike over their columns where the tile is square)
    auto place = [&](int i, int wide) { return (threadIdx.x + i * TL::kThreads) % (wide / 8) * 8; };
    auto quarter = [&](int i, int wide) { return (threadIdx.x + i * TL::kThreads) / (wide / 8); };
    auto put_a = [&](char* at, auto q) {
#pragma unroll
        for (int i = 0; i < TL::kUnitsA; ++i)
            store_a<DT, TL, q.value>(ua[i], at, place(i, TL::BM), quarter(i, TL::BM));
    };
    float scale[TL::kUnitsB][4];
    auto scales = [&] {
#pragma unroll
        for (int i = 0; i < TL::kUnitsB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) scale[i][r] = act8_scale(ub[i].exps[r]);
    };
    auto put_b = [&](char* at, auto j) {
#pragma unroll
        for (int i = 0; i < TL::kUnitsB; ++i)
            store_b<j.value>(ub[i], scale[i], at + kTermsA * kBytesA, place(i, TL::BN), quarter(i, TL::BN));
    };
    // Where a lane's operands of 16 rows t are, from the first of a wavefront's 32-column blocks.  (A block further
    // flips the third bit of column / 8, which is that of rows 32 further.)
    uint32_t at_a[kDepth / 16], at_b[kDepth / 16];
#pragma unroll
    for (int s = 0; s < kDepth / 16; ++s) {
        at_a[s] = lds_at(wm + lane % 32, 2 * s + lane / 32);
        at_b[s] = lds_at(wn + lane % 32, 2 * s + lane / 32);
    }
    bf16x8 fa[2][kTermsA][TL::WM / 32], fb[2][TL::WN / 32];
    auto fetch = [&](const char* la, auto s) {
        constexpr int S = s.value;
        const char* lb = la + kTermsA * kBytesA;
#pragma unroll
        for (int j = 0; j < TL::WN / 32; ++j)
            fb[S % 2][j] = *reinterpret_cast<const bf16x8*>(lb + at_b[S ^ 2 * (j % 2)] + j * 32 * kRowBytes);
#pragma unroll
        for (int term = 0; term < kTermsA; ++term)
#pragma unroll
            for (int i = 0; i < TL::WM / 32; ++i)
                fa[S % 2][term][i] = *reinterpret_cast<const bf16x8*>(
                    la + term * kBytesA + at_a[S ^ 2 * (i % 2)] + i * 32 * kRowBytes);
    };
    // the products of rows 16 S ... + 15 of the step that use blocks I of n
    auto multiply = [&](auto s, auto block) {
        constexpr int S = s.value, I = block.value;
#pragma unroll
        for (int term = 0; term < kTermsA; ++term)
#pragma unroll
            for (int j = 0; j < TL::WN / 32; ++j)
                acc[I][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[S % 2][term][I], fb[S % 2][j], acc[I][j],
                                                                    0, 0, 0);
    };
    if (t0 < end) {
        loader.load_a(t0, ua);
        loader.load_b(t0, ub);
        scales();
        each_of<4>([&](auto q) { put_a(lds, q); });
        each_of<8>([&](auto j) { put_b(lds, j); });
        loader.load_a(t0 + kDepth, ua);
        loader.load_b(t0 + kDepth, ub);
    }
    __syncthreads();
    int buffer = 0;
    // While a step's products run from one buffer, the next step's rows, in registers, turn into the other, and
    // the ones after that are loaded as registers fall free.  (Rows past the end are zeros.)
    constexpr int kBlocks = TL::WM / 32;
    for (int64_t t = t0; t < end; t += kDepth) {
        const char* la = lds + buffer * kBuffer;
        buffer ^= 1;
        char* next = lds + buffer * kBuffer;
        fetch(la, Type<0>{});
        fetch(la, Type<1>{});
        each_of<kBlocks>([&](auto i) {
            multiply(Type<0>{}, i);
            each_of<4 / kBlocks>([&](auto q) { put_a(next, Type<i.value * (4 / kBlocks) + q.value>{}); });
        });
        loader.load_a(t + 2 * kDepth, ua);
        scales();
        fetch(la, Type<2>{});
        each_of<kBlocks>([&](auto i) {
            multiply(Type<1>{}, i);
            each_of<4 / kBlocks>([&](auto q) { put_b(next, Type<i.value * (4 / kBlocks) + q.value>{}); });
        });
        fetch(la, Type<3>{});
        each_of<kBlocks>([&](auto i) {
            multiply(Type<2>{}, i);
            each_of<4 / kBlocks>([&](auto q) { put_b(next, Type<4 + i.value * (4 / kBlocks) + q.value>{}); });
        });
        loader.load_b(t + 2 * kDepth, ub);
        each_of<kBlocks>([&](auto i) { multiply(Type<3>{}, i); });
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
