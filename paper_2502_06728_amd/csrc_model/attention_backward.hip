// Gradients of attention: three launches.  dout . out of every query and head; then the gradients of keys and values, a
// workgroup for each 128 keys of a head of keys that walks over the queries that see them, of all heads that share it;
// then those of queries, a workgroup for each 128 queries that walks over the keys they see.  The weights are computed
// again from lse in both: two of seven products, but every sum has one owner, who adds in a fixed order.
#include "attention_device.hip.h"

namespace deto {
namespace model {
namespace attention {
namespace {

constexpr int kOwn = kWaves * kSide;        // keys, or queries, of a workgroup
template <int DT> constexpr int kKeys = DT == DETO_F32 ? 32 : 64;      // of a step of the queries' kernel
constexpr int kQueries = 32;                // of a step of the keys' kernel
// fp32 rows and sums of 128 features take the registers of two wavefronts
template <class S> constexpr int kResident = S::DT == DETO_F32 && S::DP == 128 ? 1 : 2;

// ---- delta[h][t] = dout . out
constexpr int kDotLanes = 16;

template <int DT>
__global__ __launch_bounds__(kThreads) void dots_kernel(Args a, FastDiv heads, uint32_t count) {
    const uint32_t id = blockIdx.x * (kThreads / kDotLanes) + threadIdx.x / kDotLanes;
    const bool there = id < count;
    const uint32_t t = heads.div(there ? id : 0), h = (there ? id : 0) - t * heads.d;
    const int D = a.head_dim, d = threadIdx.x % kDotLanes * 8, n = D - d >= 8 ? 8 : D - d > 0 ? D - d : 0;
    const int64_t col = int64_t{h} * D;
    float x[8], y[8], sum = 0.f;
    unpack8<DT>(load8<DT>(a.out.data + t * a.out.ld + col * kSize<DT>, 0, d, n), x);
    unpack8<DT>(load8<DT>(a.dout.data + t * a.dout.ld + col * kSize<DT>, 0, d, n), y);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fmaf(x[j], y[j], sum);
    sum = lanes_sum<kDotLanes>(sum);
    if (there && d == 0) a.delta[h * a.Tq + t] = sum;
}

// A query's lse in powers of two; one that sees nothing gets weights of zero.
__device__ __forceinline__ float stored_lse(float lse) {
    return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2E;
}

// ---- dq
template <class S, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void queries_kernel(Args a) {
    constexpr int DT = S::DT, BN = kKeys<DT>, kMatrix = BN * S::kRow;
    extern __shared__ __align__(16) char lds[];          // two buffers of keys and values
    __shared__ uint32_t bits[3][2];                      // rows of keys that hold infinities
    const uint32_t id = number_in_part();
    const int h = id / a.tiles;
    int64_t s;
    int32_t tile, tiles;
    if (!find_tile(a, a.q_starts, a.Tq, kOwn, id % a.tiles, s, tile, tiles)) return;
    if (a.causal) tile = tiles - 1 - tile;
    const Sequence seq = sequence_of(a, s);
    const int D = a.head_dim, lane = threadIdx.x % kLanes, half = lane / kSide;
    const int i0 = tile * kOwn, w0 = i0 + threadIdx.x / kLanes * kSide, i = w0 + lane % kSide;
    const bool there = i < seq.Lq;

    const auto seen = [&](int n) {
        if (!a.causal) return seq.Lk;
        const int64_t upto = int64_t{n} + seq.Lk - seq.Lq + 1;
        return static_cast<int>(upto < 0 ? 0 : upto < seq.Lk ? upto : seq.Lk);
    };
    const int last = seq.Lq - 1;
    const int upto = seen(i0 + kOwn - 1 < last ? i0 + kOwn - 1 : last);
    const int wave_upto = seen(w0 + kSide - 1 < last ? w0 + kSide - 1 : last);
    const int own = seen(i);
    const int steps = (upto + BN - 1) / BN, whole_steps = seen(i0) / BN;

    const int64_t kv = int64_t{h / a.group} * D * S::kElem, col = int64_t{h} * D * S::kElem;
    const char* const keys = a.k.data + seq.k0 * a.k.ld + kv;
    const char* const values = a.v.data + seq.k0 * a.v.ld + kv;
    const int64_t row = seq.q0 + (there ? i : last);
    u32x4 q[S::kFrags], g[S::kFrags];
    load_row<S, WHOLE>(a.q.data + row * a.q.ld + col, there, D, q);
    load_row<S, WHOLE>(a.dout.data + row * a.dout.ld + col, there, D, g);
    const float factor = a.scale * kLog2E;
    const float lse = there ? stored_lse(a.lse[h * a.Tq + row]) : __builtin_inff();
    const float delta = there ? a.delta[h * a.Tq + row] : 0.f;
    f32x16 dq[S::kBlocks] = {};

    if (threadIdx.x < 6) bits[threadIdx.x / 2][threadIdx.x % 2] = 0;
    __syncthreads();
    Stage<S, BN, WHOLE> sk, sv;
    const auto have = [&](int step) { return seq.Lk - step * BN < BN ? seq.Lk - step * BN : BN; };
    const auto load = [&](int step) {
        sk.load(keys + int64_t{step} * BN * a.k.ld, a.k.ld, have(step), D);
        sv.load(values + int64_t{step} * BN * a.v.ld, a.v.ld, have(step), D);
    };
    const auto store = [&](int step) {
        char* const at = lds + step % 2 * 2 * kMatrix;
        if (step >= whole_steps) sk.template store<true>(at, have(step), bits[step % 3]);
        else sk.template store<false>(at, have(step), nullptr);
        sv.template store<false>(at + kMatrix, have(step), nullptr);
    };
    const auto compute = [&](int step, auto masked) {
        constexpr bool MASKED = masked.value != 0;
        const char* const at = lds + step % 2 * 2 * kMatrix;
        const int left = own - step * BN - half * 4;
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b) {
            f32x16 x = rows_product<S>(at, b, q);
            const f32x16 y = rows_product<S>(at + kMatrix, b, g);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[r] = power2(fmaf(x[r], factor, -lse)) * (y[r] - delta);
                if (MASKED) x[r] = b * kSide + (r / 4) * 8 + r % 4 < left ? x[r] : 0.f;
            }
            columns_product<S>(at, b, x, dq);
            if (MASKED) {
                const uint32_t odd = bits[step % 3][b];
                if (odd)
                    add_infinities<S>(odd, keys + (int64_t{step} * BN + b * kSide) * a.k.ld, a.k.ld, D, x,
                                      [&](int n) { return step * BN + b * kSide + n < own; }, dq);
            }
        }
    };

    if (steps > 0) {
        load(0);
        store(0);
    }
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        if (threadIdx.x < 2) bits[(step + 2) % 3][threadIdx.x] = 0;
        if (step + 1 < steps) load(step + 1);
        if (step < whole_steps) compute(step, Type<0>{});
        else if (step * BN < wave_upto) compute(step, Type<1>{});
        if (step + 1 < steps) store(step + 1);
        __syncthreads();
    }
    store_columns<S>(dq, a.scale, a.dq.data + row * a.dq.ld + col, there, D);
}

// ---- dk, dv
template <class S, bool WHOLE>
__global__ __launch_bounds__(kThreads, kResident<S>) void keys_kernel(Args a) {
    constexpr int BQ = kQueries, kMatrix = BQ * S::kRow;
    extern __shared__ __align__(16) char lds[];          // two buffers of queries and gradients of outputs
    __shared__ __align__(16) float stats[2][2][BQ];      // two buffers of lse and delta
    __shared__ uint32_t bits[3][2];                      // rows of queries, of gradients that hold infinities
    const uint32_t id = number_in_part();
    const int hk = id / a.tiles;
    int64_t s;
    int32_t tile, tiles;
    if (!find_tile(a, a.k_starts, a.Tk, kOwn, id % a.tiles, s, tile, tiles)) return;
    const Sequence seq = sequence_of(a, s);
    const int D = a.head_dim, lane = threadIdx.x % kLanes, half = lane / kSide;
    const int j0 = tile * kOwn, w0 = j0 + threadIdx.x / kLanes * kSide, j = w0 + lane % kSide;
    const bool there = j < seq.Lk;

    // the first query that sees key n
    const auto seen_from = [&](int n) {
        if (!a.causal) return 0;
        const int64_t from = int64_t{n} - seq.Lk + seq.Lq;
        return static_cast<int>(from < 0 ? 0 : from < seq.Lq ? from : seq.Lq);
    };
    const int last = seq.Lk - 1;
    const int first_step = seen_from(j0) / BQ, steps = (seq.Lq + BQ - 1) / BQ - first_step;    // of a head
    const int all_from = seen_from(j0 + kOwn - 1 < last ? j0 + kOwn - 1 : last);     // seen by these queries in full
    const int wave_from = seen_from(w0 < last ? w0 : last);
    const int own = seen_from(there ? j : last);

    const int64_t kv = int64_t{hk} * D * S::kElem;
    const int64_t row = seq.k0 + (there ? j : last);
    u32x4 k[S::kFrags], v[S::kFrags];
    load_row<S, WHOLE>(a.k.data + row * a.k.ld + kv, there, D, k);
    load_row<S, WHOLE>(a.v.data + row * a.v.ld + kv, there, D, v);
    const float factor = a.scale * kLog2E;
    f32x16 dk[S::kBlocks] = {}, dv[S::kBlocks] = {};

    if (threadIdx.x < 6) bits[threadIdx.x / 2][threadIdx.x % 2] = 0;
    __syncthreads();
    Stage<S, BQ, WHOLE> sq, sg;
    float stat = 0.f;
    const int total = steps * a.group;                   // a head's steps, then the next one's
    const auto head = [&](int n) { return hk * a.group + n / steps; };
    const auto first = [&](int n) { return (first_step + n % steps) * BQ; };
    const auto have = [&](int n) { return seq.Lq - first(n) < BQ ? seq.Lq - first(n) : BQ; };
    const auto load = [&](int n) {
        const int64_t at = seq.q0 + first(n), col = int64_t{head(n)} * D * S::kElem;
        sq.load(a.q.data + at * a.q.ld + col, a.q.ld, have(n), D);
        sg.load(a.dout.data + at * a.dout.ld + col, a.dout.ld, have(n), D);
        const int t = threadIdx.x % BQ;
        if (threadIdx.x < 2 * BQ && t < have(n)) stat = (threadIdx.x < BQ ? a.lse : a.delta)[head(n) * a.Tq + at + t];
    };
    const auto store = [&](int n) {
        char* const at = lds + n % 2 * 2 * kMatrix;
        if (first(n) < all_from) {
            sq.template store<true>(at, have(n), &bits[n % 3][0]);
            sg.template store<true>(at + kMatrix, have(n), &bits[n % 3][1]);
        } else {
            sq.template store<false>(at, have(n), nullptr);
            sg.template store<false>(at + kMatrix, have(n), nullptr);
        }
        if (threadIdx.x < 2 * BQ) {
            const bool is_lse = threadIdx.x < BQ, past = static_cast<int>(threadIdx.x % BQ) >= have(n);
            stats[n % 2][!is_lse][threadIdx.x % BQ] =
                past ? (is_lse ? __builtin_inff() : 0.f) : is_lse ? stored_lse(stat) : stat;
        }
    };
    const auto compute = [&](int n, auto masked) {
        constexpr bool MASKED = masked.value != 0;
        const char* const at = lds + n % 2 * 2 * kMatrix;
        const int from = own - first(n) - half * 4;          // of the step's queries, those that see the key
        f32x16 p = rows_product<S>(at, 0, k);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = (r / 4) * 8 + r % 4;
            p[r] = power2(fmaf(p[r], factor, -stats[n % 2][0][t + half * 4]));
            if (MASKED) p[r] = t >= from ? p[r] : 0.f;
        }
        f32x16 ds = rows_product<S>(at + kMatrix, 0, v);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = (r / 4) * 8 + r % 4;
            ds[r] = p[r] * (ds[r] - stats[n % 2][1][t + half * 4]);
            if (MASKED) ds[r] = t >= from ? ds[r] : 0.f;
        }
        columns_product<S>(at + kMatrix, 0, p, dv);
        columns_product<S>(at, 0, ds, dk);
        if (MASKED) {
            const uint32_t odd_q = bits[n % 3][0], odd_g = bits[n % 3][1];
            if (odd_q | odd_g) {
                const int64_t at = seq.q0 + first(n), col = int64_t{head(n)} * D * S::kElem;
                const auto sees = [&](int t) { return first(n) + t >= own; };
                add_infinities<S>(odd_g, a.dout.data + at * a.dout.ld + col, a.dout.ld, D, p, sees, dv);
                add_infinities<S>(odd_q, a.q.data + at * a.q.ld + col, a.q.ld, D, ds, sees, dk);
            }
        }
    };

    if (total > 0) {
        load(0);
        store(0);
    }
    __syncthreads();
    for (int n = 0; n < total; ++n) {
        if (threadIdx.x < 2) bits[(n + 2) % 3][threadIdx.x] = 0;
        if (n + 1 < total) load(n + 1);
        if (first(n) >= all_from) compute(n, Type<0>{});
        else if (first(n) + BQ > wave_from) compute(n, Type<1>{});
        if (n + 1 < total) store(n + 1);
        __syncthreads();
    }
    store_columns<S>(dk, a.scale, a.dk.data + row * a.dk.ld + kv, there, D);
    store_columns<S>(dv, 1.f, a.dv.data + row * a.dv.ld + kv, there, D);
}

}  // namespace
}  // namespace attention
}  // namespace model
}  // namespace deto

using namespace deto::model;
using namespace deto::model::attention;

extern "C" {

int detonation_attention_backward(const deto_attention* cfg, int64_t Tq, int64_t Tk, const deto_rows* q,
                                  const deto_rows* k, const deto_rows* v, const deto_rows* out,
                                  const float* lse, const deto_rows* dout, const deto_rows* dq,
                                  const deto_rows* dk, const deto_rows* dv, void* workspace, void* stream) {
    int rc = check(cfg, Tq, Tk);
    if (rc) return rc;
    if (Tq == 0 && Tk == 0) return DETO_OK;
    const deto_rows* const any = Tq ? q : k;
    if (!here(any)) return DETO_ERR_NULL;
    const int H = cfg->heads, K = cfg->kv_heads, dtype = any->dtype;
    rc = first_error(check_matrix(cfg, q, Tq, H, dtype), check_matrix(cfg, k, Tk, K, dtype), check_matrix(cfg, v, Tk, K, dtype),
                     check_matrix(cfg, out, Tq, H, dtype), check_matrix(cfg, dout, Tq, H, dtype),
                     check_matrix(cfg, dq, Tq, H, dtype), check_matrix(cfg, dk, Tk, K, dtype),
                     check_matrix(cfg, dv, Tk, K, dtype));
    if (rc) return rc;
    if (Tq && (!lse || !workspace)) return DETO_ERR_NULL;
    if (!is_aligned(lse, 4) || !is_aligned(workspace, 16)) return DETO_ERR_ALIGN;
    Args a = args_of(cfg, Tq, Tk, q, k, v);
    a.lse = const_cast<float*>(lse);
    a.delta = static_cast<float*>(workspace);
    if (Tq) {
        a.out = matrix_of(out);
        a.dout = matrix_of(dout);
        a.dq = matrix_of(dq);
    }
    if (Tk) {
        a.dk = matrix_of(dk);
        a.dv = matrix_of(dv);
    }
    Args by_keys = a;
    if (!plan(a, cfg->q_starts, Tq, kOwn, H) || !plan(by_keys, cfg->k_starts, Tk, kOwn, K) || Tq * H >= (int64_t{1} << 31))
        return DETO_ERR_UNSUPPORTED;
    const hipStream_t on = static_cast<hipStream_t>(stream);
    fresh();
    by_type(dtype, [&](auto dt) {
        const uint32_t dots = static_cast<uint32_t>(Tq * H);
        constexpr uint32_t kEach = kThreads / kDotLanes;
        if (dots) dots_kernel<dt.value><<<(dots + kEach - 1) / kEach, kThreads, 0, on>>>(a, FastDiv(static_cast<uint32_t>(H)), dots);
        return by_shape<dt.value>(cfg->head_dim, [&](auto shape, auto whole) {
            using S = decltype(shape);
            if (Tk) keys_kernel<S, whole.value != 0><<<by_keys.tiles * K, kThreads, 4 * kQueries * S::kRow, on>>>(by_keys);
            if (Tq) queries_kernel<S, whole.value != 0><<<a.tiles * H, kThreads, 4 * kKeys<S::DT> * S::kRow, on>>>(a);
            return 0;
        });
    });
    return enqueued();
}

}  // extern "C"
