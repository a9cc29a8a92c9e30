// softmax(scale q k^T) v and log sum exp, one pass over the keys.
//
// A workgroup takes 128 or 256 queries of a head, 32 a wavefront, and walks over the keys they see, 64 (fp32: 32) at a
// time in LDS.  A lane has one query: its running maximum and sum are two registers, and its scores, as they come out
// of the first product, are the second product's operand.
#include "attention_device.hip.h"

namespace deto {
namespace model {
namespace attention {
namespace {

template <int DT> constexpr int kKeys = DT == DETO_F32 ? 32 : 64;      // of a step

// A query's maximum may lag behind by this much (in powers of two): its weights stay below 2^8, and the sums so far need
// not be scaled down for every new maximum.
constexpr float kLag = 8.f;

template <class S, int W, bool DIRECT>
__global__ __launch_bounds__(W * kLanes, 2) void forward_kernel(Args a) {
    constexpr int DT = S::DT, BM = W * kSide, BN = kKeys<DT>, kMatrix = BN * S::kRow, kStep = 2 * kMatrix;
    constexpr int AHEAD = kAhead<W, kStep, DIRECT>;
    extern __shared__ __align__(16) char lds[];          // AHEAD + 1 steps of keys and values
    __shared__ uint32_t odd;                             // infinities or NaNs among values that not all queries see
    Place at;
    if (!place_of(a, a.q_starts, a.Tq, BM, a.heads, a.causal, at)) return;
    const Sequence seq = sequence_of(a, at.s);
    const int D = DIRECT ? S::DP : a.head_dim, lane = threadIdx.x % kLanes, half = lane / kSide;
    const int i0 = at.tile * BM, w0 = i0 + threadIdx.x / kLanes * kSide, i = w0 + lane % kSide, last = seq.Lq - 1;
    const bool there = i <= last;

    // keys that query n sees
    const auto seen = [&](int n) {
        if (!a.causal) return seq.Lk;
        const int64_t upto = int64_t{n < last ? n : last} + seq.Lk - last;
        return static_cast<int>(upto < 0 ? 0 : upto);
    };
    const int upto = seen(i0 + BM - 1), wave_upto = seen(w0 + kSide - 1);        // by any of the workgroup's, the wavefront's
    const int own = seen(i), steps = (upto + BN - 1) / BN, whole_steps = seen(i0) / BN;

    const int64_t col = int64_t{at.head} * D * S::kElem, kv = int64_t{at.head / a.group} * D * S::kElem;
    const char* const keys = a.k.data + seq.k0 * a.k.ld + kv;
    const char* const values = a.v.data + seq.k0 * a.v.ld + kv;
    const char* const query = a.q.data + (seq.q0 + (there ? i : last)) * a.q.ld + col;

    Rows<S, BN, W, DIRECT> rk, rv;
    const auto buffer = [&](int step) { return lds + step % (AHEAD + 1) * kStep; };
    const auto begin = [&](int step) {
        const int have = seq.Lk - step * BN < BN ? seq.Lk - step * BN : BN;
        rk.begin(buffer(step), keys + int64_t{step} * BN * a.k.ld, a.k.ld, have, D);
        rv.begin(buffer(step) + kMatrix, values + int64_t{step} * BN * a.v.ld, a.v.ld, have, D);
    };
    const auto end = [&](int step) {
        rk.end(buffer(step));
        rv.end(buffer(step) + kMatrix);
    };
    if (threadIdx.x == 0) odd = 0;
#pragma unroll
    for (int n = 0; n < AHEAD; ++n)
        if (n < steps) begin(n);
    if (steps > 0) end(0);

    u32x4 q[S::kFrags];
    load_row<S>(query, there, D, q);
    const float factor = a.scale * kLog2E;       // of scores, to powers of two
    float m = -__builtin_inff(), base = 0.f, l = 0.f;
    f32x16 o[S::kBlocks] = {};

    const auto compute = [&](int step, auto masked) {
        constexpr bool MASKED = masked.value != 0;
        const char* const from = buffer(step);
        f32x16 x[BN / kSide];
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b) x[b] = rows_product<S>(from, b, q);
        const int left = own - step * BN - half * 4;         // of the keys that the query sees
        float top = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (MASKED) x[b][r] = b * kSide + (r / 4) * 8 + r % 4 < left ? x[b][r] : -__builtin_inff();
                top = fmaxf(top, x[b][r]);
            }
        top = halves_max(top);
        if (__any((top - m) * factor > kLag)) {
            m = fmaxf(m, top);
            const float before = base;
            base = m > -__builtin_inff() ? m * factor : 0.f;
            const float less = power2(before - base);
            l *= less;
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= less;
        }
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[b][r] = power2(fmaf(x[b][r], factor, -base));
                sum += x[b][r];
            }
        l += sum;
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b) columns_product<S>(from + kMatrix, b, x[b], o);
    };

    for (int step = 0; step < steps; ++step) {
        if constexpr (DIRECT) arrived_but<2 * Rows<S, BN, W, DIRECT>::kCalls>(min(AHEAD - 1, steps - 1 - step));
        meet();
        if (step + AHEAD < steps) begin(step + AHEAD);
        if (step < whole_steps) {
            compute(step, Type<0>{});
        } else {
            take_out_odd<S, BN, W>(buffer(step) + kMatrix, &odd);
            meet();
            if (step * BN < wave_upto) compute(step, Type<1>{});
        }
        if (step + AHEAD < steps) end(step + AHEAD);
    }

    if (steps > whole_steps && odd) {
        for (int j = whole_steps * BN; j < wave_upto; ++j) {
            const char* const value = values + j * a.v.ld;
            if (!row_is_odd<S>(value, D)) continue;
            const float weight = power2(fmaf(slow_dot<S>(query, keys + j * a.k.ld, D), factor, -base));
            if (j < own) add_odd<S>(value, D, weight, o);
        }
    }
    l = halves_sum(l);
    const int64_t row = seq.q0 + i;
    store_columns<S>(o, l == 0.f ? 0.f : 1.f / l, a.out.data + row * a.out.ld + col, there, D);
    if (a.lse && there && half == 0)
        a.lse[at.head * a.Tq + row] = l == 0.f ? -__builtin_inff() : (base + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

int check(const deto_attention* cfg, int64_t Tq, int64_t Tk) {
    if (!cfg) return DETO_ERR_NULL;
    constexpr int64_t kMost = (int64_t{1} << 31) - 1;
    if (Tq < 0 || Tk < 0 || Tq > kMost || Tk > kMost || cfg->sequences < 1 || cfg->sequences > kMost)
        return DETO_ERR_BAD_CONFIG;
    if (cfg->heads < 1 || cfg->heads > 65536 || cfg->kv_heads < 1 || cfg->heads % cfg->kv_heads || cfg->head_dim < 1)
        return DETO_ERR_BAD_CONFIG;
    if ((cfg->causal != 0 && cfg->causal != 1) || cfg->reserved != 0) return DETO_ERR_BAD_CONFIG;
    if (!(cfg->scale > 0.f && cfg->scale < __builtin_inff())) return DETO_ERR_BAD_CONFIG;
    if ((!cfg->q_starts && Tq % cfg->sequences) || (!cfg->k_starts && Tk % cfg->sequences)) return DETO_ERR_BAD_CONFIG;
    if (!is_aligned(cfg->q_starts, 4) || !is_aligned(cfg->k_starts, 4)) return DETO_ERR_ALIGN;
    return cfg->head_dim > 128 ? DETO_ERR_UNSUPPORTED : DETO_OK;
}

int check_matrix(const deto_attention* cfg, const deto_rows* m, int64_t T, int heads, int dtype) {
    if (T == 0) return DETO_OK;
    if (!here(m)) return DETO_ERR_NULL;
    const int rc = check_rows(m, T, int64_t{heads} * cfg->head_dim);
    return rc ? rc : m->dtype != dtype ? DETO_ERR_BAD_CONFIG : DETO_OK;
}

Args args_of(const deto_attention* cfg, int64_t Tq, int64_t Tk, const deto_rows* q, const deto_rows* k, const deto_rows* v) {
    Args a = {};
    if (Tq) a.q = matrix_of(q);
    if (Tk) {
        a.k = matrix_of(k);
        a.v = matrix_of(v);
    }
    a.q_starts = cfg->q_starts;
    a.k_starts = cfg->k_starts;
    a.Tq = Tq;
    a.Tk = Tk;
    a.sequences = cfg->sequences;
    a.heads = cfg->heads;
    a.kv_heads = cfg->kv_heads;
    a.group = cfg->heads / cfg->kv_heads;
    a.head_dim = cfg->head_dim;
    a.causal = cfg->causal;
    a.scale = cfg->scale;
    return a;
}

}  // namespace attention
}  // namespace model
}  // namespace deto

using namespace deto::model;
using namespace deto::model::attention;

extern "C" {

int64_t detonation_attention_workspace(const deto_attention* cfg, int64_t Tq, int64_t Tk) {
    if (check(cfg, Tq, Tk) != DETO_OK) return -1;
    return 2 * cfg->heads * Tq * static_cast<int64_t>(sizeof(float));
}

int detonation_attention_forward(const deto_attention* cfg, int64_t Tq, int64_t Tk, const deto_rows* q,
                                 const deto_rows* k, const deto_rows* v, const deto_rows* out,
                                 float* lse, void* workspace, void* stream) {
    int rc = check(cfg, Tq, Tk);
    if (rc) return rc;
    if (Tq == 0) return DETO_OK;
    if (!here(q)) return DETO_ERR_NULL;
    rc = first_error(check_matrix(cfg, q, Tq, cfg->heads, q->dtype), check_matrix(cfg, k, Tk, cfg->kv_heads, q->dtype),
                     check_matrix(cfg, v, Tk, cfg->kv_heads, q->dtype), check_matrix(cfg, out, Tq, cfg->heads, q->dtype));
    if (rc) return rc;
    if (!is_aligned(lse, 4)) return DETO_ERR_ALIGN;
    (void)workspace;
    Args a = args_of(cfg, Tq, Tk, q, k, v);
    a.out = matrix_of(out);
    a.lse = lse;
    int planned = DETO_OK;
    const bool wide = Tq * cfg->heads >= int64_t{256} * kCUs;
    fresh();
    by_type(q->dtype, [&](auto dt) {
        return by_shape<dt.value>(cfg->head_dim, in_pieces(a.k) && in_pieces(a.v), [&](auto shape, auto direct) {
            using S = decltype(shape);
            const auto run = [&](auto waves) {
                constexpr int W = waves.value;
                constexpr bool DIRECT = direct.value != 0;
                if (!plan(a, cfg->q_starts, Tq, W * kSide, cfg->heads)) return planned = DETO_ERR_UNSUPPORTED;
                constexpr int kStep = 2 * kKeys<S::DT> * S::kRow;
                forward_kernel<S, W, DIRECT><<<a.tiles * cfg->heads, W * kLanes, (kAhead<W, kStep, DIRECT> + 1) * kStep,
                                               static_cast<hipStream_t>(stream)>>>(a);
                return 0;
            };
            return wide ? run(Type<8>{}) : run(Type<4>{});
        });
    });
    if (planned) return planned;
    return enqueued();
}

}  // extern "C"
