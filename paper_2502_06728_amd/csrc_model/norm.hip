// x_out = x + scale * gate (.) post(f) and y = pre(x_out): the norm after a block, its gate, the residual
// sum and the norm before the next block in one pass over the rows, y also in 8 bits.
//
// Bound by memory: x and f are read once, x_out, y and the codes written once; a row stays in registers
// between its two norms, and the next row's loads go out before this one's sums (16,384 x 2,048, fp32 residual stream and
// bf16: 60 us = 6.7 TB/s; all bf16 43 us = 6.2 TB/s; one row 3 us, a chain of latencies).  LAYER takes its variance around the row's mean (two sums one after the other), so
// that a large mean costs no digits.
#include "norm_device.hip.h"

namespace deto {
namespace model {
namespace {

struct Args {
    deto_norm_residual cfg;
    int64_t T;
    int D;
    int64_t rows_per_team;
    deto_rows x, f, x_out, y;
    deto_act8 y8;
    bool once;           // the outputs are more than the caches hold: stored past them
};

template <int C>
struct Params {
    float w_post[C][8], b_post[C][8], w_pre[C][8], b_pre[C][8], gate[C][8];
};

// v <- norm(v), of a row of which this lane holds C vectors (zeros past the row's end)
template <class TM, int C>
__device__ __forceinline__ void normalise(TM& team, float (&v)[C][8], int kind, float eps, int D) {
    const float inv_d = 1.f / static_cast<float>(D);
    if (kind == DETO_NORM_LAYER) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[c][j];
        team.sum(s);
        const float mean = s[0] * inv_d;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = TM::has(c, j, D) ? v[c][j] - mean : 0.f;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[0] += v[c][j] * v[c][j];
    team.sum(q);
    const float r = 1.f / sqrtf(q[0] * inv_d + eps);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] *= r;
}

// LAYER: one of the norms is one, or has a bias.  (Without, its registers are not held.)
template <int XT, int FT, int W, int C, int L, bool WHOLE, bool LAYER>
__global__ __launch_bounds__((Team<W, C, L, WHOLE, WHOLE && XT == DETO_F32>::kThreadsWg)) void norm_residual_kernel(Args a) {
    using TM = Team<W, C, L, WHOLE, WHOLE && XT == DETO_F32>;
    __shared__ float lds[TM::kSlots];
    TM team(lds);
    const int D = a.D;
    const int64_t first = TM::index() * a.rows_per_team;
    const int64_t end = first + a.rows_per_team < a.T ? first + a.rows_per_team : a.T;
    if (first >= end) return;                // (teams of one wavefront only: no barriers)
    const bool branch = a.f.data != nullptr, post = branch && a.cfg.post != DETO_NORM_NONE,
               pre = a.cfg.pre != DETO_NORM_NONE;
    const int pre_kind = LAYER ? a.cfg.pre : DETO_NORM_RMS, post_kind = LAYER ? a.cfg.post : DETO_NORM_RMS;
    Raw8<XT> rx[C];
    Raw8<FT> rf[C];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            rx[c] = TM::template load<XT>(a.x.data, t * a.x.ld, c, D);
            if (branch) rf[c] = TM::template load<FT>(a.f.data, t * a.f.ld, c, D);
        }
    };
    if constexpr (!TM::kLean) load(first);
    // The parameters stay in registers over the team's rows; the gate (with the branch's scale) as long as its
    // row is the same.
    Params<C> p;
    auto param = [&](float (&v)[C][8], const void* at, int64_t row, float otherwise) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (at) TM::load_any(at, a.cfg.param_dtype, row, c, D, v[c]);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = otherwise;
        }
    };
    auto params_of_norms = [&](bool of_post, bool of_pre) {
        if (of_post && post) param(p.w_post, a.cfg.w_post, 0, 1.f);
        if (of_pre && pre) param(p.w_pre, a.cfg.w_pre, 0, 1.f);
        if constexpr (LAYER) {
            if (of_post && post) param(p.b_post, a.cfg.b_post, 0, 0.f);
            if (of_pre && pre) param(p.b_pre, a.cfg.b_pre, 0, 0.f);
        }
    };
    if constexpr (!TM::kLean) params_of_norms(true, true);
    int64_t gate_row = -1;
    for (int64_t t = first; t < end; ++t) {
        float v[C][8], x[C][8];
        if constexpr (TM::kLean) load(t);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            TM::template unpack<XT>(rx[c], c, D, x[c]);
            if (branch) TM::template unpack<FT>(rf[c], c, D, v[c]);
        }
        if constexpr (!TM::kLean)
            if (t + 1 < end) load(t + 1);
        if (branch) {
            const int64_t g = a.cfg.rows_per_gate ? t / a.cfg.rows_per_gate : 0;
            if (TM::kLean || g != gate_row) {
                gate_row = g;
                param(p.gate, a.cfg.gate, g * a.cfg.ld_gate, 1.f);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) p.gate[c][j] *= a.cfg.scale;
            }
            if (post) normalise(team, v, post_kind, a.cfg.eps_post, D);
            if constexpr (TM::kLean) params_of_norms(true, false);
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float u = v[c][j];
                    if (post) u *= p.w_post[c][j];
                    if constexpr (LAYER)
                        if (post) u += p.b_post[c][j];
                    x[c][j] = TM::has(c, j, D) ? x[c][j] + p.gate[c][j] * u : 0.f;
                }
            }
#pragma unroll
            for (int c = 0; c < C; ++c) TM::template store<XT>(a.x_out.data, t * a.x_out.ld, c, D, x[c], a.once);
        }
        if (!pre) continue;
        normalise(team, x, pre_kind, a.cfg.eps_pre, D);
        if constexpr (TM::kLean) params_of_norms(false, true);
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[c][j] *= p.w_pre[c][j];
                if constexpr (LAYER) x[c][j] += p.b_pre[c][j];
                if (!TM::has(c, j, D)) x[c][j] = 0.f;
            }
            if (a.y.data) TM::template store<FT>(a.y.data, t * a.y.ld, c, D, x[c], a.once);
            if (a.y8.codes) TM::put8(a.y8, t, c, D, x[c]);
        }
    }
}

// Rows a team takes one after the other.
int64_t rows_per_team(int64_t T, int teams_wg) {
    const int64_t teams = int64_t{4096} * teams_wg;
    const int64_t rows = (T + teams - 1) / teams;
    return rows < 1 ? 1 : rows;
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" int detonation_norm_residual(const deto_norm_residual* cfg, int64_t T, int64_t D,
                                        const deto_rows* x, const deto_rows* f,
                                        const deto_rows* x_out, const deto_rows* y,
                                        const deto_act8* y8, void* stream) {
    int rc = check_norm(cfg, T, D);
    if (rc || T == 0) return rc;
    const bool branch = here(f), pre = cfg->pre != DETO_NORM_NONE;
    if (!here(x) || (branch && !here(x_out)) || (pre && !here(y) && !here(y8))) return DETO_ERR_NULL;
    if ((!branch && (cfg->post != DETO_NORM_NONE || cfg->gate || here(x_out))) ||
        (!pre && (here(y) || here(y8))) || (!branch && !pre))
        return DETO_ERR_BAD_CONFIG;
    rc = first_error(check_rows(x, T, D), branch ? check_rows(f, T, D) : 0,
                     branch ? check_rows(x_out, T, D) : 0, here(y) ? check_rows(y, T, D) : 0,
                     here(y8) ? check_act8(y8, T, D) : 0);
    if (rc) return rc;
    // y has f's type; without f it may have any, without both it has x's
    const int ft = branch ? f->dtype : here(y) ? y->dtype : x->dtype;
    if ((branch && x_out->dtype != x->dtype) || (here(y) && y->dtype != ft) ||
        (x->dtype != ft && x->dtype != DETO_F32))
        return DETO_ERR_BAD_CONFIG;
    const deto_rows none = {};
    Args a = {*cfg, T, static_cast<int>(D), 0, *x, branch ? *f : none, branch ? *x_out : none,
              here(y) ? *y : none, here(y8) ? *y8 : deto_act8{}};
    // (8,192 x 4,096, fp32 and bf16, us: 80, past the caches 61; 16,384 x 768, which they hold: 25, past them 27.  With y alone
    // left there 61 as well: a product that reads it next then takes 0 to 6 % less, but 16,384 x 2,048 with the 8-bit form
    // written and decoded 91 instead of 82)
    a.once = T * D * type_size(x->dtype) >= kCacheBytes / 4;
    fresh();
    const bool layer = cfg->pre == DETO_NORM_LAYER || cfg->post == DETO_NORM_LAYER || cfg->b_pre || cfg->b_post;
    by_width(D, [&](auto w, auto c, auto l, auto whole) {
        using TM = Team<w.value, c.value, l.value, whole.value>;
        a.rows_per_team = rows_per_team(T, TM::kTeamsWg);
        const int64_t teams = (T + a.rows_per_team - 1) / a.rows_per_team;
        const unsigned grid = static_cast<unsigned>((teams + TM::kTeamsWg - 1) / TM::kTeamsWg);
        by_types(x->dtype, ft, [&](auto xt, auto fty) {
            if (layer)
                norm_residual_kernel<xt.value, fty.value, w.value, c.value, l.value, whole.value, true>
                    <<<grid, TM::kThreadsWg, 0, static_cast<hipStream_t>(stream)>>>(a);
            else
                norm_residual_kernel<xt.value, fty.value, w.value, c.value, l.value, whole.value, false>
                    <<<grid, TM::kThreadsWg, 0, static_cast<hipStream_t>(stream)>>>(a);
            return 0;
        });
    });
    return enqueued();
}
