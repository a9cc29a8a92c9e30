// Gradients of norm, gate and residual: both inputs, the gate, the norms' weights and biases.
//
// With n the normalised row, r its factor, a = dy (.) w, the gradient of a norm's input is
//     r (a - n mean(a n) [- mean(a) under LAYER])
// and those of its weight and bias are the sums over rows of dy (.) n and dy.  A team takes a run of rows, keeps
// the sums of its columns in registers and leaves them in the workspace; a second launch adds the teams'
// sums, always in the same order.  A run lies within one gate row (or holds whole ones, whose gradients the
// team then writes itself).
//
// Bound by memory: x_out, f, dy, dx_out are read once, dx and df written once.
#include "norm_device.hip.h"

namespace deto {
namespace model {
namespace {

enum { kWPre, kBPre, kWPost, kBPost, kGate, kSums };

// How rows are dealt to teams: `gates` gate rows of `rows` rows each (one of all rows without
// rows_per_gate); every gate row is cut into `cuts` runs, or a team takes `group` whole ones.
struct Deal {
    int64_t T, rows, gates, cuts, run, group, teams;
};

struct Args {
    deto_norm_residual cfg;
    int D;
    Deal deal;
    deto_rows x, f, dy, dxo, dx, df;
    deto_norm_grads grads;
    float* parts;        // [team][slot][D]
    int slot[kSums];     // of a sum in `parts`, -1: not wanted, or written by the team itself
    int slots;
};

// mean and factor of a row; v becomes what the factor multiplies
template <class TM, int C>
__device__ __forceinline__ float centre(TM& team, float (&v)[C][8], int kind, float eps, int D) {
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
        for (int c = 0; c < C; ++c) {
            const int n = TM::count(c, D);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = j < n ? v[c][j] - mean : 0.f;
        }
    }
    float q[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[0] += v[c][j] * v[c][j];
    team.sum(q);
    return 1.f / sqrtf(q[0] * inv_d + eps);
}

// v: the normalised row, a: the gradient of the norm's output times its weight; a <- gradient of the input
template <class TM, int C>
__device__ __forceinline__ void back(TM& team, const float (&v)[C][8], float (&a)[C][8], float r,
                                     int kind, int D) {
    const float inv_d = 1.f / static_cast<float>(D);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[0] += a[c][j] * v[c][j];
            s[1] += a[c][j];
        }
    team.sum(s);
    const float m0 = s[0] * inv_d, m1 = kind == DETO_NORM_LAYER ? s[1] * inv_d : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) a[c][j] = r * (a[c][j] - v[c][j] * m0 - m1);
}

template <int C>
__device__ __forceinline__ void clear(float (&v)[C][8]) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = 0.f;
}

template <int XT, int FT, int W, int C>
__global__ __launch_bounds__((Team<W, C>::kThreadsWg)) void norm_backward_kernel(Args a) {
    using TM = Team<W, C>;
    __shared__ float lds[TM::kSlots];
    TM team(lds);
    const int D = a.D;
    const Deal& deal = a.deal;
    const int64_t me = TM::index();
    if (me >= deal.teams) return;            // (teams of one wavefront only: no barriers)
    int64_t first, end;
    if (deal.group) {
        first = me * deal.group * deal.rows;
        end = first + deal.group * deal.rows;
    } else {
        const int64_t g = me / deal.cuts;
        first = g * deal.rows + me % deal.cuts * deal.run;
        end = first + deal.run;
        const int64_t last = (g + 1) * deal.rows;
        if (end > last) end = last;
    }
    if (end > deal.T) end = deal.T;
    const bool branch = a.f.data != nullptr, pre = a.cfg.pre != DETO_NORM_NONE,
               post = a.cfg.post != DETO_NORM_NONE;
    float sums[kSums][C][8];
#pragma unroll
    for (int i = 0; i < kSums; ++i) clear(sums[i]);
    for (int64_t t = first; t < end; ++t) {
        float v[C][8], G[C][8], o[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int d = TM::feature(c), n = TM::count(c, D);
            unpack8<XT>(load8<XT>(a.x.data, t * a.x.ld + d, n), v[c]);
            if (pre) unpack8<FT>(load8<FT>(a.dy.data, t * a.dy.ld + d, n), G[c]);
            if (a.dxo.data) unpack8<XT>(load8<XT>(a.dxo.data, t * a.dxo.ld + d, n), o[c]);
        }
        if (!a.dxo.data) clear(o);
        if (pre) {
            const float r = centre(team, v, a.cfg.pre, a.cfg.eps_pre, D);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int d = TM::feature(c), n = TM::count(c, D);
                float w[8];
                if (a.cfg.w_pre) load8_any(a.cfg.w_pre, a.cfg.param_dtype, d, n, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[c][j] *= r;
                    sums[kWPre][c][j] += G[c][j] * v[c][j];
                    sums[kBPre][c][j] += G[c][j];
                    if (a.cfg.w_pre) G[c][j] *= w[j];
                }
            }
            back(team, v, G, r, a.cfg.pre, D);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) G[c][j] += o[c][j];
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) G[c][j] = o[c][j];
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
            store8<XT>(a.dx.data, t * a.dx.ld + TM::feature(c), G[c], TM::count(c, D));
        if (!branch) continue;
#pragma unroll
        for (int c = 0; c < C; ++c)
            unpack8<FT>(load8<FT>(a.f.data, t * a.f.ld + TM::feature(c), TM::count(c, D)), v[c]);
        float r = 1.f;
        if (post) r = centre(team, v, a.cfg.post, a.cfg.eps_post, D);
        const int64_t gate_row = a.cfg.rows_per_gate ? t / a.cfg.rows_per_gate : 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int d = TM::feature(c), n = TM::count(c, D);
            float w[8], b[8], g[8];
            const bool has_w = post && a.cfg.w_post, has_b = post && a.cfg.b_post;
            if (has_w) load8_any(a.cfg.w_post, a.cfg.param_dtype, d, n, w);
            if (has_b) load8_any(a.cfg.b_post, a.cfg.param_dtype, d, n, b);
            if (a.cfg.gate)
                load8_any(a.cfg.gate, a.cfg.param_dtype, gate_row * a.cfg.ld_gate + d, n, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[c][j] *= r;
                const float u = v[c][j] * (has_w ? w[j] : 1.f) + (has_b ? b[j] : 0.f);
                float s = a.cfg.scale * G[c][j];
                sums[kGate][c][j] += s * u;
                if (a.cfg.gate) s *= g[j];
                sums[kWPost][c][j] += s * v[c][j];
                sums[kBPost][c][j] += s;
                G[c][j] = has_w ? s * w[j] : s;
            }
        }
        if (post) back(team, v, G, r, a.cfg.post, D);
#pragma unroll
        for (int c = 0; c < C; ++c)
            store8<FT>(a.df.data, t * a.df.ld + TM::feature(c), G[c], TM::count(c, D));
        // a gate row of this team's own ends
        if (deal.group && a.grads.gate && ((t + 1) % deal.rows == 0 || t + 1 == deal.T)) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                store8<DETO_F32>(a.grads.gate, t / deal.rows * D + TM::feature(c), sums[kGate][c],
                                 TM::count(c, D));
            clear(sums[kGate]);
        }
    }
#pragma unroll
    for (int i = 0; i < kSums; ++i)
        if (a.slot[i] >= 0) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                store8<DETO_F32>(a.parts, (me * a.slots + a.slot[i]) * D + TM::feature(c), sums[i][c],
                                 TM::count(c, D));
        }
}

// Adds the teams' sums of 64 columns: four wavefronts take the teams in turn.  blockIdx.y is the output row:
// the weights' and biases' sums over all teams, then the gate's rows, each over the teams of its own.
struct JoinArgs {
    const float* parts;
    int D, slots;
    int64_t teams;
    float* out[kSums];
    int slot[kSums];
    int outs;             // of the first four
    int64_t gate_teams;   // teams of a gate row
};

__global__ __launch_bounds__(256) void norm_join_kernel(JoinArgs a, int64_t y0) {
    __shared__ float lds[4][kLanes];
    const int col = blockIdx.x * kLanes + threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const int64_t y = y0 + blockIdx.y;
    const bool gate = y >= a.outs;
    const int i = gate ? kGate : static_cast<int>(y);
    const int64_t first = gate ? (y - a.outs) * a.gate_teams : 0;
    const int64_t end = gate ? first + a.gate_teams : a.teams;
    float s = 0.f;
    if (col < a.D)
        for (int64_t t = first + wave; t < end; t += 4)
            s += a.parts[(t * a.slots + a.slot[i]) * a.D + col];
    lds[wave][threadIdx.x % kLanes] = s;
    __syncthreads();
    if (wave == 0 && col < a.D) {
        const int l = threadIdx.x;
        a.out[i][(gate ? (y - a.outs) * a.D : 0) + col] = (lds[0][l] + lds[1][l]) + (lds[2][l] + lds[3][l]);
    }
}

// Teams that are wanted: a wavefront's worth of rows each, as many as fill the chip.
constexpr int64_t kTeams = 1024;

Deal deal_rows(const deto_norm_residual* cfg, int64_t T) {
    Deal d = {};
    d.T = T;
    d.rows = cfg->rows_per_gate ? cfg->rows_per_gate : T;
    if (d.rows > T) d.rows = T;
    if (T == 0) {
        d.rows = 1;
        return d;
    }
    d.gates = (T + d.rows - 1) / d.rows;
    if (d.gates > kTeams) {
        d.group = (d.gates + kTeams - 1) / kTeams;
        d.teams = (d.gates + d.group - 1) / d.group;
        return d;
    }
    d.cuts = kTeams / d.gates;
    if (d.cuts > d.rows) d.cuts = d.rows;
    d.run = (d.rows + d.cuts - 1) / d.cuts;
    d.cuts = (d.rows + d.run - 1) / d.run;
    d.teams = d.gates * d.cuts;
    return d;
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int64_t detonation_norm_residual_workspace(const deto_norm_residual* cfg, int64_t T, int64_t D) {
    if (check_norm(cfg, T, D)) return -1;
    return deal_rows(cfg, T).teams * kSums * D * static_cast<int64_t>(sizeof(float));
}

int detonation_norm_residual_backward(const deto_norm_residual* cfg, int64_t T, int64_t D,
                                      const deto_rows* x_out, const deto_rows* f,
                                      const deto_rows* dy, const deto_rows* dx_out,
                                      const deto_rows* dx, const deto_rows* df,
                                      const deto_norm_grads* grads, void* workspace, void* stream) {
    int rc = check_norm(cfg, T, D);
    if (rc) return rc;
    const deto_norm_grads no_grads = {};
    const deto_norm_grads g = grads ? *grads : no_grads;
    const bool pre = cfg->pre != DETO_NORM_NONE, post = cfg->post != DETO_NORM_NONE;
    // (without rows there is nothing to tell a missing matrix from an empty one by)
    const bool branch = T ? here(f) : true;
    if (((g.w_pre || g.b_pre) && !pre) || ((g.w_post || g.b_post) && !(branch && post)) ||
        (g.gate && !(branch && cfg->gate)))
        return DETO_ERR_BAD_CONFIG;
    for (const float* p : {g.w_pre, g.b_pre, g.w_post, g.b_post, g.gate})
        if (!is_aligned(p, 4)) return DETO_ERR_ALIGN;
    Args a = {};
    if (T > 0) {
        if (!here(x_out) || !here(dx) || (pre && !here(dy)) || (branch && !here(df)))
            return DETO_ERR_NULL;
        if ((!pre && here(dy)) || (!branch && (post || cfg->gate || here(df))) || (!branch && !pre))
            return DETO_ERR_BAD_CONFIG;
        rc = first_error(check_rows(x_out, T, D), check_rows(dx, T, D), branch ? check_rows(f, T, D) : 0,
                         branch ? check_rows(df, T, D) : 0, pre ? check_rows(dy, T, D) : 0,
                         here(dx_out) ? check_rows(dx_out, T, D) : 0);
        if (rc) return rc;
        const int xt = x_out->dtype, ft = branch ? f->dtype : dy->dtype;
        if (dx->dtype != xt || (here(dx_out) && dx_out->dtype != xt) || (branch && df->dtype != ft) ||
            (pre && dy->dtype != ft) || (xt != ft && xt != DETO_F32))
            return DETO_ERR_BAD_CONFIG;
    }
    a.cfg = *cfg;
    a.D = static_cast<int>(D);
    a.deal = deal_rows(cfg, T);
    a.grads = g;
    float* const outs[kSums] = {g.w_pre, g.b_pre, g.w_post, g.b_post, g.gate};
    JoinArgs j = {};
    for (int i = 0; i < kSums; ++i) {
        const bool wanted = outs[i] && !(i == kGate && a.deal.group);
        a.slot[i] = wanted ? a.slots++ : -1;
        if (!wanted) continue;
        const int at = i == kGate ? kGate : j.outs++;
        j.out[at] = outs[i];
        j.slot[at] = a.slot[i];
    }
    if (a.slots && a.deal.teams) {
        if (!workspace) return DETO_ERR_NULL;
        if (!is_aligned(workspace, 16)) return DETO_ERR_ALIGN;
    }
    if (T == 0 && a.slots == 0) return DETO_OK;
    a.parts = static_cast<float*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    fresh();
    if (T > 0) {
        const deto_rows none = {};
        a.x = *x_out;
        a.dx = *dx;
        a.f = branch ? *f : none;
        a.df = branch ? *df : none;
        a.dy = pre ? *dy : none;
        a.dxo = here(dx_out) ? *dx_out : none;
        by_width(D, [&](auto w, auto c) {
            using TM = Team<w.value, c.value>;
            const unsigned grid = static_cast<unsigned>((a.deal.teams + TM::kTeamsWg - 1) / TM::kTeamsWg);
            by_types(a.x.dtype, branch ? a.f.dtype : a.dy.dtype, [&](auto xt, auto ft) {
                norm_backward_kernel<xt.value, ft.value, w.value, c.value>
                    <<<grid, TM::kThreadsWg, 0, st>>>(a);
                return 0;
            });
        });
    }
    if (a.slots) {
        j.parts = a.parts;
        j.D = a.D;
        j.slots = a.slots;
        j.teams = a.deal.teams;
        j.gate_teams = a.deal.cuts;
        // without rows: one gate row without rows_per_gate, none with it
        const int64_t gates = a.slot[kGate] < 0 ? 0 : T ? a.deal.gates : cfg->rows_per_gate ? 0 : 1;
        const int64_t all = j.outs + gates;
        for (int64_t y0 = 0; y0 < all; y0 += 65535) {
            const unsigned rows = static_cast<unsigned>(all - y0 < 65535 ? all - y0 : 65535);
            norm_join_kernel<<<dim3(static_cast<unsigned>((D + kLanes - 1) / kLanes), rows), 256, 0, st>>>(
                j, y0);
        }
    }
    return enqueued();
}

}  // extern "C"
