// Gated residual with the norms on both sides of a block, and its backward pass:
//     v = post ? n(u; post_weight, post_bias) : u
//     h = rho x + sigma g . v                       stored in the stream's type
//     y = n(h; pre_weight, pre_bias)                of the stored h; in the branch's type, or as MXFP4 codes
// with n(a; w, b) = a r w, r = (mean a^2 + eps)^-1/2 (RMS), or (a - mu) r w + b, r = (var a + eps)^-1/2 (layer).
// Backward, with a^ the normalised input (a - mu) r:
//     b = dy pre_weight;        dh = dh_out + r_h (b - [mean b] - h^ mean(b h^));     dx = rho dh
//     dv = sigma g . dh;        c = dv post_weight;     du = r_u (c - [mean c] - u^ mean(c u^))
//     d_pre_weight = sum dy h^, d_pre_bias = sum dy, d_post_weight = sum dv u^, d_post_bias = sum dv,
//     d_gate = sum sigma dh . v        ([...]: layer only; the sums run over rows, for the gate over its rows)
//
// Both passes are bound by memory (8 to 12 bytes an element in bf16 against 40 to 60 vector instructions for eight of
// them), so a row is read once: a team of lanes holds it in registers, eight elements a lane, through both norms.
#include "mx_block.hpp"

#include <algorithm>

namespace mxl {

using namespace mxb;

namespace {

struct NormArgs {
    const void* x;
    const void* u;
    void* h;
    void* y;
    const void* pre_weight;
    const void* pre_bias;
    const void* post_weight;
    const void* post_bias;
    const void* gate;
    uint8_t* y_codes;
    uint8_t* y_scales;
    uint8_t* h8;
    uint8_t* h8_scales;
    uint8_t* u8;
    uint8_t* u8_scales;
    float4* stats;
    int64_t rows, ldx, ldu, ldh, ldy, ld_gate, gate_run;      // gate_run: rows of the stream that share a gate row
    uint32_t cols, pitch8, lanes;
    float inv_cols, rho, sigma, eps;
    bool branch, pre, post, param_bf16, gate_bf16, gate_by_row, floor_mode;
};

struct NormGradArgs {
    NormArgs f;
    const void* dh;
    const void* dy;
    void* dx;
    void* du;
    int64_t lddh, lddy, lddx, lddu;
    float* partials;          // [SUMS][parts][cols], the sums of each workgroup
    float* gate_partials;     // [gate rows x pieces][cols]
    void* dgate;              // where whole gate rows belong to one team
    int64_t gate_rows, pieces, teams, team_rows;
    bool want_gate;
};

enum { PRE_WEIGHT, POST_WEIGHT, GATE, PRE_BIAS, POST_BIAS, SUMS };

// The eight elements from `col` on: how many the row has (not positive: none).
__device__ __forceinline__ int left(uint32_t cols, uint32_t col) { return (int)cols - (int)col; }

__device__ __forceinline__ uint32_t codes4(const F8& f, bool floor_mode, uint32_t& byte)
{
    byte = mxd::scale_byte(mxd::quad_max(mxd::amax_bits8(f)), floor_mode);
    return mxd::rtn_codes8_f32(f.v, byte);
}

// Mean (0 for RMS) and reciprocal deviation of the team's row; columns past the row's end hold zeros.
template <bool LAYER, int V, typename R>
__device__ __forceinline__ float2 statistics(const R (&a)[V], Team& team, const NormArgs& g, uint32_t col0, uint32_t step)
{
    float mean = 0.0f;
    if (LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const F8 f = widen(a[v]);
#pragma unroll
            for (int t = 0; t < 8; ++t) s[0] += f.v[t];
        }
        team.sum(s);
        mean = s[0] * g.inv_cols;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int n = left(g.cols, col0 + v * step);
        const F8 f = widen(a[v]);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const float d = LAYER ? (t < n ? f.v[t] - mean : 0.0f) : f.v[t];
            q[0] = __builtin_fmaf(d, d, q[0]);
        }
    }
    team.sum(q);
    return make_float2(mean, __builtin_amdgcn_rsqf(__builtin_fmaf(q[0], g.inv_cols, g.eps)));
}

// The 8-bit checkpoint of the lane's eight elements at `col` of a row.
__device__ __forceinline__ void keep8(uint8_t* codes, uint8_t* scales, const F8& f, int64_t row, uint32_t pitch8, uint32_t col, bool live)
{
    uint32_t byte;
    const Codes8 c = pack8(f, byte);
    if (live && col < pitch8) {
        *reinterpret_cast<uint2*>(codes + row * pitch8 + col) = make_uint2(c.w[0], c.w[1]);
        if ((col & 31u) == 0) scales[row * (pitch8 >> 5) + (col >> 5)] = (uint8_t)byte;
    }
}

// Forward pass.  A team walks over rows and has the next row's loads in flight while it works on one.  With one vector a
// lane (V = 1) it also keeps the parameters, else these are read again for every row.
template <typename XT, typename UT, int V, bool LAYER, bool TAIL>
__global__ __launch_bounds__(1024) void residual_norm_fwd_kernel(const NormArgs g)
{
    __shared__ TeamScratch scratch;
    const uint32_t team_in_block = threadIdx.x / g.lanes, lane = threadIdx.x % g.lanes;
    const uint32_t teams = blockDim.x / g.lanes;
    Team team{g.lanes, team_in_block * (g.lanes >> 6), &scratch};
    const uint32_t step = g.lanes * 8u, col0 = lane * 8u;

    auto param = [&](const void* p, int v, float none) {
        const uint32_t col = col0 + v * step;
        return param8<TAIL>(p, g.param_bf16, col, left(g.cols, col), none);
    };
    const int64_t stride = (int64_t)gridDim.x * teams;
    // the gate's row of the row fetched next, and the place in its run: carried along, a division for each row costs more
    int64_t row = (int64_t)blockIdx.x * teams + team_in_block;
    int64_t gate_row = row / g.gate_run, in_run = row % g.gate_run;
    const int64_t gate_step = stride / g.gate_run, run_step = stride % g.gate_run;
    Raw<XT> xn[V];
    Raw<UT> un[V];
    F8 gn[V];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t col = col0 + v * step;
            const int n = row < g.rows ? left(g.cols, col) : 0;
            xn[v] = load_raw<TAIL>(static_cast<const XT*>(g.x) + row * g.ldx + col, n);
            if (g.branch) un[v] = load_raw<TAIL>(static_cast<const UT*>(g.u) + row * g.ldu + col, n);
            if (g.gate_by_row) gn[v] = param8<TAIL>(g.gate, g.gate_bf16, gate_row * g.ld_gate + col, n, 0.0f);
        }
        gate_row += gate_step;
        in_run += run_step;
        if (in_run >= g.gate_run) { in_run -= g.gate_run; ++gate_row; }
    };
    fetch(row);
    F8 pre_w, pre_b, post_w, post_b, gate;
    if (V == 1) {
        if (g.pre) pre_w = param(g.pre_weight, 0, 1.0f);
        if (LAYER && g.pre) pre_b = param(g.pre_bias, 0, 0.0f);
        if (g.post) post_w = param(g.post_weight, 0, 1.0f);
        if (LAYER && g.post) post_b = param(g.post_bias, 0, 0.0f);
        if (g.gate && !g.gate_by_row) gate = param8<TAIL>(g.gate, g.gate_bf16, col0, left(g.cols, col0), 0.0f);
    }

    // the workgroup's teams go through the loop together (its sums hold barriers)
    for (int64_t first = (int64_t)blockIdx.x * teams; first < g.rows; first += stride, row += stride) {
        Raw<XT> h[V];
        Raw<UT> u[V];
        F8 gr[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            h[v] = xn[v];
            if (g.branch) u[v] = un[v];
            if (g.gate_by_row) gr[v] = gn[v];
        }
        fetch(row + stride);
        const bool live = row < g.rows;
        float2 su = make_float2(0.0f, 0.0f), sh = make_float2(0.0f, 0.0f);
        if (g.branch) {
            if (g.post) su = statistics<LAYER>(u, team, g, col0, step);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t col = col0 + v * step;
                const int n = live ? left(g.cols, col) : 0;
                F8 b = widen(u[v]);
                if (g.u8 != nullptr) keep8(g.u8, g.u8_scales, b, row, g.pitch8, col, live);
                if (g.post) {
                    if (V > 1) post_w = param(g.post_weight, v, 1.0f);
                    if (V > 1 && LAYER) post_b = param(g.post_bias, v, 0.0f);
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        b.v[t] = (b.v[t] - su.x) * su.y * post_w.v[t];
                        if (LAYER) b.v[t] += post_b.v[t];
                    }
                }
                if (g.gate) {
                    if (g.gate_by_row) gate = gr[v];
                    else if (V > 1)    gate = param8<TAIL>(g.gate, g.gate_bf16, col, left(g.cols, col), 0.0f);
#pragma unroll
                    for (int t = 0; t < 8; ++t) b.v[t] *= gate.v[t];
                }
                const F8 x = widen(h[v]);
#pragma unroll
                for (int t = 0; t < 8; ++t) b.v[t] = __builtin_fmaf(g.sigma, b.v[t], g.rho * x.v[t]);
                narrow(b, h[v]);
                store_raw<TAIL>(static_cast<XT*>(g.h) + row * g.ldh + col, h[v], n);
            }
        }
        if (g.h8 != nullptr) {
#pragma unroll
            for (int v = 0; v < V; ++v) keep8(g.h8, g.h8_scales, widen(h[v]), row, g.pitch8, col0 + v * step, live);
        }
        if (g.pre) {
            sh = statistics<LAYER>(h, team, g, col0, step);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t col = col0 + v * step;
                const int n = live ? left(g.cols, col) : 0;
                if (V > 1) pre_w = param(g.pre_weight, v, 1.0f);
                if (V > 1 && LAYER) pre_b = param(g.pre_bias, v, 0.0f);
                F8 y = widen(h[v]);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    y.v[t] = (y.v[t] - sh.x) * sh.y * pre_w.v[t];
                    if (LAYER) y.v[t] += pre_b.v[t];
                }
                if (g.y_codes != nullptr) {
                    uint32_t byte;
                    const uint32_t c = codes4(y, g.floor_mode, byte);
                    if (n > 0) {
                        *reinterpret_cast<uint32_t*>(g.y_codes + row * (g.cols >> 1) + (col >> 1)) = c;
                        if ((lane & 3u) == 0) g.y_scales[row * (g.cols >> 5) + (col >> 5)] = (uint8_t)byte;
                    }
                } else {
                    store8<TAIL>(static_cast<UT*>(g.y) + row * g.ldy + col, y, n);
                }
            }
        }
        if (g.stats != nullptr && live && lane == 0) g.stats[row] = make_float4(su.x, su.y, sh.x, sh.y);
    }
}

// What a row's backward pass reads of h or u: the values as stored, or their 8-bit codes.
template <typename T, bool CKPT> struct Kept { Raw<T> raw; };
template <typename T> struct Kept<T, true> { Codes8 codes; uint32_t byte; };

template <bool TAIL, typename T, bool CKPT>
__device__ __forceinline__ void fetch_kept(Kept<T, CKPT>& k, const void* p, const uint8_t* codes, const uint8_t* scales, int64_t row, int64_t ld,
                                           uint32_t pitch8, uint32_t col, int n)
{
    if constexpr (CKPT) {
        k.codes.w[0] = k.codes.w[1] = k.byte = 0;
        if (n > 0) {
            const uint2 c = *reinterpret_cast<const uint2*>(codes + row * pitch8 + col);
            k.codes.w[0] = c.x; k.codes.w[1] = c.y;
            k.byte = scales[row * (pitch8 >> 5) + (col >> 5)];
        }
    } else {
        k.raw = load_raw<TAIL>(static_cast<const T*>(p) + row * ld + col, n);
    }
}
template <typename T> __device__ __forceinline__ F8 value_of(const Kept<T, true>& k) { return unpack8(k.codes, k.byte); }
template <typename T> __device__ __forceinline__ F8 value_of(const Kept<T, false>& k) { return widen(k.raw); }

// Backward pass.  A team owns a run of rows and adds its part of the parameters' gradients in registers, row by row; the
// teams of a workgroup are added in order at the end, and a second kernel adds the workgroups.  Gate rows: either a team's
// run is one of `pieces` parts of one gate row, or it is a number of whole ones and the team writes them out itself.
//
// Up to nine FP32 vectors of the row's length would live in registers: the sums do, the parameters are read from LDS
// (from cache where a row is too long for that, WIDE), and what a row needs again behind its sums is kept as loaded.
template <typename XT, typename UT, int V, bool WIDE, bool LAYER, bool CKPT, bool TAIL>
__global__ __launch_bounds__(WIDE ? 1024 : 512) void residual_norm_bwd_kernel(const NormGradArgs a)
{
    extern __shared__ float lds[];               // the parameters' vectors; at the end [teams][lanes * 8 * V] for the sums
    __shared__ TeamScratch scratch;
    const NormArgs& g = a.f;
    const uint32_t team_in_block = threadIdx.x / g.lanes, lane = threadIdx.x % g.lanes;
    const uint32_t teams = blockDim.x / g.lanes;
    Team team{g.lanes, team_in_block * (g.lanes >> 6), &scratch};
    const uint32_t step = g.lanes * 8u, col0 = lane * 8u, width = step * V;
    const bool read_u = g.branch && (g.post || a.want_gate);

    const int64_t k = (int64_t)blockIdx.x * teams + team_in_block;
    int64_t begin = 0, end = 0;                                          // the team's rows
    const bool whole = a.pieces == 0;
    if (k < a.teams) {
        if (whole) {
            begin = a.gate_rows * k / a.teams * g.gate_run;
            end = a.gate_rows * (k + 1) / a.teams * g.gate_run;
        } else {
            const int64_t group = k / a.pieces, piece = k % a.pieces;
            begin = group * g.gate_run + g.gate_run * piece / a.pieces;
            end = group * g.gate_run + g.gate_run * (piece + 1) / a.pieces;
        }
    }

    enum { W_PRE, W_POST, W_GATE, B_POST };
    auto from_memory = [&](int which, uint32_t col) {
        const int n = left(g.cols, col);
        if (which == W_PRE)  return param8<TAIL>(g.pre_weight, g.param_bf16, col, n, 1.0f);
        if (which == W_POST) return param8<TAIL>(g.post_weight, g.param_bf16, col, n, 1.0f);
        if (which == W_GATE) return param8<TAIL>(g.gate, g.gate_bf16, col, n, 0.0f);
        return param8<TAIL>(g.post_bias, g.param_bf16, col, n, 0.0f);
    };
    if (!WIDE) {
        for (uint32_t c = threadIdx.x * 8u; c < width; c += blockDim.x * 8u) {
            store_raw<false>(lds + c, from_memory(W_PRE, c), 8);
            if (g.post) store_raw<false>(lds + W_POST * width + c, from_memory(W_POST, c), 8);
            if (g.gate && !g.gate_by_row) store_raw<false>(lds + W_GATE * width + c, from_memory(W_GATE, c), 8);
            if (LAYER && g.post) store_raw<false>(lds + B_POST * width + c, from_memory(B_POST, c), 8);
        }
        __syncthreads();
    }
    auto param = [&](int which, int v) {
        const uint32_t col = col0 + v * step;
        if (WIDE) return from_memory(which, col);
        F8 f;
        const float4* p = reinterpret_cast<const float4*>(lds + which * width + col);
        const float4 lo = p[0], hi = p[1];
        f.v[0] = lo.x; f.v[1] = lo.y; f.v[2] = lo.z; f.v[3] = lo.w;
        f.v[4] = hi.x; f.v[5] = hi.y; f.v[6] = hi.z; f.v[7] = hi.w;
        return f;
    };

    F8 acc[SUMS][V];
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
#pragma unroll
        for (int v = 0; v < V; ++v) acc[s][v] = mxd::zero8();

    struct Row {
        Raw<UT> dy[V];
        Raw<XT> dh[V];
        Kept<XT, CKPT> h[V];
        Kept<UT, CKPT> u[V];
        float4 stats;
    };
    auto fetch = [&](Row& r, int64_t row) {
        const bool live = row < end;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t col = col0 + v * step;
            const int n = live ? left(g.cols, col) : 0;
            if (a.dy != nullptr) {
                r.dy[v] = load_raw<TAIL>(static_cast<const UT*>(a.dy) + row * a.lddy + col, n);
                fetch_kept<TAIL, XT, CKPT>(r.h[v], g.h, g.h8, g.h8_scales, row, g.ldh, g.pitch8, col, n);
            }
            if (a.dh != nullptr) r.dh[v] = load_raw<TAIL>(static_cast<const XT*>(a.dh) + row * a.lddh + col, n);
            if (read_u) fetch_kept<TAIL, UT, CKPT>(r.u[v], g.u, g.u8, g.u8_scales, row, g.ldu, g.pitch8, col, n);
        }
        r.stats = live ? g.stats[row] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    };
    int64_t gate_row = g.gate_by_row && begin < end ? begin / g.gate_run : 0, in_run = 0;
    if (!whole) in_run = begin - gate_row * g.gate_run;
    Row next;
    if (!WIDE) fetch(next, begin);
    for (int64_t i = 0; i < a.team_rows; ++i) {
        const int64_t row = begin + i;
        const bool live = row < end;
        Row r;
        if (WIDE) {
            fetch(r, row);
        } else {
            r = next;
            fetch(next, row + 1);
        }
        F8 gate_by_row[V];
        if (g.gate_by_row) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t col = col0 + v * step;
                gate_by_row[v] = param8<TAIL>(g.gate, g.gate_bf16, gate_row * g.ld_gate + col, live ? left(g.cols, col) : 0, 0.0f);
            }
        }
        const float4 st = r.stats;
        float m0 = 0.0f, m1 = 0.0f;
        if (a.dy != nullptr) {
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const F8 dy = widen(r.dy[v]), h = value_of<XT>(r.h[v]), w = param(W_PRE, v);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float n = (h.v[t] - st.z) * st.w, b = dy.v[t] * w.v[t];
                    acc[PRE_WEIGHT][v].v[t] = __builtin_fmaf(dy.v[t], n, acc[PRE_WEIGHT][v].v[t]);
                    if (LAYER) acc[PRE_BIAS][v].v[t] += dy.v[t];
                    s[0] = __builtin_fmaf(b, n, s[0]);
                    if (LAYER) s[1] += b;
                }
            }
            team.sum(s);
            m1 = s[0] * g.inv_cols;
            m0 = s[1] * g.inv_cols;
        }
        F8 dv[V];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t col = col0 + v * step;
            const int n = live ? left(g.cols, col) : 0;
            F8 dh = a.dh != nullptr ? widen(r.dh[v]) : mxd::zero8();
            if (a.dy != nullptr) {
                const F8 dy = widen(r.dy[v]), h = value_of<XT>(r.h[v]), w = param(W_PRE, v);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float hn = (h.v[t] - st.z) * st.w;
                    dh.v[t] = __builtin_fmaf(st.w, __builtin_fmaf(-hn, m1, dy.v[t] * w.v[t] - m0), dh.v[t]);
                }
            }
            if (a.dx != nullptr) {
                F8 dx;
#pragma unroll
                for (int t = 0; t < 8; ++t) dx.v[t] = g.rho * dh.v[t];
                store8<TAIL>(static_cast<XT*>(a.dx) + row * a.lddx + col, dx, n);
            }
            if (!g.branch) continue;
#pragma unroll
            for (int t = 0; t < 8; ++t) dv[v].v[t] = g.sigma * dh.v[t];
            F8 un = read_u ? value_of<UT>(r.u[v]) : mxd::zero8(), w, b;
            if (g.post) {
                w = param(W_POST, v);
                if (LAYER) b = param(B_POST, v);
#pragma unroll
                for (int t = 0; t < 8; ++t) un.v[t] = (un.v[t] - st.x) * st.y;
            }
            if (g.gate) {
                const F8 gate = g.gate_by_row ? gate_by_row[v] : param(W_GATE, v);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    float value = un.v[t];
                    if (g.post) {
                        value *= w.v[t];
                        if (LAYER) value += b.v[t];
                    }
                    acc[GATE][v].v[t] = __builtin_fmaf(dv[v].v[t], value, acc[GATE][v].v[t]);
                    dv[v].v[t] *= gate.v[t];
                }
            }
            if (g.post) {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    acc[POST_WEIGHT][v].v[t] = __builtin_fmaf(dv[v].v[t], un.v[t], acc[POST_WEIGHT][v].v[t]);
                    if (LAYER) acc[POST_BIAS][v].v[t] += dv[v].v[t];
                    dv[v].v[t] *= w.v[t];
                    s[0] = __builtin_fmaf(dv[v].v[t], un.v[t], s[0]);
                    if (LAYER) s[1] += dv[v].v[t];
                }
            }
        }
        if (g.branch) {
            if (g.post) {
                team.sum(s);
                m1 = s[0] * g.inv_cols;
                m0 = s[1] * g.inv_cols;
            }
            if (a.du != nullptr) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const uint32_t col = col0 + v * step;
                    if (g.post) {
                        const F8 u = value_of<UT>(r.u[v]);
#pragma unroll
                        for (int t = 0; t < 8; ++t) {
                            const float un = (u.v[t] - st.x) * st.y;
                            dv[v].v[t] = st.y * __builtin_fmaf(-un, m1, dv[v].v[t] - m0);
                        }
                    }
                    store8<TAIL>(static_cast<UT*>(a.du) + row * a.lddu + col, dv[v], live ? left(g.cols, col) : 0);
                }
            }
        }
        if (g.gate_by_row && ++in_run == g.gate_run) {                   // the gate's row is complete
            if (whole && a.want_gate) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const uint32_t col = col0 + v * step;
                    const int n = live ? left(g.cols, col) : 0;
                    const int64_t at = gate_row * g.cols + col;
                    if (g.gate_bf16) store8<TAIL>(static_cast<uint16_t*>(a.dgate) + at, acc[GATE][v], n);
                    else             store8<TAIL>(static_cast<float*>(a.dgate) + at, acc[GATE][v], n);
                    acc[GATE][v] = mxd::zero8();
                }
            }
            in_run = 0;
            ++gate_row;
        }
    }

#pragma unroll
    for (int s = 0; s < SUMS; ++s) {
        if (!LAYER && s >= PRE_BIAS) continue;
        if ((s == PRE_WEIGHT || s == PRE_BIAS) && a.dy == nullptr) continue;
        if ((s == POST_WEIGHT || s == POST_BIAS) && !g.post) continue;
        float* out = a.partials + ((int64_t)s * gridDim.x + blockIdx.x) * g.cols;
        if (s == GATE) {
            if (!a.want_gate || whole) continue;
            if (a.gate_rows > 1) {                                       // one row of sums for each team
                if (k < a.teams) {
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        store8<TAIL>(a.gate_partials + k * g.cols + col0 + v * step, acc[s][v], left(g.cols, col0 + v * step));
                }
                continue;
            }
            out = a.gate_partials + (int64_t)blockIdx.x * g.cols;
        }
        if (teams == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) store8<TAIL>(out + col0 + v * step, acc[s][v], left(g.cols, col0 + v * step));
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) store_raw<false>(lds + team_in_block * width + col0 + v * step, acc[s][v], 8);
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < g.cols; c += blockDim.x) {
            float t = lds[c];
            for (uint32_t i = 1; i < teams; ++i) t += lds[i * width + c];
            out[c] = t;
        }
    }
}

struct NormFinishArgs {
    const float* partials;
    const float* gate_partials;
    void* out[SUMS];
    uint32_t parts, gate_parts, cols;
    bool param_bf16, gate_bf16;
};

// Adds the workgroups' sums up: 32 columns a workgroup, its eight parts of 32 lanes each take a run of the partial rows in
// order, and the runs are added in order.
__global__ __launch_bounds__(256) void residual_norm_finish_kernel(const NormFinishArgs a)
{
    __shared__ float part[8][32];
    const uint32_t lc = threadIdx.x & 31u, p = threadIdx.x >> 5, blocks = (a.cols + 31u) / 32u;
    // the sums in order: first the four parameters (those wanted), then the gate's rows
    const uint32_t y = blockIdx.x / blocks, c = blockIdx.x % blocks * 32u + lc;
    const bool is_gate = y >= SUMS - 1;
    const uint32_t s = is_gate ? GATE : y >= GATE ? y + 1 : y;
    if (a.out[s] == nullptr) return;
    const uint32_t parts = is_gate ? a.gate_parts : a.parts;
    const float* from = is_gate ? a.gate_partials + (int64_t)(y - (SUMS - 1)) * parts * a.cols : a.partials + (int64_t)s * parts * a.cols;
    const uint32_t per = (parts + 7u) / 8u, b0 = min(parts, p * per), b1 = min(parts, b0 + per);
    float t = 0.0f;
    if (c < a.cols) {
        const float* q = from + (int64_t)b0 * a.cols + c;
        uint32_t b = b0;
        for (; b + 8u <= b1; b += 8u, q += (int64_t)8 * a.cols) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = q[(int64_t)i * a.cols];
#pragma unroll
            for (int i = 0; i < 8; ++i) t += v[i];
        }
        for (; b < b1; ++b, q += a.cols) t += *q;
    }
    part[p][lc] = t;
    __syncthreads();
    if (p == 0 && c < a.cols) {
        float sum = part[0][lc];
#pragma unroll
        for (int i = 1; i < 8; ++i) sum += part[i][lc];
        const int64_t at = (is_gate ? (int64_t)(y - (SUMS - 1)) * a.cols : 0) + c;
        if (is_gate ? a.gate_bf16 : a.param_bf16) static_cast<__bf16*>(a.out[s])[at] = (__bf16)sum;
        else                                      static_cast<float*>(a.out[s])[at] = sum;
    }
}

uint32_t lanes_for(int64_t vectors)
{
    for (uint32_t l = 8; l < 64; l *= 2)
        if (vectors <= l) return l;
    return (uint32_t)((vectors + 63) / 64 * 64);
}

// Teams of a workgroup, raised to whole waves.
uint32_t whole_waves(uint32_t teams, uint32_t lanes)
{
    const uint32_t per = lanes < 64 ? 64 / lanes : 1;
    return (teams + per - 1) / per * per;
}

NormArgs args_of(const ResidualNormParams& p, int v)
{
    NormArgs g{};
    g.x = p.x; g.u = p.u; g.h = p.h; g.y = p.y;
    g.pre_weight = p.pre_weight; g.pre_bias = p.pre_bias; g.post_weight = p.post_weight; g.post_bias = p.post_bias; g.gate = p.gate;
    g.y_codes = p.y_codes; g.y_scales = p.y_scales;
    g.h8 = p.h8; g.h8_scales = p.h8_scales; g.u8 = p.u8; g.u8_scales = p.u8_scales;
    g.stats = reinterpret_cast<float4*>(p.stats);
    g.rows = p.rows; g.ldx = p.ldx; g.ldu = p.ldu; g.ldh = p.ldh; g.ldy = p.ldy; g.ld_gate = p.ld_gate;
    g.gate_run = p.gate && p.gate_rows > 0 ? p.rows / p.gate_rows : p.rows;
    g.gate_by_row = p.gate != nullptr && p.gate_rows > 1;
    g.cols = (uint32_t)p.cols; g.pitch8 = (uint32_t)((p.cols + 31) / 32 * 32);
    g.lanes = lanes_for(((p.cols + 7) / 8 + v - 1) / v);
    g.inv_cols = (float)(1.0 / (double)p.cols);
    g.rho = p.residual_scale; g.sigma = p.branch_scale; g.eps = p.eps;
    g.branch = p.branch; g.pre = p.pre; g.post = p.post; g.param_bf16 = p.param_bf16; g.gate_bf16 = p.gate_bf16; g.floor_mode = p.floor_mode;
    return g;
}

// Calls f with the element types of the stream and the branch.
template <typename F>
void by_types(bool x_bf16, bool u_bf16, F&& f)
{
    if (x_bf16) f(uint16_t{}, uint16_t{});
    else if (u_bf16) f(float{}, uint16_t{});
    else f(float{}, float{});
}

// Calls f with three truth values as types.
template <typename F>
void by_flags(bool a, bool b, bool c, F&& f)
{
    using Y = std::true_type;
    using N = std::false_type;
    if (a) b ? (c ? f(Y{}, Y{}, Y{}) : f(Y{}, Y{}, N{})) : (c ? f(Y{}, N{}, Y{}) : f(Y{}, N{}, N{}));
    else   b ? (c ? f(N{}, Y{}, Y{}) : f(N{}, Y{}, N{})) : (c ? f(N{}, N{}, Y{}) : f(N{}, N{}, N{}));
}

constexpr uint32_t UNITS = 256;                          // compute units

template <typename XT, typename UT, int V>
void launch_fwd(const ResidualNormParams& p, hipStream_t st)
{
    const NormArgs g = args_of(p, V);
    const uint32_t most = g.lanes >= 256 ? 1 : 256 / g.lanes;
    const uint32_t teams = whole_waves((uint32_t)std::min<int64_t>(most, std::max<int64_t>(1, (p.rows + UNITS - 1) / UNITS)), g.lanes);
    const uint32_t threads = teams * g.lanes;
    const int64_t blocks = (p.rows + teams - 1) / teams;
    const uint32_t grid = (uint32_t)std::min<int64_t>(blocks, UNITS * std::max(1u, 1024 / threads));
    auto run = [&](auto kernel) { kernel<<<grid, threads, 0, st>>>(g); };
    const bool tail = p.cols % 8 != 0;
    if (p.layer) tail ? run(residual_norm_fwd_kernel<XT, UT, V, true, true>) : run(residual_norm_fwd_kernel<XT, UT, V, true, false>);
    else         tail ? run(residual_norm_fwd_kernel<XT, UT, V, false, true>) : run(residual_norm_fwd_kernel<XT, UT, V, false, false>);
}

// Shape of a backward launch, the same for every type.
struct BwdPlan {
    int v;
    bool wide;
    uint32_t lanes, teams_per_block, grid;
    int64_t teams, pieces, team_rows;        // pieces 0: teams own whole gate rows
};

BwdPlan plan_bwd(int64_t rows, int64_t cols, int64_t gate_rows)
{
    BwdPlan b{};
    const int64_t vectors = (cols + 7) / 8;
    b.v = vectors <= 512 ? 1 : 2;
    b.wide = vectors > 1024;
    b.lanes = lanes_for((vectors + b.v - 1) / b.v);
    const uint32_t most = std::max(1u, 512 / b.lanes), grid = 2 * UNITS;
    b.teams_per_block = (uint32_t)std::min<int64_t>(most, std::max<int64_t>(1, (rows + grid - 1) / grid));
    b.teams_per_block = whole_waves(b.teams_per_block, b.lanes);
    const int64_t teams = std::min<int64_t>(rows, (int64_t)grid * b.teams_per_block), run = rows / gate_rows;
    if (gate_rows == 1 || 2 * gate_rows <= teams) {
        b.pieces = std::min(run, teams / gate_rows);
        b.teams = gate_rows * b.pieces;
        b.team_rows = (run + b.pieces - 1) / b.pieces;
    } else {
        b.teams = gate_rows <= 2 * teams ? gate_rows : teams;
        b.team_rows = (gate_rows + b.teams - 1) / b.teams * run;
    }
    b.grid = (uint32_t)((b.teams + b.teams_per_block - 1) / b.teams_per_block);
    return b;
}

template <typename XT, typename UT, int V, bool WIDE>
hipError_t launch_bwd(const NormGradArgs& a, const BwdPlan& b, bool layer, bool ckpt, hipStream_t st)
{
    const uint32_t threads = b.teams_per_block * b.lanes, width = b.lanes * 8 * V;
    const uint32_t vectors = WIDE ? 0 : layer && a.f.post ? 4 : a.f.gate ? 3 : a.f.post ? 2 : 1;
    const size_t lds = std::max((size_t)vectors * width, b.teams_per_block > 1 ? (size_t)b.teams_per_block * width : 0) * sizeof(float);
    hipError_t e = hipSuccess;
    by_flags(layer, ckpt, a.f.cols % 8 != 0, [&](auto l, auto c, auto t) {
        auto kernel = residual_norm_bwd_kernel<XT, UT, V, WIDE, decltype(l)::value, decltype(c)::value, decltype(t)::value>;
        // beyond what a kernel may have without being asked; rows of up to 8192 values need 128 KB of the unit's 160
        if (lds > 65536 - sizeof(TeamScratch))
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e == hipSuccess) kernel<<<b.grid, threads, lds, st>>>(a);
    });
    return e;
}

}  // namespace

hipError_t launch_residual_norm_fwd(const ResidualNormParams& p, hipStream_t st)
{
    by_types(p.x_bf16, p.u_bf16, [&](auto xt, auto ut) {
        if (p.cols <= 8192) launch_fwd<decltype(xt), decltype(ut), 1>(p, st);
        else                launch_fwd<decltype(xt), decltype(ut), 2>(p, st);
    });
    return hipGetLastError();
}

size_t residual_norm_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_rows)
{
    const BwdPlan b = plan_bwd(rows, cols, std::max<int64_t>(1, gate_rows));
    const int64_t gate = gate_rows > 1 ? (b.pieces > 0 ? b.teams : 0) : b.grid;
    return ((size_t)SUMS * b.grid + (size_t)gate) * (size_t)cols * sizeof(float);
}

hipError_t launch_residual_norm_bwd(const ResidualNormParams& p, const ResidualNormGrads& d, hipStream_t st)
{
    const int64_t gate_rows = p.gate != nullptr ? p.gate_rows : 1;
    const BwdPlan b = plan_bwd(p.rows, p.cols, gate_rows);
    NormGradArgs a{};
    a.f = args_of(p, b.v);
    a.dh = d.dh; a.dy = d.dy; a.dx = d.dx; a.du = d.du;
    a.lddh = d.lddh; a.lddy = d.lddy; a.lddx = d.lddx; a.lddu = d.lddu;
    a.partials = static_cast<float*>(d.workspace);
    a.gate_partials = a.partials + (int64_t)SUMS * b.grid * p.cols;
    a.dgate = d.dgate;
    a.gate_rows = gate_rows; a.pieces = b.pieces; a.teams = b.teams; a.team_rows = b.team_rows;
    a.want_gate = p.gate != nullptr && d.dgate != nullptr;
    hipError_t e = hipSuccess;
    by_types(p.x_bf16, p.u_bf16, [&](auto xt, auto ut) {
        using XT = decltype(xt);
        using UT = decltype(ut);
        const bool ckpt = p.h8 != nullptr || p.u8 != nullptr;
        if (b.v == 1)     e = launch_bwd<XT, UT, 1, false>(a, b, p.layer, ckpt, st);
        else if (!b.wide) e = launch_bwd<XT, UT, 2, false>(a, b, p.layer, ckpt, st);
        else              e = launch_bwd<XT, UT, 2, true>(a, b, p.layer, ckpt, st);
    });
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess) return e;
    NormFinishArgs f{};
    f.partials = a.partials; f.gate_partials = a.gate_partials;
    f.parts = b.grid; f.gate_parts = gate_rows > 1 ? (uint32_t)b.pieces : b.grid; f.cols = (uint32_t)p.cols;
    f.param_bf16 = p.param_bf16; f.gate_bf16 = p.gate_bf16;
    f.out[PRE_WEIGHT] = d.dy ? d.dpre_weight : nullptr; f.out[PRE_BIAS] = d.dy && p.layer ? d.dpre_bias : nullptr;
    f.out[POST_WEIGHT] = p.post ? d.dpost_weight : nullptr; f.out[POST_BIAS] = p.post && p.layer ? d.dpost_bias : nullptr;
    f.out[GATE] = a.want_gate && b.pieces > 0 ? d.dgate : nullptr;
    const uint32_t gates = f.out[GATE] ? (uint32_t)gate_rows : 0;
    bool any = gates > 0;
    for (void* o : f.out) any = any || o != nullptr;
    if (!any) return hipSuccess;
    residual_norm_finish_kernel<<<(uint32_t)((p.cols + 31) / 32) * (SUMS - 1 + gates), 256, 0, st>>>(f);
    return hipGetLastError();
}

}  // namespace mxl
