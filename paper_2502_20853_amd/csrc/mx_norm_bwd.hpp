// Backward pass of the gated residual with norms (see mx_norm.hpp), compiled once for each kind of norm.
#pragma once
#include "mx_norm.hpp"

namespace mxl {

// What a row's backward pass reads of h or u: the values as stored, or their 8-bit codes.
template <typename T, bool CKPT> struct Kept { Raw<T> raw; };
template <typename T> struct Kept<T, true> { Codes8 codes; uint32_t byte; };

template <RowEnd END, int V, typename T, bool CKPT>
__device__ __forceinline__ void load_kept(Kept<T, CKPT>& k, const void* p, int64_t ld, const uint8_t* codes, const uint8_t* scales, const Place& at, int v)
{
    if constexpr (CKPT) k.codes = load_codes8<V>(codes, scales, at, v, k.byte);
    else                k.raw = load_vec<END, V, T>(p, ld, at, v);
}
template <typename T> __device__ __forceinline__ F8 value_of(const Kept<T, true>& k) { return unpack8(k.codes, k.byte); }
template <typename T> __device__ __forceinline__ F8 value_of(const Kept<T, false>& k) { return widen(k.raw); }
template <typename T> __device__ __forceinline__ void settle(Kept<T, true>&, uint32_t) {}         // codes lie in whole vectors
template <typename T> __device__ __forceinline__ void settle(Kept<T, false>& k, uint32_t back) { settle(k.raw, back); }
template <typename T> __device__ __forceinline__ void renew(Kept<T, true>& k) { renew(k.codes); }
template <typename T> __device__ __forceinline__ void renew(Kept<T, false>& k) { renew(k.raw); }

// How a team has its rows: the next row on its way while it works on one; a row in registers; or, where the sums leave no room
// for that, nothing but the sums: each of the three steps of a row loads it again, from cache then.
enum RowMode { ROW_AGAIN, ROW_HELD, ROW_AHEAD };

// By the registers that the sums, the raw row (twice) and the gradient that is passed on take, of the 256 a lane has.
// keep: also whether that gradient is kept between the second step and the third, or computed again.
// With four vectors a lane (BWD_ROWS) more registers are taken than counted here: 44 to 272 bytes of scratch a lane in whole rows
// with a post-norm, up to 892 in odd ones.
struct RowPlan {
    RowMode mode;
    bool keep;
};
template <typename XT, typename UT, int V, bool POST, bool GATE, bool LAYER, bool CKPT, bool TAIL, BwdPart PART>
constexpr RowPlan row_plan()
{
    constexpr int x = sizeof(XT) * 2, u = sizeof(UT) * 2;               // registers of eight values
    constexpr int sums = PART == BWD_ROWS ? 0 : (LAYER ? 2 : 1) * (POST ? 2 : 1) + GATE;
    constexpr int raw = u + x + (CKPT ? 3 : x) + (!POST && !GATE ? 0 : CKPT ? 3 : u);
    constexpr int fixed = V * 8 * sums + 76 + (TAIL ? 24 : 0), kept = POST ? V * 8 : 0;
    if (fixed + kept + 2 * V * raw <= 240) return {ROW_AHEAD, true};
    if (fixed + kept + V * raw <= 240) return {ROW_HELD, true};
    return {fixed + V * raw <= 240 ? ROW_HELD : ROW_AGAIN, false};
}

// Backward pass.  A team owns a run of rows and adds its part of the parameters' gradients in registers, row by row; the
// teams of a workgroup are added in order at the end, and a second kernel adds the workgroups.  Gate rows: either a team's
// run is one of `pieces` parts of one gate row, or it is a number of whole ones and the team writes them out itself.
//
// Up to nine FP32 vectors of the row's length would live in registers: the sums do, the parameters are read from LDS
// (with four vectors a lane from ParamPlanes, and from cache what has no plane there), and what a row needs again behind its
// sums is kept as loaded.  What is missing (a gradient, a weight) reads as zero or one, so that the loop has next to no branches.
template <typename XT, typename UT, int V, bool POST, bool GATE, bool LAYER, bool CKPT, RowEnd END, BwdPart PART>
__global__ __launch_bounds__(NORM_THREADS) void residual_norm_bwd_kernel(const NormGradArgs a)
{
    extern __shared__ float lds[];               // the parameters; at the end [teams][width] for the sums
    __shared__ TeamScratch scratch;
    const NormArgs& g = a.f;
    const uint32_t team_in_block = threadIdx.x / g.lanes, lane = threadIdx.x % g.lanes;
    const uint32_t teams = blockDim.x / g.lanes;
    Team team{g.lanes, team_in_block * (g.lanes >> 6), &scratch};
    const uint32_t step = g.lanes * 8u, width = step * V, vectors = g.lanes * V;
    const uint32_t base = PART == BWD_SUMS ? blockIdx.y * width : 0u, col0 = base + lane * 8u;           // of the strip
    constexpr bool READ_U = POST || GATE, TAIL = END != ROW_WHOLE;
    const bool post = POST && (!TAIL || g.post), gate_by_row = GATE && g.gate_by_row;

    // without gate rows every g.teams-th row, as in the forward pass
    const bool whole = GATE && a.pieces == 0, runs = PART != BWD_ROWS && GATE && g.row_step == 1;
    const TeamRows own(runs, team_in_block, teams, g.lanes);
    const int64_t k0 = own.k0, k = own.k;
    auto start_of = [&](int64_t k) {                                     // of a run
        if (whole) return a.gate_rows * k / g.teams * g.gate_run;
        const int64_t group = k / a.pieces, piece = k % a.pieces;
        return group * g.gate_run + g.gate_run * piece / a.pieces;
    };
    const int64_t first = runs ? start_of(k0) : k0, begin = k >= g.teams ? first : runs ? start_of(k) : k;
    const uint32_t count = k >= g.teams ? 0u : (uint32_t)(runs ? start_of(k + 1) - begin : (g.rows - k + g.teams - 1) / g.teams);

    using Params = ParamLds<POST, GATE, LAYER, true>;
    if constexpr (PART != BWD_ROWS) {
        auto fill = [&](NormParam which) {
            for (uint32_t c = threadIdx.x; c < vectors; c += blockDim.x) Params::put(lds, Params::STRIDE, which, c, norm_param<TAIL>(g, which, base + c * 8));
        };
        fill(P_PRE_WEIGHT);
        if (POST) fill(P_POST_WEIGHT);
        if (GATE && !gate_by_row) fill(P_GATE);
        if (POST && LAYER) fill(P_POST_BIAS);
        __syncthreads();
    } else {
        auto fill = [&](NormParam which) {
            if (g.plane[which] == ParamPlanes::NO_PLANE) return;
            for (uint32_t c = threadIdx.x; c < vectors; c += blockDim.x)
                ParamPlanes::put(lds, g.plane[which], vectors, c, param_is_bf16(g, which), norm_param<TAIL>(g, which, c * 8));
        };
        fill(P_PRE_WEIGHT);
        if (POST) fill(P_POST_WEIGHT);
        if (GATE) fill(P_GATE);
        __syncthreads();
    }

    F8 acc[SUMS][V];
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
#pragma unroll
        for (int v = 0; v < V; ++v) acc[s][v] = mxd::zero8();

    constexpr RowPlan PLAN = row_plan<XT, UT, V, POST, GATE, LAYER, CKPT, TAIL, PART>();
    constexpr RowMode MODE = PLAN.mode;
    struct Vec {                                                         // a lane's part of a row, as loaded
        Raw<UT> dy;
        Raw<XT> dh;
        Kept<XT, CKPT> h;
        Kept<UT, CKPT> u;
    };
    auto load = [&](Vec& r, const Place& at, int v, bool h, bool u) {
        if (h) {
            r.dy = load_vec<END, V, UT>(a.dy, a.lddy, at, v);
            load_kept<END, V, XT, CKPT>(r.h, g.h, g.ldh, g.h8, g.h8_scales, at, v);
        }
        if (u) {
            r.dh = load_vec<END, V, XT>(a.dh, a.lddh, at, v);
            if (READ_U) load_kept<END, V, UT, CKPT>(r.u, g.u, g.ldu, g.u8, g.u8_scales, at, v);
        }
    };
    // without dy the gradient of h is dh as it is: zeros for the statistics of h, which may be no numbers, leave the norm's term out
    // (where there are none of u either, the caller gives no statistics).  A mask in a vector register: a condition in the loop takes
    // scalar registers, and there are none left (50432 x 768 without a post-norm 80.2 us so, 76.5 with nothing).
    uint32_t of_h = a.dy != nullptr ? ~0u : 0u;
    if constexpr (POST) asm volatile("" : "+v"(of_h));
    const uint32_t of_u = post ? ~0u : 0u;
    Vec next[MODE == ROW_AHEAD ? V : 1];
    float4 sn;
    float2 mn = make_float2(0.0f, 0.0f);
    auto fetch = [&](const Place& at) {
        if constexpr (MODE == ROW_AHEAD) {
#pragma unroll
            for (int v = 0; v < V; ++v) load(next[v], at, v, true, true);
        }
        const u4_vec s = __builtin_amdgcn_raw_buffer_load_b128(descriptor(g.stats, at.first * (int64_t)sizeof(float4)),
                                                               at.live ? at.behind * (uint32_t)sizeof(float4) : OFF_END, 0, 0);
        sn = make_float4(__uint_as_float(s.x), __uint_as_float(s.y), __uint_as_float(s.z), __uint_as_float(s.w));
        if constexpr (PART == BWD_SUMS) {
            const u2_vec m = __builtin_amdgcn_raw_buffer_load_b64(descriptor(a.means, at.first * (int64_t)sizeof(float2)),
                                                                  at.live ? at.behind * (uint32_t)sizeof(float2) : OFF_END, 0, 0);
            mn = make_float2(__uint_as_float(m.x), __uint_as_float(m.y));
        }
    };
    int64_t gate_row = 0, in_run = 0;
    if (gate_by_row && count > 0) {
        gate_row = begin / g.gate_run;
        in_run = begin - gate_row * g.gate_run;
    }
    Place at{first, (uint32_t)(begin - first), col0, step, g.cols, g.pitch8, count > 0, back_of<END, V>(g.cols, col0, step)};
    fetch(at);
    float* own_gate = lds + vectors * Params::STRIDE + team_in_block * vectors * Params::GATE_STRIDE;     // a lane reads what it wrote
    auto gate_of_row = [&](int v) { return param8<TAIL>(g.gate, g.gate_bf16, gate_row * g.ld_gate + at.col(v), at.left(v), 0.0f); };
    auto take_gate = [&]() {
        if (PART != BWD_ROWS) {
#pragma unroll
            for (int v = 0; v < V; ++v) Params::put(own_gate + (lane + v * g.lanes) * Params::GATE_STRIDE, gate_of_row(v));
        }
    };
    if (gate_by_row) take_gate();
    auto param = [&](NormParam which, int v) {
        if constexpr (PART != BWD_ROWS) {
            if (which == P_GATE && gate_by_row) return Params::get(own_gate + (lane + v * g.lanes) * Params::GATE_STRIDE);
            return Params::get(lds, Params::STRIDE, which, lane + v * g.lanes);
        } else {
            if (which == P_GATE && gate_by_row) return gate_of_row(v);
            if (g.plane[which] != ParamPlanes::NO_PLANE) return ParamPlanes::get(lds, g.plane[which], vectors, lane + v * g.lanes, param_is_bf16(g, which));
            return norm_param<TAIL>(g, which, col0 + v * step);
        }
    };
    for (uint32_t i = 0; i < (uint32_t)g.team_rows; ++i) {
        Vec held[MODE == ROW_AGAIN ? 1 : V];
        float4 st = sn;
        const float2 means = mn;
        if (PART == BWD_ROWS && gate_by_row && at.live) gate_row = at.row() / g.gate_run;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (MODE == ROW_AHEAD) held[v] = next[v];
            if constexpr (MODE == ROW_HELD) load(held[v], at, v, true, true);
        }
        forget();
        Place ahead = at;
        ahead.first += g.row_step;
        ahead.live = i + 1 < count;
        fetch(ahead);
        if constexpr (POST) {
            st.z = __uint_as_float(__float_as_uint(st.z) & of_h);
            st.w = __uint_as_float(__float_as_uint(st.w) & of_h);
        }
        // one of the lane's vectors at a time; what a step needs of it is loaded again, or taken from its registers (first_h,
        // first_u: for the first time)
        auto each = [&](bool h, bool u, bool first_h, bool first_u, auto&& f) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Vec& r = held[MODE == ROW_AGAIN ? 0 : v];
                if constexpr (MODE == ROW_AGAIN) load(r, at, v, h, u);
                if (END == ROW_ENDS && v == V - 1) {
                    if (MODE == ROW_AGAIN ? h : first_h) {
                        settle(r.dy, at.back);
                        settle<XT>(r.h, at.back);
                    }
                    if (MODE == ROW_AGAIN ? u : first_u) {
                        settle(r.dh, at.back);
                        if (READ_U) settle<UT>(r.u, at.back);
                    }
                }
                f(r, v);
                if (V > 1) __builtin_amdgcn_sched_barrier(0);
            }
        };
        float s[2] = {0.0f, 0.0f};
        each(true, false, true, false, [&](Vec& r, int v) {
            const F8 dy = widen(r.dy), h = value_of<XT>(r.h), w = param(P_PRE_WEIGHT, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float n = (h.v[t] - st.z) * st.w, b = dy.v[t] * w.v[t];
                if constexpr (PART != BWD_ROWS) {
                    acc[PRE_WEIGHT][v].v[t] = __builtin_fmaf(dy.v[t], n, acc[PRE_WEIGHT][v].v[t]);
                    if (LAYER) acc[PRE_BIAS][v].v[t] += dy.v[t];
                }
                s[0] = __builtin_fmaf(b, n, s[0]);
                if (LAYER) s[1] += b;
            }
        });
        float h1 = means.x, h0 = means.y;
        if constexpr (PART != BWD_SUMS) {
            team.sum<LAYER ? 2 : 1>(s);
            h1 = s[0] * g.inv_cols;
            h0 = s[1] * g.inv_cols;
        }
        if (PART == BWD_ROWS && lane == 0 && at.live) a.means[at.row()] = make_float2(h1, h0);
        forget();
        s[0] = s[1] = 0.0f;
        // the gradient of h from the vector's parts
        auto gradient = [&](Vec& r, int v) {
            renew(r.dy);
            renew(r.h);
            F8 dh = widen(r.dh);
            const F8 dy = widen(r.dy), h = value_of<XT>(r.h), w = param(P_PRE_WEIGHT, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float n = (h.v[t] - st.z) * st.w;
                dh.v[t] = __builtin_fmaf(st.w, __builtin_fmaf(-n, h1, dy.v[t] * w.v[t] - h0), dh.v[t]);
            }
            return dh;
        };
        F8 dv[PLAN.keep && POST ? V : 1];
        const float ru = post ? st.y : 1.0f;                             // without a post-norm u itself takes part, its mean as 0
        if constexpr (PART != BWD_SUMS || READ_U) each(true, true, false, true, [&](Vec& r, int v) {
            const F8 dh = gradient(r, v);
            if constexpr (PART != BWD_SUMS) {
                F8 out;
#pragma unroll
                for (int t = 0; t < 8; ++t) out.v[t] = g.rho * dh.v[t];
                store_vec<END, V, XT>(a.dx, a.lddx, at, v, out);
            }
            F8 d, u, w;
#pragma unroll
            for (int t = 0; t < 8; ++t) d.v[t] = g.sigma * dh.v[t];
            if constexpr (READ_U) u = value_of<UT>(r.u);
            if constexpr (POST) {
#pragma unroll
                for (int t = 0; t < 8; ++t) u.v[t] = (u.v[t] - st.x) * ru;
                w = param(P_POST_WEIGHT, v);
            }
            if constexpr (GATE) {
                const F8 gate = param(P_GATE, v);
                F8 value = u;
                if constexpr (POST) {
#pragma unroll
                    for (int t = 0; t < 8; ++t) value.v[t] *= w.v[t];
                    if (LAYER) {
                        const F8 b = param(P_POST_BIAS, v);
#pragma unroll
                        for (int t = 0; t < 8; ++t) value.v[t] += b.v[t];
                    }
                }
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    if constexpr (PART != BWD_ROWS) acc[GATE_SUM][v].v[t] = __builtin_fmaf(d.v[t], value.v[t], acc[GATE_SUM][v].v[t]);
                    d.v[t] *= gate.v[t];
                }
            }
            if constexpr (!POST) {
                if constexpr (PART != BWD_SUMS) store_vec<END, V, UT>(a.du, a.lddu, at, v, d);
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    if constexpr (PART != BWD_ROWS) {
                        acc[POST_WEIGHT][v].v[t] = __builtin_fmaf(d.v[t], u.v[t], acc[POST_WEIGHT][v].v[t]);
                        if (LAYER) acc[POST_BIAS][v].v[t] += d.v[t];
                    }
                    d.v[t] *= w.v[t];
                    s[0] = __builtin_fmaf(d.v[t], u.v[t], s[0]);
                    if (LAYER) s[1] += d.v[t];
                }
                if constexpr (PLAN.keep) dv[v] = d;
            }
        });
        if constexpr (POST && PART != BWD_SUMS) {
            float u1 = 0.0f, u0 = 0.0f;
            if (post) {
                team.sum<LAYER ? 2 : 1>(s);
                u1 = s[0] * g.inv_cols;
                u0 = s[1] * g.inv_cols;
            }
            forget();
            each(true, true, false, false, [&](Vec& r, int v) {
                F8 d;
                if constexpr (!PLAN.keep) {
                    renew(r.dh);
                    d = gradient(r, v);
                    const F8 w = param(P_POST_WEIGHT, v);
#pragma unroll
                    for (int t = 0; t < 8; ++t) d.v[t] *= g.sigma;
                    if constexpr (GATE) {
                        const F8 gate = param(P_GATE, v);
#pragma unroll
                        for (int t = 0; t < 8; ++t) d.v[t] *= gate.v[t];
                    }
#pragma unroll
                    for (int t = 0; t < 8; ++t) d.v[t] *= w.v[t];
                } else {
                    d = dv[v];
                }
                renew(r.u);
                // without a post-norm d stays as it is, also where u is infinite: codes become those of zero, two operations; with
                // values the result is chosen (zeros for u as well: 40000 x 1001, FP32 and bf16, layer norms 225 us instead of 206)
                if constexpr (TAIL && CKPT) {
                    r.u.codes.w[0] &= of_u;
                    r.u.codes.w[1] &= of_u;
                }
                const F8 u = value_of<UT>(r.u);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float c = ru * __builtin_fmaf(-(u.v[t] - st.x) * ru, u1, d.v[t] - u0);
                    d.v[t] = post || CKPT ? c : d.v[t];
                }
                store_vec<END, V, UT>(a.du, a.lddu, at, v, d);
            });
        }
        if (PART != BWD_ROWS && gate_by_row && ++in_run == g.gate_run) {       // the gate's row is complete
            if (whole && a.want_gate) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int64_t to = gate_row * g.cols + at.col(v);
                    if (g.gate_bf16) store8<TAIL>(static_cast<uint16_t*>(a.dgate) + to, acc[GATE_SUM][v], at.left(v));
                    else             store8<TAIL>(static_cast<float*>(a.dgate) + to, acc[GATE_SUM][v], at.left(v));
                    acc[GATE_SUM][v] = mxd::zero8();
                }
            }
            in_run = 0;
            ++gate_row;
            at.live = ahead.live;                                        // its lanes in the row are the same
            take_gate();
        }
        at = ahead;
    }
    if constexpr (PART == BWD_ROWS) return;

#pragma unroll
    for (int s = 0; s < SUMS; ++s) {
        if (!LAYER && s >= PRE_BIAS) continue;
        if (!POST && (s == POST_WEIGHT || s == POST_BIAS)) continue;
        if (!GATE && s == GATE_SUM) continue;
        float* out = a.partials + ((int64_t)s * gridDim.x + blockIdx.x) * g.cols;
        if (s == GATE_SUM) {
            if (!a.want_gate || whole) continue;
            if (a.gate_rows > 1) {                                       // one row of sums for each team
                if (k < g.teams) {
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
        for (int v = 0; v < V; ++v) store_raw<false>(lds + team_in_block * width + (lane + v * g.lanes) * 8u, acc[s][v], 8);
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < width && base + c < g.cols; c += blockDim.x) {
            float t = lds[c];
            for (uint32_t i = 1; i < teams; ++i) t += lds[i * width + c];
            out[base + c] = t;
        }
    }
}

template <bool LAYER>
hipError_t launch_norm_bwd(const NormGradArgs& a, bool x_bf16, bool u_bf16, bool eight, RowEnd end, int v, BwdPart part, dim3 grid, uint32_t threads, size_t lds, hipStream_t st)
{
    hipError_t e = hipSuccess;
    by_types(x_bf16, u_bf16, [&](auto xt, auto ut) {
        by_kind(end, a.f.post, a.f.gate != nullptr, [&](auto post, auto gate, auto ends) {
            by_flag(eight, [&](auto c) {
                auto run = [&](auto n, auto which) {
                    if constexpr (decltype(ends)::value != ROW_SHORT || (decltype(n)::value == 1 && decltype(which)::value == BWD_ALL)) e = start_norm(residual_norm_bwd_kernel<decltype(xt), decltype(ut), decltype(n)::value, decltype(post)::value, decltype(gate)::value,
                                                            LAYER, decltype(c)::value, decltype(ends)::value, decltype(which)::value>, grid, threads, lds, st, a);
                };
                using One = std::integral_constant<int, 1>;
                if (part == BWD_ROWS)      run(std::integral_constant<int, 4>{}, std::integral_constant<BwdPart, BWD_ROWS>{});
                else if (part == BWD_SUMS) run(One{}, std::integral_constant<BwdPart, BWD_SUMS>{});
                else if (v == 1)           run(One{}, std::integral_constant<BwdPart, BWD_ALL>{});
                else                       run(std::integral_constant<int, 2>{}, std::integral_constant<BwdPart, BWD_ALL>{});
            });
        });
    });
    return e;
}

}  // namespace mxl
