// Device-side building blocks of the operators between the linear layers: rows of any alignment and length, FP32
// parameters from either type, the 8-bit checkpoint codec, sums over a team of lanes.
#pragma once
#include "mx_device.hpp"

namespace mxb {

using mxd::F8;

// ---- eight consecutive elements of a row ---------------------------------------------------------
// Global accesses of 16 bytes need no more than the element's own alignment here, so that rows of any pitch take the
// wide path.  Only where a row's length is no multiple of eight (TAIL) the vector that its end cuts goes in pieces of
// four, two and one elements.
typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u1_any __attribute__((aligned(2)));
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float f2_any __attribute__((ext_vector_type(2), aligned(4)));

struct RawBf16 { uint32_t w[4]; };                       // pairs, low half first
template <typename T> struct RawOf;
template <> struct RawOf<uint16_t> { typedef RawBf16 type; };
template <> struct RawOf<float> { typedef F8 type; };
template <typename T> using Raw = typename RawOf<T>::type;

// n: how many of the eight lie inside the row (none if not positive); the others read as zero.
template <bool TAIL>
__device__ __forceinline__ RawBf16 load_raw(const uint16_t* p, int n)
{
    RawBf16 r{{0, 0, 0, 0}};
    if (TAIL ? n >= 8 : n > 0) {
        const u4_any v = __builtin_nontemporal_load(reinterpret_cast<const u4_any*>(p));
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    } else if (TAIL && n > 0) {
        uint32_t two = 0, one = 0;
        if (n & 4) {
            const u2_any v = *reinterpret_cast<const u2_any*>(p);
            r.w[0] = v.x; r.w[1] = v.y;
        }
        if (n & 2) two = *reinterpret_cast<const u1_any*>(p + (n & 4));
        if (n & 1) one = p[n & 6];
        if (n & 4) { r.w[2] = n & 2 ? two : one; r.w[3] = n & 2 ? one : 0; }
        else       { r.w[0] = n & 2 ? two : one; r.w[1] = n & 2 ? one : 0; }
    }
    return r;
}

template <bool TAIL>
__device__ __forceinline__ F8 load_raw(const float* p, int n)
{
    F8 r = mxd::zero8();
    if (TAIL ? n >= 8 : n > 0) {
        const f4_any a = __builtin_nontemporal_load(reinterpret_cast<const f4_any*>(p));
        const f4_any b = __builtin_nontemporal_load(reinterpret_cast<const f4_any*>(p) + 1);
        r.v[0] = a.x; r.v[1] = a.y; r.v[2] = a.z; r.v[3] = a.w;
        r.v[4] = b.x; r.v[5] = b.y; r.v[6] = b.z; r.v[7] = b.w;
    } else if (TAIL && n > 0) {
        f2_any two = {0.0f, 0.0f};
        float one = 0.0f;
        if (n & 4) {
            const f4_any a = *reinterpret_cast<const f4_any*>(p);
            r.v[0] = a.x; r.v[1] = a.y; r.v[2] = a.z; r.v[3] = a.w;
        }
        if (n & 2) two = *reinterpret_cast<const f2_any*>(p + (n & 4));
        if (n & 1) one = p[n & 6];
        const float a = n & 2 ? two.x : one, b = two.y, c = n & 2 ? one : 0.0f;
        if (n & 4) { r.v[4] = a; r.v[5] = b; r.v[6] = c; }
        else       { r.v[0] = a; r.v[1] = b; r.v[2] = c; }
    }
    return r;
}

__device__ __forceinline__ F8 widen(const F8& r) { return r; }
__device__ __forceinline__ F8 widen(const RawBf16& r)
{
    F8 f;
#pragma unroll
    for (int t = 0; t < 8; ++t) f.v[t] = __uint_as_float((t & 1) ? r.w[t >> 1] & 0xFFFF0000u : r.w[t >> 1] << 16);
    return f;
}

// Rounded to nearest even where the type is bf16.
__device__ __forceinline__ void narrow(const F8& f, F8& r) { r = f; }
__device__ __forceinline__ void narrow(const F8& f, RawBf16& r)
{
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        mxd::bf16x2_hw p;
        p.x = (__bf16)f.v[2 * t];
        p.y = (__bf16)f.v[2 * t + 1];
        r.w[t] = mxd::bits_as<uint32_t>(p);
    }
}

template <bool TAIL>
__device__ __forceinline__ void store_raw(uint16_t* p, const RawBf16& r, int n)
{
    if (TAIL ? n >= 8 : n > 0) {
        u4_any v;
        v.x = r.w[0]; v.y = r.w[1]; v.z = r.w[2]; v.w = r.w[3];
        *reinterpret_cast<u4_any*>(p) = v;
    } else if (TAIL && n > 0) {
        if (n & 4) {
            u2_any v;
            v.x = r.w[0]; v.y = r.w[1];
            *reinterpret_cast<u2_any*>(p) = v;
        }
        const uint32_t w0 = r.w[0], w1 = r.w[1], w2 = r.w[2], w3 = r.w[3];         // by value: no indexed registers
        const uint32_t a = n & 4 ? w2 : w0, b = n & 4 ? w3 : w1;
        if (n & 2) *reinterpret_cast<u1_any*>(p + (n & 4)) = a;
        if (n & 1) p[n & 6] = (uint16_t)(n & 2 ? b : a);
    }
}

template <bool TAIL>
__device__ __forceinline__ void store_raw(float* p, const F8& r, int n)
{
    if (TAIL ? n >= 8 : n > 0) {
        f4_any a, b;
        a.x = r.v[0]; a.y = r.v[1]; a.z = r.v[2]; a.w = r.v[3];
        b.x = r.v[4]; b.y = r.v[5]; b.z = r.v[6]; b.w = r.v[7];
        reinterpret_cast<f4_any*>(p)[0] = a;
        reinterpret_cast<f4_any*>(p)[1] = b;
    } else if (TAIL && n > 0) {
        if (n & 4) {
            f4_any a;
            a.x = r.v[0]; a.y = r.v[1]; a.z = r.v[2]; a.w = r.v[3];
            *reinterpret_cast<f4_any*>(p) = a;
        }
        f2_any two;
        two.x = n & 4 ? r.v[4] : r.v[0];
        two.y = n & 4 ? r.v[5] : r.v[1];
        if (n & 2) *reinterpret_cast<f2_any*>(p + (n & 4)) = two;
        if (n & 1) p[n & 6] = n & 2 ? (n & 4 ? r.v[6] : r.v[2]) : two.x;
    }
}

template <bool TAIL, typename T>
__device__ __forceinline__ void store8(T* p, const F8& f, int n)
{
    Raw<T> r;
    narrow(f, r);
    store_raw<TAIL>(p, r, n);
}

// Eight values of a parameter vector of either type; `none` inside the row where there is no vector, 0 past its end.
template <bool TAIL>
__device__ __forceinline__ F8 param8(const void* p, bool bf16, int64_t at, int n, float none)
{
    if (p == nullptr) {
        F8 f;
#pragma unroll
        for (int t = 0; t < 8; ++t) f.v[t] = t < n ? none : 0.0f;
        return f;
    }
    return bf16 ? widen(load_raw<TAIL>(static_cast<const uint16_t*>(p) + at, n)) : load_raw<TAIL>(static_cast<const float*>(p) + at, n);
}

// ---- 8-bit checkpoints ----------------------------------------------------------------------------
// Groups of 32 (four neighbouring lanes of eight) share a power of two 2^s, the smallest that leaves no magnitude above
// E4M3's largest, 448 = 1.75 * 2^8: with M = m * 2^e that is s = e - 8, one more where m > 1.75; byte = s + 127, not
// below 0.  The scaled conversion divides by 2^s and rounds to nearest even in one step, so a value is off by at most
// 2^-4 of itself (or half a step of 2^(s-9) near zero).  A NaN stays one, under a scale taken from the others; a group
// that holds an infinity becomes NaN as a whole.
__device__ __forceinline__ uint32_t scale_byte8(uint32_t amax_bits)
{
    // adding 0x1FFFFF carries into the exponent field exactly when the mantissa exceeds 0x600000
    const uint32_t field = (amax_bits + 0x1FFFFFu) >> 23;
    uint32_t b;
    asm("v_sub_u32_e64 %0, %1, 8 clamp" : "=v"(b) : "v"(field));
    return b;
}

typedef short s16x2_any __attribute__((ext_vector_type(2)));

struct Codes8 { uint32_t w[2]; };

__device__ __forceinline__ uint32_t cvt4_fp8(float a, float b, float c, float d, float scale)
{
    s16x2_any r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
    return mxd::bits_as<uint32_t>(r);
}

// Codes and scale byte of the lane's eight elements; all four lanes of the group take part.
__device__ __forceinline__ Codes8 pack8(const F8& f, uint32_t& byte)
{
    const uint32_t amax = mxd::quad_max(mxd::amax_bits8(f));
    byte = scale_byte8(amax);
    const float s = mxd::scale_operand(byte);
    Codes8 c;
    c.w[0] = cvt4_fp8(f.v[0], f.v[1], f.v[2], f.v[3], s);
    c.w[1] = cvt4_fp8(f.v[4], f.v[5], f.v[6], f.v[7], s);
    if (amax >= 0x7F800000u) c.w[0] = c.w[1] = 0x7F7F7F7Fu;
    return c;
}

__device__ __forceinline__ F8 unpack8(const Codes8& c, uint32_t byte)
{
    const float s = mxd::scale_operand(byte);
    F8 f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const mxd::f32x2_hw lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.w[i], s, false);
        const mxd::f32x2_hw hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.w[i], s, true);
        f.v[4 * i] = lo.x; f.v[4 * i + 1] = lo.y; f.v[4 * i + 2] = hi.x; f.v[4 * i + 3] = hi.y;
    }
    return f;
}

// ---- sums over a team of lanes --------------------------------------------------------------------
// A team is 8, 16, 32 or 64 neighbouring lanes, or whole waves.  Every lane gets the sum, formed in one fixed order.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}

__device__ __forceinline__ float sum16(float v)
{
    v = dpp_add<0xB1>(v);                                // lane ^ 1
    v = dpp_add<0x4E>(v);                                // lane ^ 2
    v = dpp_add<0x141>(v);                               // the other half of 8 lanes
    return dpp_add<0x140>(v);                            // the other half of 16
}

__device__ __forceinline__ float wave_part_sum(float v, uint32_t lanes)
{
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    if (lanes >= 16) v = dpp_add<0x140>(v);
    if (lanes >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if (lanes >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

constexpr int TEAM_WAVES_MAX = 16;
struct TeamScratch { float part[2][2][TEAM_WAVES_MAX]; };        // [parity][value][wave of the workgroup]

struct Team {
    uint32_t lanes;          // 8, 16, 32, 64 or a multiple of 64
    uint32_t first_wave;     // of the workgroup's waves
    TeamScratch* scratch;
    uint32_t parity = 0;

    // Consecutive sums use the two halves of the scratch in turn: a wave writes a half again only behind the barrier
    // of the sum between, which every wave reaches after its last read of that half.
    template <int N>
    __device__ __forceinline__ void sum(float* v)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = wave_part_sum(v[i], lanes);
        if (lanes <= 64) return;
        const uint32_t waves = lanes >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) scratch->part[parity][i][wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t w = lane & 15u;
            v[i] = sum16(w < waves ? scratch->part[parity][i][first_wave + w] : 0.0f);
        }
        parity ^= 1u;
    }
};

}  // namespace mxb
