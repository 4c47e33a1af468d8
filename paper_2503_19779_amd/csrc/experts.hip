// experts.hip -- routing to experts, the experts' products and their weighted sum, products of 8-bit weights with a scale per block of
// 128, and the quantisation of rows.  gfx950 only.
#include "device.h"

#include <algorithm>
#include <iterator>
#include <type_traits>

namespace pgk {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef v4u v4u_1 __attribute__((aligned(1)));

template <typename T> __device__ __forceinline__ const T* operand(const void* p, unsigned slots, int j) {
    return (const T*)resolve_rt(p, (slots >> j) & 1u);
}
__device__ __forceinline__ int up_to(int x, int to) { return (x + to - 1) / to * to; }

// ---- PG_QUANTIZE -------------------------------------------------------------------------------------------
// q = x 2^-e rounded to e4m3 (the one rounding), e the least with max |x| <= 448 * 2^e: the maximum's exponent, and one more above 1.75.  Memory bounds it: each
// value is read once and written once.  16 lanes take a block of 128 values, 8 each; their maximum goes round in four steps of a DPP row.
__device__ __forceinline__ float row16_max(float v) {
    v = __builtin_fmaxf(v, dpp_take<0xB1>(v));
    v = __builtin_fmaxf(v, dpp_take<0x4E>(v));
    v = __builtin_fmaxf(v, dpp_take<0x141>(v));
    return __builtin_fmaxf(v, dpp_take<0x140>(v));
}

// Eight values from element c of a row on, zeros beyond its last one
template <typename T>
__device__ __forceinline__ void eight_of(const T* row, int c, int cols, float* f) {
    if (c + 8 <= cols) {
        unsigned w[sizeof(T) * 2];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; i++) {
            const v4u v = *(const v4u_any PG_GLOBAL*)(uintptr_t)(row + c + 4 * i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = sizeof(T) == 4 ? __uint_as_float(w[sizeof(T) == 4 ? i : 0]) : __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = c + i < cols ? load_elem(row + c + i) : 0.f;
    }
}

// 16 lanes take four neighbouring blocks of a row, whose exponents are one word: four loads (eight for fp32) in flight a lane.
// 8192 rows of 4096 bf16 columns: 21.7 us, 4.66 TB/s (47 us with one block each and narrower loads); a copy of 1 GB reaches 4.8.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_quantize(QuantizeArgs p) {
    const T* x = operand<T>(p.x, p.slots, 0);
    const unsigned nb = (unsigned)(p.cols + kScaleBlock - 1) / kScaleBlock, quads = (nb + 3) / 4, lane = threadIdx.x & 15;
    const unsigned long long total = (unsigned long long)p.rows * quads;
    const unsigned unit = blockIdx.x * (kBlock / 16) + (threadIdx.x >> 4);          // (fewer than 2^31: plan_experts)
    const bool live = unit < total;
    const unsigned row = live ? unit / quads : 0u, quad = live ? unit - row * quads : 0u;
    const T* from = x + (long long)row * p.cols;
    float f[4][8];
#pragma unroll
    for (int u = 0; u < 4; u++) eight_of(from, (int)(quad * 512 + u * 128 + lane * 8), p.cols, f[u]);
    unsigned char* out = (unsigned char*)p.out;
    const long long kp = (long long)nb * kScaleBlock;
    unsigned exps = 0;
#pragma unroll
    for (int u = 0; u < 4; u++) {
        float top = 0.f;
        bool fine = true;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float a = __builtin_fabsf(f[u][i]);
            const bool is = a < __builtin_inff();
            fine = fine && is;
            top = __builtin_fmaxf(top, is ? a : 0.f);
        }
        top = row16_max(top);
        // 448 = 1.75 * 2^8
        const unsigned bits = __float_as_uint(top);
        int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
        e = e < -126 ? -126 : e;
        const float by = __uint_as_float((unsigned)(127 - e) << 23);
        unsigned w[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            int q = __builtin_amdgcn_cvt_pk_fp8_f32(f[u][4 * i] * by, f[u][4 * i + 1] * by, 0, false);
            w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[u][4 * i + 2] * by, f[u][4 * i + 3] * by, q, true);
        }
        if (!fine)
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (!(__builtin_fabsf(f[u][i]) < __builtin_inff())) w[i / 4] = (w[i / 4] & ~(0xffu << (8 * (i & 3)))) | 0x7fu << (8 * (i & 3));
        const unsigned kb = quad * 4 + u;
        exps |= (unsigned)(kb < nb ? e + 127 : 127) << (8 * u);
        if (live && kb < nb) *(uint2*)(out + row * kp + kb * 128 + lane * 8) = uint2{w[0], w[1]};
    }
    if (live && lane == 0) *(unsigned*)(out + (long long)p.rows * kp + ((long long)row * quads + quad) * 4) = exps;
}

// ---- PG_EXPERT_SUM -----------------------------------------------------------------------------------------
// fp32 sums, the slots in their order, then x; one rounding at the store.  Memory bounds it.  A lane takes 16 bytes of a row, with up to eight slots' loads in
// flight.  A row goes to as many lanes as it has such pieces, rounded up to a power of two, or to several workgroups.  4096 rows of 8 slots of 2048 bf16
// outputs: 31 us, 5.4 TB/s (131 us with one slot's load at a time).
__host__ __device__ inline int sum_lanes(int pieces) {
    int l = 1;
    while (l < pieces && l < kBlock) l *= 2;
    return l;
}
template <typename T>
__global__ __launch_bounds__(kBlock) void k_expert_sum(ExpertSumArgs p) {
    constexpr int NV = 16 / (int)sizeof(T), kAt = 8;
    const T* z = operand<T>(p.z, p.slots, 0);
    const Routed* r = operand<Routed>(p.r, p.slots, 1);
    const T* x = p.x ? operand<T>(p.x, p.slots, 2) : nullptr;
    const int pieces = (p.n + NV - 1) / NV, lanes = sum_lanes(pieces), per_row = (pieces + lanes - 1) / lanes;
    const unsigned line = blockIdx.x / (unsigned)per_row;
    const long long row = lanes == kBlock ? (long long)line : (long long)blockIdx.x * (kBlock / lanes) + threadIdx.x / lanes;
    const int piece = lanes == kBlock ? (int)(blockIdx.x - line * per_row) * kBlock + threadIdx.x : threadIdx.x % lanes;
    if (row >= p.rows || piece >= pieces) return;
    const int j = piece * NV, have = p.n - j < NV ? p.n - j : NV;
    auto fetch = [&](const T* at, unsigned* w) {
        if (have == NV) {
            const v4u v = *(const v4u_any PG_GLOBAL*)(uintptr_t)at;
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = 0u;
#pragma unroll
            for (int i = 0; i < NV; i++)
                if (i < have) { if constexpr (sizeof(T) == 4) w[i] = load_raw(at + i); else w[i / 2] |= load_raw(at + i) << (16 * (i & 1)); }
        }
    };
    float acc[NV], f[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) acc[i] = 0.f;
    const Routed* rr = r + row * p.k;
    const T* zr = z + row * p.k * p.n + j;
    unsigned wx[4];
    if (x) fetch(x + row * p.n + j, wx);
    for (int t0 = 0; t0 < p.k; t0 += kAt) {
        Routed q[kAt];
        unsigned w[kAt][4];
        const int more = p.k - t0;
#pragma unroll
        for (int t = 0; t < kAt; t++) q[t] = rr[t0 + (t < more ? t : 0)];
        // (an empty slot, and what lies behind the last one, is left out of the sum, whatever is fetched in its place)
#pragma unroll
        for (int t = 0; t < kAt; t++) if (t < more) fetch(zr + (long long)(t0 + t) * p.n, w[t]);
#pragma unroll
        for (int t = 0; t < kAt; t++) {
            if (t >= more) break;
            Vec<T, 16>::unpack(w[t], f);
#pragma unroll
            for (int i = 0; i < NV; i++) acc[i] = q[t].expert >= 0 ? __builtin_fmaf(q[t].weight, f[i], acc[i]) : acc[i];
        }
    }
    if (x) {
        Vec<T, 16>::unpack(wx, f);
#pragma unroll
        for (int i = 0; i < NV; i++) acc[i] += f[i];
    }
    T* o = (T*)p.out + row * p.n + j;
    unsigned w[4];
    Vec<T, 16>::pack(acc, w);
    if (have == NV) *(v4u_any*)o = v4u{w[0], w[1], w[2], w[3]};
    else
#pragma unroll
        for (int i = 0; i < NV; i++) if (i < have) store_elem(o + i, acc[i]);
}

// ---- PG_ROUTE ----------------------------------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ double dpp_take64(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, 0xf, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double read_lane64(double v, int lane) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), lane);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ float read_lane(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ double read_lane_k(double v, int lane) { return read_lane64(v, lane); }
__device__ __forceinline__ float read_lane_k(float v, int lane) { return read_lane(v, lane); }
template <int CTRL> __device__ __forceinline__ double dpp_take_k(double v) { return dpp_take64<CTRL>(v); }
template <int CTRL> __device__ __forceinline__ float dpp_take_k(float v) { return dpp_take<CTRL>(v); }
__device__ __forceinline__ double wave_sum64(double v) {
    v += dpp_take64<0xB1>(v);
    v += dpp_take64<0x4E>(v);
    v += dpp_take64<0x141>(v);
    v += dpp_take64<0x140>(v);
    return (read_lane64(v, 0) + read_lane64(v, 16)) + (read_lane64(v, 32) + read_lane64(v, 48));
}
__device__ __forceinline__ float wave_max(float v) {
    v = row16_max(v);
    return __builtin_fmaxf(__builtin_fmaxf(read_lane(v, 0), read_lane(v, 16)), __builtin_fmaxf(read_lane(v, 32), read_lane(v, 48)));
}
// exp(x) in fp32 within two half steps, x <= 0 or finite: 2^k exp(r), ln 2 in two pieces
__device__ __forceinline__ float exp_f32(float x) {
    constexpr float kLog2e = 1.4426950408889634f, kLn2Hi = 0.693145751953125f, kLn2Lo = 1.42860682030941723212e-6f;
    const float kf = __builtin_rintf(__builtin_fmaxf(__builtin_fminf(x, 100.f), -200.f) * kLog2e);
    const float r = __builtin_fmaf(kf, -kLn2Lo, __builtin_fmaf(kf, -kLn2Hi, __builtin_fmaxf(__builtin_fminf(x, 100.f), -200.f)));
    return __builtin_ldexpf(__builtin_amdgcn_exp2f(r * kLog2e), (int)kf);
}
// exp of N values in fp64 within about 3e-16, zero and infinite where fp64 is: the sum of r^n / n! to n = 13, |r| <= 0.347 (the next term is below
// 5e-18).  Side by side: each coefficient takes two moves.
template <int N>
__device__ __forceinline__ void exp_f64(double (&x)[N]) {
    constexpr double kLog2e = 1.4426950408889634, kLn2Hi = 0x1.62e42fefa0000p-1, kLn2Lo = 1.6465949582897082e-12;
    constexpr double c[] = {1.0 / 6227020800.0, 1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0,
                            1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
    double v[N];
    int e[N];
#pragma unroll
    for (int n = 0; n < N; n++) {
        const double y = __builtin_fmin(__builtin_fmax(x[n], -800.0), 800.0), kf = __builtin_rint(y * kLog2e);
        x[n] = __builtin_fma(kf, -kLn2Lo, __builtin_fma(kf, -kLn2Hi, y));
        e[n] = (int)kf;
        v[n] = c[0];
    }
#pragma unroll
    for (int i = 1; i < 14; i++)
#pragma unroll
        for (int n = 0; n < N; n++) v[n] = __builtin_fma(v[n], x[n], c[i]);
#pragma unroll
    for (int n = 0; n < N; n++) x[n] = __builtin_ldexp(v[n], e[n]);
}
// p of N scores, up to the factor `over`: 1 / (1 + exp(-x)), the reciprocal by two Newton steps and zero below -708, or exp(x - top)
template <int N>
__device__ __forceinline__ void scores_p(bool sigmoid, double top, double (&x)[N]) {
    double d[N];
#pragma unroll
    for (int n = 0; n < N; n++) d[n] = sigmoid ? __builtin_fmin(-x[n], 709.0) : x[n] - top;
    exp_f64(d);
#pragma unroll
    for (int n = 0; n < N; n++) {
        const double q = 1.0 + d[n];
        double y = __builtin_amdgcn_rcp(q);
        y = __builtin_fma(__builtin_fma(-q, y, 1.0), y, y);
        y = __builtin_fma(__builtin_fma(-q, y, 1.0), y, y);
        x[n] = !sigmoid ? d[n] : x[n] < -708.0 ? 0.0 : y;
    }
}

// A wave takes a row, lane l the experts l * V .. l * V + V - 1.  HIGH: where the choice goes by p itself -- a bias, or sums of two -- p is worked out in
// fp64; without it the scores are in the order of p, and only the chosen ones need it.  Either way a round of the choice goes by the values rounded to
// fp32, one instruction a step: what is largest in fp64 is among those that are largest then, mostly the only one.  Each lane keeps its experts sorted, best
// first, so that a round looks at heads only.  Latency bounds it: a round of the choice is a maximum over the wave and a ballot.  4096 rows, 8 of 256
// experts by bias and groups: 9.5 us; one row, 8 of 64: the launch, 2.4 us of its 4.1.
template <typename T, int V, bool HIGH>
__global__ __launch_bounds__(kBlock) void k_route(RouteArgs p) {
    using K = std::conditional_t<HIGH, double, float>;
    __shared__ K shared_keys[kBlock / 64][V * 64 < 128 ? 128 : V * 64];
    const T* s = operand<T>(p.s, p.slots, 0);
    const float* bias = p.bias ? operand<float>(p.bias, p.slots, 1) : nullptr;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = blockIdx.x * (kBlock / 64) + wave, e0 = lane * V;
    const bool sigmoid = (p.flags & 1) != 0, two = (p.flags & 4) != 0;
    if (row >= p.rows) return;                            // (waves share nothing)
    const T* sr = s + (long long)row * p.experts;
    constexpr float kNone = -__builtin_inff();
    float x[V];
    if (e0 + V <= p.experts) {
        constexpr int kBytes = V * (int)sizeof(T);
        unsigned w[kBytes < 4 ? 1 : kBytes / 4];
        if constexpr (kBytes >= 16) {
#pragma unroll
            for (int i = 0; i < kBytes / 16; i++) {
                const v4u v = *(const v4u_any PG_GLOBAL*)(uintptr_t)((const char*)(sr + e0) + 16 * i);
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else if constexpr (kBytes >= 4) {
#pragma unroll
            for (int i = 0; i < kBytes / 4; i++) w[i] = *(const u32_any PG_GLOBAL*)(uintptr_t)((const char*)(sr + e0) + 4 * i);
        } else {
            w[0] = load_raw_global(sr + e0);
        }
#pragma unroll
        for (int i = 0; i < V; i++) x[i] = sizeof(T) == 4 ? __uint_as_float(w[i * (int)sizeof(T) / 4]) : __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < V; i++) x[i] = e0 + i < p.experts ? load_elem(sr + e0 + i) : kNone;
    }
    float top = kNone;
#pragma unroll
    for (int i = 0; i < V; i++) {
        x[i] = x[i] > kNone ? __builtin_fminf(x[i], 3.40282347e38f) : kNone;       // (what is not a number as well)
        top = __builtin_fmaxf(top, x[i]);
    }
    top = wave_max(top);
    // key: what experts are compared by; -inf: never chosen.  p = sigmoid, or exp(x - top) * over
    K key[V];
    double pr[HIGH ? V : 1], over = 1.;
    if constexpr (HIGH) {
        double total = 0.;
#pragma unroll
        for (int i = 0; i < V; i++) pr[i] = (double)x[i];
        scores_p(sigmoid, (double)top, pr);
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (!(x[i] > kNone)) pr[i] = 0.;
            total += pr[i];
        }
        if (!sigmoid) {
            over = 1. / wave_sum64(total);
#pragma unroll
            for (int i = 0; i < V; i++) pr[i] = x[i] > kNone ? pr[i] * over : 0.;
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
            const double c = bias ? pr[i] + (double)bias[e0 + i < p.experts ? e0 + i : 0] : (double)x[i];
            key[i] = x[i] > kNone && c > (double)kNone ? c : (double)kNone;
        }
    } else {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) {
            key[i] = x[i];
            if (!sigmoid) z += x[i] > kNone ? exp_f32(x[i] - top) : 0.f;
        }
        if (!sigmoid) over = 1. / (double)wave_sum(z);
    }
    if (p.groups > 1) {
        const int per = p.experts / p.groups;
        K* const keys = shared_keys[wave];
        K best = (K)kNone, second = (K)kNone;
        auto take = [&](K a) {
            second = a > best ? best : a > second ? a : second;
            best = a > best ? a : best;
        };
        auto counts = [&](int i) -> K {                   // what expert i counts in its group
            if constexpr (HIGH) { if (two && !bias) return key[i] > (K)kNone ? pr[i] : (K)kNone; }
            return key[i];
        };
        const bool whole = per % V == 0;                  // a group is so many lanes'
        const int lanes = per / V;
        const bool rows16 = whole && lanes <= 16 && (lanes & (lanes - 1)) == 0;        // ... of one DPP row
        if (whole) {
#pragma unroll
            for (int i = 0; i < V; i++) take(counts(i));
        }
        int from = 1;                                     // the lane that has group g's count: g * from
        if (rows16) {
            auto join = [&](K b, K s) {
                const K low = b < best ? b : best, most = s > second ? s : second;
                best = b > best ? b : best;
                second = low > most ? low : most;
            };
            if (lanes > 1) join(dpp_take_k<0xB1>(best), dpp_take_k<0xB1>(second));
            if (lanes > 2) join(dpp_take_k<0x4E>(best), dpp_take_k<0x4E>(second));
            if (lanes > 4) join(dpp_take_k<0x141>(best), dpp_take_k<0x141>(second));
            if (lanes > 8) join(dpp_take_k<0x140>(best), dpp_take_k<0x140>(second));
            from = lanes;
        } else {
            if (whole) {
                keys[2 * lane] = best;
                keys[2 * lane + 1] = second;
            } else {
#pragma unroll
                for (int i = 0; i < V; i++) keys[e0 + i] = counts(i);
            }
            __builtin_amdgcn_wave_barrier();
            best = second = (K)kNone;
            if (lane < p.groups) {
                const K* at = keys + lane * (whole ? 2 * lanes : per);
                const int n = whole ? 2 * lanes : per;
#pragma unroll 4
                for (int i = 0; i < n; i++) take(at[i]);
            }
        }
        if (two && second > (K)kNone) best += second;
        int before = 0;                                   // groups that come before lane g's; lane g: group g from here on
        K mine_g = (K)kNone;
        for (int g = 0; g < p.groups; g++) {
            const K v = read_lane_k(best, g * from);
            if (lane == g) mine_g = v;
        }
        for (int g = 0; g < p.groups; g++) {
            const K v = read_lane_k(best, g * from);
            before += v > mine_g || (v == mine_g && g < lane);
        }
        const unsigned long long kept = __ballot(lane < p.groups && before < p.kept);
        if (whole) {
            const bool in = (kept >> (lane / lanes & 63)) & 1ull;
#pragma unroll
            for (int i = 0; i < V; i++) key[i] = in ? key[i] : (K)kNone;
        } else {
#pragma unroll
            for (int i = 0; i < V; i++) key[i] = (kept >> ((e0 + i) / per & 63)) & 1ull ? key[i] : (K)kNone;
        }
    }
    // the lane's experts, best first, equal ones in their order
    int of[V];
#pragma unroll
    for (int i = 0; i < V; i++) of[i] = e0 + i;
#pragma unroll
    for (int j = 1; j < V; j++)
#pragma unroll
        for (int i = 0; i + j < V; i++)                   // neighbours only: what is equal keeps its order
            if (key[i + 1] > key[i]) {
                const K k = key[i];
                key[i] = key[i + 1];
                key[i + 1] = k;
                const int o = of[i];
                of[i] = of[i + 1];
                of[i + 1] = o;
            }
    int mine = -1;
    for (int t = 0; t < p.k; t++) {
        const float head = (float)key[0], best = wave_max(head);
        if (!(best > kNone)) break;
        unsigned long long at = __ballot(head == best);
        if (HIGH && (at & (at - 1))) {                    // equal in fp32: compared in fp64
            double all = (double)kNone;
            for (unsigned long long left = at; left; left &= left - 1) all = __builtin_fmax(all, read_lane64(key[0], __builtin_ctzll(left)));
            at &= __ballot(key[0] == all);
        }
        const int l = __builtin_ctzll(at), e = __builtin_amdgcn_readlane(of[0], l);
        if (lane == t) mine = e;
        if (lane == l) {
#pragma unroll
            for (int i = 0; i + 1 < V; i++) { key[i] = key[i + 1]; of[i] = of[i + 1]; }
            key[V - 1] = (K)kNone;
        }
    }
    // the weights in fp64: a few lanes' one value each
    double weight = 0.;
    if (mine >= 0) {
        double score[1] = {(double)__builtin_fminf(load_elem(sr + mine), 3.40282347e38f)};
        scores_p(sigmoid, (double)top, score);
        weight = score[0] * over;
    }
    if (p.flags & 2) {
        const double all = wave_sum64(weight);
        weight = all > 0. ? weight / all : 0.;
    }
    Routed q;
    q.expert = mine;
    q.weight = (float)(weight * (double)p.factor);
    if (lane < p.k) ((Routed*)p.out)[(long long)row * p.k + lane] = q;
}

// ---- PG_EXPERT_GEMV: the slots in the order of their experts ---------------------------------------------------
constexpr int kSortThreads = 1024, kSortMostExperts = 1024, kSortHeld = 32;
__device__ __forceinline__ SortedTile* sorted_tiles(void* area) { return (SortedTile*)((SortedSlots*)area + 1); }
__device__ __forceinline__ int* sorted_order(void* area, int tiles) { return (int*)(sorted_tiles(area) + tiles); }

// One workgroup: a slot's place among its expert's is what a count in LDS says when it is counted, and from the counts follow the places of the
// experts.  Counts are kept in kCopies for neighbouring lanes to add to (lanes of a wave that add to one place wait for each other: 32768 slots of 64
// experts 14 us with one).  Slots of an expert come in no fixed order, and a product's rows do not depend on it: each is a row of its own in a tile.
// Whole tiles come first, so that the small ones fill what is left of the chip at the end.  Bucket `experts` takes the empty slots.  32768 slots of 64
// experts: 9 us, of which reading the slots through one compute unit and the counting take most; 513 slots: 6.
__global__ __launch_bounds__(kSortThreads) void k_sort_slots(ExpertArgs p) {
    constexpr int kCopies = 8;
    __shared__ int cnt[kCopies][kSortMostExperts + 1];
    __shared__ int sums[3][kSortThreads / 64];
    __shared__ unsigned short ordered[kSortThreads * kSortHeld];
    const Routed* r = operand<Routed>(p.r, p.slots, 2);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, buckets = p.experts + 1;
    const int slots = p.rows * p.k;
    const bool few = slots <= kSortThreads * kSortHeld;      // slots and places stay in registers
    int* const mine = cnt[lane % kCopies];
    auto bucket = [&](int e) { return (unsigned)e < (unsigned)p.experts ? e : p.experts; };
    for (int c = 0; c < kCopies; c++)
        for (int i = tid; i < buckets; i += kSortThreads) cnt[c][i] = 0;
    // two neighbouring slots a load: slots (i / 2 * kSortThreads + tid) * 2 + i % 2
    int id[kSortHeld], place[kSortHeld];
    auto slot = [&](int i) { return (i / 2 * kSortThreads + tid) * 2 + i % 2; };
    if (few) {
#pragma unroll
        for (int i = 0; i < kSortHeld; i += 2) {
            const int s = slot(i);
            v4u v = {0u, 0u, 0u, 0u};
            if (s + 1 < slots) v = *(const v4u_any PG_GLOBAL*)(uintptr_t)(r + s);
            else if (s < slots) v.x = (unsigned)r[s].expert;
            id[i] = (int)v.x;
            id[i + 1] = (int)v.z;
        }
    }
    __syncthreads();
    if (few) {
#pragma unroll
        for (int i = 0; i < kSortHeld; i++)
            if (slot(i) < slots) {
                id[i] = bucket(id[i]);
                place[i] = atomicAdd(&mine[id[i]], 1);
            }
    } else {
        for (int s = tid; s < slots; s += kSortThreads) atomicAdd(&mine[bucket(r[s].expert)], 1);
    }
    __syncthreads();
    // in front of each bucket: slots, whole tiles, others.  A thread takes two neighbouring buckets (1025 of 1024 threads).
    int c[2], v[3] = {0, 0, 0}, before[3];
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int b = tid * 2 + q;
        c[q] = 0;
        if (b < buckets)
#pragma unroll
            for (int u = 0; u < kCopies; u++) c[q] += cnt[u][b];
        v[0] += c[q];
        v[1] += c[q] / p.tile;
        v[2] += c[q] % p.tile != 0;
    }
#pragma unroll
    for (int w = 0; w < 3; w++) {
        before[w] = v[w];
        for (int d = 1; d < 64; d <<= 1) {
            const int a = __shfl_up(before[w], d);
            if (lane >= d) before[w] += a;
        }
        if (lane == 63) sums[w][wave] = before[w];
        before[w] -= v[w];
    }
    __syncthreads();
    int whole = 0, all = 0;
    for (int u = 0; u < kSortThreads / 64; u++) {
        if (u < wave) for (int w = 0; w < 3; w++) before[w] += sums[w][u];
        whole += sums[1][u];
        all += sums[1][u] + sums[2][u];
    }
    SortedTile* tiles = sorted_tiles(p.sorted);
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int b = tid * 2 + q;
        if (b >= buckets) break;
        const int first = before[0], expert = b < p.experts ? b : -1, n = c[q] / p.tile;
        for (int i = 0; i < n; i++) tiles[before[1]++] = SortedTile{expert, first + i * p.tile, first + (i + 1) * p.tile, 0};
        if (c[q] % p.tile) tiles[whole + before[2]++] = SortedTile{expert, first + n * p.tile, first + c[q], 0};
        int at = first;
#pragma unroll
        for (int u = 0; u < kCopies; u++) {
            const int n_u = cnt[u][b];
            cnt[u][b] = at;
            at += n_u;
        }
        before[0] += c[q];
    }
    if (tid == 0) ((SortedSlots*)p.sorted)->n_tiles = all;
    __syncthreads();
    int* order = sorted_order(p.sorted, p.tiles);
    if (few) {                       // (by way of LDS: 64 scattered stores of a wave take 64 lines' time)
#pragma unroll
        for (int i = 0; i < kSortHeld; i++)
            if (slot(i) < slots) ordered[mine[id[i]] + place[i]] = (unsigned short)slot(i);
        __syncthreads();
        for (int s = tid; s < slots; s += kSortThreads) order[s] = ordered[s];
    } else {
        for (int s = tid; s < slots; s += kSortThreads) order[atomicAdd(&mine[bucket(r[s].expert)], 1)] = s;
    }
}

// ---- products ----------------------------------------------------------------------------------------------
// Eight bf16 values from column c of a row of cols >= 8 on, at any element boundary, zeros beyond its last one: what 16 bytes load from inside the row, and the
// shift that puts it in place
__device__ __forceinline__ v4u row8_raw(const bf16_t* row, int c, int cols) {
    return *(const v4u_any PG_GLOBAL*)(uintptr_t)(row + (c + 8 <= cols ? c : cols - 8));
}
__device__ __forceinline__ v4u row8_fix(v4u v, int c, int cols) {
    const int over = c + 8 - cols, s = over < 0 ? 0 : over > 8 ? 8 : over, b = 16 * (s & 3);
    unsigned long long lo = (unsigned long long)v.y << 32 | v.x, hi = (unsigned long long)v.w << 32 | v.z;
    if (s >= 4) { lo = s == 8 ? 0 : hi; hi = 0; }
    if (b) { lo = lo >> b | hi << (64 - b); hi >>= b; }
    v.x = (unsigned)lo; v.y = (unsigned)(lo >> 32); v.z = (unsigned)hi; v.w = (unsigned)(hi >> 32);
    return v;
}
// ... of a row of any length, one by one
__device__ __forceinline__ v4u row8_short(const bf16_t* row, int c, int cols) {
    unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; i++) if (c + i < cols) w[i / 2] |= (unsigned)row[c + i] << (16 * (i & 1));
    return v4u{w[0], w[1], w[2], w[3]};
}
template <bool HI> __device__ __forceinline__ unsigned f8_to_bf16(unsigned w) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}
// eight e4m3 values (two words) as bf16: exact
__device__ __forceinline__ v4u f8x8_to_bf16(unsigned a, unsigned b) {
    v4u v;
    v.x = f8_to_bf16<false>(a); v.y = f8_to_bf16<true>(a); v.z = f8_to_bf16<false>(b); v.w = f8_to_bf16<true>(b);
    return v;
}
__device__ __forceinline__ v4u half_to_bf16(v4u v, int high) { return high ? f8x8_to_bf16(v.z, v.w) : f8x8_to_bf16(v.x, v.y); }
__device__ __forceinline__ f32x4 mfma_bf16(v4u a, v4u b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// Sums that the matrix instructions themselves carry over a loop, before their first use behind it: 32 idle cycles, since the compiler was seen to omit the
// wait states where the last of those instructions and the use lie in different blocks (gemv.hip, mm_drained)
template <int M, int J>
__device__ __forceinline__ void sums_drained(f32x4 (&acc)[M][J]) {
    asm volatile("s_nop 15\n\ts_nop 15" : "+v"(acc[M - 1][J - 1]));
#pragma unroll
    for (int m = 0; m < M; m++)
#pragma unroll
        for (int j = 0; j < J; j++) asm volatile("" : "+v"(acc[m][j]));
}

// What the operands are.  8-bit rows go two ways.  The 8-bit matrix instruction lines up the products of eight neighbouring columns with the
// largest of them and drops what lies below 2^-13 of its binade (found with one large and one small product at every pair of places; between
// the groups, and onto the accumulator, it adds in fp32): rms 1.5e-5 to 5e-5 of the result, which a bf16 output with its half step of 2^-8 does not
// show.  An fp32 output would, so there both operands become bf16, exactly, and the bf16 instruction, which sums in fp32, takes them.
enum Form : int { kW16H16, kW8H16, kW8H8, kW8H8Wide };

// The tile of slots that a workgroup of a routed product takes: its expert and how many slots.  From the sorted slots, or, up to kFewSlots of them,
// worked out by each wave for itself (a dispatch in front costs more): slot i, in lane i, is the rank-th of its expert; the slots whose rank is a
// multiple of the tile open a tile each, and those are numbered in the order of the slots.  expert -2: there is no tile t.
constexpr int kFewSlots = 64;
struct TileOf { int expert, used; int begin; unsigned long long members; };
template <int TILE>
__device__ __forceinline__ TileOf routed_tile(const ExpertArgs& p, int t) {
    if (p.sorted) {
        const int n = ((const SortedSlots*)p.sorted)->n_tiles;
        const SortedTile st = sorted_tiles(p.sorted)[t < p.tiles ? t : p.tiles - 1];       // (asked for beside the number of tiles, not behind it)
        return t < n ? TileOf{st.expert, st.end - st.begin, st.begin, 0} : TileOf{-2, 0, 0, 0};
    }
    const Routed* r = operand<Routed>(p.r, p.slots, 2);
    const int slots = p.rows * p.k, lane = threadIdx.x & 63;
    const int e = lane < slots ? r[lane].expert : 0, id = (unsigned)e < (unsigned)p.experts ? e : p.experts;
    unsigned long long same = slots < 64 ? (1ull << slots) - 1ull : ~0ull;
    const unsigned long long all = same, before = (1ull << lane) - 1ull;
    for (int b = 0; b < 32 - __builtin_clz(p.experts); b++) {
        const unsigned long long on = __ballot((id >> b) & 1);
        same &= ((id >> b) & 1) ? on : ~on;
    }
    const int rank = __popcll(same & before);
    const unsigned long long opens = __ballot(rank % TILE == 0) & all;
    const unsigned long long mine = __ballot((int)__popcll(opens & before) == t) & opens;
    if (!mine) return TileOf{-2, 0, 0, 0};
    const int at = __builtin_ctzll(mine), expert = __builtin_amdgcn_readlane(id, at), first = __builtin_amdgcn_readlane(rank, at);
    const unsigned long long members = __ballot(id == expert && rank >= first && rank < first + TILE) & all;
    return TileOf{expert < p.experts ? expert : -1, (int)__popcll(members), 0, members};
}
// Its slots to `list`, the last one again where there are fewer than TILE: by each wave for itself, all the same
template <int TILE>
__device__ __forceinline__ void tile_slots(const ExpertArgs& p, const TileOf& tile, int* list) {
    const int lane = threadIdx.x & 63;
    if (p.sorted) {
        const int* order = sorted_order(p.sorted, p.tiles) + tile.begin;
        for (int i = lane; i < TILE; i += 64) list[i] = order[i < tile.used ? i : tile.used - 1];
    } else {
        const int place = __popcll(tile.members & ((1ull << lane) - 1ull)), last = 63 - __builtin_clzll(tile.members);
        if ((tile.members >> lane) & 1ull) list[place] = lane;
        for (int i = lane; i < TILE; i += 64) if (i >= tile.used) list[i] = last;
    }
    __builtin_amdgcn_wave_barrier();
}

// The i-th of its slots to lane i, the last one again where there are fewer than 64
__device__ __forceinline__ int tile_slot(const ExpertArgs& p, const TileOf& tile) {
    const int lane = threadIdx.x & 63;
    if (p.sorted) return sorted_order(p.sorted, p.tiles)[tile.begin + (lane < tile.used ? lane : tile.used - 1)];
    const unsigned long long before = (1ull << lane) - 1ull;
    const int to = (tile.members >> lane) & 1ull ? __popcll(tile.members & before) : tile.used + __popcll(~tile.members & before);       // (a place for every lane)
    const int slot = __builtin_amdgcn_ds_permute(to * 4, lane);
    return lane < tile.used ? slot : __builtin_amdgcn_readlane(slot, tile.used - 1);
}
// The same for up to kSomeSlots, by the workgroup: the slots of each expert are counted (cnt: experts + 1 places, the last for empty slots), tiles are
// numbered by expert, and the slots of a tile follow in their order.  Against the sorting's dispatch: 8 of 64 experts of 2048 columns, 1536 outputs in 8
// bits, 72 slots 34 -> 27 us, 512 slots 46 -> 42; with more than a round of workgroups to count for themselves 1024 slots in bf16 87 -> 90, and with 1024
// experts' counts 35 -> 56; in one round 1000 slots of 8 experts of 512 columns, 512 outputs 13.4 -> 9.1.
constexpr int kSomeSlots = 1024;
template <int TILE, int THREADS>
__device__ __forceinline__ TileOf counted_tile(const ExpertArgs& p, int t, int* cnt, unsigned short* ids, int* list, int& slot) {
    constexpr int kEach = kSomeSlots / THREADS;
    static_assert(kEach * THREADS == kSomeSlots && TILE <= 64, "slots, lanes");
    const Routed* r = operand<Routed>(p.r, p.slots, 2);
    const int slots = p.rows * p.k, lane = threadIdx.x & 63, buckets = p.experts + 1;
    int e[kEach];
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        const int s = i * THREADS + threadIdx.x;
        e[i] = s < slots ? r[s].expert : 0;
    }
    for (int i = threadIdx.x; i < buckets; i += THREADS) cnt[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        const int s = i * THREADS + threadIdx.x, id = (unsigned)e[i] < (unsigned)p.experts ? e[i] : p.experts;
        if (s >= slots) continue;
        ids[s] = (unsigned short)id;
        atomicAdd(&cnt[id], 1);
    }
    __syncthreads();
    int expert = -2, first = 0, used = 0, base = 0;
    for (int b0 = 0; b0 < buckets && expert == -2; b0 += 64) {       // (uniform)
        const int c = b0 + lane < buckets ? cnt[b0 + lane] : 0, n = (c + TILE - 1) / TILE;
        int upto = n;
        for (int d = 1; d < 64; d <<= 1) {
            const int a = __shfl_up(upto, d);
            if (lane >= d) upto += a;
        }
        const unsigned long long beyond = __ballot(base + upto > t);
        if (beyond) {
            const int l = __builtin_ctzll(beyond);
            expert = b0 + l;
            first = (t - base - __builtin_amdgcn_readlane(upto - n, l)) * TILE;
            used = __builtin_amdgcn_readlane(c, l) - first;
            used = used < TILE ? used : TILE;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    if (expert == -2) return TileOf{-2, 0, 0, 0};
    int rank = -first;
    for (int s0 = 0; s0 < slots; s0 += 64) {
        const int id = s0 + lane < slots ? ids[s0 + lane] : -1;
        const unsigned long long same = __ballot(id == expert);
        const int at = rank + __popcll(same & ((1ull << lane) - 1ull));
        if (id == expert && at >= 0 && at < used) list[at] = s0 + lane;          // (by each wave, the same)
        rank += __popcll(same);
    }
    __syncthreads();                                         // (what comes next takes the counts' place)
    slot = list[lane < used ? lane : used - 1];
    return TileOf{expert < p.experts ? expert : -1, used, 0, 0};
}

__device__ const v4u kZeros[1] = {{0u, 0u, 0u, 0u}};
// 16 bytes a lane from global memory into LDS, lane l's at `to` + 16 l
__device__ __forceinline__ void direct_to_lds(const unsigned char* base /* uniform */, unsigned off, char* to /* uniform */) {
    __builtin_amdgcn_global_load_lds((const void PG_GLOBAL*)((const char PG_GLOBAL*)(uintptr_t)base + off), (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
__device__ __forceinline__ void word_to_lds(const unsigned char* base /* uniform */, unsigned off, char* to /* uniform */) {
    __builtin_amdgcn_global_load_lds((const void PG_GLOBAL*)((const char PG_GLOBAL*)(uintptr_t)base + off), (__attribute__((address_space(3))) void*)to, 4, 0, 0);
}
__device__ __forceinline__ void word_to_lds(const unsigned char* from, char* to /* uniform */) {
    __builtin_amdgcn_global_load_lds((const void PG_GLOBAL*)(uintptr_t)from, (__attribute__((address_space(3))) void*)to, 4, 0, 0);
}
// (the address as it is: some lanes' is not the tensor's)
__device__ __forceinline__ void direct_to_lds(const unsigned char* from, char* to /* uniform */) {
    __builtin_amdgcn_global_load_lds((const void PG_GLOBAL*)(uintptr_t)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
__device__ __forceinline__ v4u row8_shifted(const bf16_t* row, int c, int cols) {
    const v4u v = row8_raw(row, c, cols);
    return c + 8 <= cols ? v : row8_fix(v, c, cols);
}
// The fragments of N tiles of 16 rows, 2 KB apart, of pieces at `a` and at `b`: read and waited for in one piece of assembly (reads of LDS that the
// compiler places behind loads into LDS wait for all of those first)
template <int N>
__device__ __forceinline__ void lds_frags(unsigned a, unsigned b, v4u (&f)[N][2]) {
    static_assert(N == 1 || N == 2 || N == 4, "tiles");
    if constexpr (N == 1)
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(f[0][0]), "=&v"(f[0][1]) : "v"(a), "v"(b) : "memory");
    else if constexpr (N == 2)
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:2048\n\tds_read_b128 %3, %5 offset:2048\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0][0]), "=&v"(f[0][1]), "=&v"(f[1][0]), "=&v"(f[1][1]) : "v"(a), "v"(b) : "memory");
    else
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %8 offset:2048\n\tds_read_b128 %3, %9 offset:2048\n\t"
                     "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %9 offset:4096\n\tds_read_b128 %6, %8 offset:6144\n\tds_read_b128 %7, %9 offset:6144\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(f[0][0]), "=&v"(f[0][1]), "=&v"(f[1][0]), "=&v"(f[1][1]), "=&v"(f[2][0]), "=&v"(f[2][1]), "=&v"(f[3][0]), "=&v"(f[3][1])
                     : "v"(a), "v"(b) : "memory");
}
__device__ __forceinline__ unsigned lds_address(const char* p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }

// N bytes, 64 bytes apart
template <int N>
__device__ __forceinline__ void lds_bytes(unsigned at, unsigned (&v)[N]) {
    static_assert(N == 1 || N == 2 || N == 4, "tiles");
    if constexpr (N == 1) asm volatile("ds_read_u8 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v[0]) : "v"(at) : "memory");
    else if constexpr (N == 2)
        asm volatile("ds_read_u8 %0, %2\n\tds_read_u8 %1, %2 offset:64\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v[0]), "=&v"(v[1]) : "v"(at) : "memory");
    else
        asm volatile("ds_read_u8 %0, %4\n\tds_read_u8 %1, %4 offset:64\n\tds_read_u8 %2, %4 offset:128\n\tds_read_u8 %3, %4 offset:192\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]) : "v"(at) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Products with few rows for an expert, where what bounds it is the way of the weights: a workgroup takes 16 * JT outputs of up to 16 * MT rows of h, its NW
// waves the steps of K in turn (128 columns; 64 where the weights are bf16), each through a ring of S steps in its own part of LDS, with no barrier
// until the partial sums meet.  Loads go by whole lines of eight rows, straight into LDS: as fragments in registers, neighbouring lanes took
// 16 bytes of a row each, and a load the time of 64 lines (64 rows of 4096 columns 16 us for any number of outputs).  With 8-bit weights 16 rows of 4096
// columns, 16384 outputs 12.6 us, 5.4 TB/s; 256 slots of 64 experts of 2048 columns, 1536 outputs 37 us, 5.4 TB/s, and 73 in bf16, 5.5 TB/s.
template <Form FORM, bool ROUTED, int MT, int JT, int S, int NW>
__global__ __launch_bounds__(NW * 64, (150 * 1024 / (S * NW * ((FORM == kW8H16 ? 2 : 1) * MT + JT) * 2048) > 1 ? 2 : 1) * NW / 4) void k_product(ExpertArgs p) {
    constexpr bool W8 = FORM != kW16H16, H8 = FORM == kW8H8 || FORM == kW8H8Wide;
    constexpr int TILE = 16 * MT, OUTS = 16 * JT, kStep = W8 ? 128 : 64;
    constexpr int HS = W8 && !H8 ? 2 : 1;                     // pieces of 128 bytes that a row of h has of a step
    constexpr int QH = HS * MT * 2, QW = JT * 2, kLoads = QH + QW + (H8 ? 1 : 0);
    constexpr int kHBytes = QH * 1024, kStage = (QH + QW) * 1024 + (H8 ? 256 : 0);
    constexpr int kRing = NW * S * kStage, kParts = NW * TILE * (OUTS + 1) * 4;
    __shared__ __attribute__((aligned(128))) char lds[kRing > kParts ? kRing : kParts];
    __shared__ int list[TILE];
    __shared__ unsigned short ids[ROUTED ? kSomeSlots : 1];
    static_assert(sizeof lds >= (kSortMostExperts + 1) * sizeof(int), "counts");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, quad = lane >> 4;
    const int jt = (p.n + OUTS - 1) / OUTS;
    const int t = (int)(blockIdx.x / (unsigned)jt), j0 = (int)(blockIdx.x % (unsigned)jt) * OUTS;
    TileOf tile{0, p.rows - t * TILE < TILE ? p.rows - t * TILE : TILE, 0, 0};
    int slot = 0;                                             // lane i: the tile's i-th
    if constexpr (ROUTED) {
        const bool counted = !p.sorted && p.rows * p.k > kFewSlots;
        tile = counted ? counted_tile<TILE, NW * 64>(p, t, (int*)lds, ids, list, slot) : routed_tile<TILE>(p, t);
        if (tile.expert == -2) return;
        if (!counted) slot = tile_slot(p, tile);            // (of the sorted ones: waited for when the weights are on their way)
    }
    f32x4 acc[MT][JT];
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int j = 0; j < JT; j++) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!ROUTED || tile.expert >= 0) {
        const int nk = (p.cols + kStep - 1) / kStep, nb = (p.cols + kScaleBlock - 1) / kScaleBlock, nb4 = up_to(nb, 4);
        const long long kp = (long long)nb * kScaleBlock, wpitch = W8 ? kp : 2ll * p.cols, hpitch = H8 ? kp : 2ll * p.cols;
        const unsigned char* W = operand<unsigned char>(p.W, p.slots, 0);
        const unsigned char* h = operand<unsigned char>(p.h, p.slots, 1);
        const float* scales = (const float*)(W + (long long)p.experts * p.n * kp) + ((long long)tile.expert * ((p.n + kScaleBlock - 1) / kScaleBlock) + j0 / kScaleBlock) * nb;
        const int hrows = ROUTED && p.per_slot ? p.rows * p.k : p.rows;
        // (from the register: a read of LDS would wait for the weights)
        const int lane_row = ROUTED && !p.per_slot ? slot / p.k : ROUTED ? slot : t * TILE + (lane < tile.used ? lane : tile.used - 1);
        auto hrow = [&](int i) { return (long long)__shfl(lane_row, i); };
        // lane l of a load takes the 16-byte piece (l & 7) ^ (l >> 3) of row l >> 3 of its eight: fragment reads of eight lanes touch every bank once
        const int piece = (lane & 7) ^ (lane >> 3);
        const unsigned char *hp[MT * 2], *wp[QW], *hs = h;
#pragma unroll
        for (int q = 0; q < QW; q++) {
            const int j = j0 + q * 8 + (lane >> 3);
            wp[q] = W + ((long long)tile.expert * p.n + (j < p.n ? j : p.n - 1)) * wpitch;
        }
        char* const mine = lds + wave * (S * kStage);
        const unsigned mine0 = lds_address(mine);
        const int f0 = l16 * 128 + ((quad ^ (l16 & 7)) * 16), f1 = l16 * 128 + (((quad + 4) ^ (l16 & 7)) * 16);
        const int g0 = HS == 1 ? f0 : l16 * 128 + (((2 * quad) ^ (l16 & 7)) * 16), g1 = HS == 1 ? f1 : l16 * 128 + (((2 * quad + 1) ^ (l16 & 7)) * 16);
        // The wave's steps: wave, wave + NW, ..., begun at another place by neighbouring workgroups of an XCD (rows of a power of two long have a
        // column in few memory channels).  By the outputs alone: a slot's sums may not depend on the tile that it is sorted into.
        const int turn = (int)((unsigned)(j0 / OUTS >> 3) * NW % (unsigned)nk), mine_n = (nk - wave + NW - 1) / NW;
        auto step = [&](int b) { const int k = wave + NW * b + turn; return k < nk ? k : k - nk; };
        // way: 0 straight into LDS; 1 by way of registers; 2 the same, rows shorter than 16 bytes
        constexpr int kRegs = (W8 ? 0 : QW) + (H8 ? 0 : QH);
        auto bf16_piece = [&](auto way, const unsigned char* row, int k, int more, char* dst, v4u* held) {
            constexpr int kWay = decltype(way)::value;
            const int c = k * kStep + more + piece * 8;
            if constexpr (kWay == 0) direct_to_lds((k + 1) * kStep <= p.cols || c < p.cols ? row + 2ll * c : (const unsigned char*)kZeros, dst);
            else *held = kWay == 1 ? row8_shifted((const bf16_t*)row, c, p.cols) : row8_short((const bf16_t*)row, c, p.cols);
        };
        auto issue_weights = [&](auto way, int b, char* to, v4u* held) {
            const int k = step(b);
#pragma unroll
            for (int q = 0; q < QW; q++) {
                if constexpr (W8) direct_to_lds(wp[q] + (long long)k * 128 + piece * 16, to + kHBytes + q * 1024);
                else bf16_piece(way, wp[q], k, 0, to + kHBytes + q * 1024, held + q);
            }
        };
        auto issue_rows = [&](auto way, int b, char* to, v4u* held) {
            const int k = step(b);
            if constexpr (H8) word_to_lds(hs + (k & ~3), to + kHBytes + QW * 1024);
#pragma unroll
            for (int q = 0; q < QH; q++) {
                if constexpr (H8) direct_to_lds(hp[q] + (long long)k * 128 + piece * 16, to + q * 1024);
                else bf16_piece(way, hp[q % (MT * 2)], k, q / (MT * 2) * 64, to + q * 1024, held + (W8 ? 0 : QW) + q);
            }
        };
        auto put = [&](char* to, const v4u* held) {            // what came through registers
#pragma unroll
            for (int q = 0; q < kRegs; q++) {
                const int at = W8 ? q : q < QW ? QH + q : q - QW;          // (weights first)
                *(v4u*)(to + at * 1024 + lane * 16) = held[q];
            }
        };
        float scale64 = 0.f;                                   // lane l: the scale of the wave's step l of 64
        auto load_scales = [&](int b) { if (W8) scale64 = *(const float PG_GLOBAL*)(uintptr_t)(scales + step(b + lane < mine_n ? b + lane : mine_n - 1)); };
        auto stream = [&](auto way) {
            constexpr bool kDirect = decltype(way)::value == 0;
            // Steps on their way: a ring of S in LDS; or in registers, as many as they have room for, and 8-bit weights beside them in the ring's places
            constexpr int kAhead = kDirect ? S : kRegs <= 10 && S >= 2 ? 2 : 1;
            v4u held[kDirect ? 1 : kAhead][kRegs ? kRegs : 1];
            if (mine_n > 0) {
                load_scales(0);
#pragma unroll
                for (int b = 0; b < kAhead; b++) if (b < mine_n) issue_weights(way, b, mine + b * kStage, held[kDirect ? 0 : b]);
            }
#pragma unroll
            for (int q = 0; q < MT * 2; q++) hp[q] = h + hrow(q * 8 + (lane >> 3)) * hpitch;
            if constexpr (H8) hs = h + hrows * kp + hrow(lane % TILE) * nb4;
#pragma unroll
            for (int b = 0; b < kAhead; b++) if (b < mine_n) issue_rows(way, b, mine + b * kStage, held[kDirect ? 0 : b]);
            asm volatile("" : "+v"(scale64));                  // (waits for the scales here, not at each use for whatever was loaded behind them)
            int at = 0;
#pragma unroll 1
            for (int b0 = 0; b0 < mine_n; b0 += kDirect ? 1 : kAhead)
#pragma unroll
            for (int u = 0; u < (kDirect ? 1 : kAhead); u++) {
                const int b = b0 + u;
                if (!kDirect && b >= mine_n) break;
                if (W8 && b && (b & 63) == 0) {
                    load_scales(b);
                    asm volatile("" : "+v"(scale64));
                }
                if constexpr (kDirect) {
                    if (kAhead > 1 && b && b + kAhead <= mine_n) wait_loads<(kAhead - 1) * kLoads>();      // (at first rows come behind all steps' weights)
                    else wait_loads<0>();
                } else {
                    put(mine + at, held[u]);                   // (waits for this step's registers; 8-bit weights came before them)
                    if constexpr (W8) {
                        if (b + 1 < mine_n && kAhead > 1) wait_loads<QW + kRegs>();
                        else wait_loads<0>();
                    }
                }
                const unsigned now = mine0 + (unsigned)at;
                unsigned exps[MT];
                if constexpr (H8) lds_bytes<MT>(now + kHBytes + QW * 1024 + l16 * 4 + (step(b) & 3), exps);
                v4u hf[HS][MT][2], wf[JT][2];
#pragma unroll
                for (int q = 0; q < HS; q++) lds_frags<MT>(now + q * MT * 2048 + g0, now + q * MT * 2048 + g1, hf[q]);
                lds_frags<JT>(now + kHBytes + f0, now + kHBytes + f1, wf);
                if (b + kAhead < mine_n) {                     // (what was there has been read)
                    issue_weights(way, b + kAhead, mine + at, held[kDirect ? 0 : u]);
                    issue_rows(way, b + kAhead, mine + at, held[kDirect ? 0 : u]);
                }
                at = at + kStage == (kDirect ? S : kAhead) * kStage ? 0 : at + kStage;
                const float s = W8 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(scale64), b & 63)) : 1.f;
#pragma unroll
                for (int j = 0; j < JT; j++) {
                    if constexpr (FORM == kW8H8) {
                        const v4u a0 = wf[j][0], a1 = wf[j][1];
                        const v8i A = {(int)a0.x, (int)a0.y, (int)a0.z, (int)a0.w, (int)a1.x, (int)a1.y, (int)a1.z, (int)a1.w};
#pragma unroll
                        for (int m = 0; m < MT; m++) {
                            const v4u b0 = hf[0][m][0], b1 = hf[0][m][1];
                            const v8i B = {(int)b0.x, (int)b0.y, (int)b0.z, (int)b0.w, (int)b1.x, (int)b1.y, (int)b1.z, (int)b1.w};
                            const f32x4 sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 127, 0, (int)exps[m]);
#pragma unroll
                            for (int i = 0; i < 4; i++) acc[m][j][i] = __builtin_fmaf(s, sum[i], acc[m][j][i]);
                        }
                    } else if constexpr (FORM == kW16H16) {
#pragma unroll
                        for (int m = 0; m < MT; m++)
#pragma unroll
                            for (int q = 0; q < 2; q++) acc[m][j] = mfma_bf16(wf[j][q], hf[0][m][q], acc[m][j]);
                    } else {
                        v4u A[4];
#pragma unroll
                        for (int q = 0; q < 4; q++) A[q] = half_to_bf16(wf[j][q >> 1], q & 1);
#pragma unroll
                        for (int m = 0; m < MT; m++) {
                            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int q = 0; q < 4; q++) sum = mfma_bf16(A[q], H8 ? half_to_bf16(hf[0][m][q >> 1], q & 1) : hf[HS == 2 ? q >> 1 : 0][m][q & 1], sum);
                            const float by = H8 ? __builtin_ldexpf(s, (int)exps[m] - 127) : s;
#pragma unroll
                            for (int i = 0; i < 4; i++) acc[m][j][i] = __builtin_fmaf(by, sum[i], acc[m][j][i]);
                        }
                    }
                }
            }
        };
        // (uniform) can 16-byte loads into LDS reach the bf16 rows?
        if ((W8 && H8) || (p.cols % 8 == 0 && aligned_to(h, 16) && (W8 || aligned_to(W, 16)))) stream(std::integral_constant<int, 0>{});
        else if constexpr (!(W8 && H8)) {
            if (MT > 1 || JT > 1 || p.cols >= 8) stream(std::integral_constant<int, 1>{});
            else if constexpr (MT == 1 && JT == 1) stream(std::integral_constant<int, 2>{});         // (plan_experts)
        }
    }
    if constexpr (FORM == kW16H16) sums_drained(acc);
    if (ROUTED && (int)threadIdx.x < TILE) list[threadIdx.x] = slot;
    __syncthreads();                                           // every wave has read its steps
    float* const part = (float*)lds;                           // [NW][TILE][OUTS + 1]
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int j = 0; j < JT; j++)
#pragma unroll
            for (int i = 0; i < 4; i++) part[(wave * TILE + m * 16 + l16) * (OUTS + 1) + j * 16 + quad * 4 + i] = acc[m][j][i];
    __syncthreads();
    for (int i = threadIdx.x; i < TILE * OUTS; i += NW * 64) {
        const int m = i / OUTS, c = i % OUTS;
        if (m >= tile.used || j0 + c >= p.n) continue;
        float y = part[m * (OUTS + 1) + c];
#pragma unroll
        for (int w = 1; w < NW; w++) y += part[(w * TILE + m) * (OUTS + 1) + c];
        const long long at = (long long)(ROUTED ? list[m] : t * TILE + m) * p.n + j0 + c;
        if (p.out_f32) ((float*)p.out)[at] = y;
        else ((bf16_t*)p.out)[at] = (bf16_t)f32_to_bf16(y);
    }
}

// ---- large products -----------------------------------------------------------------------------------------
// Workgroup b of `total` in an order that gives each of the eight XCDs (workgroups go to them in turn) a stretch of neighbours: they share
// rows and weights in its L2.
__device__ __forceinline__ unsigned neighbours(unsigned b, unsigned total) {
    const unsigned x = b & 7u, each = total >> 3, more = total & 7u;
    return x * each + (x < more ? x : more) + (b >> 3);
}
// WR x WJ waves, each RM x JN tiles of 16 rows x 16 outputs, over K in steps of 128 columns (64 where the weights are bf16), S steps in LDS: S - 1 on
// their way while one is multiplied.  A block's sum comes from the matrix instruction, times the rows' exponents, and the weights' scale joins it on its way
// to the fp32 accumulator.  4096 x 4096 x 4096 with both operands in 8 bits: 67 us, 2.04 PFLOP/s of the 2.6 that a large product without scales reaches;
// the matrix cores are busy 45 % of it.  What bounds it: a step of 256 x 256 takes its fragments through LDS in about the time that it multiplies
// (256 KB at 128 bytes a clock, 2048 clocks either way), and the two overlap in part; and 16 us before the first step and behind the last, the store of 33 MB
// among them.  bf16 rows beside 8-bit weights become twice the LDS bytes and half the rate: 130 us, 1.06 PFLOP/s; an fp32 output of 8-bit rows 135 us.
template <Form FORM, bool ROUTED, int RM, int JN, int WR, int WJ, int S>
__global__ __launch_bounds__(WR * WJ * 64, 2) void k_product_tile(ExpertArgs p) {
    constexpr bool W8 = FORM != kW16H16, H8 = FORM == kW8H8 || FORM == kW8H8Wide;
    constexpr int NW = WR * WJ, BM = RM * 16 * WR, BN = JN * 16 * WJ;
    constexpr int kStep = W8 ? 128 : 64;                      // columns
    constexpr int HS = W8 && !H8 ? 2 : 1;                     // pieces of 128 bytes that a row of h has of a step
    constexpr int kHBytes = HS * BM * 128, kStage = kHBytes + BN * 128;
    constexpr int QH = HS * BM / 8 / NW, QW = BN / 8 / NW;    // loads of eight rows for each wave
    static_assert(QH * 8 * NW == HS * BM && QW * 8 * NW == BN && (128 % (JN * 16)) == 0, "whole loads; a wave's outputs share their scale");
    constexpr int kLoads = QH + QW + (H8 ? 1 : 0);            // a wave's loads of a step
    static_assert(S >= 2 && S <= 8 && BM % 64 == 0, "exponents: of four steps at a time, in four places");
    __shared__ __attribute__((aligned(128))) char lds[S * kStage];
    __shared__ int slot_of[BM];
    __shared__ __attribute__((aligned(16))) char lds_exps[4][H8 ? BM * 4 : 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quad = lane >> 4;
    const int jt = (p.n + BN - 1) / BN;
    int t = 0, jb = 0;
    {
        if (ROUTED) {
            // Sixteen tiles at a time, two to each XCD, which mostly are one expert's, with all their outputs; the last ones, fewer than sixteen, in
            // stretches like a plain product's.  How many there are at least follows from the slots; the others ask.
            unsigned b = blockIdx.x, of16 = (unsigned)(p.rows * p.k / BM / 16 * 16) * jt;
            if (b >= of16) {
                const int n = p.sorted ? ((const SortedSlots*)p.sorted)->n_tiles : p.tiles;
                of16 = (unsigned)(n / 16 * 16) * jt;
                if (b >= (unsigned)n * jt) return;
                if (b >= of16) {
                    const unsigned u = neighbours(b - of16, (unsigned)n * jt - of16), pair = u / (2u * jt), in = u % (2u * jt), first = n / 16 * 16 + 2u * pair;
                    const unsigned two = (unsigned)n - first < 2u ? 1u : 2u;
                    t = (int)(first + in % two);
                    jb = (int)(in / two);
                }
            }
            if (b < of16) {
                const unsigned in = (b >> 3) % (2u * jt);
                t = (int)((b >> 3) / (2u * jt) * 16 + (b & 7u) * 2 + (in & 1u));
                jb = (int)(in >> 1);
            }
        } else {                                             // four tiles of rows, then the next outputs: a stretch is about square
            const unsigned u = neighbours(blockIdx.x, gridDim.x);
            const unsigned group = u / (4u * jt), in = u % (4u * jt), first = 4u * group, rows4 = (unsigned)p.tiles - first < 4u ? (unsigned)p.tiles - first : 4u;
            t = (int)(first + in % rows4);
            jb = (int)(in / rows4);
        }
    }
    const int begin = t * BM;
    TileOf tile{0, p.rows - begin < BM ? p.rows - begin : BM, 0, 0};
    if constexpr (ROUTED) {
        tile = routed_tile<BM>(p, t);
        if (tile.expert == -2) return;
        tile_slots<BM>(p, tile, slot_of);
    } else {
        for (int i = lane; i < BM; i += 64) slot_of[i] = begin + (i < tile.used ? i : tile.used - 1);
        __builtin_amdgcn_wave_barrier();
    }
    const int expert = tile.expert, used = tile.used;
    const int j0 = jb * BN, wr = wave / WJ, wj = wave % WJ;      // (waves w and w + 4 share a SIMD: other rows, of which a small tile may have none)
    const int nk = (p.cols + kStep - 1) / kStep, nb = (p.cols + kScaleBlock - 1) / kScaleBlock, nb4 = up_to(nb, 4);
    const long long kp = (long long)nb * kScaleBlock;
    f32x4 acc[RM][JN];
#pragma unroll
    for (int i = 0; i < RM; i++)
#pragma unroll
        for (int j = 0; j < JN; j++) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!ROUTED || expert >= 0) {
        const long long wpitch = W8 ? kp : 2ll * p.cols, hpitch = H8 ? kp : 2ll * p.cols;
        const unsigned char* W = operand<unsigned char>(p.W, p.slots, 0);
        const unsigned char* h = operand<unsigned char>(p.h, p.slots, 1);
        const int jblocks = (p.n + kScaleBlock - 1) / kScaleBlock, jblock = (j0 + wj * JN * 16) / kScaleBlock;
        const float* scales = (const float*)(W + (long long)p.experts * p.n * kp) + ((long long)expert * jblocks + (jblock < jblocks ? jblock : jblocks - 1)) * nb;
        const int hrows = ROUTED && p.per_slot ? p.rows * p.k : p.rows;
        // rows as offsets of 32 bits from the first row of the tile, or where rows are gathered from that of the tensor (plan_experts)
        const long long first = ROUTED ? 0 : begin;
        auto hrow = [&](int i) { const int s = slot_of[i]; return (unsigned)(ROUTED && !p.per_slot ? s / p.k : ROUTED ? s : s - begin); };
        W += ((long long)expert * p.n + j0) * wpitch;
        const unsigned char* hs = h + hrows * kp + first * nb4;
        h += first * hpitch;
        // loading: lane l of a load takes the 16-byte piece (l & 7) ^ (l >> 3) of row l >> 3 of its eight, and puts it to place l & 7: fragment
        // reads of eight neighbouring lanes touch every bank once
        const int piece = (lane & 7) ^ (lane >> 3);
        unsigned hp[QH], wp[QW];
#pragma unroll
        for (int q = 0; q < QH; q++) hp[q] = hrow(((wave * QH + q) * 8 + (lane >> 3)) % BM) * (unsigned)hpitch + (H8 ? piece * 16 : 0);
#pragma unroll
        for (int q = 0; q < QW; q++) {
            const int j = (wave * QW + q) * 8 + (lane >> 3), last = p.n - 1 - j0;
            wp[q] = (unsigned)(j < last ? j : last) * (unsigned)wpitch + (W8 ? piece * 16 : 0);
        }
        // the word of a row's exponents that step k's is in; every wave has a load of every step, so that all count the same
        const int exps_rows = wave % (BM / 64);
        const unsigned exps_at = H8 ? hrow(exps_rows * 64 + lane) * (unsigned)nb4 : 0u;
        auto load_exps = [&](int k) { word_to_lds(hs + (k & ~3), exps_at, lds_exps[(k >> 2) & 3] + exps_rows * 256); };
        // (uniform) can 16-byte loads into LDS reach the bf16 rows?
        const bool direct = (W8 && H8) || (p.cols % 8 == 0 && aligned_to(h, 16) && (W8 || aligned_to(W, 16)));
        constexpr int kRegs = (H8 ? 0 : QH) + (W8 ? 0 : QW);
        v4u held[kRegs ? kRegs : 1];
        auto issue = [&](auto way, int k, char* to) {
            constexpr bool kDirect = decltype(way)::value;
            const bool inside = (k + 1) * kStep <= p.cols;     // (uniform)
            if constexpr (H8) load_exps(k);
#pragma unroll
            for (int q = 0; q < QH; q++) {
                const int at = (wave * QH + q) * 8;          // of HS * BM pieces of rows
                char* const dst = to + at * 128;
                if constexpr (H8) {
                    direct_to_lds(h + (long long)k * 128, hp[q], dst);
                } else {
                    const int c = k * kStep + (at / BM) * 64 + piece * 8;
                    if constexpr (kDirect) {
                        if (inside) direct_to_lds(h + 2ll * k * kStep, hp[q] + (unsigned)((at / BM) * 128 + piece * 16), dst);
                        else direct_to_lds(c < p.cols ? h + hp[q] + 2ll * c : (const unsigned char*)kZeros, dst);
                    } else held[q] = row8_shifted((const bf16_t*)(h + hp[q]), c, p.cols);
                }
            }
#pragma unroll
            for (int q = 0; q < QW; q++) {
                char* const dst = to + kHBytes + (wave * QW + q) * 1024;
                if constexpr (W8) {
                    direct_to_lds(W + (long long)k * 128, wp[q], dst);
                } else {
                    const int c = k * kStep + piece * 8;
                    if constexpr (kDirect) {
                        if (inside) direct_to_lds(W + 2ll * k * kStep, wp[q] + piece * 16u, dst);
                        else direct_to_lds(c < p.cols ? W + wp[q] + 2ll * c : (const unsigned char*)kZeros, dst);
                    } else held[(H8 ? 0 : QH) + q] = row8_shifted((const bf16_t*)(W + wp[q]), c, p.cols);
                }
            }
        };
        auto put_held = [&](auto way, char* to) {
            if constexpr (kRegs && !decltype(way)::value) {
                {
                    if constexpr (!H8)
#pragma unroll
                        for (int q = 0; q < QH; q++) *(v4u*)(to + (wave * QH + q) * 1024 + lane * 16) = held[q];
                    if constexpr (!W8)
#pragma unroll
                        for (int q = 0; q < QW; q++) *(v4u*)(to + kHBytes + (wave * QW + q) * 1024 + lane * 16) = held[(H8 ? 0 : QH) + q];
                }
            }
        };
        // where a lane finds its fragments: row l16 of a tile, pieces quad and quad + 4
        const int f0 = l16 * 128 + ((quad ^ (l16 & 7)) * 16), f1 = l16 * 128 + (((quad + 4) ^ (l16 & 7)) * 16);
        // ... and in rows of h in bf16 beside 8-bit weights the columns of those pieces: two pieces in each half of the step
        const int g0 = HS == 1 ? f0 : l16 * 128 + (((2 * quad) ^ (l16 & 7)) * 16), g1 = HS == 1 ? f1 : l16 * 128 + (((2 * quad + 1) ^ (l16 & 7)) * 16);
        // lane l: the scale of step l of 64
        float scale64 = 0.f;
        auto load_scales = [&](int k) { if (W8) scale64 = *(const float PG_GLOBAL*)(uintptr_t)(scales + (k + lane < nb ? k + lane : nb - 1)); };
        load_scales(0);
        const unsigned lds0 = lds_address(lds), exps0 = lds_address(lds_exps[0]) + (wr * RM * 16 + l16) * 4;
        constexpr int kPer = FORM == kW8H8 || FORM == kW16H16 ? 2 : 1;       // tiles of weights that are read at a time
        auto stream = [&](auto way) {
        constexpr int kAhead = decltype(way)::value ? S - 1 : 1;             // (rows that come through registers: one step)
#pragma unroll
        for (int k = 0; k < kAhead; k++) if (k < nk) issue(way, k, lds + k * kStage);
        put_held(way, lds);
        // (the compiler waits for the scales here, and not at each of their uses for whatever was loaded behind them)
        asm volatile("" : "+v"(scale64));
        int now_at = 0, next_at = kAhead * kStage;             // in LDS: this step, and the one to load
#pragma unroll 1
        for (int k = 0; k < nk; k++) {
            char* const next = lds + next_at;
            if (W8 && k && (k & 63) == 0) {
                load_scales(k);
                asm volatile("" : "+v"(scale64));
            }
            // this wave's loads of this step, which came before those of the steps behind it
            if (kAhead > 1 && k + kAhead - 1 < nk) wait_loads<(kAhead - 1) * kLoads>();
            else wait_loads<0>();
            lds_barrier();                                     // all waves' loads of this step are in, and the step before has been read
            if (k + kAhead < nk) issue(way, k + kAhead, next);
            const float s = W8 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(scale64), k & 63)) : 1.f;
            const unsigned now = lds0 + (unsigned)now_at;
            now_at = now_at + kStage == S * kStage ? 0 : now_at + kStage;
            next_at = next_at + kStage == S * kStage ? 0 : next_at + kStage;
            unsigned exps[RM];
            if constexpr (H8) lds_bytes<RM>(exps0 + ((k >> 2) & 3) * (BM * 4) + (k & 3), exps);
            if (wr * RM * 16 < used) {
            v4u hf[HS][RM][2];
#pragma unroll
            for (int q = 0; q < HS; q++) lds_frags<RM>(now + (q * BM + wr * RM * 16) * 128 + g0, now + (q * BM + wr * RM * 16) * 128 + g1, hf[q]);
#pragma unroll
            for (int jp = 0; jp < JN; jp += kPer) {
                v4u wf[kPer][2];
                const unsigned at = now + kHBytes + (wj * JN + jp) * 16 * 128;
                lds_frags<kPer>(at + f0, at + f1, wf);
#pragma unroll
                for (int jj = 0; jj < kPer; jj++) {
                    const int j = jp + jj;
                    if constexpr (FORM == kW8H8) {
                        const v4u a0 = wf[jj][0], a1 = wf[jj][1];
                        const v8i A = {(int)a0.x, (int)a0.y, (int)a0.z, (int)a0.w, (int)a1.x, (int)a1.y, (int)a1.z, (int)a1.w};
#pragma unroll
                        for (int i = 0; i < RM; i++) {
                            const v4u b0 = hf[0][i][0], b1 = hf[0][i][1];
                            const v8i B = {(int)b0.x, (int)b0.y, (int)b0.z, (int)b0.w, (int)b1.x, (int)b1.y, (int)b1.z, (int)b1.w};
                            const f32x4 sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 127, 0, (int)exps[i]);
#pragma unroll
                            for (int e = 0; e < 4; e++) acc[i][j][e] = __builtin_fmaf(s, sum[e], acc[i][j][e]);
                        }
                    } else if constexpr (FORM == kW16H16) {
#pragma unroll
                        for (int i = 0; i < RM; i++)
#pragma unroll
                            for (int q = 0; q < 2; q++) acc[i][j] = mfma_bf16(wf[jj][q], hf[0][i][q], acc[i][j]);
                    } else {
                        v4u A[4];
#pragma unroll
                        for (int q = 0; q < 4; q++) A[q] = half_to_bf16(wf[jj][q >> 1], q & 1);
#pragma unroll
                        for (int i = 0; i < RM; i++) {
                            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int q = 0; q < 4; q++) sum = mfma_bf16(A[q], H8 ? half_to_bf16(hf[0][i][q >> 1], q & 1) : hf[HS == 2 ? q >> 1 : 0][i][q & 1], sum);
                            const float by = H8 ? __builtin_ldexpf(s, (int)exps[i] - 127) : s;
#pragma unroll
                            for (int e = 0; e < 4; e++) acc[i][j][e] = __builtin_fmaf(by, sum[e], acc[i][j][e]);
                        }
                    }
                }
            }
            }
            put_held(way, next);
        }
        };
        if ((W8 && H8) || direct) stream(std::true_type{});
        else if constexpr (!(W8 && H8)) stream(std::false_type{});
    }
    // Out by whole pieces of rows: 16 rows of a wave at a time go through its own part of LDS (16 bytes between rows: other banks), 16 bytes a lane from there.
    if constexpr (FORM == kW16H16) sums_drained(acc);
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();                                           // the last step has been read
    auto emit = [&](auto* out) {
        using O = std::remove_pointer_t<decltype(out)>;
        constexpr int NV = 16 / (int)sizeof(O), kPitch = JN * 16 * (int)sizeof(O) + 16, kLanes = JN * 16 / NV, kRowsAt = 64 / kLanes;
        static_assert(NW * 16 * kPitch <= S * kStage, "the waves' parts");
        char* const mine = lds + wave * 16 * kPitch;
        const int c = j0 + wj * JN * 16 + lane % kLanes * NV;
#pragma unroll
        for (int i = 0; i < RM; i++) {
            if ((wr * RM + i) * 16 >= used) break;
#pragma unroll
            for (int j = 0; j < JN; j++) {
                char* const at = mine + l16 * kPitch + (j * 16 + quad * 4) * (int)sizeof(O);
                const f32x4 v = acc[i][j];
                if constexpr (sizeof(O) == 4) *(f32x4*)at = v;
                else *(uint2*)at = uint2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int q = 0; q < 16 / kRowsAt; q++) {
                const int r = q * kRowsAt + lane / kLanes, row = (wr * RM + i) * 16 + r;
                const v4u v = *(const v4u*)(mine + r * kPitch + lane % kLanes * 16);
                if (row >= used || c >= p.n) continue;
                O* o = out + (long long)slot_of[row] * p.n + c;
                if (c + NV <= p.n) *(v4u_any PG_GLOBAL*)(uintptr_t)o = v;
                else
#pragma unroll
                    for (int e = 0; e < NV; e++)
                        if (c + e < p.n) o[e] = (O)(sizeof(O) == 4 ? v[e & 3] : v[(e / 2) & 3] >> (16 * (e & 1)));
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (p.out_f32) emit((unsigned*)p.out);
    else emit((bf16_t*)p.out);
}

template <typename T, bool HIGH> const void* route_kernel(long long experts) {
    return experts <= 64 ? PG_FN(k_route<T, 1, HIGH>) : experts <= 128 ? PG_FN(k_route<T, 2, HIGH>) : experts <= 256 ? PG_FN(k_route<T, 4, HIGH>)
         : experts <= 512 ? PG_FN(k_route<T, 8, HIGH>) : PG_FN(k_route<T, 16, HIGH>);
}

constexpr long long kComputeUnits = 256;
struct TileKernel {
    Form form;
    const void* plain;
    const void* routed;
    int rows, outputs, threads;
    int round, both;        // what a round of up to 256 workgroups takes, and one of up to 512 where two fit a compute unit (0: they don't)
    long long workgroups(long long slots, long long experts, long long n) const {        // (slots that are spread evenly, and half a tile more for each expert)
        return (experts > 1 ? (2 * slots / rows + experts) / 2 : (slots + rows - 1) / rows) * ((n + outputs - 1) / outputs);
    }
    long long cost(long long wgs) const {
        const long long cap = both ? 2 * kComputeUnits : kComputeUnits, rest = wgs % cap;
        return wgs / cap * (both ? both : round) + (!rest ? 0 : rest <= kComputeUnits ? round : both);
    }
};
#define PG_TILE(F, RM, JN, WR, WJ, S, ROUND, BOTH) {F, PG_FN(k_product_tile<F, false, RM, JN, WR, WJ, S>), PG_FN(k_product_tile<F, true, RM, JN, WR, WJ, S>), RM * 16 * WR, JN * 16 * WJ, WR * WJ * 64, ROUND, BOTH}
// The large tiles do the most work to a byte that they load, but a round of them that the chip cannot fill takes as long as a full one.  What a round
// takes is measured, in us: 8-bit rows and bf16 beside 8-bit weights with 4096 columns, bf16 with 1024.  The cheapest of a form is taken.  4096 outputs:
// 1024 rows 30 us (8 waves), 2048 rows 41 (4 waves, two workgroups to a compute unit; 56 with 8 waves, 64 with the large tile), 4096 rows 67 (large; 79
// with 4 waves, 109 with 8).  bf16 slots: 5 of 7 experts for 2000 rows of 1024 columns, 512 outputs 30 (4 waves; 38 with 8), for 4086 rows of 3456 columns,
// 128 outputs 60 (8 waves; 74 with 4).
const TileKernel kTileKernels[] = {
    PG_TILE(kW8H8, 4, 8, 4, 2, 2, 67, 0), PG_TILE(kW8H8, 4, 4, 2, 2, 2, 32, 41), PG_TILE(kW8H8, 2, 4, 4, 2, 4, 30, 0),
    PG_TILE(kW8H16, 4, 4, 2, 4, 2, 65, 0), PG_TILE(kW8H16, 2, 4, 4, 2, 3, 45, 0),
    PG_TILE(kW16H16, 4, 8, 4, 2, 2, 36, 0), PG_TILE(kW16H16, 4, 4, 2, 2, 2, 20, 24), PG_TILE(kW16H16, 2, 4, 4, 2, 4, 16, 0),
    PG_TILE(kW8H8Wide, 4, 4, 2, 2, 2, 50, 65), PG_TILE(kW8H8Wide, 2, 4, 4, 2, 4, 48, 0),
};
// Where an expert has few rows, or a product makes fewer workgroups of the smallest tile than tiles_from, k_product, which splits K, is faster.  8 of 64 experts,
// 1536 outputs, k_product and these: 8 bits, 36 rows on the mean, 4096 columns 126 and 126 us, 50 rows 157 and 120; bf16, 50 rows 185 and 200, 62 rows 233
// and 203.  A short K leaves nothing to split: 256 columns, 17 rows 24 and 21 (bf16 beside 8 bits), 50 rows 37 and 24; 1024 columns, 25 rows 40 and 41
// (in a plain product not: 20 rows of 256 columns, 32768 outputs 5.7 and 6.0).  4096 x
// 4096 in 8 bits, 512 rows (128 workgroups): k_product 20 us, these 29; with bf16 rows 31 and 45.  Routed, 4 of 4 experts for 1133 rows of 768 columns, 512
// outputs (144 workgroups): 24 and 19; 2 of 4 for 300 of 2944 columns, 5760 outputs (270) 46 and 37, with an fp32 output 51 and 59.
constexpr int kTilesRows = 128;
constexpr long long tiles_mean(bool routed, Form form, long long cols) { return routed && cols <= 512 ? 16 : form == kW16H16 ? 57 : 43; }
constexpr long long tiles_from(bool routed, Form form) { return form == kW8H16 ? 256 : !routed ? 192 : form == kW8H8Wide ? 320 : 128; }

struct RowsKernel {
    Form form;
    const void* plain;
    const void* routed;
    int rows, outputs, threads;
};
#define PG_ROWS(F, MT, JT, S, NW) {F, PG_FN(k_product<F, false, MT, JT, S, NW>), PG_FN(k_product<F, true, MT, JT, S, NW>), 16 * MT, 16 * JT, NW * 64}
const RowsKernel kRowsKernels[] = {
    // MT, JT, S: steps in the ring, as many as leave three workgroups (two beside four tiles of both) room in a compute unit's LDS: more steps with fewer
    // workgroups are slower (64 slots of 64 experts in 8 bits, two steps of one workgroup 25 us, one step of three 17.5).
    PG_ROWS(kW16H16, 1, 1, 4, 4), PG_ROWS(kW16H16, 1, 2, 2, 4), PG_ROWS(kW16H16, 1, 4, 1, 4), PG_ROWS(kW16H16, 2, 1, 2, 4), PG_ROWS(kW16H16, 2, 2, 2, 4), PG_ROWS(kW16H16, 2, 4, 1, 4), PG_ROWS(kW16H16, 4, 1, 1, 4), PG_ROWS(kW16H16, 4, 2, 1, 4), PG_ROWS(kW16H16, 4, 4, 1, 4),
    PG_ROWS(kW8H16, 1, 1, 3, 4), PG_ROWS(kW8H16, 1, 2, 2, 4), PG_ROWS(kW8H16, 1, 4, 1, 4), PG_ROWS(kW8H16, 2, 1, 1, 4), PG_ROWS(kW8H16, 2, 2, 1, 4), PG_ROWS(kW8H16, 2, 4, 1, 4),
    PG_ROWS(kW8H8, 1, 1, 2, 4), PG_ROWS(kW8H8, 1, 2, 2, 4), PG_ROWS(kW8H8, 1, 4, 1, 4), PG_ROWS(kW8H8, 2, 1, 2, 4), PG_ROWS(kW8H8, 2, 2, 2, 4), PG_ROWS(kW8H8, 2, 4, 1, 4), PG_ROWS(kW8H8, 4, 1, 1, 4), PG_ROWS(kW8H8, 4, 2, 1, 4), PG_ROWS(kW8H8, 4, 4, 1, 4),
    PG_ROWS(kW8H8Wide, 1, 1, 2, 4), PG_ROWS(kW8H8Wide, 1, 2, 2, 4), PG_ROWS(kW8H8Wide, 1, 4, 1, 4), PG_ROWS(kW8H8Wide, 2, 1, 2, 4), PG_ROWS(kW8H8Wide, 2, 2, 2, 4), PG_ROWS(kW8H8Wide, 2, 4, 1, 4), PG_ROWS(kW8H8Wide, 4, 1, 1, 4), PG_ROWS(kW8H8Wide, 4, 2, 1, 4), PG_ROWS(kW8H8Wide, 4, 4, 1, 4),
};

// Several tiles of outputs share their rows' loads, as long as every compute unit has a workgroup.  4096 x 4096 in 8 bits, 64 rows: 7.4 us with 32 outputs (256
// workgroups), 8.9 with 16, 9.5 with 64; 512 rows in bf16: 32 us with 64 outputs, 56 with 16.
constexpr long long kRowsFrom = 256;
constexpr long long kSmallestTile = 16;
long long most_tiles(long long slots, long long experts, long long tile) { return slots / tile + std::min(slots, experts + 1); }

}  // namespace

size_t sorted_bytes(int op, const Shape& s) {
    if (op != kExpertGemv || s.rows < 1 || s.m < 1 || s.m > (1 << 24) / s.rows || s.inner < 1 || s.inner > kSortMostExperts) return 0;
    const long long slots = s.rows * s.m;
    if (slots <= kFewSlots) return 0;
    return sizeof(SortedSlots) + (size_t)most_tiles(slots, s.inner, kSmallestTile) * sizeof(SortedTile) + (size_t)slots * sizeof(int);
}

static bool plan_kernel(int op, int dtype, const Shape& s, Launch* out, Launch* pre) {
    *out = Launch();
    *pre = Launch();
    out->block = dim3(kBlock);
    const bool f32 = dtype == kF32;
    switch (op) {
    case kQuantize: {
        const long long units = s.rows * (((s.cols + kScaleBlock - 1) / kScaleBlock + 3) / 4);
        if (units >= 1ll << 31) return false;
        out->fn = f32 ? PG_FN(k_quantize<float>) : PG_FN(k_quantize<bf16_t>);
        out->arg_bytes = sizeof(QuantizeArgs);
        out->grid = dim3(blocks_for(units, kBlock / 16));
        return true;
    }
    case kRoute:
        out->fn = s.high ? (f32 ? route_kernel<float, true>(s.cols) : route_kernel<bf16_t, true>(s.cols)) : f32 ? route_kernel<float, false>(s.cols) : route_kernel<bf16_t, false>(s.cols);
        out->arg_bytes = sizeof(RouteArgs);
        out->grid = dim3(blocks_for(s.rows, kBlock / 64));
        return true;
    case kExpertSum: {
        const int pieces = (int)((s.n + (f32 ? 4 : 8) - 1) / (f32 ? 4 : 8)), lanes = sum_lanes(pieces);
        const long long grid = lanes == kBlock ? s.rows * blocks_for(pieces, kBlock) : (s.rows + kBlock / lanes - 1) / (kBlock / lanes);
        if (grid > 0x7fffffffll) return false;
        out->fn = f32 ? PG_FN(k_expert_sum<float>) : PG_FN(k_expert_sum<bf16_t>);
        out->arg_bytes = sizeof(ExpertSumArgs);
        out->grid = dim3((unsigned)grid);
        return true;
    }
    case kGemvF8: case kExpertGemv: {
        const bool routed = op == kExpertGemv, w8 = s.in_dtype[0] == kF8Weight, h8 = s.in_dtype[1] == kF8Rows;
        const long long slots = routed ? s.rows * s.m : s.rows, experts = routed ? s.inner : 1, mean = slots / experts;
        const Form form = !w8 ? kW16H16 : !h8 ? kW8H16 : f32 ? kW8H8Wide : kW8H8;
        auto with = [&](int tile, int outputs) {
            out->tile = tile;
            out->tiles = (int)(routed ? most_tiles(slots, s.inner, tile) : (slots + tile - 1) / tile);
            const long long grid = out->tiles * ((s.n + outputs - 1) / outputs);
            out->grid = dim3((unsigned)grid);
            return grid <= 0x7fffffffll;
        };
        out->arg_bytes = sizeof(ExpertArgs);
        const TileKernel* fit = nullptr;
        // (their offsets within a tile, and of gathered rows within h, have 32 bits)
        const long long pitch = w8 ? (s.cols + kScaleBlock - 1) / kScaleBlock * kScaleBlock : 2 * s.cols, hpitch = h8 ? pitch : 2 * s.cols;
        const bool fits = s.cols >= 8 && 256 * std::max(pitch, hpitch) < (1ll << 32) && (!routed || slots * hpitch < (1ll << 32));
        if (fits && mean >= tiles_mean(routed, form, s.cols)) {
            long long least = 0, smallest = 0;
            for (const TileKernel& k : kTileKernels) {
                if (k.form != form) continue;
                const long long wgs = k.workgroups(slots, experts, s.n), cost = k.cost(wgs);
                if ((2 * mean >= k.rows || k.rows == kTilesRows) && (!fit || cost < least)) { fit = &k; least = cost; }
                smallest = wgs;                          // (the last of a form)
            }
            if (smallest < tiles_from(routed, form)) fit = nullptr;
        }
        if (fit) {
            if (!with(fit->rows, fit->outputs)) return false;
            out->fn = routed ? fit->routed : fit->plain;
            out->block = dim3(fit->threads);
        } else {
            const long long each = routed ? (3 * slots + 2 * std::min(slots, s.inner) - 1) / (2 * std::min(slots, s.inner)) : slots;      // slots of an expert: half as many again as the mean
            // The smallest tile that holds an expert's rows, with as many outputs as leave kRowsFrom workgroups.  64 rows where they come in the weights' type:
            // 16-bit rows beside 8-bit weights take twice the LDS.  In 8 bits 32 are faster up to 128 rows: 64 rows of 4096 x 4096 7.5 and 9.3 us, 128 rows
            // 9.7 and 10.2, 256 rows 13.9 and 12.9.
            const RowsKernel* k = kRowsKernels;
            const int most = form == kW8H16 || (form != kW16H16 && each <= 128) ? 32 : 64;
            while (k->form != form || (s.cols >= 8 && each > k->rows && k->rows < most)) k++;
            const long long about = routed ? std::min(slots, s.inner) * ((each + k->rows - 1) / k->rows) : (slots + k->rows - 1) / k->rows;
            while (s.cols >= 8 && k->outputs < 64 && about * ((s.n + k[1].outputs - 1) / k[1].outputs) >= kRowsFrom) k++;
            if (!with(k->rows, k->outputs)) return false;
            out->fn = routed ? k->routed : k->plain;
            out->block = dim3(k->threads);
        }
        if (routed && slots > (fit ? kFewSlots : out->grid.x <= 2 * kComputeUnits ? kSomeSlots : kSomeSlots / 2)) {       // (half of them where more than a round of workgroups counts)
            pre->fn = PG_FN(k_sort_slots);
            pre->arg_bytes = sizeof(ExpertArgs);
            pre->block = dim3(kSortThreads);
        }
        return true;
    }
    default: return false;
    }
}

bool plan_experts(int op, int dtype, const Shape& s, Launch* out, Launch* pre) {
    return plan_kernel(op, dtype, s, out, pre) && (unsigned long long)out->grid.x * out->block.x < 1ull << 32;       // (threads of a launch)
}

}  // namespace pgk
