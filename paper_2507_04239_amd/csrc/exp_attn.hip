// Exponential (softmax) attention on grouped heads, the weight that arXiv 2507.04239 compares power attention with (Sec. 2 Eq. 1),
// forward and backward:
//     x_ij = scale q_i . k_j      s_ij = cap tanh(x_ij / cap) - slope_h |pos_i - j|      pos_i = i + Tk - T
//     L_i = log sum_j exp s_ij    P_ij = exp(s_ij - L_i)    O_i = sum_j P_ij v_j         over the keys lo_i <= j < hi_i
//     D_i = dO_i . O_i            t_ij = P_ij (dO_i . v_j - D_i) (1 - tanh^2(x_ij / cap))
//     dQ_i = scale sum_j t_ij k_j     dK_j = scale sum_i t_ij q_i     dV_j = sum_i P_ij dO_i
// The last two sum over the query heads that share the key head too.
//
// The kernels have the shape of the attention form's (mfma_attn.hip): a workgroup of 4 waves owns a block of rows (queries for the
// forward pass and dQ, keys for dK / dV) and walks over the other side in tiles of 64 rows staged in LDS.  Every mask here
// is an interval of keys per query row; blocks of rows know the least and greatest ends of their intervals, so a tile that
// no row sees is not read, one that every row sees whole has no comparison in it, and only the ones between select.
//
// Scores are in units of log 2 from the first multiplication on, so a weight is one multiply-add and one v_exp_f32.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_tile.hpp"

namespace pa {
namespace mfma {
namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float NEG_INF = -__builtin_inff();

// ---- the score --------------------------------------------------------------------------------------
// cap tanh(x / cap) = cap - 2 cap / (exp(2 x / cap) + 1): one exponential and one reciprocal, exact at both ends (exp 0 and
// infinity), its absolute error a few float32 roundings of cap.
struct Score {
    float sl;           // scale log2 e
    float kc, capl;     // 2 scale log2 e / cap; cap log2 e
};
Score score_of(const pa_exp_problem& pr) {
    Score s{pr.scale * LOG2E, 0.f, 0.f};
    if (pr.cap > 0.f) {
        s.kc = (float)(2.0 * pr.scale / pr.cap * 1.44269504088896340736);
        s.capl = pr.cap * LOG2E;
    }
    return s;
}
// 1 / (exp(2 x / cap) + 1) = r:  s = capl - 2 capl r,  1 - tanh^2 = 4 r (1 - r)
__device__ __forceinline__ float cap_r(float c, const Score& sc) {
    return __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(c * sc.kc) + 1.f);
}

// ---- masks --------------------------------------------------------------------------------------------
struct Rows {
    const int *lo, *hi;
    int window, off, T, Tk;     // off = Tk - T
};
struct Range {
    int lo, hi;         // keys lo .. hi - 1; lo = Tk, hi = 0: none
};
__device__ __forceinline__ Range row_range(const Rows& m, int b, int i) {
    const int pos = i + m.off;
    const size_t at = (size_t)b * m.T + i;
    Range r{m.lo != nullptr ? m.lo[at] : 0, m.hi != nullptr ? m.hi[at] : pos + 1};
    if (m.window > 0) r.lo = max(r.lo, pos - m.window + 1);
    r.lo = max(r.lo, 0);
    r.hi = min(r.hi, m.Tk);
    if (r.lo >= r.hi) r = {m.Tk, 0};
    return r;
}
// key - lo < hi - lo, unsigned, for keys that are not negative
__device__ __forceinline__ bool sees(int key, const Range& r) { return (unsigned)(key - r.lo) < (unsigned)max(r.hi - r.lo, 0); }

// least and greatest ends over a set of rows
struct Ends {
    int lo_min, hi_max, lo_max, hi_min;
    __device__ __forceinline__ bool none(int first, int n) const { return hi_max <= first || lo_min >= first + n; }   // of n keys from `first`
    __device__ __forceinline__ bool all(int first, int n) const { return lo_max <= first && hi_min >= first + n; }
};
__device__ __forceinline__ Ends join(const Ends& a, const Ends& b) {
    return {min(a.lo_min, b.lo_min), max(a.hi_max, b.hi_max), max(a.lo_max, b.lo_max), min(a.hi_min, b.hi_min)};
}
__device__ __forceinline__ Ends wave_ends(Range r) {
    Ends e{r.lo, r.hi, r.lo, r.hi};
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const Ends o{__shfl_xor(e.lo_min, off), __shfl_xor(e.hi_max, off), __shfl_xor(e.lo_max, off), __shfl_xor(e.hi_min, off)};
        e = join(e, o);
    }
    e.lo_min = __builtin_amdgcn_readfirstlane(e.lo_min);
    e.hi_max = __builtin_amdgcn_readfirstlane(e.hi_max);
    e.lo_max = __builtin_amdgcn_readfirstlane(e.lo_max);
    e.hi_min = __builtin_amdgcn_readfirstlane(e.hi_min);
    return e;
}

// Infinities and NaN of rows that are masked for some row of the other side must not reach it, and in a matrix product they would
// (0 x NaN).  So in tiles that are not seen whole by the whole workgroup such values enter LDS as zeros and their tile row is
// marked; a wave that finds a mark adds what the pairs that are seen would have received.
__device__ __forceinline__ uint32_t nonfinite2(uint32_t u) { return ((u & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ bool nonfinite8(uint4 u) {
    return (nonfinite2(u.x) | nonfinite2(u.y) | nonfinite2(u.z) | nonfinite2(u.w)) != 0;
}
__device__ __forceinline__ uint32_t finite2(uint32_t u) { return u & ~((nonfinite2(u) >> 15) * 0xffffu); }
struct Marks {
    uint32_t row[3][2];     // of the tile in use, the one being staged, and the one cleared for the next
};
__device__ __forceinline__ void clean(uint4& u, uint32_t (&marks)[2], int row) {
    if (!nonfinite8(u)) return;
    u = make_uint4(finite2(u.x), finite2(u.y), finite2(u.z), finite2(u.w));
    atomicOr(&marks[row >> 5], 1u << (row & 31));
}
#define PA_TILE_CLEAN(REGS, MARKS) \
    _Pragma("unroll") for (int q_ = 0; q_ < HD / 32; ++q_) clean(REGS[q_], MARKS, (tid + 256 * q_) / (HD / 8));
__device__ __forceinline__ uint64_t marked(const uint32_t (&m)[2]) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)m[0]) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)m[1]) << 32;
}

// ---- the order of the workgroups ------------------------------------------------------------------------
// Workgroups with the longest walk of all heads of a group come first.  Consecutive workgroups go to the 8 XCDs in turn, so the
// heads that share a key head are `group` apart: with a group that 8 divides, or that divides 8, they meet on one XCD's L2.
struct Order {
    int H, Hk, G, BHk;      // query heads, key heads, query heads per key head, key heads of the batch
    int group, nblk;        // key heads of a group; blocks of rows of a head
};
struct Place {
    int kv, g, rank;
};
template <bool PER_KEY_HEAD>
__device__ __forceinline__ bool place(const Order& o, Place& p) {
    const unsigned per = (unsigned)o.group * (PER_KEY_HEAD ? 1u : (unsigned)o.G);
    const unsigned row = blockIdx.x / per, x = blockIdx.x - row * per;
    const unsigned z = row / (unsigned)o.nblk;
    p.rank = (int)(row - z * (unsigned)o.nblk);
    p.g = (int)(x / (unsigned)o.group);
    p.kv = (int)(z * (unsigned)o.group + x % (unsigned)o.group);
    return p.kv < o.BHk;
}

// ---- forward --------------------------------------------------------------------------------------------
// acc[vb][ib] = O^T: value columns 32 vb + .., query 32 ib + r32 of the wave's OWN queries.  One pass: m is the reference of the
// running sum, in units of log 2; it follows the row's maximum only once that is 8 above it (weights up to 256 lose nothing,
// and most tiles then rescale nothing).
template <int HD>
struct FwdShared {
    AttnTile<HD> k[2], v[2];
    Ends ends[4];
    Marks marks;
};
template <int HD, int OWN, int WPE, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, WPE) void k_exp_fwd(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K,
                                                      const bf16_t* __restrict__ V, const float* __restrict__ slopes,
                                                      bf16_t* __restrict__ O, float* __restrict__ L, Order order, Rows rows, Score sc) {
    constexpr int NI = OWN / 32, NK = HD / 16, NV = HD / 32, WG = 4 * OWN;
    constexpr bool RAW = !CAP && !BIAS;     // the products themselves are compared, and scaled with the subtraction
    __shared__ FwdShared<HD> sm;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, h = lane >> 5;
    Place at;
    if (!place<false>(order, at)) return;
    const int T = rows.Tk;          // rows of the streamed side, for the tile loads
    const int i0 = (order.nblk - 1 - at.rank) * WG, q0 = i0 + OWN * w;
    const int b = at.kv / order.Hk, head = b * order.H + (at.kv - b * order.Hk) * order.G + at.g;
    const bf16_t* Kh = K + (size_t)at.kv * T * HD;
    const bf16_t* Vh = V + (size_t)at.kv * T * HD;
    const size_t row0 = (size_t)head * rows.T;

    bf16x8 qf[NI][NK];
    f32x16 acc[NV][NI];
    float lsum[NI], m[NI];
    Range rg[NI];
    Ends mine{T, 0, 0, T};
#pragma unroll
    for (int ib = 0; ib < NI; ++ib) {
        const int i = min(q0 + 32 * ib + r32, rows.T - 1);
        lsum[ib] = 0.f;
        m[ib] = NEG_INF;
        rg[ib] = row_range(rows, b, i);
        mine = join(mine, wave_ends(rg[ib]));
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) qf[ib][ks] = row_frag_global<HD>(Q, row0 + i, ks, h);
#pragma unroll
        for (int vb = 0; vb < NV; ++vb) acc[vb][ib] = splat16(0.f);
    }
    const float slope = BIAS ? slopes[head - b * order.H] * LOG2E : 0.f;

    if (lane == 0) sm.ends[w] = mine;
    if (tid < 6) (&sm.marks.row[0][0])[tid] = 0;
    __syncthreads();
    Ends all = join(join(sm.ends[0], sm.ends[1]), join(sm.ends[2], sm.ends[3]));
    const int t_lo = __builtin_amdgcn_readfirstlane(all.lo_min) / AT, t_hi = (__builtin_amdgcn_readfirstlane(all.hi_max) + AT - 1) / AT;

    auto tile = [&](auto mask_c, int buf, int key0, uint64_t bad) {
        constexpr bool MASK = decltype(mask_c)::value;
        f32x16 c[2][NI];        // S^T: key 32 kb + 8 k + 4 h + r, query 32 ib + r32
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int ib = 0; ib < NI; ++ib) c[kb][ib] = splat16(0.f);
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
                const bf16x8 kf = row_frag<HD>(sm.k[buf], kb, ks, lane);
#pragma unroll
                for (int ib = 0; ib < NI; ++ib) c[kb][ib] = mfma32(kf, qf[ib][ks], c[kb][ib]);
            }
        }
        float mm[NI];
#pragma unroll
        for (int ib = 0; ib < NI; ++ib) {
            const float far = BIAS ? (float)(q0 + 32 * ib + r32 + rows.off - key0 - 4 * h) : 0.f;
            float top[2] = {NEG_INF, NEG_INF};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = 32 * kb + 8 * (i >> 2) + (i & 3);       // of the tile, less 4 h
                    float x = c[kb][ib][i];
                    if (CAP) x = fmaf(-2.f * sc.capl, cap_r(x, sc), sc.capl);
                    else if (BIAS) x *= sc.sl;
                    if (BIAS) x = fmaf(-slope, fabsf(far - (float)key), x);
                    if (MASK && !sees(key0 + 4 * h + key, rg[ib])) x = NEG_INF;
                    c[kb][ib][i] = x;
                    top[kb] = fmaxf(top[kb], x);
                }
            float lo, hi;
            halves(fmaxf(top[0], top[1]), lo, hi);
            const float t = RAW ? fmaxf(lo, hi) * sc.sl : fmaxf(lo, hi);
            if (__any(t > m[ib] + 8.f)) {
                const float to = fmaxf(t, m[ib]);
                const float f = to == NEG_INF ? 1.f : __builtin_amdgcn_exp2f(m[ib] - to);
                m[ib] = to;
                lsum[ib] *= f;
#pragma unroll
                for (int vb = 0; vb < NV; ++vb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[vb][ib][i] *= f;
            }
            mm[ib] = m[ib] == NEG_INF ? 0.f : m[ib];
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            Frag pf[NI][2];
#pragma unroll
            for (int ib = 0; ib < NI; ++ib) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = c[kb][ib][i];
                    pf[ib][i >> 3].v[i & 7] = (__bf16)__builtin_amdgcn_exp2f(RAW ? fmaf(x, sc.sl, -mm[ib]) : x - mm[ib]);
                }
                // the denominator sums the rounded weights, the ones that the numerator uses
#pragma unroll
                for (int j = 0; j < 2; ++j) lsum[ib] = sum_bf16x8(pf[ib][j], lsum[ib]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int vb = 0; vb < NV; ++vb) {
                    const bf16x8 vf = col_frag<HD>(sm.v[buf], 2 * kb + j, vb, lane);
#pragma unroll
                    for (int ib = 0; ib < NI; ++ib) acc[vb][ib] = mfma32(vf, pf[ib][j].v, acc[vb][ib]);
                }
        }
        for (; bad != 0; bad &= bad - 1) {      // values that entered as zeros
            const int key = key0 + __builtin_ctzll(bad);
            const bf16_t* v = Vh + (size_t)min(key, T - 1) * HD;
#pragma unroll
            for (int ib = 0; ib < NI; ++ib)
                if (sees(key, rg[ib]))
#pragma unroll
                    for (int vb = 0; vb < NV; ++vb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t u = v[32 * vb + 8 * (i >> 2) + 4 * h + (i & 3)];
                            if (nonfinite2(u) != 0) acc[vb][ib][i] += __uint_as_float(u << 16);
                        }
        }
    };

    uint4 kr[HD / 32], vr[HD / 32];
    if (t_lo < t_hi) {
        PA_TILE_LOAD(kr, Kh, t_lo * AT, false)
        PA_TILE_LOAD(vr, Vh, t_lo * AT, false)
        if (!all.all(t_lo * AT, AT)) PA_TILE_CLEAN(vr, sm.marks.row[0])
        PA_TILE_STORE(sm.k[0], kr)
        PA_TILE_STORE(sm.v[0], vr)
    }
    __syncthreads();
    int slot = 0;
    for (int t = t_lo; t < t_hi; ++t) {
        const int buf = (t - t_lo) & 1, key0 = t * AT, next = slot == 2 ? 0 : slot + 1;
        if (t + 1 < t_hi) {
            PA_TILE_LOAD(kr, Kh, key0 + AT, false)
            PA_TILE_LOAD(vr, Vh, key0 + AT, false)
        }
        if (!mine.none(key0, AT)) {
            const uint64_t bad = all.all(key0, AT) ? 0 : marked(sm.marks.row[slot]);
            if (mine.all(key0, AT)) tile(std::false_type{}, buf, key0, bad);
            else tile(std::true_type{}, buf, key0, bad);
        }
        if (t + 1 < t_hi) {
            if (!all.all(key0 + AT, AT)) PA_TILE_CLEAN(vr, sm.marks.row[next])
            PA_TILE_STORE(sm.k[buf ^ 1], kr)
            PA_TILE_STORE(sm.v[buf ^ 1], vr)
        }
        if (tid < 2) sm.marks.row[next == 2 ? 0 : next + 1][tid] = 0;   // read last one tile ago, marked next one tile on
        slot = next;
        __syncthreads();
    }

#pragma unroll
    for (int ib = 0; ib < NI; ++ib) {
        const int i = q0 + 32 * ib + r32;
        const bool in = i < rows.T;
        const size_t row = row0 + min(i, rows.T - 1);
        const float z = xor32_sum(lsum[ib]), f = z != 0.f ? 1.f / z : 0.f;
#pragma unroll
        for (int vb = 0; vb < NV; ++vb) store_block(O + row * HD + 32 * vb, acc[vb][ib], f, h, in);
        if (L != nullptr && h == 0 && in) L[row] = z != 0.f ? (m[ib] + __builtin_amdgcn_logf(z)) * LN2 : NEG_INF;
    }
}

// ---- backward: preparation --------------------------------------------------------------------------------
// stat[row] = {L log2 e, -dO . O}: what the weights and their gradients are formed from.  A workgroup takes 64 rows of a head, HD / 8 lanes a row;
// the first head of a batch entry also leaves the rows' intervals and, per 64 rows, their ends.
struct BwdScratch {
    float2* stat;       // [B H][T]
    int2* range;        // [B][T]
    int4* ends;         // [B][tiles]: of the 64 rows of a tile
};
template <int HD>
__global__ __launch_bounds__(256) void k_exp_prep(const bf16_t* __restrict__ dO, const bf16_t* __restrict__ O, const float* __restrict__ L,
                                                  BwdScratch to, Rows rows, int H, int ntile) {
    constexpr int LPR = HD / 8, RPP = 256 / LPR;
    const unsigned head = blockIdx.x / (unsigned)ntile;
    const int t = (int)(blockIdx.x - head * (unsigned)ntile), b = (int)(head / (unsigned)H);
    const int tid = threadIdx.x, c8 = tid % LPR;
#pragma unroll
    for (int p = 0; p < 64; p += RPP) {
        const int i = t * AT + p + tid / LPR;
        const size_t row = (size_t)head * rows.T + min(i, rows.T - 1);
        const uint4 g = *(const uint4*)(dO + row * HD + 8 * c8), o = *(const uint4*)(O + row * HD + 8 * c8);
        const uint32_t gu[4] = {g.x, g.y, g.z, g.w}, ou[4] = {o.x, o.y, o.z, o.w};
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) d += bf_lo(gu[e]) * bf_lo(ou[e]) + bf_hi(gu[e]) * bf_hi(ou[e]);
#pragma unroll
        for (int off = 1; off < LPR; off <<= 1) d += __shfl_xor(d, off);
        const float l = L[row];
        if (c8 == 0 && i < rows.T) to.stat[row] = make_float2(l == NEG_INF ? 0.f : l * LOG2E, -d);
    }
    if (head != (unsigned)(b * H) || tid >= 64) return;
    const int i = t * AT + tid;
    const Range r = i < rows.T ? row_range(rows, b, i) : Range{rows.Tk, 0};
    if (i < rows.T) to.range[(size_t)b * rows.T + i] = make_int2(r.lo, r.hi);
    const Ends e = wave_ends(r);
    if (tid == 0) to.ends[(size_t)b * ntile + t] = make_int4(e.lo_min, e.hi_max, e.lo_max, e.hi_min);
}

// weight of a pair and, times (dO . v - D), the gradient of its product: p and t from the product c and e = dO . v - D
template <bool CAP, bool BIAS>
__device__ __forceinline__ void pair_grad(float c, float e, float l2, float slope, float dist, const Score& sc, float& p, float& t) {
    float r = 0.f, s;
    if (CAP) {
        r = cap_r(c, sc);
        s = fmaf(-2.f * sc.capl, r, sc.capl - l2);
    } else {
        s = fmaf(c, sc.sl, -l2);
    }
    if (BIAS) s = fmaf(-slope, fabsf(dist), s);
    p = __builtin_amdgcn_exp2f(s);
    t = p * e;
    if (CAP) t *= 4.f * fmaf(-r, r, r);
}

// ---- backward: dQ -------------------------------------------------------------------------------------------
// acc[fb][ib] = dQ^T / scale: features 32 fb + .., query 32 ib + r32.
template <int HD, int OWN, int WPE, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, WPE) void k_exp_dq(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K,
                                                     const bf16_t* __restrict__ V, const float* __restrict__ slopes,
                                                     const bf16_t* __restrict__ dO, const float2* __restrict__ stat,
                                                     bf16_t* __restrict__ dQ, Order order, Rows rows, Score sc, float scale) {
    constexpr int NI = OWN / 32, NK = HD / 16, NF = HD / 32, WG = 4 * OWN;
    __shared__ FwdShared<HD> sm;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, h = lane >> 5;
    Place at;
    if (!place<false>(order, at)) return;
    const int T = rows.Tk;
    const int i0 = (order.nblk - 1 - at.rank) * WG, q0 = i0 + OWN * w;
    const int b = at.kv / order.Hk, head = b * order.H + (at.kv - b * order.Hk) * order.G + at.g;
    const bf16_t* Kh = K + (size_t)at.kv * T * HD;
    const bf16_t* Vh = V + (size_t)at.kv * T * HD;
    const size_t row0 = (size_t)head * rows.T;

    bf16x8 qf[NI][NK], gf[NI][NK];
    f32x16 acc[NF][NI];
    float2 st[NI];
    Range rg[NI];
    Ends mine{T, 0, 0, T};
#pragma unroll
    for (int ib = 0; ib < NI; ++ib) {
        const int i = min(q0 + 32 * ib + r32, rows.T - 1);
        st[ib] = stat[row0 + i];
        rg[ib] = row_range(rows, b, i);
        mine = join(mine, wave_ends(rg[ib]));
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
            qf[ib][ks] = row_frag_global<HD>(Q, row0 + i, ks, h);
            gf[ib][ks] = row_frag_global<HD>(dO, row0 + i, ks, h);
        }
#pragma unroll
        for (int fb = 0; fb < NF; ++fb) acc[fb][ib] = splat16(0.f);
    }
    const float slope = BIAS ? slopes[head - b * order.H] * LOG2E : 0.f;

    if (lane == 0) sm.ends[w] = mine;
    if (tid < 6) (&sm.marks.row[0][0])[tid] = 0;
    __syncthreads();
    Ends all = join(join(sm.ends[0], sm.ends[1]), join(sm.ends[2], sm.ends[3]));
    const int t_lo = __builtin_amdgcn_readfirstlane(all.lo_min) / AT, t_hi = (__builtin_amdgcn_readfirstlane(all.hi_max) + AT - 1) / AT;

    auto tile = [&](auto mask_c, int buf, int key0, uint64_t bad) {
        constexpr bool MASK = decltype(mask_c)::value;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            f32x16 c[NI], e[NI];        // S^T and (dO V^T - D)^T: key 32 kb + 8 k + 4 h + r, query 32 ib + r32
#pragma unroll
            for (int ib = 0; ib < NI; ++ib) {
                c[ib] = splat16(0.f);
                e[ib] = splat16(st[ib].y);
            }
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
                const bf16x8 kf = row_frag<HD>(sm.k[buf], kb, ks, lane), vf = row_frag<HD>(sm.v[buf], kb, ks, lane);
#pragma unroll
                for (int ib = 0; ib < NI; ++ib) {
                    c[ib] = mfma32(kf, qf[ib][ks], c[ib]);
                    e[ib] = mfma32(vf, gf[ib][ks], e[ib]);
                }
                if (ks & 1) __builtin_amdgcn_sched_barrier(0);
            }
            Frag tf[NI][2];
#pragma unroll
            for (int ib = 0; ib < NI; ++ib) {
                const float far = BIAS ? (float)(q0 + 32 * ib + r32 + rows.off - key0 - 32 * kb - 4 * h) : 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = 8 * (i >> 2) + (i & 3);
                    float p, t;
                    pair_grad<CAP, BIAS>(c[ib][i], e[ib][i], st[ib].x, slope, far - (float)key, sc, p, t);
                    if (MASK && !sees(key0 + 32 * kb + 4 * h + key, rg[ib])) t = 0.f;
                    tf[ib][i >> 3].v[i & 7] = (__bf16)t;
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int fb = 0; fb < NF; ++fb) {
                    const bf16x8 kc = col_frag<HD>(sm.k[buf], 2 * kb + j, fb, lane);   // K^T
#pragma unroll
                    for (int ib = 0; ib < NI; ++ib) acc[fb][ib] = mfma32(kc, tf[ib][j].v, acc[fb][ib]);
                }
        }
        for (; bad != 0; bad &= bad - 1) {      // a key that is no finite vector: nothing is left of the rows that see it
            const int key = key0 + __builtin_ctzll(bad);
#pragma unroll
            for (int ib = 0; ib < NI; ++ib)
                if (sees(key, rg[ib]))
#pragma unroll
                    for (int fb = 0; fb < NF; ++fb) acc[fb][ib] = splat16(__builtin_nanf(""));
        }
    };

    uint4 kr[HD / 32], vr[HD / 32];
    if (t_lo < t_hi) {
        PA_TILE_LOAD(kr, Kh, t_lo * AT, false)
        PA_TILE_LOAD(vr, Vh, t_lo * AT, false)
        if (!all.all(t_lo * AT, AT)) PA_TILE_CLEAN(kr, sm.marks.row[0])
        PA_TILE_STORE(sm.k[0], kr)
        PA_TILE_STORE(sm.v[0], vr)
    }
    __syncthreads();
    int slot = 0;
    for (int t = t_lo; t < t_hi; ++t) {
        const int buf = (t - t_lo) & 1, key0 = t * AT, next = slot == 2 ? 0 : slot + 1;
        if (t + 1 < t_hi) {
            PA_TILE_LOAD(kr, Kh, key0 + AT, false)
            PA_TILE_LOAD(vr, Vh, key0 + AT, false)
        }
        if (!mine.none(key0, AT)) {
            const uint64_t bad = all.all(key0, AT) ? 0 : marked(sm.marks.row[slot]);
            if (mine.all(key0, AT)) tile(std::false_type{}, buf, key0, bad);
            else tile(std::true_type{}, buf, key0, bad);
        }
        if (t + 1 < t_hi) {
            if (!all.all(key0 + AT, AT)) PA_TILE_CLEAN(kr, sm.marks.row[next])
            PA_TILE_STORE(sm.k[buf ^ 1], kr)
            PA_TILE_STORE(sm.v[buf ^ 1], vr)
        }
        if (tid < 2) sm.marks.row[next == 2 ? 0 : next + 1][tid] = 0;
        slot = next;
        __syncthreads();
    }

#pragma unroll
    for (int ib = 0; ib < NI; ++ib) {
        const int i = q0 + 32 * ib + r32;
        const size_t row = row0 + min(i, rows.T - 1);
#pragma unroll
        for (int fb = 0; fb < NF; ++fb) store_block(dQ + row * HD + 32 * fb, acc[fb][ib], scale, h, i < rows.T);
    }
}

// ---- backward: dK, dV -----------------------------------------------------------------------------------------
// dk[fb][kb] = dK^T / scale: features 32 fb + .., key 32 kb + r32 of the wave's OWN keys; dv likewise.  The walk goes over the
// query rows of every head that reads the key head; tiles of rows that see none of the block's keys are found 64 at a time from the
// ends that the preparation left.
template <int HD>
struct BwdShared {
    AttnTile<HD> q[2], g[2];
    float l2[2][AT], d[2][AT];
    int lo[2][AT], hi[2][AT];
    Marks marks;
};
template <int HD, int OWN, int WPE, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, WPE) void k_exp_dkdv(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K,
                                                       const bf16_t* __restrict__ V, const float* __restrict__ slopes,
                                                       const bf16_t* __restrict__ dO, BwdScratch from, bf16_t* __restrict__ dK,
                                                       bf16_t* __restrict__ dV, Order order, Rows rows, Score sc, float scale) {
    constexpr int NJ = OWN / 32, NK = HD / 16, NF = HD / 32, WG = 4 * OWN;
    __shared__ BwdShared<HD> sm;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, h = lane >> 5;
    Place at;
    if (!place<true>(order, at)) return;
    const int T = rows.T, ntile = (T + AT - 1) / AT;
    const int j0 = at.rank * WG, k0 = j0 + OWN * w;
    const int b = at.kv / order.Hk, head0 = b * order.H + (at.kv - b * order.Hk) * order.G;
    const size_t key_row0 = (size_t)at.kv * rows.Tk;
    const int4* ends = from.ends + (size_t)b * ntile;
    const int2* range = from.range + (size_t)b * T;

    bf16x8 kf[NJ][NK], vf[NJ][NK];
    f32x16 dk[NF][NJ], dv[NF][NJ];
#pragma unroll
    for (int kb = 0; kb < NJ; ++kb) {
        const size_t row = key_row0 + min(k0 + 32 * kb + r32, rows.Tk - 1);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
            kf[kb][ks] = row_frag_global<HD>(K, row, ks, h);
            vf[kb][ks] = row_frag_global<HD>(V, row, ks, h);
        }
#pragma unroll
        for (int fb = 0; fb < NF; ++fb) {
            dk[fb][kb] = splat16(0.f);
            dv[fb][kb] = splat16(0.f);
        }
    }
    if (tid < 6) (&sm.marks.row[0][0])[tid] = 0;
    __syncthreads();

    auto tile = [&](auto mask_c, int buf, int q0, float slope, uint64_t bad) {
        constexpr bool MASK = decltype(mask_c)::value;
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            float l2[16], g0[16];
            row_values(l2, &sm.l2[buf][32 * qb], h);
            row_values(g0, &sm.d[buf][32 * qb], h);
            f32x16 c[NJ], e[NJ];        // S and dO V^T - D: query 32 qb + 8 k + 4 h + r, key 32 kb + r32
#pragma unroll
            for (int kb = 0; kb < NJ; ++kb) {
                c[kb] = splat16(0.f);
#pragma unroll
                for (int i = 0; i < 16; ++i) e[kb][i] = g0[i];
            }
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
                const bf16x8 qa = row_frag<HD>(sm.q[buf], qb, ks, lane), ga = row_frag<HD>(sm.g[buf], qb, ks, lane);
#pragma unroll
                for (int kb = 0; kb < NJ; ++kb) {
                    c[kb] = mfma32(qa, kf[kb][ks], c[kb]);
                    e[kb] = mfma32(ga, vf[kb][ks], e[kb]);
                }
            }
            Frag tf[NJ][2], pf[NJ][2];
#pragma unroll
            for (int kb = 0; kb < NJ; ++kb) {
                const int key = k0 + 32 * kb + r32;
                const float far = BIAS ? (float)(q0 + 32 * qb + 4 * h + rows.off - key) : 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = 8 * (i >> 2) + (i & 3);
                    float p, t;
                    pair_grad<CAP, BIAS>(c[kb][i], e[kb][i], l2[i], slope, far + (float)r, sc, p, t);
                    if (MASK) {
                        const int i_row = 32 * qb + 4 * h + r;
                        if (!sees(key, {sm.lo[buf][i_row], sm.hi[buf][i_row]})) p = t = 0.f;
                    }
                    pf[kb][i >> 3].v[i & 7] = (__bf16)p;
                    tf[kb][i >> 3].v[i & 7] = (__bf16)t;
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int fb = 0; fb < NF; ++fb) {
                    const bf16x8 qc = col_frag<HD>(sm.q[buf], 2 * qb + j, fb, lane);   // Q^T
                    const bf16x8 gc = col_frag<HD>(sm.g[buf], 2 * qb + j, fb, lane);   // dO^T
#pragma unroll
                    for (int kb = 0; kb < NJ; ++kb) {
                        dk[fb][kb] = mfma32(qc, tf[kb][j].v, dk[fb][kb]);
                        dv[fb][kb] = mfma32(gc, pf[kb][j].v, dv[fb][kb]);
                    }
                }
        }
        for (; bad != 0; bad &= bad - 1) {      // a query or a gradient that is no finite vector
            const int r = __builtin_ctzll(bad);
            const Range rg{sm.lo[buf][r], sm.hi[buf][r]};
#pragma unroll
            for (int kb = 0; kb < NJ; ++kb)
                if (sees(k0 + 32 * kb + r32, rg))
#pragma unroll
                    for (int fb = 0; fb < NF; ++fb) dk[fb][kb] = dv[fb][kb] = splat16(__builtin_nanf(""));
        }
    };

    // the tiles of rows that see a key of the block, for one head after the other, 64 tiles at a time
    int base = -64, g = order.G;
    uint64_t seen = 0, left = 0;
    auto advance = [&]() -> int {
        while (left == 0) {
            if (++g < order.G) {
                left = seen;
            } else {
                base += 64;
                if (base >= ntile) return -1;
                const int t = base + lane;
                const int4 e = ends[min(t, ntile - 1)];
                seen = left = __ballot(t < ntile && !Ends{e.x, e.y, e.z, e.w}.none(j0, WG));
                g = seen != 0 ? 0 : order.G;
            }
        }
        const int t = base + __builtin_ctzll(left);
        left &= left - 1;
        return t;
    };
    uint4 qr[HD / 32], gr[HD / 32];
    float2 str = make_float2(0.f, 0.f);
    int2 rgr = make_int2(0, 0);
    auto load = [&](int t, int head) {
        const size_t base_row = (size_t)head * T;
        PA_TILE_LOAD(qr, Q + base_row * HD, t * AT, false)
        PA_TILE_LOAD(gr, dO + base_row * HD, t * AT, false)
        if (tid < AT) {
            const int i = min(t * AT + tid, T - 1);
            str = from.stat[base_row + i];
            rgr = t * AT + tid < T ? range[i] : make_int2(rows.Tk, 0);
        }
    };
    auto store = [&](int buf, uint32_t (&marks)[2], const Ends& e) {
        if (!e.all(j0, WG)) {
            PA_TILE_CLEAN(qr, marks)
            PA_TILE_CLEAN(gr, marks)
        }
        PA_TILE_STORE(sm.q[buf], qr)
        PA_TILE_STORE(sm.g[buf], gr)
        if (tid < AT) {
            sm.l2[buf][tid] = str.x;
            sm.d[buf][tid] = str.y;
            sm.lo[buf][tid] = rgr.x;
            sm.hi[buf][tid] = rgr.y;
        }
    };
    auto ends_of = [&](int t) {
        const int4 e = ends[t];
        return Ends{__builtin_amdgcn_readfirstlane(e.x), __builtin_amdgcn_readfirstlane(e.y), __builtin_amdgcn_readfirstlane(e.z),
                    __builtin_amdgcn_readfirstlane(e.w)};
    };
    int t = advance(), gt = g, buf = 0, slot = 0;
    Ends e{0, 0, 0, 0};
    if (t >= 0) {
        e = ends_of(t);
        load(t, head0 + gt);
        store(0, sm.marks.row[0], e);
    }
    __syncthreads();
    while (t >= 0) {
        const int tn = advance(), gn = g, next = slot == 2 ? 0 : slot + 1;
        Ends en{0, 0, 0, 0};
        if (tn >= 0) {
            en = ends_of(tn);
            load(tn, head0 + gn);
        }
        if (!e.none(k0, OWN)) {
            const float slope = BIAS ? slopes[head0 + gt - b * order.H] * LOG2E : 0.f;
            const uint64_t bad = e.all(j0, WG) ? 0 : marked(sm.marks.row[slot]);
            if (e.all(k0, OWN)) tile(std::false_type{}, buf, t * AT, slope, bad);
            else tile(std::true_type{}, buf, t * AT, slope, bad);
        }
        if (tn >= 0) store(buf ^ 1, sm.marks.row[next], en);
        if (tid < 2) sm.marks.row[next == 2 ? 0 : next + 1][tid] = 0;
        slot = next;
        buf ^= 1;
        t = tn;
        gt = gn;
        e = en;
        __syncthreads();
    }

#pragma unroll
    for (int kb = 0; kb < NJ; ++kb) {
        const int key = k0 + 32 * kb + r32;
        const size_t row = key_row0 + min(key, rows.Tk - 1);
#pragma unroll
        for (int fb = 0; fb < NF; ++fb) {
            store_block(dK + row * HD + 32 * fb, dk[fb][kb], scale, h, key < rows.Tk);
            store_block(dV + row * HD + 32 * fb, dv[fb][kb], 1.f, h, key < rows.Tk);
        }
    }
}

// ---- launches -----------------------------------------------------------------------------------------------
// Key heads whose K and V fit half of the memory-side cache go together (attention form: 184 ms a step with all heads, 156 so).
Order order_of(const pa_exp_problem& pr, int rows_per_block, int len) {
    Order o{pr.H, pr.Hk, pr.H / pr.Hk, pr.B * pr.Hk, pr.B * pr.Hk, (len + rows_per_block - 1) / rows_per_block};
    const long long fit = std::max(8LL, (128LL << 20) / (4LL * std::max(pr.T, pr.Tk) * pr.d));
    if (o.BHk > fit) {
        int g = 8;
        while (2 * g <= fit) g *= 2;
        o.group = g;
    }
    return o;
}
long long blocks_of(const Order& o, bool per_key_head) {
    return (long long)((o.BHk + o.group - 1) / o.group) * o.group * (per_key_head ? 1 : o.G) * o.nblk;
}

template <int HD>
struct Shape {
    static constexpr int FWD_OWN = 32, FWD_WPE = 2, DQ_WPE = 2, DKDV_WPE = HD == 128 ? 1 : 2;
};

template <int HD, bool CAP, bool BIAS>
pa_status fwd_t(const pa_exp_problem& pr, const bf16_t* Q, const bf16_t* K, const bf16_t* V, const ExpMask& mk, const Rows& rows, bf16_t* O,
                float* L, hipStream_t s) {
    constexpr int OWN = Shape<HD>::FWD_OWN;
    const Order o = order_of(pr, 4 * OWN, pr.T);
    LaunchScope ls("exp_fwd", s);
    hipLaunchKernelGGL((k_exp_fwd<HD, OWN, Shape<HD>::FWD_WPE, CAP, BIAS>), dim3((unsigned)blocks_of(o, false)), dim3(256), 0, s, Q, K, V,
                       mk.slopes, O, L, o, rows, score_of(pr));
    return launch_ok() ? PA_OK : PA_ERR_HIP;
}
BwdScratch bwd_scratch(const pa_exp_problem& pr, char* ws) {
    const size_t BHT = (size_t)pr.B * pr.H * pr.T, BT = (size_t)pr.B * pr.T;
    char* range = ws + align_up(BHT * sizeof(float2), 256);
    return {(float2*)ws, (int2*)range, (int4*)(range + align_up(BT * sizeof(int2), 256))};
}
template <int HD, bool CAP, bool BIAS>
pa_status bwd_t(const pa_exp_problem& pr, const bf16_t* Q, const bf16_t* K, const bf16_t* V, const ExpMask& mk, const Rows& rows,
                const bf16_t* O, const float* L, const bf16_t* dO, bf16_t* dQ, bf16_t* dK, bf16_t* dV, char* ws, hipStream_t s) {
    const BwdScratch sc = bwd_scratch(pr, ws);
    const int ntile = (pr.T + AT - 1) / AT;
    {
        LaunchScope ls("exp_bwd_prep", s);
        hipLaunchKernelGGL((k_exp_prep<HD>), dim3((unsigned)(pr.B * pr.H * (long long)ntile)), dim3(256), 0, s, dO, O, L, sc, rows, pr.H,
                           ntile);
        if (!launch_ok()) return PA_ERR_HIP;
    }
    {
        const Order o = order_of(pr, 128, pr.Tk);
        LaunchScope ls("exp_bwd_dkdv", s);
        hipLaunchKernelGGL((k_exp_dkdv<HD, 32, Shape<HD>::DKDV_WPE, CAP, BIAS>), dim3((unsigned)blocks_of(o, true)), dim3(256), 0, s, Q, K,
                           V, mk.slopes, dO, sc, dK, dV, o, rows, score_of(pr), pr.scale);
        if (!launch_ok()) return PA_ERR_HIP;
    }
    const Order o = order_of(pr, 128, pr.T);
    LaunchScope ls("exp_bwd_dq", s);
    hipLaunchKernelGGL((k_exp_dq<HD, 32, Shape<HD>::DQ_WPE, CAP, BIAS>), dim3((unsigned)blocks_of(o, false)), dim3(256), 0, s, Q, K, V,
                       mk.slopes, dO, sc.stat, dQ, o, rows, score_of(pr), pr.scale);
    return launch_ok() ? PA_OK : PA_ERR_HIP;
}

// the instance of a problem
template <typename F>
pa_status dispatch(const pa_exp_problem& pr, const ExpMask& mk, F f) {
    auto with = [&](auto hd) {
        const bool cap = pr.cap > 0.f, bias = mk.slopes != nullptr;
        if (cap) return bias ? f(hd, std::true_type{}, std::true_type{}) : f(hd, std::true_type{}, std::false_type{});
        return bias ? f(hd, std::false_type{}, std::true_type{}) : f(hd, std::false_type{}, std::false_type{});
    };
    switch (pr.d) {
        case 32: return with(std::integral_constant<int, 32>{});
        case 64: return with(std::integral_constant<int, 64>{});
        case 128: return with(std::integral_constant<int, 128>{});
    }
    return PA_ERR_UNSUPPORTED;
}
Rows rows_of(const pa_exp_problem& pr, const ExpMask& mk) {
    return {mk.lo, mk.hi, std::min(pr.window, 1 << 30), pr.Tk - pr.T, pr.T, pr.Tk};
}

}  // namespace
}  // namespace mfma

using namespace mfma;

bool exp_grid_ok(const pa_exp_problem& pr) {
    const long long most = 0x7fffffffLL;
    return blocks_of(order_of(pr, 128, pr.T), false) <= most && blocks_of(order_of(pr, 128, pr.Tk), true) <= most &&
           (long long)pr.B * pr.H * ((pr.T + AT - 1) / AT) <= most;
}

size_t exp_workspace_bytes(const pa_exp_problem& pr, bool backward) {
    if (!backward) return 0;
    const BwdScratch sc = bwd_scratch(pr, nullptr);
    return (size_t)(char*)sc.ends + align_up((size_t)pr.B * ((pr.T + AT - 1) / AT) * sizeof(int4), 256);
}

pa_status exp_fwd(const pa_exp_problem& pr, const bf16_t* Q, const bf16_t* K, const bf16_t* V, ExpMask mk, bf16_t* O, float* L, char*,
                  hipStream_t s) {
    return dispatch(pr, mk, [&](auto hd, auto cap, auto bias) {
        return fwd_t<decltype(hd)::value, decltype(cap)::value, decltype(bias)::value>(pr, Q, K, V, mk, rows_of(pr, mk), O, L, s);
    });
}

pa_status exp_bwd(const pa_exp_problem& pr, const bf16_t* Q, const bf16_t* K, const bf16_t* V, ExpMask mk, const bf16_t* O,
                  const float* L, const bf16_t* dO, bf16_t* dQ, bf16_t* dK, bf16_t* dV, char* ws, hipStream_t s) {
    return dispatch(pr, mk, [&](auto hd, auto cap, auto bias) {
        return bwd_t<decltype(hd)::value, decltype(cap)::value, decltype(bias)::value>(pr, Q, K, V, mk, rows_of(pr, mk), O, L, dO, dQ, dK,
                                                                                     dV, ws, s);
    });
}

}  // namespace pa
