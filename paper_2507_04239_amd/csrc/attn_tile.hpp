// What the attention-form kernels share (bf16, 32x32x16 MFMA): the streamed tile of 64 rows in LDS, its operands, the rows of a
// result.  Layouts of the MFMAs: mfma_common.hpp.
#pragma once

#include "mfma_common.hpp"

namespace pa {
namespace mfma {
namespace {

constexpr int AT = 64;   // rows per streamed tile

template <int HD>
struct AttnTile {
    bf16_t r[AT][HD + 8];   // pitch (HD + 8) / 2 dwords = 4 (mod 8): the 16 rows of a fragment read hit distinct banks
};

// z + the sum of 8 bf16 values (exact products with one, float32 sums)
__device__ __forceinline__ float sum_bf16x8(const Frag& f, float z) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int i = 0; i < 8; i += 2) z = __builtin_amdgcn_fdot2_f32_bf16((bf16x2){f.v[i], f.v[i + 1]}, one, z, false);
    return z;
}

// Staging of a 64-row tile of a row-major [.][HD] array: HD / 32 pieces of 16 bytes per thread,
// piece id = tid + 256 q is row id / (HD / 8), features 8 (id % (HD / 8)) .. + 7.  The pieces wait
// in registers while the tile before them is being used (plain arrays and unrolled loops in the
// kernels: wrapped in a struct they end up in scratch memory).
// T need not be a multiple of the tile: rows past the end are read as row T - 1 (keys and queries
// there are masked out by causality, or never stored) or, with ZERO, as zeros (ghat, whose rows
// past the end must not contribute to dK, dV).
template <int HD, bool ZERO>
__device__ __forceinline__ uint4 piece_load(const bf16_t* __restrict__ head_base, int row0, int id, int T) {
    const int row = row0 + id / (HD / 8);
    const uint4 u = *(const uint4*)(head_base + (size_t)min(row, T - 1) * HD + 8 * (id % (HD / 8)));
    return ZERO && row >= T ? make_uint4(0, 0, 0, 0) : u;
}
template <int HD>
__device__ __forceinline__ void piece_store(AttnTile<HD>& dst, int id, uint4 u) {
    *(uint4*)&dst.r[id / (HD / 8)][8 * (id % (HD / 8))] = u;
}
#define PA_TILE_LOAD(REGS, BASE, ROW0, ZERO)        \
    _Pragma("unroll") for (int q_ = 0; q_ < HD / 32; ++q_) REGS[q_] = piece_load<HD, ZERO>(BASE, ROW0, tid + 256 * q_, T);
#define PA_TILE_STORE(DST, REGS)                    \
    _Pragma("unroll") for (int q_ = 0; q_ < HD / 32; ++q_) piece_store<HD>(DST, tid + 256 * q_, REGS[q_]);

// row 32 blk + r32, features 16 ks + 8 h .. + 7: A operand (rows x features) or B operand
// (features x rows) of a contraction over the features
template <int HD>
__device__ __forceinline__ bf16x8 row_frag(const AttnTile<HD>& t, int blk, int ks, int lane) {
    Frag f;
    f.u = *(const uint4*)&t.r[32 * blk + (lane & 31)][16 * ks + 8 * (lane >> 5)];
    return f.v;
}
template <int HD>
__device__ __forceinline__ bf16x8 row_frag_global(const bf16_t* __restrict__ X, size_t row, int ks, int h) {
    Frag f;
    f.u = *(const uint4*)(X + row * HD + 16 * ks + 8 * h);
    return f.v;
}

// A operand of a contraction over the tile's rows: column 32 cb + r32, k-slots = rows 16 j + 4 h .. + 3 and 8 further.
// The transposing read hands lane n of a 16-lane group column n of the 4 x 16 block whose row i the lanes 4 i .. 4 i + 3
// point at (4 columns each).
template <int HD>
__device__ __forceinline__ bf16x8 col_frag(const AttnTile<HD>& t, int j, int cb, int lane) {
    typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
    const int r16 = lane & 15, h = lane >> 5, odd = (lane >> 4) & 1;
    const bf16_t* p = &t.r[16 * j + 4 * h + (r16 >> 2)][32 * cb + 16 * odd + 4 * (r16 & 3)];
    union {
        bf16x8 v;
        bf16x4 h[2];
    } f;
    f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
    f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 8 * (HD + 8)));
    return f.v;
}
__device__ __forceinline__ f32x16 splat16(float x) {
    f32x16 v;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = x;
    return v;
}
// four values per accumulator quad k: rows 8 k + 4 h + r of a per-row float array
__device__ __forceinline__ void row_values(float (&o)[16], const float* base, int h) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float4 q = *(const float4*)(base + 8 * k + 4 * h);
        o[4 * k] = q.x; o[4 * k + 1] = q.y; o[4 * k + 2] = q.z; o[4 * k + 3] = q.w;
    }
}
// one 32-row block of an output row's columns: dst[8 k + 4 h + r] = f acc[4 k + r] (bf16); two lanes 32 apart exchange
// halves so that each stores whole 16-byte runs
__device__ __forceinline__ void store_block(bf16_t* dst, const f32x16& acc, float f, int h, bool in) {
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        union {
            bf16x4 v;
            uint2 u;
        } x, y;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x.v[r] = (__bf16)(f * acc[4 * k + r]);
            y.v[r] = (__bf16)(f * acc[4 * k + 4 + r]);
        }
        const auto d0 = __builtin_amdgcn_permlane32_swap(x.u.x, y.u.x, false, false);
        const auto d1 = __builtin_amdgcn_permlane32_swap(x.u.y, y.u.y, false, false);
        if (in) *(u32x4*)(dst + 8 * (k + h)) = (u32x4){d0[0], d1[0], d0[1], d1[1]};
    }
}

}  // namespace
}  // namespace mfma
}  // namespace pa
