// attention.hpp -- what the attention kernels share: tiles of rows in LDS, matrix-core operands from them, scores.
//
// Every product is formed "transposed", with the rows a wave owns (queries in the forward and for dQ, keys for dK and dV) as the
// COLUMNS of 32x32x16 MFMAs: a lane then holds one column, so that maxima, sums, log-sum-exps and masks of a row are one
// value per lane, and a result tile, rounded to 16 bits, is in place as the B operand of the next product -- if the
// contracted index is counted in the order in which the accumulator has it:
//   accumulator register i of lane l:  row 8*(i/4) + 4*(l/32) + i%4,  column l%32
//   B operand element e of lane l, registers 8g..8g+7 packed:  index 16g + 8*(e/4) + 4*(l/32) + e%4
// and the A operand of that product is read from LDS in the same order: two transposing reads of four rows each, at
// rows 16g + 4*(l/32) and 8 further on.
//
// A tile's rows are DP elements (DP: head_dim padded to 64 or 128 with zeros), in pieces of 16 bytes, piece c of row r
// at place c ^ turn(r), so that rows' pieces c (plain reads) and four rows' 32-byte pairs of pieces (transposing reads) lie in
// different banks.  Measured per wave and read, for ten such orders: plain 2.2 ns and transposing 1.1 ns at best, and so for the order
// of 64 elements; for 128 the one that takes 3.5 and 1.7 ns, whose turns repeat every eight rows: the kernels are not bound by these reads,
// and the best order's many addresses cost the walk over rows 711 -> 775 us (4 x 4096 x 16 heads).  Without any: 27 and 3.7 ns.
#pragma once
#include <hip/hip_runtime.h>

#include "api_util.hpp"
#include "common.hpp"

namespace mesa {

typedef float at_acc __attribute__((ext_vector_type(16)));
typedef __bf16 at_v8b __attribute__((ext_vector_type(8)));
typedef _Float16 at_v8h __attribute__((ext_vector_type(8)));
typedef short at_v4s __attribute__((ext_vector_type(4)));
typedef __bf16 at_v2b __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kAtLow = -3.0e38f;      // a running maximum before anything is seen; finite, so that (-inf) - it is -inf
constexpr float kAtMostCap = 256.0f;    // tanh is formed with an absolute error, 2^-23 or so, which a score has cap-fold
constexpr int kAtDrop = 8;              // binary16 probabilities of the backward carry this power of two, clear of subnormal values

template <typename T> struct AtNum;
template <> struct AtNum<_Float16> {
    static constexpr bool kHalf = true;
    __device__ static __forceinline__ at_acc mfma(u32x4 a, u32x4 b, at_acc c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(at_v8h, a), __builtin_bit_cast(at_v8h, b), c, 0, 0, 0);
    }
    __device__ static __forceinline__ uint32_t pack(float a, float b)      // round to nearest even
    {
        h2 p;
        p.x = _Float16(a);
        p.y = _Float16(b);
        return as_u32(p);
    }
    __device__ static __forceinline__ uint32_t rest(float a, float b, uint32_t w)      // what pack left of them
    {
        const h2 p = as_h2(w);
        return pack(a - float(p.x), b - float(p.y));
    }
};
template <> struct AtNum<__bf16> {
    static constexpr bool kHalf = false;
    __device__ static __forceinline__ at_acc mfma(u32x4 a, u32x4 b, at_acc c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(at_v8b, a), __builtin_bit_cast(at_v8b, b), c, 0, 0, 0);
    }
    __device__ static __forceinline__ uint32_t pack(float a, float b)
    {
        at_v2b p;
        p.x = __bf16(a);
        p.y = __bf16(b);
        return __builtin_bit_cast(uint32_t, p);
    }
    __device__ static __forceinline__ uint32_t rest(float a, float b, uint32_t w) { return pack(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xFFFF0000u)); }
};

// a tensor (B, tokens, heads, D) as the kernels see it; strides in bytes
struct AtView {
    const char *p;
    int64_t batch, token, head;
};
struct AtOut {
    char *p;
    int64_t batch, token, head;
};

// the shape: rows of a (sequence, key head) pair are its tokens times the G query heads of the group, token by token
struct AtShape {
    int32_t B, Nq, Nk, Hq, Hk, G, D;
    uint32_t R;                         // Nq * G
    FastDiv div_g;
    float c;                            // scores to powers of two: scale * log2(e); with a cap 2 log2(e) scale / cap
    float cap2;                         // cap * log2(e)
    float scale;
    const int32_t *lo, *hi, *q_start;
    const float *slopes;
};

struct AtRow {
    uint32_t token, g;
};
__device__ __forceinline__ AtRow at_row(const AtShape &s, uint32_t r)
{
    AtRow w;
    w.token = s.G == 1 ? r : fastdiv(r, s.div_g);
    w.g = r - w.token * uint32_t(s.G);
    return w;
}
// the interval of row `token` of sequence b, cut to the keys that there are; 0, 0 where it holds none
__device__ __forceinline__ void at_interval(const AtShape &s, int b, uint32_t token, int &lo, int &hi)
{
    lo = 0;
    hi = s.Nk;
    if (s.lo) {
        lo = s.lo[int64_t(b) * s.Nq + token];
        hi = s.hi[int64_t(b) * s.Nq + token];
        lo = lo < 0 ? 0 : lo;
        hi = hi > s.Nk ? s.Nk : hi;
    }
    if (lo >= hi) lo = hi = 0;
}
__device__ __forceinline__ int at_place(const AtShape &s, int b, uint32_t token)
{
    return int(token + uint32_t(s.q_start ? s.q_start[b] : s.Nk - s.Nq));
}

// linear in the row's bits: turn(a ^ b) = turn(a) ^ turn(b)
template <int DP> __device__ __forceinline__ constexpr int at_turn(int row) { return ((row & 3) << 1) ^ ((row >> 2) & (DP == 128 ? 1 : 7)); }

// ROWS x DP elements from memory to LDS by NT threads, by way of registers.  Rows past `rows` and pieces past D become zeros: they lie
// outside of the span, whose end is the last row's (rows that overlap in memory, as where one key stands for all, come again instead).
template <int NT, int ROWS, int DP> struct AtTile {
    static constexpr int kPieces = DP / 8, kN = ROWS * kPieces / NT, kBytes = ROWS * DP * 2;
    static_assert(ROWS * kPieces % NT == 0 && NT % kPieces == 0, "whole rows per step of the threads");
    u32x4 r[kN];
    __device__ static __forceinline__ uint32_t place(uint32_t stride, int D)       // of this thread's first piece
    {
        const int piece = int(threadIdx.x) % kPieces;
        return piece * 8 < D ? uint32_t(int(threadIdx.x) / kPieces) * stride + piece * 16 : kNowhere;
    }
    __device__ __forceinline__ void load(const char *base, int rows, uint32_t stride, int D, uint32_t at)
    {
        const Span s(base, uint32_t((rows < ROWS ? rows : ROWS) - 1) * stride + uint32_t(D) * 2);
#pragma unroll
        for (int k = 0; k < kN; ++k) s.load_kept(at == kNowhere ? kNowhere : at + uint32_t(k * (NT / kPieces)) * stride, r[k]);
    }
    __device__ __forceinline__ void keep(uint64_t rows)      // rows without a bit become zeros
    {
#pragma unroll
        for (int k = 0; k < kN; ++k)
            if (!(rows >> ((int(threadIdx.x) + k * NT) / kPieces) & 1u)) r[k] = u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void store(char *lds) const
    {
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const int i = int(threadIdx.x) + k * NT, row = i / kPieces, piece = i % kPieces;
            *reinterpret_cast<u32x4 *>(lds + row * (DP * 2) + ((piece ^ at_turn<DP>(row)) << 4)) = r[k];
        }
    }
};

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Wint-to-pointer-cast"      // the host pass counts pointers in 64 bits
// LDS by its 32-bit address: a lane's place in a tile is one register for plain reads and one for transposing ones; which
// piece a read takes is an exclusive-or with a constant (tiles start at multiples of 128 bytes, whose turns stay within them), the row an immediate offset.
__device__ __forceinline__ uint32_t at_address(const char *lds) { return uint32_t(uintptr_t((__attribute__((address_space(3))) const char *)lds)); }
template <int DP> __device__ __forceinline__ uint32_t at_plain_lane(int lane) { return (lane & 31) * (DP * 2) + (((lane >> 5) ^ at_turn<DP>(lane & 31)) << 4); }
template <int DP> __device__ __forceinline__ uint32_t at_trans_lane(int lane)
{
    const int sl = lane & 15, row = 4 * (lane >> 5) + (sl >> 2), piece = ((lane >> 4) & 1) * 2 + ((sl & 3) >> 1);
    return row * (DP * 2) + ((piece ^ at_turn<DP>(row)) << 4) + (sl & 1) * 8;
}
// A operand, rows as they lie: rows row0..row0+31 of the tile (row0 a multiple of 32), elements 16*ks ..+15; at: tile's address + at_plain_lane
template <int DP> __device__ __forceinline__ u32x4 at_plain(uint32_t at, int row0, int ks)
{
    typedef __attribute__((address_space(3))) const u32x4 *lds_p;
    return *(lds_p)((at ^ uint32_t((ks & 3) << 5)) + uint32_t(row0 * (DP * 2) + (ks >> 2) * 128));
}
// A operand, transposed: elements d0..d0+31 (d0 a multiple of 32) as its rows, the tile's rows row0..row0+15 (a multiple of 16) as the
// contracted index; at: tile's address + at_trans_lane
template <int DP> __device__ __forceinline__ u32x4 at_transposed(uint32_t at, int row0, int d0)
{
    typedef __attribute__((address_space(3))) at_v4s *lds_p;
    const uint32_t p = (at ^ uint32_t((((d0 >> 3) & 7) ^ at_turn<DP>(row0 & 31)) << 4)) + uint32_t(row0 * (DP * 2) + (d0 >> 6) * 128);
    const uint32_t q = (at ^ uint32_t((((d0 >> 3) & 7) ^ at_turn<DP>((row0 & 31) + 8)) << 4)) + uint32_t((row0 + 8) * (DP * 2) + (d0 >> 6) * 128);
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)p));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)q));
    return u32x4{a[0], a[1], b[0], b[1]};
}

#pragma clang diagnostic pop

// B operand straight from memory: elements 16*ks + 8*(lane/32) ..+7 of the lane's row, zeros past D
__device__ __forceinline__ u32x4 at_column(const char *row, int ks, int lane, int D)
{
    const int d = ks * 16 + (lane >> 5) * 8;
    return d < D ? *reinterpret_cast<const u32x4 *>(row + d * 2) : u32x4{0u, 0u, 0u, 0u};
}

// the partner's value of the same column (lane ^ 32) beside the lane's own
__device__ __forceinline__ float at_pair_max(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float at_pair_sum(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ int at_wave_min(int v)      // over the 32 columns; uniform
{
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) { const int o = __shfl_xor(v, m, 64); v = o < v ? o : v; }
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int at_wave_max(int v)
{
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) { const int o = __shfl_xor(v, m, 64); v = o > v ? o : v; }
    return __builtin_amdgcn_readfirstlane(v);
}

__device__ __forceinline__ float at_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// tanh of x, for u = 2 log2(e) x.  EXACT:  (1 - 2^-|u|) / (1 + 2^-|u|) with the sign of u -- the difference is exact where it is small, so that
// what is left of an error is that of the power; times the cap it is a score's, which the forward hands on in lse.  Else  1 - 2 / (2^u + 1),
// two instructions less and off by twice that, 1e-7: for the backward, whose probabilities are rounded to 16 bits.  Both hand NaN on.
template <bool EXACT> __device__ __forceinline__ float at_tanh(float u)
{
    if (!EXACT) return fmaf(-2.0f, __builtin_amdgcn_rcpf(at_exp2(u) + 1.0f), 1.0f);
    const float e = at_exp2(-fabsf(u));
    return __builtin_copysignf((1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e), u);
}

// index within a 32-row accumulator tile of register i, without the lane's part 4*(lane/32)
__device__ __forceinline__ constexpr int at_reg_row(int i) { return 8 * (i / 4) + i % 4; }

// Tiles of keys at the edge of what a workgroup's rows see: keys that none of them sees are stored as zeros, so that what they hold
// (padding; infinities and NaN there) enters no product as 0 * NaN.  lo, hi: this lane's row; the waves' answers meet in `seen`.
// A bit per key of the tile; ends in a barrier's worth of order, so every wave of the workgroup has to come.
template <int NW> __device__ __forceinline__ uint64_t at_seen(uint64_t *seen, int wave, int lane, int j0, int lo, int hi)
{
    bool any = false;
#pragma unroll 8
    for (int i = 0; i < 32; ++i) {
        const int l = __builtin_amdgcn_readlane(lo, i), h = __builtin_amdgcn_readlane(hi, i);
        any |= uint32_t(j0 + lane - l) < uint32_t(h - l);
    }
    uint64_t m = __ballot(any);
    if (NW == 1) return m;
    __syncthreads();                               // the last answers have been read
    if (lane == 0) seen[wave] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) m |= seen[w];
    return m;
}

// four consecutive elements of a result row
template <typename T> __device__ __forceinline__ void at_store4(char *p, float a, float b, float c, float d)
{
    *reinterpret_cast<u32x2 *>(p) = u32x2{AtNum<T>::pack(a, b), AtNum<T>::pack(c, d)};
}

// ---- host side ----
inline bool at_valid(const mesa_attention &a)
{
    const int64_t top = int64_t(1) << 30;
    return a.B >= 0 && a.Nq >= 0 && a.Nk >= 0 && a.Hk >= 1 && a.Hq >= 1 && a.Hq % a.Hk == 0 && a.D >= 1 && a.scale > 0.0f && a.scale < __builtin_inff() && a.cap >= 0.0f &&
           a.cap < __builtin_inff() && a.scale < 1.0e37f && (a.cap == 0.0f || a.scale / a.cap < 1.0e37f) && a.B < top && a.Nq < top && a.Nk < top && a.Hq < top && a.Hk < top;
}
// MESA_OK, or why the kernels do not take this shape
inline mesa_status at_supported(const mesa_attention &a, mesa_dtype dt)
{
    if (!valid_dtype(dt) || !at_valid(a)) return MESA_ERR_INVALID_ARG;
    if (dt == MESA_F32 || a.D % 8 != 0 || a.D > 128 || a.cap > kAtMostCap) return MESA_ERR_UNSUPPORTED;
    // rows and pieces of a head are counted in 32 bits, workgroups by what a launch takes; below these, products of two sizes fit 64 bits
    const int64_t top = int64_t(1) << 31;
    if (a.Nq >= top / (a.Hq / a.Hk) || a.Nq >= top * 8 / a.D || a.Nk >= top * 8 / a.D || a.B > most_workgroups(256) / a.Hk) return MESA_ERR_UNSUPPORTED;
    return MESA_OK;
}
AtShape at_shape(const mesa_attention &a, const mesa_attention_mask &m);

}  // namespace mesa
