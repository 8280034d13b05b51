// attention_bwd.hip -- the backward of attention over intervals of keys, at operands that were saved as codes.
//   p = exp(s - lse),  delta_i = do_i.o_i,  ds = p (do.v - delta) (times the cap's derivative 1 - tanh^2)
//   dv_j = sum_i p_ij do_i,   dk_j = scale sum_i ds_ij q_i,   dq_i = scale sum_j ds_ij k_j
//
// Three steps on the stream: a pass over the rows leaves delta, log-sum-exps and intervals, row by row, and turns codes into 16-bit
// operands in the workspace (they are read many times over); then keys (dk and dv: a wave owns 32 keys and walks over
// the rows) and queries (dq: a wave owns 32 rows and walks over the keys).  The scores are formed in both, seven products instead
// of five: dq added up across workgroups would need atomics, whose order changes the result.  A group's heads are rows of
// the same walk, so the gradients of a shared key head add up in registers.
//
// binary16 storage: p goes into its products 2^8-fold, and ds with a power of two from the norms of do and v that keeps it
// below 2^15 and as far as it can from the subnormal values, where products of long rows' probabilities and of small
// gradients would lose their bits.  bfloat16 has the exponents of binary32 and needs neither.
// Measured, 4 x 4096 x 16 heads of 128 on 4, causal, bfloat16: rows 29 us (145 MB, 5 TB/s), dk and dv 600 (four products, 0.92 PFLOP/s),
// dq 405 (three products, 1.0 PFLOP/s; a large library product 1.2).  32 x 12 heads of 197 keys, all codes: 13.5 and 43, by latency.
#include "attention.hpp"

namespace mesa {

bool at_strides(const mesa_attention &a, int64_t tokens, int64_t heads, int64_t batch, int64_t token, int64_t head);

constexpr int kAbRows = 128;           // rows of a workgroup of the row pass, and keys of one of its value norms
constexpr int kAbTile = 32;            // rows per step of the walk over rows
constexpr int kAbKeys = 128;           // keys of a workgroup

// The walk over rows takes them in tiles of 32 places: as many whole tokens of a group's G heads as fit, or 32 of one token's
// heads where G is larger, so that a place's token and head within its tile are the same in every tile.
struct AbOrder {
    int32_t tokens, heads, parts;      // of a tile: tokens, heads; tiles per token (1 where a token fits)
    uint32_t tiles;                    // of a (sequence, key head) pair; always even
    FastDiv div_heads, div_parts;
};
enum { kAbLse = 0, kAbDelta, kAbLo, kAbHi, kAbSlope, kAbPlace, kAbEmpty, kAbWords };   // 32 words of each per tile
struct AbRows {                        // what the row pass leaves
    uint32_t *info;                    // [b * Hk + key head][tile][word][place]: log-sum-exp in powers of two (3e38 where nothing is seen), -delta,
                                       // interval, slope in powers of two, place of the query, 1.0f where nothing is seen
    int4 *tiles;                       // [..][tile]: least lo, largest hi of the rows that see something; largest lo, least hi of all
    float2 *most;                      // [..][four tiles]: largest |do|, largest |delta|   (binary16 only)
    float *values;                     // [..][128 keys]: largest |v|                       (binary16 only)
    uint32_t blocks, key_blocks;       // of four tiles, of 128 keys
};
struct AbPlace {
    int64_t token;
    int32_t g;
    bool live;
};
__device__ __forceinline__ AbPlace ab_place(const AtShape &s, const AbOrder &w, uint32_t tile, int x)   // the row of a tile's place x
{
    const uint32_t t = w.parts == 1 ? tile : fastdiv(tile, w.div_parts), dt = fastdiv(uint32_t(x), w.div_heads);
    AbPlace p;
    p.token = int64_t(t) * w.tokens + dt;
    p.g = int(tile - t * w.parts) * 32 + (x - int(dt) * w.heads);
    p.live = int(dt) < w.tokens && p.token < s.Nq && p.g < s.G;
    return p;
}
__device__ __forceinline__ int64_t ab_info(const AbOrder &w, uint32_t head, uint32_t token, uint32_t g)   // where a row's words are
{
    const uint32_t t = token / uint32_t(w.tokens), x = (token - t * w.tokens) * w.heads + (g & 31u);
    return (int64_t(head) * w.tiles + t * w.parts + (w.parts == 1 ? 0 : g >> 5)) * (kAbWords * 32) + (w.parts == 1 ? (token - t * w.tokens) * w.heads + g : x);
}
struct AtBwd {
    AtShape s;
    AtView q, k, v, o, dO;
    AtOut dq, dk, dv;
    const float *lse;
    AbRows w;
    AbOrder order;
    float *part;                       // [split][b * Hk + head][Nk][2][D]; null: no split
    float *part_q;                     // [row split][b * Hk + head][row][D]; null: no split
    uint32_t heads, key_blocks, splits, row_blocks, row_splits;
};

// codes to contiguous (B, heads, tokens, D) elements, as mesa_dequantize; eight per thread
struct AbCodes {
    AtView q;
    const float *alpha, *beta;
    char *out;
    int32_t heads, tokens;
    uint32_t first, per_head;          // workgroups: the operand's first one, those of a (sequence, head)
};
struct AbOperands {
    AbCodes c[3], v;                   // v: values that the row pass has to read anyway
    int32_t count;
    bool values;
    FastDiv div_d;                     // by D / 8
};
template <typename T> __device__ __forceinline__ typename Store<T>::raw_t ab_operand(const AbCodes &c, int D, uint32_t b, uint32_t h, uint32_t t, uint32_t e)
{
    const u32x2 v = *reinterpret_cast<const u32x2 *>(c.q.p + int64_t(b) * c.q.batch + int64_t(t) * c.q.token + int64_t(h) * c.q.head + e);
    float f[8];
    codes_to_float(v, f);
    const float s = c.alpha[h] / 255.0f, z = c.beta[h];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float y = f[k] * s;
        f[k] = y + z;
    }
    const typename Store<T>::raw_t r = Store<T>::pack(f);
    Store<T>::store(c.out, ((int64_t(b) * c.heads + h) * c.tokens + t) * D + e, r);
    return r;
}

// The row pass.  Workgroups [0, blocks) of a head: the deltas of 128 places, log-sum-exps, intervals and the summaries of their four
// tiles; further ones (binary16): the largest norm of 128 keys' values, which become elements there if they are codes.  Eight or sixteen
// lanes per row.  Behind all heads' the workgroups of the other operands that are codes.
template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void k_attn_rows(const AtBwd a, const AbOperands in)
{
    constexpr int kLanes = DP / 8, kPer = kThreads / kLanes;
    const AtShape &s = a.s;
    const uint32_t mine = a.heads * (a.w.blocks + (AtNum<T>::kHalf ? a.w.key_blocks : 0));
    if (blockIdx.x >= mine) {
        const uint32_t at = blockIdx.x - mine;
        const int n = in.count > 2 && at >= in.c[2].first ? 2 : in.count > 1 && at >= in.c[1].first ? 1 : 0;
        const AbCodes &c = n == 0 ? in.c[0] : n == 1 ? in.c[1] : in.c[2];
        const uint32_t blk = at - c.first, bh = blk / c.per_head, b = bh / uint32_t(c.heads), h = bh - b * uint32_t(c.heads);
        const uint32_t i = (blk - bh * c.per_head) * kThreads + threadIdx.x, t = fastdiv(i, in.div_d), e = (i - t * uint32_t(s.D / 8)) * 8;
        if (t < uint32_t(c.tokens)) ab_operand<T>(c, s.D, b, h, t, e);
        return;
    }
    const uint32_t head = blockIdx.x % a.heads, blk = blockIdx.x / a.heads;
    const int b = int(head / uint32_t(s.Hk)), hk = int(head) - b * s.Hk;
    const int tid = threadIdx.x, part = tid % kLanes, first = tid / kLanes;
    __shared__ float top[2][kThreads / 64];
    float most = 0.0f, most_delta = 0.0f;
    if (blk >= a.w.blocks) {                               // values
        const uint32_t kb = blk - a.w.blocks;
        for (int r = first; r < kAbRows; r += kPer) {
            const int j = int(kb) * kAbRows + r;
            float ss = 0.0f;
            if (j < s.Nk && part * 8 < s.D) {
                float f[8];
                Store<T>::unpack(in.values ? ab_operand<T>(in.v, s.D, uint32_t(b), uint32_t(hk), uint32_t(j), uint32_t(part) * 8)
                                                : Store<T>::load(a.v.p + int64_t(b) * a.v.batch + int64_t(j) * a.v.token + int64_t(hk) * a.v.head, part * 8), f);
#pragma unroll
                for (int k = 0; k < 8; ++k) ss = fmaf(f[k], f[k], ss);
            }
            ss = lanes_sum_dpp<kLanes>(ss);
            if (ss < __builtin_inff()) most = fmaxf(most, ss);   // not finite: a row that no query sees
        }
    } else {
        __shared__ uint32_t empty[kAbRows / 32];
        if (tid < kAbRows) {
            const uint32_t tile = blk * 4 + (tid >> 5);
            const int x = tid & 31;
            const AbPlace row = ab_place(s, a.order, tile, x);
            int lo = 0, hi = 0, place = 0;
            float lse2 = 3.0e38f, slope2 = 0.0f;
            if (row.live) {
                at_interval(s, b, uint32_t(row.token), lo, hi);
                if (hi > 0) {
                    lse2 = a.lse[(int64_t(b) * s.Hq + hk * s.G + row.g) * s.Nq + row.token] * kLog2e;
                    if (AtNum<T>::kHalf) lse2 -= float(kAtDrop);
                }
                place = at_place(s, b, uint32_t(row.token));
                if (s.slopes) slope2 = s.slopes[hk * s.G + row.g] * kLog2e;
            }
            const uint64_t none = __ballot(hi == 0);
            int l0 = hi > 0 ? lo : 0x7FFFFFFF, h1 = hi, l1 = lo, h0 = hi;
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) {
                int y = __shfl_xor(l0, m, 64); l0 = y < l0 ? y : l0;
                y = __shfl_xor(h1, m, 64); h1 = y > h1 ? y : h1;
                y = __shfl_xor(l1, m, 64); l1 = y > l1 ? y : l1;
                y = __shfl_xor(h0, m, 64); h0 = y < h0 ? y : h0;
            }
            if (tile < a.order.tiles) {
                const int64_t at = int64_t(head) * a.order.tiles + tile;
                uint32_t *p = a.w.info + at * (kAbWords * 32) + x;
                p[kAbLse * 32] = __float_as_uint(lse2);
                p[kAbLo * 32] = uint32_t(lo);
                p[kAbHi * 32] = uint32_t(hi);
                p[kAbSlope * 32] = __float_as_uint(slope2);
                p[kAbPlace * 32] = uint32_t(place);
                p[kAbEmpty * 32] = __float_as_uint(hi == 0 ? 1.0f : 0.0f);
                if (x == 0) a.w.tiles[at] = make_int4(l0, h1, l1, h0);
            }
            if (x == 0) empty[tid >> 5] = uint32_t(none >> (tid & 32));
        }
        __syncthreads();
        for (int y = first; y < kAbRows; y += kPer) {
            const uint32_t tile = blk * 4 + (y >> 5);
            const AbPlace row = ab_place(s, a.order, tile, y & 31);
            const bool live = row.live && !(empty[y >> 5] >> (y & 31) & 1u);
            float dot = 0.0f, ss = 0.0f;
            if (live && part * 8 < s.D) {
                const int64_t h = hk * s.G + row.g;
                float f[8], g[8];
                Store<T>::unpack(Store<T>::load(a.o.p + int64_t(b) * a.o.batch + row.token * a.o.token + h * a.o.head, part * 8), f);
                Store<T>::unpack(Store<T>::load(a.dO.p + int64_t(b) * a.dO.batch + row.token * a.dO.token + h * a.dO.head, part * 8), g);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    dot = fmaf(f[k], g[k], dot);
                    ss = fmaf(g[k], g[k], ss);
                }
            }
            dot = lanes_sum_dpp<kLanes>(dot);
            if (part == 0 && tile < a.order.tiles) a.w.info[(int64_t(head) * a.order.tiles + tile) * (kAbWords * 32) + kAbDelta * 32 + (y & 31)] = __float_as_uint(-dot);
            if (AtNum<T>::kHalf) {
                ss = lanes_sum_dpp<kLanes>(ss);
                if (ss < __builtin_inff()) most = fmaxf(most, ss);             // not finite: keys that the row sees get no better, others are to
                if (fabsf(dot) < __builtin_inff()) most_delta = fmaxf(most_delta, fabsf(dot));
            }
        }
    }
    if (!AtNum<T>::kHalf) return;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        most = fmaxf(most, __shfl_xor(most, m, 64));
        most_delta = fmaxf(most_delta, __shfl_xor(most_delta, m, 64));
    }
    if ((tid & 63) == 0) {
        top[0][tid >> 6] = most;
        top[1][tid >> 6] = most_delta;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kThreads / 64; ++w) {
            most = fmaxf(most, top[0][w]);
            most_delta = fmaxf(most_delta, top[1][w]);
        }
        if (blk >= a.w.blocks) a.w.values[int64_t(head) * a.w.key_blocks + (blk - a.w.blocks)] = sqrtf(most);
        else a.w.most[int64_t(head) * a.w.blocks + blk] = make_float2(sqrtf(most), most_delta);
    }
}

// the exponent e with 2^e * bound within [2^13, 2^14): |ds| stays below 2^15 with a bound on |do.v| + |delta|, rounding included
__device__ __forceinline__ int ab_exponent(float bound)
{
    if (!(bound > 0.0f)) return 0;
    const int e = 13 - (int(__float_as_uint(bound) >> 23) - 127);
    return e < -60 ? -60 : e > 100 ? 100 : e;
}
__device__ __forceinline__ float ab_pow2(int e) { return __uint_as_float(uint32_t(127 + e) << 23); }   // -126 <= e <= 127

// A wave's 32 result rows of accumulators (columns), by way of its own 32 * DP * 2 bytes of LDS: whole lines leave in 16-byte pieces, not eight bytes
// a row (32 x 12 heads of 512 keys 168 -> 161 us).  row(i): where row i goes, null where there is none.
template <typename T, int DP, typename Row> __device__ __forceinline__ void ab_put(char *lds, const at_acc *x, float mul, int lane, int D, Row row)
{
    constexpr int kPieces = DP / 8;
    char *own = lds + (lane & 31) * (DP * 2) + (lane >> 5) * 8;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int w = 0; w < 4; ++w) at_store4<T>(own + (((d * 4 + w) ^ (lane & 7)) << 4), x[d][4 * w] * mul, x[d][4 * w + 1] * mul, x[d][4 * w + 2] * mul, x[d][4 * w + 3] * mul);
    __builtin_amdgcn_wave_barrier();
    const int piece = lane % kPieces;
#pragma unroll
    for (int k = 0; k < kPieces / 2; ++k) {
        const int i = k * (64 / kPieces) + lane / kPieces;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + i * (DP * 2) + ((piece ^ (i & 7)) << 4));
        char *p = row(i);
        if (p && piece * 8 < D) *reinterpret_cast<u32x4 *>(p + piece * 16) = v;
    }
    __builtin_amdgcn_wave_barrier();
}

// scores of one accumulator in powers of two and, with a cap, the cap's derivative; away: place - key for register 0
// ALONG: the registers count keys (a lane is a row), else rows (a lane is a key)
template <bool CAP> __device__ __forceinline__ float ab_score(const AtShape &s, float x, float &slope)
{
    if (!CAP) return x * s.c;
    const float t = at_tanh<false>(x * s.c);
    slope = fmaf(-t, t, 1.0f);
    return s.cap2 * t;
}

// ---------------------------------------------------------------------------------------------
// dq: a wave owns 32 rows
// ---------------------------------------------------------------------------------------------
template <typename T, int DP, int NW, int BN, bool CAP, bool BIAS, bool FINE> __device__ __forceinline__ void ab_dq(const AtBwd &a, uint32_t block)
{
    typedef AtNum<T> Num;
    typedef AtTile<NW * 64, BN, DP> Tile;
    constexpr int kKs = DP / 16, kDt = DP / 32, kSub = BN / 32;
    __shared__ __attribute__((aligned(256))) char lds[4 * Tile::kBytes];
    __shared__ int range[4][NW];
    __shared__ uint64_t seen[NW];
    const AtShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), half = lane >> 5;
    const uint32_t head = block % a.heads, rest = block / a.heads, split = rest % a.row_splits, rb = a.row_blocks - 1 - rest / a.row_splits;
    const int b = int(head / uint32_t(s.Hk)), hk = int(head) - b * s.Hk;
    const uint32_t r_own = (rb * NW + wave) * 32 + (lane & 31), r = r_own < s.R ? r_own : s.R - 1;
    const AtRow row = at_row(s, r);
    const int hq = hk * s.G + int(row.g);
    const uint32_t *info = a.w.info + ab_info(a.order, head, row.token, row.g);
    const int lo = int(info[kAbLo * 32]), hi = int(info[kAbHi * 32]);
    float lse2 = __uint_as_float(info[kAbLse * 32]);
    const float delta = __uint_as_float(info[kAbDelta * 32]);      // with the sign that the sums do.v start from
    const int wlo = at_wave_min(hi > 0 ? lo : 0x7FFFFFFF), whi = at_wave_max(hi), flo = at_wave_max(lo), fhi = at_wave_min(hi);
    if (lane == 0) {
        range[0][wave] = wlo;
        range[1][wave] = whi;
        range[2][wave] = flo;
        range[3][wave] = fhi;
    }
    u32x4 qf[kKs], gf[kKs];
    {
        const char *p = a.q.p + int64_t(b) * a.q.batch + int64_t(row.token) * a.q.token + int64_t(hq) * a.q.head;
        const char *g = a.dO.p + int64_t(b) * a.dO.batch + int64_t(row.token) * a.dO.token + int64_t(hq) * a.dO.head;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            qf[ks] = at_column(p, ks, lane, s.D);
            gf[ks] = at_column(g, ks, lane, s.D);
        }
    }
    const float slope2 = BIAS ? s.slopes[hq] * kLog2e : 0.0f;
    const int place = BIAS ? at_place(s, b, row.token) : 0;
    __syncthreads();
    int blo = 0x7FFFFFFF, bhi = 0, full_lo[NW], full_hi[NW];      // the same of the workgroup's rows; what each wave's rows see, all of them
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        blo = range[0][w] < blo ? range[0][w] : blo;
        bhi = range[1][w] > bhi ? range[1][w] : bhi;
        full_lo[w] = __builtin_amdgcn_readfirstlane(range[2][w]);
        full_hi[w] = __builtin_amdgcn_readfirstlane(range[3][w]);
    }
    int t0 = bhi > 0 ? blo / BN : 0, t1 = bhi > 0 ? (bhi + BN - 1) / BN : 0;
    if (a.row_splits > 1) {
        const int per = (t1 - t0 + int(a.row_splits) - 1) / int(a.row_splits);
        t0 += int(split) * per;
        t1 = t0 + per < t1 ? t0 + per : t1;
    }
    t0 = __builtin_amdgcn_readfirstlane(t0);
    t1 = __builtin_amdgcn_readfirstlane(t1);

    const char *kbase = a.k.p + int64_t(b) * a.k.batch + int64_t(hk) * a.k.head, *vbase = a.v.p + int64_t(b) * a.v.batch + int64_t(hk) * a.v.head;
    Tile tk, tv;
    const uint32_t k_step = uint32_t(a.k.token), v_step = uint32_t(a.v.token), k_at = Tile::place(k_step, s.D), v_at = Tile::place(v_step, s.D);
    kbase += int64_t(t0) * BN * a.k.token;
    vbase += int64_t(t0) * BN * a.v.token;
    auto fetch = [&](int t) __attribute__((always_inline)) {        // t0, t0 + 1, ...
        tk.load(kbase, s.Nk - t * BN, k_step, s.D, k_at);
        tv.load(vbase, s.Nk - t * BN, v_step, s.D, v_at);
        kbase += int64_t(BN) * a.k.token;
        vbase += int64_t(BN) * a.v.token;
    };
    if (t0 < t1) fetch(t0);
    float undo = s.scale;                             // of the sums; the factor of ds goes into p, which nothing else here takes
    if (Num::kHalf) {
        float ss = 0.0f, vmax = 0.0f;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            float f[8];
            Store<T>::unpack(gf[ks], f);
#pragma unroll
            for (int k = 0; k < 8; ++k) ss = fmaf(f[k], f[k], ss);
        }
        ss = at_pair_sum(ss);
        for (int kb = t0 * BN / kAbRows; kb * kAbRows < t1 * BN && kb < int(a.w.key_blocks); ++kb) vmax = fmaxf(vmax, a.w.values[int64_t(head) * a.w.key_blocks + kb]);
        const int e = ab_exponent(sqrtf(ss) * vmax + fabsf(delta));
        lse2 -= float(e - kAtDrop);
        undo = s.scale * ab_pow2(-e);
    }

    at_acc dq[kDt];
#pragma unroll
    for (int d = 0; d < kDt; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] = 0.0f;

    const uint32_t plain_at = at_address(lds) + at_plain_lane<DP>(lane), trans_at = at_address(lds) + at_trans_lane<DP>(lane);
    auto work = [&](int cur, int j0, bool whole) __attribute__((always_inline)) {
        const uint32_t ka = plain_at + cur * 2 * Tile::kBytes, va = ka + Tile::kBytes, kt = trans_at + cur * 2 * Tile::kBytes;
#pragma unroll
        for (int t = 0; t < kSub; ++t) {
            at_acc x, y;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = 0.0f;
                y[i] = delta;
            }
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) {
                x = Num::mfma(at_plain<DP>(ka, t * 32, ks), qf[ks], x);
                y = Num::mfma(at_plain<DP>(va, t * 32, ks), gf[ks], y);
                if (ks % 2 == 1) __builtin_amdgcn_sched_barrier(0);
            }
            const int first = j0 + t * 32 + 4 * half;
            const float away = BIAS ? float(place - first) : 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float slope = 1.0f, p;
                if (!CAP && !BIAS) {
                    p = at_exp2(fmaf(x[i], s.c, -lse2));
                } else {
                    float sc = ab_score<CAP>(s, x[i], slope);
                    if (BIAS) sc = fmaf(-slope2, fabsf(away - float(at_reg_row(i))), sc);
                    p = at_exp2(sc - lse2);
                }
                x[i] = p * y[i];
                if (CAP) x[i] *= slope;
            }
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = uint32_t(first + at_reg_row(i) - lo) < uint32_t(hi - lo) ? x[i] : 0.0f;
            }
            u32x4 ds[2];
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int w = 0; w < 4; ++w) ds[g][w] = Num::pack(x[8 * g + 2 * w], x[8 * g + 2 * w + 1]);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int d = 0; d < kDt; ++d) {
                    const u32x4 f = at_transposed<DP>(kt, t * 32 + g * 16, d * 32);
                    dq[d] = Num::mfma(f, ds[g], dq[d]);
                    if (FINE) {
                        u32x4 rest;
#pragma unroll
                        for (int w = 0; w < 4; ++w) rest[w] = Num::rest(x[8 * g + 2 * w], x[8 * g + 2 * w + 1], ds[g][w]);
                        dq[d] = Num::mfma(f, rest, dq[d]);
                    }
                    if (d == kDt - 1) __builtin_amdgcn_sched_barrier(0);
                }
        }
    };
    for (int t = t0, cur = 0; t < t1; ++t, cur ^= 1) {
        char *lk = lds + cur * 2 * Tile::kBytes, *lv = lk + Tile::kBytes;
        const int j0 = t * BN;
        bool known = false;                         // some wave's rows see the whole tile: no key of it is unseen
#pragma unroll
        for (int w = 0; w < NW; ++w) known |= j0 >= full_lo[w] && j0 + BN <= full_hi[w];
        if (!known) {
            const uint64_t some = at_seen<NW>(seen, wave, lane, j0, lo, hi);
            tk.keep(some);
            tv.keep(some);
        }
        tk.store(lk);
        tv.store(lv);
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1);
        if (j0 + BN <= wlo || j0 >= whi) continue;
        work(cur, j0, j0 >= flo && j0 + BN <= fhi);
    }
    if (a.part_q) {
        if (r_own >= s.R) return;
        float *p = a.part_q + ((int64_t(split) * a.heads + head) * s.R + r_own) * s.D;
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int e = d * 32 + 8 * w + 4 * half;
                if (e < s.D) *reinterpret_cast<float4 *>(p + e) = make_float4(dq[d][4 * w] * undo, dq[d][4 * w + 1] * undo, dq[d][4 * w + 2] * undo, dq[d][4 * w + 3] * undo);
            }
        return;
    }
    __syncthreads();                                // the last tiles are done with
    const uint32_t r0 = (rb * NW + wave) * 32;
    char *out = a.dq.p + int64_t(b) * a.dq.batch + int64_t(hk) * s.G * a.dq.head;
    ab_put<T, DP>(lds + wave * 32 * DP * 2, dq, undo, lane, s.D, [&](int i) __attribute__((always_inline)) -> char * {
        const AtRow w = at_row(s, r0 + i);
        return r0 + i < s.R ? out + int64_t(w.token) * a.dq.token + int64_t(w.g) * a.dq.head : nullptr;
    });
}

// ---------------------------------------------------------------------------------------------
// dk, dv: a wave owns 32 keys
// ---------------------------------------------------------------------------------------------
// A step is two tiles of 32 rows.  Where a tile lies at the edge of what its rows see, probabilities are set to zero element by
// element; rows that see nothing are zeros in LDS, so that what they hold does not enter.
template <typename T, int DP, bool CAP, bool BIAS, bool FINE> __device__ __forceinline__ void ab_dkv(const AtBwd &a, uint32_t block)
{
    typedef AtNum<T> Num;
    constexpr int kKs = DP / 16, kDt = DP / 32, kPieces = DP / 8;
    constexpr int kTile = kAbTile * DP * 2;           // bytes: 32 rows of q, or of do
    constexpr int kOff = kAbTile * kPieces / 256;     // rows of a tile per thread
    constexpr int kInfo = BIAS ? 6 : 4;               // words per row that are used here
    __shared__ __attribute__((aligned(256))) char lds[2 * 4 * kTile];          // [buffer][tile][q, do]
    __shared__ __attribute__((aligned(16))) uint32_t info[2][2][kInfo * 32];   // [buffer][tile][word][row]
    const AtShape &s = a.s;
    const AbOrder &order = a.order;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const uint32_t head = block % a.heads, rest = block / a.heads, split = rest % a.splits, kb = rest / a.splits;   // the keys that most rows see first
    const int b = int(head / uint32_t(s.Hk)), hk = int(head) - b * s.Hk;
    const int k0 = int(kb) * kAbKeys, j0 = k0 + wave * 32, j_own = j0 + (lane & 31), j = j_own < s.Nk ? j_own : s.Nk - 1;
    u32x4 kf[kKs], vf[kKs];
    {
        const char *p = a.k.p + int64_t(b) * a.k.batch + int64_t(j) * a.k.token + int64_t(hk) * a.k.head;
        const char *v = a.v.p + int64_t(b) * a.v.batch + int64_t(j) * a.v.token + int64_t(hk) * a.v.head;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            kf[ks] = at_column(p, ks, lane, s.D);
            vf[ks] = at_column(v, ks, lane, s.D);
        }
    }
    const char *qbase = a.q.p + int64_t(b) * a.q.batch + int64_t(hk) * s.G * a.q.head, *gbase = a.dO.p + int64_t(b) * a.dO.batch + int64_t(hk) * s.G * a.dO.head;
    const int4 *tiles = a.w.tiles + int64_t(head) * order.tiles;
    const uint32_t *words = a.w.info + int64_t(head) * order.tiles * (kAbWords * 32);
    const int pairs = int(order.tiles / 2), mine = (pairs - int(split) + int(a.splits) - 1) / int(a.splits);   // this workgroup's: split, split + splits, ...

    // this thread's pieces of a tile: the rows' places within it.  A tile is cut short by the tokens that are left or, where a token's
    // heads are more than a tile, by the heads: `cut` counts what the cut goes by.
    const bool long_tokens = order.parts > 1;
    uint32_t q_at[kOff], g_at[kOff], lds_at[kOff];
    int cut[kOff];
    const int piece = tid % kPieces;
#pragma unroll
    for (int k = 0; k < kOff; ++k) {
        const int x = tid / kPieces + k * (256 / kPieces), dt = int(fastdiv(uint32_t(x), order.div_heads)), dg = x - dt * order.heads;
        q_at[k] = uint32_t(dt) * uint32_t(a.q.token) + uint32_t(dg) * uint32_t(a.q.head) + piece * 16;
        g_at[k] = uint32_t(dt) * uint32_t(a.dO.token) + uint32_t(dg) * uint32_t(a.dO.head) + piece * 16;
        lds_at[k] = x * (DP * 2) + ((piece ^ at_turn<DP>(x)) << 4);
        cut[k] = dt < order.tokens && piece * 8 < s.D ? (long_tokens ? dg : dt) : 0x40000000;
    }

    // the next pair of tiles that this workgroup's keys meet: 64 summaries at a time, one per lane, and what this wave makes of them
    enum { kMine = 1, kWhole = 4, kSome = 16 };       // (twice) the wave's keys are met; are seen by all rows; some row sees nothing
    int base = -64, flags = 0;
    uint64_t meets = 0;
    auto next = [&]() __attribute__((always_inline)) {
        while (meets == 0) {
            base += 64;
            if (base >= mine) return -1;
            const int n = base + lane;
            int4 t[2] = {make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
            if (n < mine) {
                const int4 *p = tiles + 2 * (int(split) + n * int(a.splits));
                t[0] = p[0];
                t[1] = p[1];
            }
            bool in = false;
            flags = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                in |= t[u].y > k0 && t[u].x < k0 + kAbKeys;
                if (t[u].y > j0 && t[u].x < j0 + 32) flags |= kMine << u;
                if (t[u].w >= j0 + 32 && t[u].z <= j0) flags |= kWhole << u;
                if (t[u].w == 0) flags |= kSome;
            }
            meets = __ballot(in);
        }
        const int bit = __builtin_ctzll(meets);
        meets &= meets - 1;
        return ((int(split) + (base + bit) * int(a.splits)) << 5) | __builtin_amdgcn_readlane(flags, bit);
    };
    u32x4 tq[2][kOff], tg[2][kOff];
    uint32_t word, word2 = 0;
    const int64_t q_tile = int64_t(order.tokens) * a.q.token, g_tile = int64_t(order.tokens) * a.dO.token;
    const uint32_t word_at = (tid >> 7) * (kAbWords * 128) + (tid & 127) * 4, word2_at = ((tid >> 6) & 1) * (kAbWords * 128) + (128 + (tid & 63)) * 4;
    auto fetch = [&](int what) __attribute__((always_inline)) {
        const uint32_t pair = uint32_t(what >> 5);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t tile = pair * 2 + u;
            const char *qp = qbase, *gp = gbase;
            int left;
            if (!long_tokens) {
                qp += int64_t(tile) * q_tile;
                gp += int64_t(tile) * g_tile;
                left = s.Nq - int(tile) * order.tokens;
            } else {
                const uint32_t t = fastdiv(tile, order.div_parts), g0 = (tile - t * uint32_t(order.parts)) * 32;
                qp += int64_t(t) * a.q.token + int64_t(g0) * a.q.head;
                gp += int64_t(t) * a.dO.token + int64_t(g0) * a.dO.head;
                left = int(t) < s.Nq ? s.G - int(g0) : 0;
            }
            const Span q(qp, kNowhere), g(gp, kNowhere);
#pragma unroll
            for (int k = 0; k < kOff; ++k) {
                q.load_kept(cut[k] < left ? q_at[k] : kNowhere, tq[u][k]);
                g.load_kept(cut[k] < left ? g_at[k] : kNowhere, tg[u][k]);
            }
        }
        const Span p(words + int64_t(pair) * 2 * (kAbWords * 32), 2 * kAbWords * 128);
        word = __float_as_uint(p.load_f32(word_at));
        if (BIAS) word2 = __float_as_uint(p.load_f32(word2_at));
    };
    at_acc dk[kDt], dv[kDt];
#pragma unroll
    for (int d = 0; d < kDt; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.0f;

    const uint32_t plain_at = at_address(lds) + at_plain_lane<DP>(lane), trans_at = at_address(lds) + at_trans_lane<DP>(lane);
    float mul = 1.0f, undo = s.scale, undo_v = 1.0f;
    // A wave issues in order, and at 128 elements it is alone on its SIMD: what is to run beside a product has to stand between
    // products, and what a product reads has to be on its way well before.  Fences keep the order below: scores; do.v with the
    // exponentials between its products and dv's operands read meanwhile; dv with ds between; dk, with the next tile's rows read.
    constexpr int kPer = 16 / kKs;                   // scores per product
    u32x4 fq[kKs], fg[kKs], l4[4], d4[4], sl4[BIAS ? 4 : 1], pl4[BIAS ? 4 : 1];
    auto read = [&](int at, const uint32_t *in, int ks) __attribute__((always_inline)) {      // a part of the rows and of what is known of them
        fq[ks] = at_plain<DP>(plain_at + at, 0, ks);
        fg[ks] = at_plain<DP>(plain_at + at + kTile, 0, ks);
        if (ks < 4) {
            const uint32_t *q = in + 8 * ks + 4 * half;                // rows of registers 4ks..4ks+3
            l4[ks] = *reinterpret_cast<const u32x4 *>(q + kAbLse * 32);
            d4[ks] = *reinterpret_cast<const u32x4 *>(q + kAbDelta * 32);
            if (BIAS) {
                sl4[ks] = *reinterpret_cast<const u32x4 *>(q + kAbSlope * 32);
                pl4[ks] = *reinterpret_cast<const u32x4 *>(q + kAbPlace * 32);
            }
        }
    };
    static_assert(kKs >= 4, "four parts of what is known of the rows");
    // at_next: the tile to read meanwhile, if any
    auto work = [&](int at, const uint32_t *in, bool whole, bool more, int at_next, const uint32_t *in_next) __attribute__((always_inline)) {
        const uint32_t qt = trans_at + at, gt = qt + kTile;
        at_acc x, y;
        float slope[CAP ? 16 : 1];
        u32x4 p[2], ds[2], p_rest[2], ds_rest[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = 0.0f;
            y[i] = __uint_as_float(d4[i / 4][i % 4]);      // the sums do.v start from -delta
        }
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) x = Num::mfma(fq[ks], kf[ks], x);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            y = Num::mfma(fg[ks], vf[ks], y);
            fq[ks] = at_transposed<DP>(gt, ks / kDt * 16, ks % kDt * 32);     // dv's operands, 2 * kDt = kKs of them
#pragma unroll
            for (int i = ks * kPer; i < ks * kPer + kPer; ++i) {
                const float lse2 = __uint_as_float(l4[i / 4][i % 4]);
                if (!CAP && !BIAS) {
                    x[i] = at_exp2(fmaf(x[i], s.c, -lse2));
                } else {
                    float sl = 1.0f, sc = ab_score<CAP>(s, x[i], sl);
                    if (CAP) slope[i] = sl;
                    if (BIAS) sc = fmaf(-__uint_as_float(sl4[i / 4][i % 4]), fabsf(float(int(pl4[i / 4][i % 4]) - j_own)), sc);
                    x[i] = at_exp2(sc - lse2);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!whole) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const u32x4 lo4 = *reinterpret_cast<const u32x4 *>(in + kAbLo * 32 + 8 * w + 4 * half), hi4 = *reinterpret_cast<const u32x4 *>(in + kAbHi * 32 + 8 * w + 4 * half);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const bool vis = uint32_t(j_own - int(lo4[c])) < hi4[c] - lo4[c];
                    x[4 * w + c] = vis ? x[4 * w + c] : 0.0f;
                    y[4 * w + c] = vis ? y[4 * w + c] : 0.0f;
                }
            }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                p[g][w] = Num::pack(x[8 * g + 2 * w], x[8 * g + 2 * w + 1]);
                if (FINE) p_rest[g][w] = Num::rest(x[8 * g + 2 * w], x[8 * g + 2 * w + 1], p[g][w]);
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < kKs; ++n) {
            dv[n % kDt] = Num::mfma(fq[n], p[n / kDt], dv[n % kDt]);
            if (FINE) dv[n % kDt] = Num::mfma(fq[n], p_rest[n / kDt], dv[n % kDt]);
            fg[n] = at_transposed<DP>(qt, n / kDt * 16, n % kDt * 32);        // dk's operands
#pragma unroll
            for (int i = n * kPer; i < n * kPer + kPer; ++i) {
                y[i] *= x[i];
                if (CAP) y[i] *= slope[i];
                if (Num::kHalf) y[i] *= mul;
            }
#pragma unroll
            for (int w = n * kPer / 2; w < (n + 1) * kPer / 2; ++w) {
                ds[w / 4][w % 4] = Num::pack(y[2 * w], y[2 * w + 1]);
                if (FINE) ds_rest[w / 4][w % 4] = Num::rest(y[2 * w], y[2 * w + 1], ds[w / 4][w % 4]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < kKs; ++n) {
            dk[n % kDt] = Num::mfma(fg[n], ds[n / kDt], dk[n % kDt]);
            if (FINE) dk[n % kDt] = Num::mfma(fg[n], ds_rest[n / kDt], dk[n % kDt]);
            if (more) read(at_next, in_next, n);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    float2 first_most = make_float2(0.0f, 0.0f);
    if (Num::kHalf && uint32_t(lane) < a.w.blocks) first_most = a.w.most[int64_t(head) * a.w.blocks + lane];
    int t = __builtin_amdgcn_readfirstlane(next());
    if (t >= 0) fetch(t);                            // on its way while the factors below are formed
    if (Num::kHalf) {
        float ss = 0.0f, most = first_most.x, most_delta = first_most.y;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            float f[8];
            Store<T>::unpack(vf[ks], f);
#pragma unroll
            for (int k = 0; k < 8; ++k) ss = fmaf(f[k], f[k], ss);
        }
        ss = at_pair_sum(ss);
        for (uint32_t k = lane + 64; k < a.w.blocks; k += 64) {
            const float2 m = a.w.most[int64_t(head) * a.w.blocks + k];
            most = fmaxf(most, m.x);
            most_delta = fmaxf(most_delta, m.y);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            most = fmaxf(most, __shfl_xor(most, m, 64));
            most_delta = fmaxf(most_delta, __shfl_xor(most_delta, m, 64));
        }
        const int e = ab_exponent(sqrtf(ss) * most + most_delta);
        mul = ab_pow2(e - kAtDrop);
        undo = s.scale * ab_pow2(-e);
        undo_v = ab_pow2(-kAtDrop);
    }
    for (int cur = 0; t >= 0; cur ^= 1) {
        char *p = lds + cur * 4 * kTile;
        const int at = cur * 4 * kTile;
        if (t & kSome) {
            const Span e(words + int64_t(t >> 5) * 2 * (kAbWords * 32), 2 * kAbWords * 128);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < kOff; ++k)
                    if (e.load_f32(((u * kAbWords + kAbEmpty) * 32 + tid / kPieces + k * (256 / kPieces)) * 4) != 0.0f) tq[u][k] = tg[u][k] = u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < kOff; ++k) {
                *reinterpret_cast<u32x4 *>(p + u * 2 * kTile + lds_at[k]) = tq[u][k];
                *reinterpret_cast<u32x4 *>(p + u * 2 * kTile + kTile + lds_at[k]) = tg[u][k];
            }
        info[cur][tid >> 7][tid & 127] = word;
        if (BIAS && tid < 128) info[cur][tid >> 6][(128 + (tid & 63)) % (kInfo * 32)] = word2;
        __syncthreads();
        const int u0 = t & 1 ? 0 : 1;                // the first of the two tiles that this wave's keys meet (the other one is read for nothing where there is none)
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) read(at + u0 * 2 * kTile, info[cur][u0], ks);
        __builtin_amdgcn_sched_barrier(0);
        const int after = __builtin_amdgcn_readfirstlane(next());
        if (after >= 0) fetch(after);
        __builtin_amdgcn_sched_barrier(0);
        if (t & 1) work(at, info[cur][0], t >> 2 & 1, true, at + 2 * kTile, info[cur][1]);
        if (t & 2) work(at + 2 * kTile, info[cur][1], t >> 3 & 1, false, 0, nullptr);
        t = after;
    }
    if (a.part) {
        if (j_own >= s.Nk) return;
        float *p = a.part + ((int64_t(split) * a.heads + head) * s.Nk + j_own) * 2 * s.D;
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int e = d * 32 + 8 * w + 4 * half;
                if (e < s.D) {
                    *reinterpret_cast<float4 *>(p + e) = make_float4(dk[d][4 * w] * undo, dk[d][4 * w + 1] * undo, dk[d][4 * w + 2] * undo, dk[d][4 * w + 3] * undo);
                    *reinterpret_cast<float4 *>(p + s.D + e) = make_float4(dv[d][4 * w] * undo_v, dv[d][4 * w + 1] * undo_v, dv[d][4 * w + 2] * undo_v, dv[d][4 * w + 3] * undo_v);
                }
            }
        return;
    }
    __syncthreads();                                // the last tiles are done with
    char *pk = a.dk.p + int64_t(b) * a.dk.batch + int64_t(j0) * a.dk.token + int64_t(hk) * a.dk.head;
    char *pv = a.dv.p + int64_t(b) * a.dv.batch + int64_t(j0) * a.dv.token + int64_t(hk) * a.dv.head;
    char *mid = lds + wave * 32 * DP * 2;
    ab_put<T, DP>(mid, dk, undo, lane, s.D, [&](int i) __attribute__((always_inline)) { return j0 + i < s.Nk ? pk + int64_t(i) * a.dk.token : nullptr; });
    ab_put<T, DP>(mid, dv, undo_v, lane, s.D, [&](int i) __attribute__((always_inline)) { return j0 + i < s.Nk ? pv + int64_t(i) * a.dv.token : nullptr; });
}

// Both walks in one launch: the rows' workgroups fill in where the keys' run out (8 x 12 heads of 197 keys 23.6 -> 15.1 us, 2 x 4 heads of 4001
// keys in documents 327 -> 225, 4 x 4 of 4096 543 -> 517).  With more workgroups there is less to fill in, and dq alone has more waves (4 x 4 heads of
// 4001 keys, at the border: 390 us in two launches, 400 in one).  Tiles of 64 keys for dq here, whose waves are few and wait for them (2 x 12 heads of
// 4096 keys 405 -> 395 us; 8 x 12 of 197 15.0 -> 15.4).
template <typename T, int DP, bool CAP, bool BIAS, bool FINE>
__global__ __launch_bounds__(256, DP == 64 ? 2 : 1) void k_attn_both(const AtBwd a)
{
    const uint32_t keys = a.heads * a.key_blocks * a.splits;
    if (blockIdx.x < keys) ab_dkv<T, DP, CAP, BIAS, FINE>(a, blockIdx.x);
    else ab_dq<T, DP, 4, 64, CAP, BIAS, FINE>(a, blockIdx.x - keys);
}
template <typename T, int DP, bool CAP, bool BIAS, bool FINE>
__global__ __launch_bounds__(256, DP == 64 ? 2 : 1) void k_attn_dkv(const AtBwd a)
{
    ab_dkv<T, DP, CAP, BIAS, FINE>(a, blockIdx.x);
}
template <typename T, int DP, bool CAP, bool BIAS, bool FINE>
__global__ __launch_bounds__(256, 2) void k_attn_dq(const AtBwd a)
{
    ab_dq<T, DP, 4, 32, CAP, BIAS, FINE>(a, blockIdx.x);
}

// the splits added up in their order, four elements per thread: of dk or dv, behind those of dq
__device__ __forceinline__ float4 ab_sum(const float *p, int64_t step, uint32_t splits)
{
    float4 v = *reinterpret_cast<const float4 *>(p);
    for (uint32_t k = 1; k < splits; ++k) {
        const float4 u = *reinterpret_cast<const float4 *>(p + k * step);
        v.x += u.x;
        v.y += u.y;
        v.z += u.z;
        v.w += u.w;
    }
    return v;
}
template <typename T>
__global__ __launch_bounds__(kThreads) void k_attn_add(const AtBwd a, int64_t pieces, int64_t row_pieces)
{
    const AtShape &s = a.s;
    int64_t id = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (id < pieces) {
        const int quads = s.D / 2;                              // of a key: D/4 of dk, D/4 of dv
        const int64_t at = id / quads, head = at / s.Nk;
        const int x = int(id - at * quads), j = int(at - head * s.Nk);
        const float4 v = ab_sum(a.part + at * 2 * s.D + x * 4, int64_t(a.heads) * s.Nk * 2 * s.D, a.splits);
        const int b = int(head) / s.Hk, hk = int(head) - b * s.Hk;
        const bool key = x < s.D / 4;
        const AtOut &o = key ? a.dk : a.dv;
        at_store4<T>(o.p + int64_t(b) * o.batch + int64_t(j) * o.token + int64_t(hk) * o.head + (key ? x : x - s.D / 4) * 8, v.x, v.y, v.z, v.w);
        return;
    }
    id -= pieces;
    if (id >= row_pieces) return;
    const int quads = s.D / 4;
    const int64_t at = id / quads, head = at / s.R;
    const int x = int(id - at * quads), b = int(head) / s.Hk, hk = int(head) - b * s.Hk;
    const AtRow row = at_row(s, uint32_t(at - head * s.R));
    const float4 v = ab_sum(a.part_q + at * s.D + x * 4, int64_t(a.heads) * s.R * s.D, a.row_splits);
    at_store4<T>(a.dq.p + int64_t(b) * a.dq.batch + int64_t(row.token) * a.dq.token + int64_t(hk * s.G + int(row.g)) * a.dq.head + x * 8, v.x, v.y, v.z, v.w);
}

// zeros: dq where there are no keys, dk and dv where there are no queries
template <typename T>
__global__ __launch_bounds__(kThreads) void k_attn_zero(AtOut o, int heads, int tokens, int D, int64_t pieces)
{
    const int64_t id = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (id >= pieces) return;
    const int per = D / 4;
    const int64_t row = id / per, bt = row / heads, b = bt / tokens;
    at_store4<T>(o.p + b * o.batch + (bt - b * tokens) * o.token + (row - bt * heads) * o.head + (id - row * per) * 8, 0.0f, 0.0f, 0.0f, 0.0f);
}

struct AtBwdPlan {
    AbOrder order;
    uint32_t blocks, key_blocks, splits, row_blocks, row_splits;
    size_t info, part, part_q, operand[3], total;       // bytes
};
static size_t ab_up(size_t n) { return (n + 255) & ~size_t(255); }
static AtBwdPlan at_bwd_plan(const mesa_attention &a, const bool codes[3])
{
    AtBwdPlan p;
    const int64_t R = a.Nq * (a.Hq / a.Hk), heads = a.B * a.Hk;
    const int64_t G = a.Hq / a.Hk;
    AbOrder &o = p.order;
    o.heads = int32_t(G > 32 ? 32 : G);
    o.tokens = int32_t(G > 32 ? 1 : 32 / G);
    o.parts = int32_t(ceil_div(G, 32));
    const int64_t tiles = ceil_div(a.Nq, o.tokens) * o.parts;
    o.tiles = uint32_t(tiles + (tiles & 1));
    o.div_heads = make_fastdiv(uint32_t(o.heads));
    o.div_parts = make_fastdiv(uint32_t(o.parts));
    p.blocks = uint32_t(ceil_div(o.tiles, 4));
    p.key_blocks = uint32_t(ceil_div(a.Nk, kAbKeys));
    p.row_blocks = uint32_t(ceil_div(R, 128));
    // Few keys and long walks: the rows' tiles are dealt out to several workgroups and their sums added up, so that there is a round of 512 (heads of 128,
    // 4 x 4 of 4096 keys: one split 1038 us, two 1080; 3 x 4: two 817, one 889); two rounds where up to 64 elements one is full, as walks
    // differ in length (4 x 4 heads of 4001 keys in documents 446 -> 432 us).
    const int64_t have = heads * p.key_blocks, most = o.tiles / 16;
    int64_t n = have > 0 ? (a.D <= 64 && have >= 512 ? 1024 / have : ceil_div(512, have)) : 1, m = 1;
    n = n > most ? most : n;
    // So few workgroups of either walk that compute units have nothing to do, and walks long enough to pay for the addition's launch (4 us): both
    // are dealt out, down to four tiles of rows or 192 keys each.  Two heads of 64, causal: 911 keys 32 -> 23 us, 2000 60 -> 33, 4000 111 -> 46;
    // of 128, 4000 keys 187 -> 90; where a window leaves nothing to deal out, 20 -> 21.5.
    const int64_t rows = heads * p.row_blocks;
    if (have > 0 && have + rows <= 512 && o.tiles >= 24 && a.Nk >= 768) {
        const int64_t few = 256 / have < o.tiles / 4 ? 256 / have : o.tiles / 4;
        n = n > few ? n : few;
        m = 512 / rows < a.Nk / 192 ? 512 / rows : a.Nk / 192;
    }
    n = n > 32 ? 32 : n < 1 ? 1 : n;
    p.splits = uint32_t(n);
    p.row_splits = uint32_t(m > 8 ? 8 : m);
    const size_t h = size_t(heads);
    p.info = ab_up(h * o.tiles * kAbWords * 128) + ab_up(h * o.tiles * sizeof(int4)) + ab_up(h * p.blocks * sizeof(float2)) + ab_up(h * p.key_blocks * sizeof(float));
    p.part = n > 1 ? ab_up(size_t(n) * h * size_t(a.Nk) * 2 * size_t(a.D) * sizeof(float)) : 0;
    p.part_q = p.row_splits > 1 ? ab_up(size_t(p.row_splits) * h * size_t(R) * size_t(a.D) * sizeof(float)) : 0;
    const int64_t tokens[3] = {a.Nq, a.Nk, a.Nk}, hs[3] = {a.Hq, a.Hk, a.Hk};
    p.total = p.info + p.part + p.part_q;
    for (int k = 0; k < 3; ++k) {
        p.operand[k] = codes[k] ? ab_up(size_t(a.B) * size_t(tokens[k]) * size_t(hs[k]) * size_t(a.D) * 2) : 0;
        p.total += p.operand[k];
    }
    return p;
}

template <typename T, int DP, bool CAP, bool BIAS, bool FINE> static mesa_status at_bwd_launch(const AtBwd &a, hipStream_t s)
{
    const uint32_t keys = a.heads * a.key_blocks * a.splits, rows = a.heads * a.row_blocks * a.row_splits;
    const bool both = DP == 64 ? keys <= 1024 : keys + rows <= 256;      // two rounds of workgroups; one to a compute unit
    if (both) hipLaunchKernelGGL((k_attn_both<T, DP, CAP, BIAS, FINE>), dim3(keys + rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_attn_dkv<T, DP, CAP, BIAS, FINE>), dim3(keys), dim3(256), 0, s, a);
    if (const mesa_status st = launch_status()) return st;
    if (!both) {
        hipLaunchKernelGGL((k_attn_dq<T, DP, CAP, BIAS, FINE>), dim3(rows), dim3(256), 0, s, a);
        if (const mesa_status st = launch_status()) return st;
    }
    const int64_t pieces = a.splits > 1 ? int64_t(a.heads) * a.s.Nk * (a.s.D / 2) : 0, row_pieces = a.row_splits > 1 ? int64_t(a.heads) * a.s.R * (a.s.D / 4) : 0;
    if (pieces + row_pieces == 0) return MESA_OK;
    hipLaunchKernelGGL(k_attn_add<T>, dim3(uint32_t(ceil_div(pieces + row_pieces, kThreads))), dim3(kThreads), 0, s, a, pieces, row_pieces);
    return launch_status();
}
// Up to kAbFine keys the call is bound by what it reads and writes (14 products of 64 keys to a row's four vectors), and with so few terms to
// a sum the products' roundings do not average out: there probabilities and score gradients enter in two 16-bit parts.
constexpr int kAbFine = 64;
template <typename T, int DP, bool CAP, bool BIAS> static mesa_status at_bwd_parts(const AtBwd &a, hipStream_t s)
{
    return a.s.Nk <= kAbFine ? at_bwd_launch<T, DP, CAP, BIAS, true>(a, s) : at_bwd_launch<T, DP, CAP, BIAS, false>(a, s);
}
template <typename T, int DP> static mesa_status at_bwd_forms(const AtBwd &a, const AbOperands &in, uint32_t in_blocks, bool cap, bool bias, hipStream_t s)
{
    hipLaunchKernelGGL((k_attn_rows<T, DP>), dim3(a.heads * (a.w.blocks + (AtNum<T>::kHalf ? a.w.key_blocks : 0)) + in_blocks), dim3(kThreads), 0, s, a, in);
    if (const mesa_status st = launch_status()) return st;
    if (cap && bias) return at_bwd_parts<T, DP, true, true>(a, s);
    if (cap) return at_bwd_parts<T, DP, true, false>(a, s);
    if (bias) return at_bwd_parts<T, DP, false, true>(a, s);
    return at_bwd_parts<T, DP, false, false>(a, s);
}
template <typename T> static mesa_status at_zero(const AtOut &o, int64_t B, int64_t tokens, int64_t heads, int64_t D, hipStream_t s)
{
    const int64_t pieces = B * tokens * heads * (D / 4);
    if (pieces == 0) return MESA_OK;
    hipLaunchKernelGGL(k_attn_zero<T>, dim3(uint32_t(ceil_div(pieces, kThreads))), dim3(kThreads), 0, s, o, int(heads), int(tokens), int(D), pieces);
    return launch_status();
}

template <typename T>
static mesa_status at_bwd(const mesa_attention &m, AtBwd &a, const AtBwdPlan &p, const mesa_attention_in *in, const bool codes[3], char *ws, bool bias, hipStream_t s)
{
    if (m.Nk == 0) return at_zero<T>(a.dq, m.B, m.Nq, m.Hq, m.D, s);
    if (m.Nq == 0) {
        if (const mesa_status st = at_zero<T>(a.dk, m.B, m.Nk, m.Hk, m.D, s)) return st;
        return at_zero<T>(a.dv, m.B, m.Nk, m.Hk, m.D, s);
    }
    AtView *view[3] = {&a.q, &a.k, &a.v};
    const int64_t tokens[3] = {m.Nq, m.Nk, m.Nk}, heads[3] = {m.Hq, m.Hk, m.Hk};
    char *out = ws + p.info + p.part + p.part_q;
    AbOperands ops;
    ops.count = 0;
    ops.values = false;
    ops.div_d = make_fastdiv(uint32_t(m.D / 8));
    int64_t blocks = 0;
    for (int k = 0; k < 3; ++k) {
        if (!codes[k]) continue;
        AbCodes c;
        c.q = AtView{static_cast<const char *>(in[k].data), in[k].batch, in[k].token, in[k].head};
        c.alpha = in[k].alpha;
        c.beta = in[k].beta;
        c.out = out;
        c.heads = int32_t(heads[k]);
        c.tokens = int32_t(tokens[k]);
        c.first = uint32_t(blocks);
        c.per_head = uint32_t(ceil_div(tokens[k] * (m.D / 8), kThreads));
        if (k == 2 && AtNum<T>::kHalf) {
            ops.v = c;
            ops.values = true;
        } else {
            ops.c[ops.count++] = c;
            blocks += m.B * heads[k] * int64_t(c.per_head);
        }
        *view[k] = AtView{out, heads[k] * tokens[k] * m.D * 2, m.D * 2, tokens[k] * m.D * 2};
        out += p.operand[k];
    }
    return m.D <= 64 ? at_bwd_forms<T, 64>(a, ops, uint32_t(blocks), m.cap > 0.0f, bias, s) : at_bwd_forms<T, 128>(a, ops, uint32_t(blocks), m.cap > 0.0f, bias, s);
}

}  // namespace mesa

using namespace mesa;

extern "C" MESA_EXPORT size_t mesa_attention_bwd_q_workspace_bytes(mesa_attention a, int q_codes, int k_codes, int v_codes, mesa_dtype dt)
{
    const bool codes[3] = {q_codes != 0, k_codes != 0, v_codes != 0};
    return at_supported(a, dt) == MESA_OK && a.B > 0 && a.Nq > 0 && a.Nk > 0 ? at_bwd_plan(a, codes).total : 0;
}

extern "C" MESA_EXPORT mesa_status mesa_attention_bwd_q(mesa_attention a, mesa_attention_in q, mesa_attention_in k, mesa_attention_in v, mesa_attention_in o, const float *lse,
                                                        mesa_attention_in dO, mesa_attention_out dq, mesa_attention_out dk, mesa_attention_out dv, mesa_attention_mask m, void *ws,
                                                        size_t ws_bytes, mesa_dtype dt, void *stream)
{
    if (const mesa_status st = at_supported(a, dt)) return st;
    if (a.B == 0 || (a.Nq == 0 && a.Nk == 0)) return MESA_OK;
    const mesa_attention_in in[3] = {q, k, v};
    const int64_t tokens[3] = {a.Nq, a.Nk, a.Nk}, group = a.Hq / a.Hk;
    bool codes[3];
    for (int n = 0; n < 3; ++n) {
        codes[n] = in[n].alpha != nullptr;
        if (codes[n] != (in[n].beta != nullptr) || !aligned4(in[n].alpha) || !aligned4(in[n].beta)) return MESA_ERR_INVALID_ARG;
        if (tokens[n] && !in[n].data) return MESA_ERR_INVALID_ARG;
        if ((reinterpret_cast<uintptr_t>(in[n].data) & (codes[n] ? 7u : 15u)) != 0 || !at_strides(a, tokens[n], n == 0 ? group : 1, in[n].batch, in[n].token, in[n].head))
            return MESA_ERR_INVALID_ARG;
    }
    if (a.Nq && (!o.data || !dO.data || !dq.data || !lse)) return MESA_ERR_INVALID_ARG;
    if (a.Nk && (!dk.data || !dv.data)) return MESA_ERR_INVALID_ARG;
    if (o.alpha || dO.alpha || (m.lo == nullptr) != (m.hi == nullptr) || !aligned16(o.data) || !aligned16(dO.data) || !aligned16(dq.data) || !aligned16(dk.data) ||
        !aligned16(dv.data) || !aligned4(lse) || !aligned4(m.lo) || !aligned4(m.hi) || !aligned4(m.slopes) || !aligned4(m.q_start))
        return MESA_ERR_INVALID_ARG;
    if (!at_strides(a, a.Nq, group, o.batch, o.token, o.head) || !at_strides(a, a.Nq, group, dO.batch, dO.token, dO.head) ||
        !at_strides(a, a.Nq, group, dq.batch, dq.token, dq.head) || !at_strides(a, a.Nk, 1, dk.batch, dk.token, dk.head) || !at_strides(a, a.Nk, 1, dv.batch, dv.token, dv.head))
        return MESA_ERR_INVALID_ARG;
    const AtBwdPlan p = at_bwd_plan(a, codes);
    const int64_t heads = a.B * a.Hk, most = most_workgroups(256), rows = heads * a.Nq * group, keys = heads * a.Nk, operands = (rows + 2 * keys) * (a.D / 8) / kThreads + heads * (group + 2);
    if (heads * (int64_t(p.key_blocks) * p.splits + p.row_blocks) > most || heads * (int64_t(p.blocks) + p.key_blocks) + operands > most ||
        (rows > 2 * keys ? rows : 2 * keys) * (a.D / 4) > most * kThreads)
        return MESA_ERR_UNSUPPORTED;
    if (a.Nq > 0 && a.Nk > 0 && (!ws || !aligned16(ws) || ws_bytes < p.total)) return MESA_ERR_WORKSPACE;
    if (a.Nq > 0 && a.Nk > 0) {                       // operands are read again after the first results
        const void *r[3] = {dq.data, dk.data, dv.data}, *x[5] = {q.data, k.data, v.data, o.data, dO.data};
        for (int n = 0; n < 3; ++n) {
            if (r[n] == r[(n + 1) % 3]) return MESA_ERR_INVALID_ARG;
            for (const void *y : x)
                if (r[n] == y) return MESA_ERR_INVALID_ARG;
        }
    }
    AtBwd f;
    f.s = at_shape(a, m);
    auto view = [](const mesa_attention_in &x) { return AtView{static_cast<const char *>(x.data), x.batch * 2, x.token * 2, x.head * 2}; };
    auto result = [](const mesa_attention_out &x) { return AtOut{static_cast<char *>(x.data), x.batch * 2, x.token * 2, x.head * 2}; };
    f.q = view(q);
    f.k = view(k);
    f.v = view(v);
    f.o = view(o);
    f.dO = view(dO);
    f.dq = result(dq);
    f.dk = result(dk);
    f.dv = result(dv);
    f.lse = lse;
    f.heads = uint32_t(heads);
    f.key_blocks = p.key_blocks;
    f.splits = p.splits;
    f.row_blocks = p.row_blocks;
    f.row_splits = p.row_splits;
    char *w = static_cast<char *>(ws);
    const size_t h = size_t(heads), tiles_at = ab_up(h * p.order.tiles * kAbWords * 128), most_at = tiles_at + ab_up(h * p.order.tiles * sizeof(int4));
    f.order = p.order;
    f.w.info = reinterpret_cast<uint32_t *>(w);
    f.w.tiles = reinterpret_cast<int4 *>(w + tiles_at);
    f.w.most = reinterpret_cast<float2 *>(w + most_at);
    f.w.values = reinterpret_cast<float *>(w + most_at + ab_up(h * p.blocks * sizeof(float2)));
    f.w.blocks = p.blocks;
    f.w.key_blocks = p.key_blocks;
    f.part = p.splits > 1 ? reinterpret_cast<float *>(w + p.info) : nullptr;
    f.part_q = p.row_splits > 1 ? reinterpret_cast<float *>(w + p.info + p.part) : nullptr;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bias = m.slopes != nullptr;
    return dt == MESA_F16 ? at_bwd<_Float16>(a, f, p, in, codes, w, bias, s) : at_bwd<__bf16>(a, f, p, in, codes, w, bias, s);
}
