// qkv_norm_rope.hip -- the packed query/key/value projection of a language model's attention block: the norm of each query
// and key head and the rotation by position in one pass that also leaves the codes of every head and moves the running
// estimates; queries and keys again from the codes; and the backward from the codes.
//   r = 1/sqrt(sum x^2/D + eps),  z = gamma x r,  y = R(pos) z;     g = R(pos)^T dy,  n = x_hat r,  u = gamma g,
//   dx = r (u - n mean(u n)),  dgamma = sum g n
// R turns pairs of elements, so its transpose is the same rotation by the negative angle.
//
// Bound by memory: per element of a 16-bit tensor the forward moves 2 bytes in and 2 + 1 out, the backward 2 + 1 in and 2 out.
// A head is a group of LPH lanes with eight elements each (LPH: the power of two from D/8), a wave holds 64/LPH heads side by
// side ("slot") and walks over the tokens of its tile with the same heads, so that the extrema accumulate in registers.  Cosines and sines depend on token and pair, not on the head: a workgroup
// forms them once per tile into LDS -- angle and reduction in binary64, as positions times frequencies have more than 24
// bits -- and all heads read them there.
// Measured, 32768 tokens of 32 + 8 + 8 heads of 128, bfloat16 (a copy of as many bytes runs at 5.0 TB/s): forward 196 us (939 MB, 4.8 TB/s),
// queries and keys again 109 us (503 MB, 4.6 TB/s), backward 171 us (839 MB, 4.9 TB/s).  One token of 24 heads of 64: 4.5 us.
#include <hip/hip_runtime.h>

#include "api_util.hpp"
#include "common.hpp"
#include "quantize.hpp"

namespace mesa {

constexpr int kQkvTile = 16;        // tokens of a tile at most; 32 left no other workgroup to load while one forms its angles (forward 207 -> 198 us)
constexpr int kQkvGrid = 1024;      // workgroups at most: four per compute unit
constexpr int kQkvMaxHeads = 512;
constexpr int kQkvAlone = 16384;    // elements at most that one workgroup takes

struct QkvGeom {
    int64_t T;
    uint32_t Hq, Hn, H, D, rot, lph_log2;   // Hn = Hq + Hk, H = Hn + Hv
    uint32_t tile, phases_log2;             // tokens per tile; into how many parts the four waves share out a tile's tokens
    uint32_t end[4];                        // first pair behind each axis
    uint32_t parts, angles;                 // lanes that hold pairs to turn; angles of a token in LDS
    FastDiv div_half;
    int interleaved;
    float eps;
};

static QkvGeom qkv_geom(const mesa_qkv_heads &h)
{
    QkvGeom g;
    g.T = h.T;
    g.Hq = uint32_t(h.Hq);
    g.Hn = uint32_t(h.Hq + h.Hk);
    g.H = uint32_t(h.Hq + h.Hk + h.Hv);
    g.D = uint32_t(h.D);
    g.rot = uint32_t(h.rot);
    g.lph_log2 = 0;
    while ((8u << g.lph_log2) < g.D) ++g.lph_log2;
    // few tokens: tiles of fewer, so that there are workgroups for every compute unit
    int64_t t = ceil_div(h.T, kQkvGrid);
    // so few that one workgroup does them: it moves the estimates, or adds up the gains' gradients, itself -- a second, dependent launch
    // costs as much as the first
    if (h.T <= kQkvTile && h.T * int64_t(g.H) * h.D <= kQkvAlone) t = h.T;
    g.tile = uint32_t(t < 1 ? 1 : t > kQkvTile ? kQkvTile : t);
    const uint32_t slots = (g.H << g.lph_log2) / 64 + (((g.H << g.lph_log2) % 64) != 0);
    g.phases_log2 = slots >= 4 || g.tile < 2 ? 0 : slots >= 2 || g.tile < 4 ? 1 : 2;      // no more parts than tokens
    uint32_t e = 0;
    for (int a = 0; a < 4; ++a) {
        if (a < h.axes) e += uint32_t(h.section[a]);
        g.end[a] = a < h.axes - 1 ? e : 0xFFFFFFFFu;
    }
    g.interleaved = h.interleaved;
    const uint32_t per = h.interleaved ? 4 : 8;
    g.parts = (g.rot / 2 + per - 1) / per;
    g.angles = g.parts * per;
    g.div_half = make_fastdiv(g.rot ? g.rot / 2 : 1);
    g.eps = h.eps;
    return g;
}

static int qkv_grid(const QkvGeom &g)
{
    const int64_t n = ceil_div(g.T, g.tile);
    return int(n < kQkvGrid ? n : kQkvGrid);
}

// cosines and sines of a tile's tokens.  A lane reads those of its own part of a head in 16-byte pieces of two pairs, and the pieces of
// neighbouring lanes lie side by side: pair i of a token is at [token][(i % per) / 2][i / per][i % 2], per pairs to a lane (side
// by side in a lane's own order the pieces lay 64 bytes apart and met in a quarter of the banks).
__device__ __forceinline__ uint32_t qkv_pair_at(const QkvGeom &g, uint32_t lane_part, uint32_t k)   // of a lane's pair k
{
    return ((k >> 1) * g.parts + lane_part) * 2 + (k & 1);
}
__device__ __forceinline__ void qkv_angles(float2 *cs, const QkvGeom &g, const float *__restrict__ freq, const int32_t *__restrict__ pos, int64_t t0, uint32_t tokens)
{
    const uint32_t half = g.rot / 2, per_log2 = g.interleaved ? 2 : 3;
    for (uint32_t k = threadIdx.x; k < tokens * half; k += kThreads) {
        const uint32_t tk = fastdiv(k, g.div_half), i = k - tk * half;
        const uint32_t axis = (i >= g.end[0]) + (i >= g.end[1]) + (i >= g.end[2]);
        // in turns, the whole ones taken off: what is left is below a half and exact enough in binary32 (2^-25 turns)
        double turns = double(pos[int64_t(axis) * g.T + t0 + tk]) * double(freq[i]) * 0.15915494309189535;
        turns -= rint(turns);
        float s, c;
        sincospif(float(2.0 * turns), &s, &c);
        cs[tk * g.angles + qkv_pair_at(g, i >> per_log2, i & ((1u << per_log2) - 1))] = make_float2(c, s);
    }
}

// The other half of each pair, from the lane `hop` further on or back, by data-parallel-primitive moves where the hop is a power of two
// below 16 (the LDS crossbar, which serves the whole compute unit, was what bound the backward: 250 us with it, 218 without, when the rest was
// still to come).
template <int CTRL, int BANKS> __device__ __forceinline__ float qkv_move(float old, float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v), CTRL, 0xf, BANKS, false));
}
__device__ __forceinline__ void qkv_partner(const float f[8], float o[8], uint32_t hop, int partner)
{
    if (hop == 8) {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = qkv_move<0x128, 0xf>(f[k], f[k]);                              // row_ror:8
    } else if (hop == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = qkv_move<0x114, 0xa>(qkv_move<0x104, 0x5>(f[k], f[k]), f[k]);  // row_shl:4 and row_shr:4, each to every other four lanes
    } else if (hop == 2) {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = qkv_move<0x4E, 0xf>(f[k], f[k]);                               // quad_perm [2,3,0,1]
    } else if (hop == 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = qkv_move<0xB1, 0xf>(f[k], f[k]);                               // quad_perm [1,0,3,2]
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = __shfl(f[k], partner, 64);
    }
}

// f[0..7] of this lane's part of a head, turned by the token's angles; d0: the part's first element.  sign -1: turned back.
// Every lane of the wave takes part (the partner's elements come from its registers).
__device__ __forceinline__ void qkv_turn(float f[8], const float2 *cs, const QkvGeom &g, uint32_t d0, int partner, float sign)
{
    if (g.interleaved) {
        const uint32_t part = d0 / 8 < g.parts ? d0 / 8 : 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 w = cs[qkv_pair_at(g, part, k)];
            const float a = f[2 * k], b = f[2 * k + 1], s = sign * w.y;
            const bool turned = d0 + 2 * k < g.rot;
            f[2 * k] = turned ? fmaf(a, w.x, -(b * s)) : a;
            f[2 * k + 1] = turned ? fmaf(b, w.x, a * s) : b;
        }
        return;
    }
    const bool second = d0 >= g.rot / 2, turned = d0 < g.rot;
    const uint32_t part = turned ? (second ? d0 - g.rot / 2 : d0) / 8 : 0;
    const float sg = second ? sign : -sign;
    float o[8];
    qkv_partner(f, o, g.rot / 16, partner);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float2 w = cs[qkv_pair_at(g, part, k)];
        const float v = fmaf(f[k], w.x, o[k] * (sg * w.y));
        f[k] = turned ? v : f[k];
    }
}

__device__ __forceinline__ float qkv_head_sum(float v, uint32_t lph_log2)      // over the lanes of a head
{
    switch (lph_log2) {
    case 0: return v;
    case 1: return v + dpp_move<0xB1>(v);
    case 2: return lanes_sum_dpp<4>(v);
    case 3: return lanes_sum_dpp<8>(v);
    case 4: return lanes_sum_dpp<16>(v);
    }
    return lanes_sum_dpp<32>(v);
}

__device__ __forceinline__ void qkv_hat(u32x2 c, float s, float b, float f[8])
{
    codes_to_float(c, f);
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = fmaf(f[k], s, b);
}

// What the kernels below share: a workgroup's heads' parameters in LDS -- (scale, offset) of the codes, gains in binary32 -- and the walk of a
// wave over its items: U tokens of a slot, slot by slot, tile by tile.  An item's loads are requested while the item before it is worked
// on, the first one's before the parameters and angles are formed: with a few tokens per workgroup these latencies are most of its time
// (forward of one token 6.7 -> 4.5 us, of 2000 tokens 24 -> 16 us; of 32768 no change).
struct QkvItem {
    int64_t t0;                        // the tile's first token; at or past T: no item
    uint32_t slot, base;               // base: the item's first token within the tile
};
struct QkvWave {
    uint32_t lane, wave, lph, hpw, d0, sub, phase, phases, slots, slot0, slot_step;
    int partner;
    __device__ __forceinline__ QkvWave(const QkvGeom &g, uint32_t heads)
    {
        lane = threadIdx.x & 63u;
        wave = uint32_t(__builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)));
        lph = 1u << g.lph_log2;
        hpw = 64u >> g.lph_log2;
        d0 = (lane & (lph - 1)) * 8;
        sub = lane >> g.lph_log2;
        const int hop = int(g.rot / 16);
        partner = int(lane) + (d0 < g.rot / 2 ? hop : d0 < g.rot ? -hop : 0);
        slots = (heads + hpw - 1) / hpw;
        phases = 1u << g.phases_log2;
        phase = wave & (phases - 1);
        slot0 = wave >> g.phases_log2;
        slot_step = (kThreads / 64) >> g.phases_log2;
    }
    __device__ __forceinline__ uint32_t tokens(const QkvGeom &g, int64_t t0) const { return g.T - t0 < g.tile ? uint32_t(g.T - t0) : g.tile; }
    // the first item of the tile at t0 or of the first one behind it that has any for this wave
    __device__ __forceinline__ QkvItem first(const QkvGeom &g, int64_t t0) const
    {
        QkvItem i = {t0, slot0, phase};
        while (i.t0 < g.T && (slot0 >= slots || phase >= tokens(g, i.t0))) i.t0 += int64_t(gridDim.x) * g.tile;
        return i;
    }
    template <int U> __device__ __forceinline__ QkvItem next(const QkvGeom &g, QkvItem i) const
    {
        i.base += phases * U;
        if (i.base < tokens(g, i.t0)) return i;
        i.base = phase;
        i.slot += slot_step;
        return i.slot < slots ? i : first(g, i.t0 + int64_t(gridDim.x) * g.tile);
    }
};
__host__ __device__ inline uint32_t qkv_even(uint32_t n) { return (n + 1) & ~1u; }      // gains start at 16 bytes
// params: [heads] (scale, offset), then gains [2][D]; CODES: 255 / alpha, else alpha / 255
template <typename T, bool CODES>
__device__ __forceinline__ void qkv_params(float2 *params, const QkvGeom &g, uint32_t heads, const float *alpha, const float *beta, const void *gamma_q, const void *gamma_k)
{
    for (uint32_t h = threadIdx.x; h < heads; h += kThreads) {
        const float a = alpha[h];
        params[h] = make_float2(CODES ? (a > 0.0f ? 255.0f / a : 0.0f) : a / 255.0f, beta[h]);
    }
    float *gain = reinterpret_cast<float *>(params + qkv_even(heads));
    if (gamma_q)
        for (uint32_t i = threadIdx.x; i < 2 * g.D; i += kThreads) gain[i] = i < g.D ? Store<T>::load1(gamma_q, i) : Store<T>::load1(gamma_k, i - g.D);
}
__device__ __forceinline__ void qkv_gain(const float *gain, uint32_t at, bool take, float gam[8])     // at: a multiple of 8
{
    const float4 *p = reinterpret_cast<const float4 *>(gain + at);
    const float4 a = p[0], b = p[1];
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int k = 0; k < 8; ++k) gam[k] = take ? v[k] : 1.0f;
}

// The forward (AGAIN false: from x, with codes and extrema) or queries and keys once more (AGAIN: from the codes and rstd).
// Both round y once, from binary32.  Lanes without an element and tokens past the tile lie outside of their spans: no access is
// conditional.
template <typename T, bool SR, bool AGAIN>
__global__ __launch_bounds__(kThreads, 4) void k_qkv_fwd(QkvGeom g, const void *__restrict__ x, int64_t x_row, const int8_t *__restrict__ qin, const void *__restrict__ gamma_q,
                                                      const void *__restrict__ gamma_k, const float *__restrict__ freq, const int32_t *__restrict__ pos,
                                                      float *alpha, float *beta, float lambda, void *__restrict__ y, float *__restrict__ rstd,
                                                      int8_t *__restrict__ q, uint64_t seed, uint64_t offset, float *__restrict__ part)
{
    typedef typename Store<T>::raw_t Raw;
    constexpr uint32_t kEb = sizeof(T);
    constexpr int U = AGAIN ? 4 : 2;                           // codes are half as many bytes to request (two: 117 us, four: 109)
    extern __shared__ float4 smem[];
    const uint32_t heads = AGAIN ? g.Hn : g.H, wide = g.H * g.D, slim = g.Hn * g.D;       // wide, slim: elements of a token, in codes and in y
    float2 *params = reinterpret_cast<float2 *>(smem), *cs = params + qkv_even(heads) + g.D;
    float *gain = reinterpret_cast<float *>(params + qkv_even(heads));
    int *lmn = reinterpret_cast<int *>(cs + g.tile * g.angles), *lmx = lmn + g.H;
    const QkvWave w(g, heads);
    const uint32_t d0 = w.d0;
    struct Loads {
        Raw raw[U];
        u32x2 cin[U];
        float rs[U];
    };
    auto load = [&](const QkvItem &i, Loads &l) __attribute__((always_inline)) {
        if (i.t0 >= g.T) return;                               // uniform; nothing is behind it
        const uint32_t n = w.tokens(g, i.t0), hd = i.slot * w.hpw + w.sub;
        const bool act = hd < heads && d0 < g.D;
        const Span sx(AGAIN ? nullptr : static_cast<const char *>(x) + i.t0 * x_row * kEb, AGAIN ? 0 : kNowhere), sq(AGAIN ? qin + i.t0 * wide : nullptr, AGAIN ? n * wide : 0);
        const Span sr(AGAIN && rstd ? rstd + i.t0 * g.Hn : nullptr, AGAIN && rstd ? n * g.Hn * 4 : 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t tk = i.base + u * w.phases;
            if (AGAIN) {
                const bool live = act && tk < n;
                l.cin[u] = sq.load8(live ? tk * wide + hd * g.D + d0 : kNowhere);
                l.rs[u] = sr.load_f32(live ? (tk * g.Hn + hd) * 4 : kNowhere);
            } else {
                // past the tile: the item's first token again, so that extrema stay what they are
                sx.load(act ? ((tk < n ? tk : i.base) * uint32_t(x_row) + hd * g.D + d0) * kEb : kNowhere, l.raw[u]);
            }
        }
    };
    QkvItem item = w.first(g, int64_t(blockIdx.x) * g.tile);
    Loads now, then;
    load(item, now);
    qkv_params<T, !AGAIN>(params, g, heads, alpha, beta, gamma_q, gamma_k);
    if (!AGAIN)
        for (uint32_t h = threadIdx.x; h < g.H; h += kThreads) {
            lmn[h] = order_key(__builtin_inff());
            lmx[h] = order_key(-__builtin_inff());
        }
    const float inv_d = 1.0f / float(g.D);
    float mn = __builtin_inff(), mx = -__builtin_inff();
    for (int64_t t0 = int64_t(blockIdx.x) * g.tile; t0 < g.T; t0 += int64_t(gridDim.x) * g.tile) {
        const uint32_t tokens = w.tokens(g, t0);
        if (t0 != int64_t(blockIdx.x) * g.tile) __syncthreads();      // the last tile's angles are done with
        qkv_angles(cs, g, freq, pos, t0, tokens);
        __syncthreads();
        const Span sq(AGAIN ? nullptr : q + t0 * wide, AGAIN ? 0 : tokens * wide);
        const Span sy(static_cast<char *>(y) + t0 * slim * kEb, tokens * slim * kEb), sr(!AGAIN && rstd ? rstd + t0 * g.Hn : nullptr, !AGAIN && rstd ? tokens * g.Hn * 4 : 0);
        while (item.t0 == t0) {
            const QkvItem after = w.next<U>(g, item);
            load(after, then);
            __builtin_amdgcn_sched_barrier(0);                 // requested before this item is worked on
            const uint32_t hd = item.slot * w.hpw + w.sub, at = hd * g.D + d0;
            const bool act = hd < heads && d0 < g.D, turn = act && hd < g.Hn;
            const bool any_turn = item.slot * w.hpw < g.Hn;     // uniform
            const float2 prm = params[act ? hd : 0];
            float gam[8];
            if (gamma_q) qkv_gain(gain, (hd < g.Hq ? 0 : g.D) + (d0 < g.D ? d0 : 0), turn, gam);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t tk = item.base + u * w.phases;
                const bool live = act && tk < tokens;
                float f[8];
                if (AGAIN) {
                    qkv_hat(now.cin[u], prm.x, prm.y, f);
                    if (gamma_q)
#pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] *= now.rs[u] * gam[k];
                } else {
                    Store<T>::unpack(now.raw[u], f);
                    const uint32_t e = tk * wide + at;
                    float v[8], bits[8];
                    if (SR) sr_bits(seed, offset + uint64_t((t0 * wide + e) >> 3), bits);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        v[k] = quantize_real<SR>(f[k], prm.x, prm.y, SR ? bits[k] : 0.0f);
                        mn = vmin(mn, f[k]);
                        mx = vmax(mx, f[k]);
                    }
                    const u32x2 c = round_pack_codes<SR>(v);
                    sq.store8(live ? e : kNowhere, c);
                    if (!any_turn) continue;
                    if (gamma_q) {
                        float ss = 0.0f;
#pragma unroll
                        for (int k = 0; k < 8; ++k) ss = fmaf(f[k], f[k], ss);
                        const float rr = 1.0f / sqrtf(fmaf(qkv_head_sum(ss, g.lph_log2), inv_d, g.eps));
                        sr.store_f32(live && turn && d0 == 0 ? (tk * g.Hn + hd) * 4 : kNowhere, rr);
#pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] *= rr * gam[k];
                    }
                }
                if (g.rot) qkv_turn(f, cs + (tk < tokens ? tk : 0) * g.angles, g, d0, w.partner, 1.0f);
                sy.store(live && turn ? (tk * slim + at) * kEb : kNowhere, Store<T>::pack(f));
            }
            if (!AGAIN && (after.slot != item.slot || after.t0 != t0)) {
                if (act) {
                    atomicMin(&lmn[hd], order_key(mn));
                    atomicMax(&lmx[hd], order_key(mx));
                }
                mn = __builtin_inff();
                mx = -__builtin_inff();
            }
            item = after;
            now = then;
        }
    }
    if (!AGAIN) {
        __syncthreads();
        if (gridDim.x == 1) {
            for (uint32_t h = threadIdx.x; h < g.H; h += kThreads)
                ema_update(order_val(lmn[h]), order_val(lmx[h]), alpha[h], beta[h], alpha, beta, h, lambda, 0);
            return;
        }
        for (uint32_t h = threadIdx.x; h < g.H; h += kThreads) {
            part[int64_t(blockIdx.x) * 2 * g.H + h] = order_val(lmn[h]);
            part[int64_t(blockIdx.x) * 2 * g.H + g.H + h] = order_val(lmx[h]);
        }
    }
}

// The backward; part[workgroup][2][D] takes the gains' gradients of its tokens, of query heads and of key heads.
template <typename T, bool NORM>
__global__ __launch_bounds__(kThreads, 4) void k_qkv_bwd(QkvGeom g, const int8_t *__restrict__ q, const void *__restrict__ gamma_q, const void *__restrict__ gamma_k,
                                                      const float *__restrict__ freq, const int32_t *__restrict__ pos, const float *__restrict__ alpha,
                                                      const float *__restrict__ beta, const float *__restrict__ rstd, const void *dy, void *dx, int64_t dx_row,
                                                      float *__restrict__ part, float *__restrict__ dgamma_q, float *__restrict__ dgamma_k)
{
    typedef typename Store<T>::raw_t Raw;
    constexpr uint32_t kEb = sizeof(T);
    constexpr int U = 2;
    extern __shared__ float4 smem[];
    const uint32_t heads = g.Hn, wide = g.H * g.D, slim = g.Hn * g.D;
    float2 *params = reinterpret_cast<float2 *>(smem), *cs = params + (NORM ? qkv_even(heads) + g.D : 0);
    float *gain = reinterpret_cast<float *>(params + qkv_even(heads));
    // the gains' gradients of this lane's elements, of query and of key heads: in LDS, where only this lane reaches them
    float *sums = reinterpret_cast<float *>(cs + g.tile * g.angles), *mine_q = sums + threadIdx.x * 8, *mine_k = mine_q + kThreads * 8;
    const QkvWave w(g, heads);
    const uint32_t d0 = w.d0;
    struct Loads {
        Raw raw[U];
        u32x2 cin[U];
        float rs[U];
    };
    auto load = [&](const QkvItem &i, Loads &l) __attribute__((always_inline)) {
        if (i.t0 >= g.T) return;
        const uint32_t n = w.tokens(g, i.t0), hd = i.slot * w.hpw + w.sub;
        const bool act = hd < heads && d0 < g.D;
        const Span sdy(static_cast<const char *>(dy) + i.t0 * slim * kEb, n * slim * kEb);
        const Span sq(NORM ? q + i.t0 * wide : nullptr, NORM ? n * wide : 0), sr(NORM ? rstd + i.t0 * g.Hn : nullptr, NORM ? n * g.Hn * 4 : 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t tk = i.base + u * w.phases;
            const bool live = act && tk < n;
            sdy.load(live ? (tk * slim + hd * g.D + d0) * kEb : kNowhere, l.raw[u]);
            if (NORM) {
                l.cin[u] = sq.load8(live ? tk * wide + hd * g.D + d0 : kNowhere);
                l.rs[u] = sr.load_f32(live ? (tk * g.Hn + hd) * 4 : kNowhere);
            }
        }
    };
    QkvItem item = w.first(g, int64_t(blockIdx.x) * g.tile);
    Loads now, then;
    load(item, now);
    if (NORM) {
        qkv_params<T, false>(params, g, heads, alpha, beta, gamma_q, gamma_k);
#pragma unroll
        for (int k = 0; k < 8; ++k) mine_q[k] = mine_k[k] = 0.0f;
    }
    const float inv_d = 1.0f / float(g.D);
    float mine[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) mine[k] = 0.0f;
    for (int64_t t0 = int64_t(blockIdx.x) * g.tile; t0 < g.T; t0 += int64_t(gridDim.x) * g.tile) {
        const uint32_t tokens = w.tokens(g, t0);
        if (t0 != int64_t(blockIdx.x) * g.tile) __syncthreads();
        qkv_angles(cs, g, freq, pos, t0, tokens);
        __syncthreads();
        const Span sdx(static_cast<char *>(dx) + t0 * dx_row * kEb, kNowhere);
        while (item.t0 == t0) {
            const QkvItem after = w.next<U>(g, item);
            load(after, then);
            __builtin_amdgcn_sched_barrier(0);
            const uint32_t hd = item.slot * w.hpw + w.sub, at = hd * g.D + d0;
            const bool act = hd < heads && d0 < g.D, key = hd >= g.Hq;
            float2 prm = make_float2(0.0f, 0.0f);
            float gam[8];
            if (NORM) {
                prm = params[act ? hd : 0];
                qkv_gain(gain, (key ? g.D : 0) + (d0 < g.D ? d0 : 0), true, gam);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t tk = item.base + u * w.phases;
                const bool live = act && tk < tokens;
                float f[8];
                Store<T>::unpack(now.raw[u], f);           // zeros where nothing was loaded
                if (g.rot) qkv_turn(f, cs + (tk < tokens ? tk : 0) * g.angles, g, d0, w.partner, -1.0f);
                if (NORM) {
                    float n[8], dot = 0.0f;
                    qkv_hat(now.cin[u], prm.x, prm.y, n);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        n[k] *= now.rs[u];
                        mine[k] = fmaf(f[k], n[k], mine[k]);
                        f[k] *= gam[k];
                        dot = fmaf(f[k], n[k], dot);
                    }
                    const float mean = qkv_head_sum(dot, g.lph_log2) * inv_d;
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] = now.rs[u] * fmaf(-n[k], mean, f[k]);
                }
                __builtin_amdgcn_sched_barrier(0);
                sdx.store(live ? (tk * uint32_t(dx_row) + at) * kEb : kNowhere, Store<T>::pack(f));
            }
            if (NORM && (after.slot != item.slot || after.t0 != t0)) {
                float *to = key ? mine_k : mine_q;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    to[k] += mine[k];
                    mine[k] = 0.0f;
                }
            }
            item = after;
            now = then;
        }
    }
    if (!NORM) return;
    // threads that hold the same elements of different heads, in their order (exchanges between lanes before that took 3 us more)
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 2 * g.D; i += kThreads) {
        const uint32_t c = i >= g.D, d = i - c * g.D;
        const float *p = sums + c * (kThreads * 8) + d;
        float v = 0.0f;
#pragma unroll 8
        for (uint32_t k = 0; k < kThreads; k += w.lph) v += p[k * 8];
        if (gridDim.x > 1) part[int64_t(blockIdx.x) * 2 * g.D + i] = v;
        else (c ? dgamma_k : dgamma_q)[d] = v;
    }
}

// columns of part[nwg][2*D]: a workgroup takes 32 of them, 32 rows at a time
constexpr int kQkvCols = 32;
__global__ __launch_bounds__(1024) void k_qkv_gains(const float *__restrict__ part, int nwg, uint32_t D, float *__restrict__ dgamma_q, float *__restrict__ dgamma_k)
{
    __shared__ float s[32][kQkvCols + 1];
    const uint32_t col = blockIdx.x * kQkvCols + (threadIdx.x & 31u), row = threadIdx.x >> 5;
    float v = 0.0f;
    if (col < 2 * D)
#pragma unroll 8
        for (int w = int(row); w < nwg; w += 32) v += part[int64_t(w) * 2 * D + col];
    s[row][threadIdx.x & 31u] = v;
    __syncthreads();
    if (row == 0 && col < 2 * D) {
        float a = 0.0f;
        for (int k = 0; k < 32; ++k) a += s[k][threadIdx.x & 31u];
        if (col < D) dgamma_q[col] = a;
        else dgamma_k[col - D] = a;
    }
}

static mesa_status check_qkv(const mesa_qkv_heads &h, mesa_dtype dt)
{
    if (!valid_dtype(dt) || h.T < 0 || h.Hq < 0 || h.Hk < 0 || h.Hv < 0 || h.Hq + h.Hk < 1 || h.D < 1 || h.rot < 0 || h.rot > h.D || (h.rot & 1)) return MESA_ERR_INVALID_ARG;
    if (h.axes < 1 || h.axes > 4 || !(h.eps >= 0.0f) || !(h.eps <= 3.0e38f)) return MESA_ERR_INVALID_ARG;
    int64_t pairs = 0;
    for (int a = 0; a < h.axes; ++a) {
        if (h.section[a] < 0 || h.section[a] > h.rot / 2) return MESA_ERR_INVALID_ARG;
        pairs += h.section[a];
    }
    if (pairs != h.rot / 2) return MESA_ERR_INVALID_ARG;
    if (h.Hq > kQkvMaxHeads || h.Hk > kQkvMaxHeads || h.Hv > kQkvMaxHeads || h.Hq + h.Hk + h.Hv > kQkvMaxHeads) return MESA_ERR_UNSUPPORTED;
    if (h.D % 8 != 0 || h.D > 256 || (!h.interleaved && h.rot % 16 != 0) || h.T >= (int64_t(1) << 31)) return MESA_ERR_UNSUPPORTED;
    return MESA_OK;
}

static size_t qkv_lds_fwd(const QkvGeom &g, bool again)
{
    return (qkv_even(again ? g.Hn : g.H) + g.D + g.tile * g.angles) * sizeof(float2) + (again ? 0 : size_t(g.H) * 8);
}
static size_t qkv_lds_bwd(const QkvGeom &g, bool norm)
{
    return (size_t(norm ? qkv_even(g.Hn) + g.D : 0) + g.tile * g.angles) * sizeof(float2) + (norm ? 2 * kThreads * 32 : 0);
}

}  // namespace mesa

using namespace mesa;

extern "C" MESA_EXPORT size_t mesa_qkv_norm_rope_fwd_q_workspace_bytes(mesa_qkv_heads h, mesa_dtype dt)
{
    if (check_qkv(h, dt) != MESA_OK) return 0;
    const QkvGeom g = qkv_geom(h);
    return size_t(qkv_grid(g) < 1 ? 1 : qkv_grid(g)) * 2 * g.H * sizeof(float);
}

extern "C" MESA_EXPORT size_t mesa_qkv_norm_rope_bwd_q_workspace_bytes(mesa_qkv_heads h, mesa_dtype dt)
{
    if (check_qkv(h, dt) != MESA_OK) return 0;
    const QkvGeom g = qkv_geom(h);
    return size_t(qkv_grid(g) < 1 ? 1 : qkv_grid(g)) * 2 * g.D * sizeof(float);
}

extern "C" MESA_EXPORT mesa_status mesa_qkv_norm_rope_fwd_q(const void *x, int64_t x_row, mesa_qkv_heads h, const void *gamma_q, const void *gamma_k, const float *freq,
                                                            const int32_t *pos, float *alpha, float *beta, float lambda, void *y, float *rstd, int8_t *q, mesa_round mode,
                                                            uint64_t seed, uint64_t offset, void *ws, size_t ws_bytes, mesa_dtype dt, void *stream)
{
    if (mode != MESA_ROUND_NEAREST_EVEN && mode != MESA_ROUND_STOCHASTIC) return MESA_ERR_INVALID_ARG;
    if (!(lambda >= 0.0f && lambda <= 1.0f)) return MESA_ERR_INVALID_ARG;
    if (const mesa_status st = check_qkv(h, dt)) return st;
    if (x_row % 8 != 0 || x_row < (h.Hq + h.Hk + h.Hv) * h.D || (gamma_q == nullptr) != (gamma_k == nullptr)) return MESA_ERR_INVALID_ARG;
    if (h.T == 0) return MESA_OK;
    if (x_row >= (int64_t(1) << 24)) return MESA_ERR_UNSUPPORTED;
    if (!x || !y || !q || !alpha || !beta || x == y || !aligned16(x) || !aligned16(y) || !aligned16(q) || !aligned16(gamma_q) || !aligned16(gamma_k) || !aligned4(alpha) ||
        !aligned4(beta) || (gamma_q && !rstd) || !aligned4(rstd) || (h.rot && (!freq || !pos)) || !aligned4(freq) || !aligned4(pos))
        return MESA_ERR_INVALID_ARG;
    const QkvGeom g = qkv_geom(h);
    const int grid = qkv_grid(g);
    if (!ws || !aligned4(ws) || ws_bytes < mesa_qkv_norm_rope_fwd_q_workspace_bytes(h, dt)) return MESA_ERR_WORKSPACE;
    const size_t lds = qkv_lds_fwd(g, false);
    hipStream_t s = static_cast<hipStream_t>(stream);
#define MESA_QKV(T) \
    do { \
        auto *k = mode == MESA_ROUND_STOCHASTIC ? k_qkv_fwd<T, true, false> : k_qkv_fwd<T, false, false>; \
        hipLaunchKernelGGL(k, dim3(grid), dim3(kThreads), lds, s, g, x, x_row, nullptr, gamma_q, gamma_k, freq, pos, alpha, beta, lambda, y, rstd, q, seed, offset, static_cast<float *>(ws)); \
    } while (0)
    MESA_FOR_DTYPE(dt, MESA_QKV);
#undef MESA_QKV
    if (const mesa_status st = launch_status()) return st;
    if (grid == 1) return MESA_OK;
    launch_ema_finalize(static_cast<const float *>(ws), grid, g.H, alpha, beta, lambda, 0, 0, 0.0f, s);
    return launch_status();
}

extern "C" MESA_EXPORT mesa_status mesa_qkv_norm_rope_recompute_q(const int8_t *q, mesa_qkv_heads h, const void *gamma_q, const void *gamma_k, const float *freq,
                                                                  const int32_t *pos, const float *alpha, const float *beta, const float *rstd, void *y, mesa_dtype dt,
                                                                  void *stream)
{
    if (const mesa_status st = check_qkv(h, dt)) return st;
    if ((gamma_q == nullptr) != (gamma_k == nullptr)) return MESA_ERR_INVALID_ARG;
    if (h.T == 0) return MESA_OK;
    if (!q || !y || !alpha || !beta || !aligned16(q) || !aligned16(y) || !aligned16(gamma_q) || !aligned16(gamma_k) || !aligned4(alpha) || !aligned4(beta) ||
        (gamma_q && !rstd) || !aligned4(rstd) || (h.rot && (!freq || !pos)) || !aligned4(freq) || !aligned4(pos))
        return MESA_ERR_INVALID_ARG;
    const QkvGeom g = qkv_geom(h);
    const size_t lds = qkv_lds_fwd(g, true);
#define MESA_QKV(T) \
    hipLaunchKernelGGL((k_qkv_fwd<T, false, true>), dim3(qkv_grid(g)), dim3(kThreads), lds, static_cast<hipStream_t>(stream), g, nullptr, 0, q, gamma_q, gamma_k, freq, pos, \
                       const_cast<float *>(alpha), const_cast<float *>(beta), 0.0f, y, const_cast<float *>(rstd), nullptr, 0, 0, nullptr)
    MESA_FOR_DTYPE(dt, MESA_QKV);
#undef MESA_QKV
    return launch_status();
}

extern "C" MESA_EXPORT mesa_status mesa_qkv_norm_rope_bwd_q(const int8_t *q, mesa_qkv_heads h, const void *gamma_q, const void *gamma_k, const float *freq, const int32_t *pos,
                                                            const float *alpha, const float *beta, const float *rstd, const void *dy, void *dx, int64_t dx_row,
                                                            float *dgamma_q, float *dgamma_k, void *ws, size_t ws_bytes, mesa_dtype dt, void *stream)
{
    if (const mesa_status st = check_qkv(h, dt)) return st;
    const bool norm = gamma_q != nullptr;
    if (norm != (gamma_k != nullptr) || dx_row % 8 != 0 || dx_row < (h.Hq + h.Hk) * h.D || (norm && (!dgamma_q || !dgamma_k)) || !aligned4(dgamma_q) || !aligned4(dgamma_k))
        return MESA_ERR_INVALID_ARG;
    if (dx == dy && dx_row != (h.Hq + h.Hk) * h.D) return MESA_ERR_INVALID_ARG;
    if (dx_row >= (int64_t(1) << 24)) return MESA_ERR_UNSUPPORTED;
    if (h.T > 0) {
        if (!dy || !dx || !aligned16(dy) || !aligned16(dx) || (h.rot && (!freq || !pos)) || !aligned4(freq) || !aligned4(pos)) return MESA_ERR_INVALID_ARG;
        if (norm && (!q || !alpha || !beta || !rstd || !aligned16(q) || !aligned16(gamma_q) || !aligned16(gamma_k) || !aligned4(alpha) || !aligned4(beta) || !aligned4(rstd)))
            return MESA_ERR_INVALID_ARG;
    }
    if (h.T == 0 && !norm) return MESA_OK;
    const QkvGeom g = qkv_geom(h);
    const int grid = qkv_grid(g);
    if (norm && (!ws || !aligned4(ws) || ws_bytes < mesa_qkv_norm_rope_bwd_q_workspace_bytes(h, dt))) return MESA_ERR_WORKSPACE;
    const size_t lds = qkv_lds_bwd(g, norm);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (h.T > 0) {
#define MESA_QKV(T) \
    do { \
        auto *k = norm ? k_qkv_bwd<T, true> : k_qkv_bwd<T, false>; \
        hipLaunchKernelGGL(k, dim3(grid), dim3(kThreads), lds, s, g, q, gamma_q, gamma_k, freq, pos, alpha, beta, rstd, dy, dx, dx_row, static_cast<float *>(ws), dgamma_q, dgamma_k); \
    } while (0)
        MESA_FOR_DTYPE(dt, MESA_QKV);
#undef MESA_QKV
        if (const mesa_status st = launch_status()) return st;
    }
    if (norm && (h.T == 0 || grid > 1)) {   // no tokens: zeros
        hipLaunchKernelGGL(k_qkv_gains, dim3(uint32_t(ceil_div(2 * h.D, kQkvCols))), dim3(1024), 0, s, static_cast<const float *>(ws), h.T > 0 ? grid : 0, g.D, dgamma_q, dgamma_k);
        return launch_status();
    }
    return MESA_OK;
}
