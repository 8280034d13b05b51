// attention_fwd.hip -- the forward of attention over intervals of keys, and the intervals themselves.
//   s = scale q.k (capped, biased by distance),  p = softmax over lo <= j < hi,  o = p v,  lse = log sum exp s
//
// One pass over the keys with a running maximum and sum (powers of two): a wave owns 32 rows -- queries of the heads that share
// a key head, token by token, so that a group's heads read each tile once -- and keeps q and the sums of o in registers;
// the workgroup's waves share tiles of k and v in LDS, the next tile on its way while one is worked on.  Scores come out
// transposed (attention.hpp), so a row's maximum and sum are a lane's own business but for one swap of half-waves.
// Tiles that no row of the workgroup sees are not loaded, tiles that all rows of a wave see in full are not masked.
// Measured: 8 x 4096 x 16 heads of 64, causal, binary16, 359 us (0.77 PFLOP/s; vector instructions issue for 0.8 of the cycles: an
// exponential and four more a score); 2 x 8192 x 16 heads of 128, capped, bfloat16, 676 us (0.81; eight and three at a quarter of the rate); a token
// of 16 sequences, 396 MB of keys and values, 88 us with the join (4.5 TB/s; a copy 5.0).
#include "attention.hpp"

namespace mesa {

AtShape at_shape(const mesa_attention &a, const mesa_attention_mask &m)
{
    AtShape s;
    s.B = int32_t(a.B);
    s.Nq = int32_t(a.Nq);
    s.Nk = int32_t(a.Nk);
    s.Hq = int32_t(a.Hq);
    s.Hk = int32_t(a.Hk);
    s.G = int32_t(a.Hq / a.Hk);
    s.D = int32_t(a.D);
    s.R = uint32_t(a.Nq * s.G);
    s.div_g = make_fastdiv(uint32_t(s.G));
    s.c = a.cap > 0.0f ? 2.0f * kLog2e * a.scale / a.cap : kLog2e * a.scale;
    s.cap2 = a.cap * kLog2e;
    s.scale = a.scale;
    s.lo = m.lo;
    s.hi = m.hi;
    s.q_start = m.q_start;
    s.slopes = m.slopes;
    return s;
}

// ---------------------------------------------------------------------------------------------
// intervals
// ---------------------------------------------------------------------------------------------
// A workgroup takes kAtStretch consecutive queries of a sequence, whose places are consecutive keys.  Documents: where the number
// changes within the stretch is one bit per place in LDS, and each query finds its run's ends among those; only the run that the
// first place lies in, and the one of the last, may reach out of the stretch, and two waves search for those ends, 64 keys at a time.
// Every query searching for itself took 51 us where this takes 8.8 (64 x 32768 queries, 61 documents a row; 63 such rows 10.7), of which 5.4 are
// spent without documents: 16.8 MB written, as fast as memory takes them.
constexpr int kAtStretch = 1024;

// the first x of [l, h] with x == h or not below(x), for a row where below() holds up to there and no further; 64 probes a round
template <typename Below> __device__ __forceinline__ int at_search(int l, int h, int lane, Below below)
{
    while (l < h) {
        const int step = (h - l + 63) / 64;
        const int64_t x = l + int64_t(lane) * step;
        const int n = __popcll(__ballot(x < h && below(int(x))));
        if (n == 0) {
            h = l;
        } else {
            const int64_t up = l + int64_t(n) * step;
            l += (n - 1) * step + 1;
            h = up < h ? int(up) : h;
        }
    }
    return l;
}

template <bool DOC>
__global__ __launch_bounds__(kThreads) void k_attn_bounds(int32_t *__restrict__ lo, int32_t *__restrict__ hi, int Nq, int Nk, int causal, int window,
                                                          const int32_t *__restrict__ kv_len, const int32_t *__restrict__ q_start, const int32_t *__restrict__ prefix,
                                                          const int32_t *__restrict__ doc, uint32_t B)
{
    constexpr int kU = kAtStretch / kThreads, kWords = kAtStretch / 64;
    __shared__ uint64_t change[kWords];
    __shared__ int end[2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int64_t b = blockIdx.x % uint32_t(B);     // the sequences first: where they are a multiple of 8, a sequence's workgroups share one XCD's cache
    const int i0 = int(blockIdx.x / uint32_t(B)) * kAtStretch, count = Nq - i0 < kAtStretch ? Nq - i0 : kAtStretch;
    int n = Nk;
    if (kv_len) n = kv_len[b] < n ? kv_len[b] : n;
    const int64_t from = (q_start ? int64_t(q_start[b]) : int64_t(Nk) - Nq) + i0;    // the place of the stretch's first query
    const bool some = n > 0 && from < n && from + count > 0;                           // of any of its queries among the keys; -kAtStretch < from < n then, and 32 bits do
    const int p0 = some ? int(from) : 0, p1 = p0 + count - 1, first = p0 > 0 ? p0 : 0, last = p1 < n - 1 ? p1 : n - 1;
    const int32_t *d = DOC ? doc + b * Nk : nullptr;
    uint32_t words = 0;
    if (DOC && some) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int x = p0 + u * kThreads + int(threadIdx.x);
            const bool differs = x > first && x <= last && d[x] != d[x - 1];
            const uint64_t m = __ballot(differs);
            if (lane == 0) change[u * (kThreads / 64) + wave] = m;
        }
        if (wave == 0) {
            const int mine = d[first], at = at_search(0, first, lane, [&](int x) { return d[x] < mine; });
            if (lane == 0) end[0] = at;
        } else if (wave == 1) {
            const int mine = d[last], at = at_search(last + 1, n, lane, [&](int x) { return d[x] <= mine; });
            if (lane == 0) end[1] = at;
        }
        __syncthreads();
        words = uint32_t(__ballot(lane < kWords && change[lane & (kWords - 1)] != 0));
    }
    const int top = prefix ? prefix[b] : 0;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const int w = u * (kThreads / 64) + wave, k = w * 64 + lane;
        if (k >= count) break;
        const int p = p0 + k;
        int l = 0, h = 0;
        if (some && p >= 0 && p < n) {
            h = n;
            if (causal) {
                const int seen = p + 1 > top ? p + 1 : top;
                h = seen < h ? seen : h;
            }
            if (window > 0) {
                l = p - window + 1 > 0 ? p - window + 1 : 0;
                if (!causal && p + window < h) h = p + window;
            }
        }
        if (DOC && some) {
            // the last change among the words before and the first among those behind: one answer per wave; then this word's own
            const uint64_t c = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(change[w] >> 32))))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(change[w]))));
            const uint32_t before = words & ((1u << w) - 1), behind = words >> w >> 1;
            int x = end[0], y = end[1];
            if (before) {
                const int v = 31 - __clz(before);
                x = p0 + v * 64 + 63 - __clzll(change[v]);
            }
            if (behind) {
                const int v = w + 1 + __builtin_ctz(behind);
                y = p0 + v * 64 + __builtin_ctzll(change[v]);
            }
            if (c) {
                const uint64_t below = c & (~uint64_t(0) >> (63 - lane)), above = c & ~(~uint64_t(0) >> (63 - lane));
                if (below) x = p0 + w * 64 + 63 - __clzll(below);
                if (above) y = p0 + w * 64 + __builtin_ctzll(above);
            }
            l = x > l ? x : l;
            h = y < h ? y : h;
        }
        if (l >= h) l = h = 0;
        lo[b * Nq + i0 + k] = l;
        hi[b * Nq + i0 + k] = h;
    }
}

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
struct AtFwd {
    AtShape s;
    AtView q, k, v;
    AtOut o;
    float *lse;
    float *part_o, *part_lse;    // [split][(b, key head, row)][D] and [split][...]; null: no split
    uint32_t heads, row_blocks, splits;   // heads: B * Hk
};

// NW waves of 32 rows, tiles of BN keys
// CAP: kAtCapped takes at_tanh<true>.  kAtCappedLong leaves r = -1 / (2^u + 1) in a score's place, u = 2 log2(e) s / cap, whose score is
// cap + 2 cap r: both go into the exponent's one multiply-add, three instructions less of eleven a score where vector instructions are
// what binds (2 x 8192 x 16 heads of 128 717 -> 670 us, of 64 486 -> 423).  Such a score is off by 2^-23 of the cap or so, whatever its
// size; lse over 600 keys then by 1.3e-7 of itself (4e-8 with tanh), where a query sees one key of them by 1.5e-6 (cap 30): so only from kAtLong keys on and for
// caps up to kAtLongCap.
enum { kAtUncapped = 0, kAtCapped, kAtCappedLong };
constexpr int kAtLong = 512;
constexpr float kAtLongCap = 64.0f;
template <typename T, int DP, int NW, int BN, int CAP, bool BIAS>
__global__ __launch_bounds__(NW * 64, NW == 1 ? 1 : DP == 64 && !BIAS ? 4 : 2) void k_attn_fwd(const AtFwd a)
{
    typedef AtNum<T> Num;
    typedef AtTile<NW * 64, BN, DP> Tile;
    constexpr int kKs = DP / 16, kDt = DP / 32, kSub = BN / 32;
    __shared__ __attribute__((aligned(256))) char lds[4 * Tile::kBytes];      // two tiles of k, two of v
    __shared__ int range[4][NW];
    __shared__ uint64_t seen[NW];
    const AtShape &s = a.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), half = lane >> 5;
    const uint32_t head = blockIdx.x % a.heads, rest = blockIdx.x / a.heads;     // the heads first: a head's workgroups stay on one XCD where they are a multiple of 8
    const uint32_t split = rest % a.splits, rb = a.row_blocks - 1 - rest / a.splits;   // the longest rows of a causal order first
    const int b = int(head / uint32_t(s.Hk)), hk = int(head) - b * s.Hk;
    const uint32_t r_own = (rb * NW + wave) * 32 + (lane & 31), r = r_own < s.R ? r_own : s.R - 1;
    const AtRow row = at_row(s, r);
    const int hq = hk * s.G + int(row.g);
    int lo, hi;
    at_interval(s, b, row.token, lo, hi);
    const bool none = lo >= hi;
    const int wlo = at_wave_min(none ? 0x7FFFFFFF : lo), whi = at_wave_max(hi);   // of what the wave's rows see, any
    const int flo = at_wave_max(lo), fhi = at_wave_min(hi);                        // and all
    if (lane == 0) {
        range[0][wave] = wlo;
        range[1][wave] = whi;
        range[2][wave] = flo;
        range[3][wave] = fhi;
    }
    u32x4 qf[kKs];
    {
        const char *p = a.q.p + int64_t(b) * a.q.batch + int64_t(row.token) * a.q.token + int64_t(hq) * a.q.head;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) qf[ks] = at_column(p, ks, lane, s.D);
    }
    const float slope2 = BIAS ? s.slopes[hq] * kLog2e : 0.0f;
    const int place = BIAS ? at_place(s, b, row.token) : 0;
    const float to_score = CAP == kAtCappedLong ? 2.0f * s.cap2 : CAP ? s.cap2 : s.c;      // to powers of two, from r, tanh or the product
    const float more = CAP == kAtCappedLong ? s.cap2 : 0.0f;
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
    if (a.splits > 1) {
        const int per = (t1 - t0 + int(a.splits) - 1) / int(a.splits);
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

    at_acc o[kDt];
#pragma unroll
    for (int d = 0; d < kDt; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = kAtLow, l = 0.0f;

    const uint32_t plain_at = at_address(lds) + at_plain_lane<DP>(lane), trans_at = at_address(lds) + at_trans_lane<DP>(lane);
    auto work = [&](int cur, int j0, bool whole) __attribute__((always_inline)) {
        const uint32_t ka = plain_at + cur * 2 * Tile::kBytes, va = trans_at + cur * 2 * Tile::kBytes + Tile::kBytes;
        at_acc x[kSub];
#pragma unroll
        for (int t = 0; t < kSub; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[t][i] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) {
                x[t] = Num::mfma(at_plain<DP>(ka, t * 32, ks), qf[ks], x[t]);
                if (ks % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
        const int first = j0 + 4 * half;           // the key of register 0
        if (CAP || BIAS) {
            const float away = float(place - first);
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (CAP == kAtCappedLong) x[t][i] = __builtin_amdgcn_rcpf(-1.0f - at_exp2(x[t][i] * s.c));
                    else if (CAP) x[t][i] = at_tanh<true>(x[t][i] * s.c);
                    if (BIAS) x[t][i] = fmaf(x[t][i], to_score, fmaf(-slope2, fabsf(away - float(t * 32 + at_reg_row(i))), more));
                }
        }
        if (!whole) {
#pragma unroll
            for (int t = 0; t < kSub; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[t][i] = uint32_t(first + t * 32 + at_reg_row(i) - lo) < uint32_t(hi - lo) ? x[t][i] : -__builtin_inff();
        }
        float top = x[0][0];
#pragma unroll
        for (int t = 0; t < kSub; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[t][i]);
        top = at_pair_max(top);
        constexpr bool kRaw = !BIAS;               // the factor is then still to come (it is positive)
        if (kRaw) top = fmaf(top, to_score, more);
        // the sums are scaled anew only where a row's maximum has grown by more than 2^8: probabilities up to 2^8 are as exact
        if (__ballot(top > m + 8.0f)) {
            const float m1 = fmaxf(m, top), f = at_exp2(m - m1);
            m = m1;
            l *= f;
#pragma unroll
            for (int d = 0; d < kDt; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        u32x4 p[2 * kSub];
        float l1 = 0.0f;
        const float less = more - m;
#pragma unroll
        for (int t = 0; t < kSub; ++t)
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int i = 8 * g + 2 * w;
                    const float e0 = at_exp2(kRaw ? fmaf(x[t][i], to_score, less) : x[t][i] - m), e1 = at_exp2(kRaw ? fmaf(x[t][i + 1], to_score, less) : x[t][i + 1] - m);
                    l += e0;
                    l1 += e1;
                    p[2 * t + g][w] = Num::pack(e0, e1);
                }
        l += l1;
#pragma unroll
        for (int g = 0; g < 2 * kSub; ++g)
#pragma unroll
            for (int d = 0; d < kDt; ++d) {
                o[d] = Num::mfma(at_transposed<DP>(va, g * 16, d * 32), p[g], o[d]);
                if (d == kDt - 1) __builtin_amdgcn_sched_barrier(0);
            }
    };

    if (t0 < t1) fetch(t0);
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
        __syncthreads();                            // the other pair of tiles is behind every wave then
        if (t + 1 < t1) fetch(t + 1);
        if (j0 + BN <= wlo || j0 >= whi) continue;
        work(cur, j0, j0 >= flo && j0 + BN <= fhi);
    }

    l = at_pair_sum(l);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;       // not a number where a score is none, lse then too
    if (r_own >= s.R) return;
    if (a.part_o) {
        const int64_t at = int64_t(split) * a.heads * s.R + int64_t(head) * s.R + r;
        if (half == 0) a.part_lse[at] = l == 0.0f ? -__builtin_inff() : m + __log2f(l);
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int e = d * 32 + 8 * w + 4 * half;
                if (e < s.D) *reinterpret_cast<float4 *>(a.part_o + at * s.D + e) = make_float4(o[d][4 * w] * inv, o[d][4 * w + 1] * inv, o[d][4 * w + 2] * inv, o[d][4 * w + 3] * inv);
            }
        return;
    }
    if (half == 0) a.lse[(int64_t(b) * s.Hq + hq) * s.Nq + row.token] = l == 0.0f ? -__builtin_inff() : (m + __log2f(l)) * kLn2;
    char *op = a.o.p + int64_t(b) * a.o.batch + int64_t(row.token) * a.o.token + int64_t(hq) * a.o.head;
#pragma unroll
    for (int d = 0; d < kDt; ++d)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int e = d * 32 + 8 * w + 4 * half;
            if (e < s.D) at_store4<T>(op + e * 2, o[d][4 * w] * inv, o[d][4 * w + 1] * inv, o[d][4 * w + 2] * inv, o[d][4 * w + 3] * inv);
        }
}

// The splits of a row joined, with weights 2^(lse_s - max): 32 threads with four elements each.  FEW: a workgroup per row, whose eight such groups
// share out the splits and meet in LDS; else a row to each of
// them, or to 16 threads up to 64 elements (32768 rows of four splits 24.7 -> 7.5 us).
template <typename T, bool FEW>
__global__ __launch_bounds__(kThreads) void k_attn_join(const AtFwd a)
{
    constexpr int kU = 4, kGroups = kThreads / 32;
    static_assert(kThreads == 256, "8 - log2 rows of a workgroup");
    const AtShape &s = a.s;
    __shared__ float sums[FEW ? kGroups : 1][32][5];
    __shared__ float tops[FEW ? kGroups : 1];
    const int log2 = FEW || s.D > 64 ? 5 : 4, quad = threadIdx.x & ((1 << log2) - 1), group = threadIdx.x >> log2, e = quad * 4;
    const int64_t step = int64_t(a.heads) * s.R, at = FEW ? int64_t(blockIdx.x) : (int64_t(blockIdx.x) << (8 - log2)) + group;     // (b, key head, row)
    if (!FEW && at >= step) return;
    const int first = FEW ? group : 0, stride = FEW ? kGroups : 1;
    const bool act = e < s.D;
    float top = kAtLow, total = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = first; k0 < int(a.splits); k0 += stride * kU) {
        float z[kU];
        float4 v[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {                                // four requested together; behind the last one this group's first again, without weight
            const int64_t k = (k0 + u * stride < int(a.splits) ? k0 + u * stride : k0) * step + at;
            z[u] = a.part_lse[k];
            v[u] = act ? *reinterpret_cast<const float4 *>(a.part_o + k * s.D + e) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        float m = top;
#pragma unroll
        for (int u = 0; u < kU; ++u) m = fmaxf(m, z[u]);
        const float f = at_exp2(top - m);
        top = m;
        total *= f;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] *= f;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const float w = k0 + u * stride < int(a.splits) ? at_exp2(z[u] - m) : 0.0f;      // a split that saw nothing: -infinity, no weight
            total += w;
            x[0] = fmaf(w, v[u].x, x[0]);
            x[1] = fmaf(w, v[u].y, x[1]);
            x[2] = fmaf(w, v[u].z, x[2]);
            x[3] = fmaf(w, v[u].w, x[3]);
        }
    }
    float m = top;
    if (FEW) {
        if (quad == 0) tops[group] = top;
#pragma unroll
        for (int k = 0; k < 4; ++k) sums[group][quad][k] = x[k];
        sums[group][quad][4] = total;
        __syncthreads();
        if (group > 0) return;
        m = kAtLow;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) m = fmaxf(m, tops[g]);
        total = x[0] = x[1] = x[2] = x[3] = 0.0f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const float w = at_exp2(tops[g] - m);
            total = fmaf(w, sums[g][quad][4], total);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = fmaf(w, sums[g][quad][k], x[k]);
        }
    }
    if (!act) return;
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const uint32_t head = uint32_t(at / s.R), r = uint32_t(at - int64_t(head) * s.R);
    const int b = int(head) / s.Hk, hk = int(head) - b * s.Hk;
    const AtRow row = at_row(s, r);
    const int hq = hk * s.G + int(row.g);
    at_store4<T>(a.o.p + int64_t(b) * a.o.batch + int64_t(row.token) * a.o.token + int64_t(hq) * a.o.head + e * 2, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    if (e == 0) a.lse[(int64_t(b) * s.Hq + hq) * s.Nq + row.token] = total == 0.0f ? -__builtin_inff() : (m + __log2f(total)) * kLn2;
}

struct AtFwdPlan {
    int waves, keys;             // of a workgroup; of a tile
    uint32_t row_blocks, splits;
    size_t ws;
};
// Rows that fit one wave get workgroups of one wave with small tiles (a single token's reading is all latency and bandwidth, and
// four waves would load for one); few workgroups share out the keys.
static AtFwdPlan at_fwd_plan(const mesa_attention &a)
{
    AtFwdPlan p;
    const int64_t R = a.Nq * (a.Hq / a.Hk), heads = a.B * a.Hk;
    p.waves = R <= 32 ? 1 : 4;
    p.keys = p.waves == 1 ? 32 : 64;
    p.row_blocks = uint32_t(ceil_div(R, p.waves * 32));
    // One wave per SIMD fits the wide heads' registers: 1024 workgroups at a time.  Two rounds of them even out lengths that differ (16 x 4
    // heads over 16381 keys or fewer: 24 splits 90 us, 32 85, 64 88); with less than 256 keys each the rounds' own cost takes more
    // than that (3001 keys: 23 splits 21.7 us, 16 17.5).  Of four waves, one round as registers have it, four workgroups to a compute unit up to
    // 64 elements and two above (8 heads of 4096 tokens 67 -> 41 us and 103 -> 70; 16 x 64 tokens after 16381 376 -> 296); down to 192 keys
    // where workgroups are few (2 heads of 911 tokens 19 -> 12.5, 8 of 800 18 -> 14.5), 512 where the join's rows are many (8 key heads of 4 x
    // 1000 rows: 21 us whole, 29 in splits of 250).
    const int64_t have = heads * p.row_blocks, most = a.Nk / (p.waves == 1 ? 128 : have <= 64 ? 192 : 512);
    int64_t n = have > 0 ? (p.waves == 1 ? 2048 : a.D > 64 ? 512 : 1024) / have : 1;
    if (p.waves == 1 && n * 256 > a.Nk) n = 1024 / have;
    n = n > most ? most : n;
    n = n > 128 ? 128 : n < 1 ? 1 : n;
    p.splits = uint32_t(n);
    p.ws = n > 1 ? size_t(n) * size_t(heads) * size_t(R) * size_t(a.D + 1) * sizeof(float) : 0;
    return p;
}

template <typename T, int DP, bool CAP, bool BIAS> static void at_fwd_launch(const AtFwd &a, const AtFwdPlan &p, hipStream_t s)
{
    const dim3 grid(a.heads * a.row_blocks * a.splits);
    constexpr int kCap = CAP ? kAtCapped : kAtUncapped, kLong = CAP ? kAtCappedLong : kAtUncapped;
    if (p.waves == 1) hipLaunchKernelGGL((k_attn_fwd<T, DP, 1, 32, kCap, BIAS>), grid, dim3(64), 0, s, a);     // what it reads takes longer
    else if (a.s.Nk < kAtLong || a.s.cap2 > kAtLongCap * kLog2e) hipLaunchKernelGGL((k_attn_fwd<T, DP, 4, 64, kCap, BIAS>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_attn_fwd<T, DP, 4, 64, kLong, BIAS>), grid, dim3(256), 0, s, a);
}
template <typename T, int DP> static void at_fwd_forms(const AtFwd &a, const AtFwdPlan &p, bool cap, bool bias, hipStream_t s)
{
    if (cap && bias) at_fwd_launch<T, DP, true, true>(a, p, s);
    else if (cap) at_fwd_launch<T, DP, true, false>(a, p, s);
    else if (bias) at_fwd_launch<T, DP, false, true>(a, p, s);
    else at_fwd_launch<T, DP, false, false>(a, p, s);
}

// zero output where there are no keys
template <typename T> __global__ __launch_bounds__(kThreads) void k_attn_nothing(const AtFwd a, int64_t pieces)
{
    const AtShape &s = a.s;
    const int64_t id = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (id >= pieces) return;
    const int quads = s.D / 4;
    const int64_t at = id / quads, t = at / s.Hq, b = t / s.Nq;
    const int h = int(at - t * s.Hq), e = int(id - at * quads) * 4, i = int(t - b * s.Nq);
    at_store4<T>(a.o.p + b * a.o.batch + int64_t(i) * a.o.token + int64_t(h) * a.o.head + e * 2, 0.0f, 0.0f, 0.0f, 0.0f);
    if (e == 0) a.lse[(b * s.Hq + h) * s.Nq + i] = -__builtin_inff();
}

}  // namespace mesa

using namespace mesa;

extern "C" MESA_EXPORT mesa_status mesa_attention_bounds(int32_t *lo, int32_t *hi, int64_t B, int64_t Nq, int64_t Nk, int causal, int64_t window, const int32_t *kv_len,
                                                         const int32_t *q_start, const int32_t *prefix, const int32_t *doc, void *stream)
{
    const int64_t top = int64_t(1) << 30;
    if (B < 0 || Nq < 0 || Nk < 0 || window < 0) return MESA_ERR_INVALID_ARG;
    if (B == 0 || Nq == 0) return MESA_OK;
    if (!lo || !hi || lo == hi || !aligned4(lo) || !aligned4(hi) || !aligned4(kv_len) || !aligned4(q_start) || !aligned4(prefix) || !aligned4(doc)) return MESA_ERR_INVALID_ARG;
    if (Nq >= top || Nk >= top || B >= (int64_t(1) << 40) / Nq || B * ceil_div(Nq, kAtStretch) > most_workgroups(kThreads)) return MESA_ERR_UNSUPPORTED;
    const uint32_t per = uint32_t(ceil_div(Nq, kAtStretch));
    hipLaunchKernelGGL(doc ? k_attn_bounds<true> : k_attn_bounds<false>, dim3(uint32_t(B) * per), dim3(kThreads), 0, static_cast<hipStream_t>(stream), lo, hi, int(Nq), int(Nk),
                       causal, int(window < top ? window : top), kv_len, q_start, prefix, doc, uint32_t(B));
    return launch_status();
}

extern "C" MESA_EXPORT size_t mesa_attention_fwd_workspace_bytes(mesa_attention a, mesa_dtype dt)
{
    return at_supported(a, dt) == MESA_OK && a.B > 0 && a.Nq > 0 ? at_fwd_plan(a).ws : 0;
}

namespace mesa {
bool at_strides(const mesa_attention &a, int64_t tokens, int64_t heads, int64_t batch, int64_t token, int64_t head)
{
    const int64_t top = int64_t(1) << 30;
    if (((batch | token | head) & 7) || batch < 0 || token < 0 || head < 0) return false;
    return token <= top / 256 && head <= top / heads && 256 * token + heads * head + a.D < top && (tokens == 0 || batch < (int64_t(1) << 50));
}
}

extern "C" MESA_EXPORT mesa_status mesa_attention_fwd(mesa_attention a, mesa_attention_in q, mesa_attention_in k, mesa_attention_in v, mesa_attention_out o, float *lse,
                                                      mesa_attention_mask m, void *ws, size_t ws_bytes, mesa_dtype dt, void *stream)
{
    if (const mesa_status st = at_supported(a, dt)) return st;
    if (a.B == 0 || a.Nq == 0) return MESA_OK;
    if (!q.data || !o.data || !lse || (a.Nk && (!k.data || !v.data)) || q.alpha || k.alpha || v.alpha || (m.lo == nullptr) != (m.hi == nullptr)) return MESA_ERR_INVALID_ARG;
    if (!aligned16(q.data) || !aligned16(k.data) || !aligned16(v.data) || !aligned16(o.data) || !aligned4(lse) || !aligned4(m.lo) || !aligned4(m.hi) || !aligned4(m.slopes) ||
        !aligned4(m.q_start))
        return MESA_ERR_INVALID_ARG;
    const int64_t group = a.Hq / a.Hk;
    if (!at_strides(a, a.Nq, group, q.batch, q.token, q.head) || !at_strides(a, a.Nk, 1, k.batch, k.token, k.head) || !at_strides(a, a.Nk, 1, v.batch, v.token, v.head) ||
        !at_strides(a, a.Nq, group, o.batch, o.token, o.head))
        return MESA_ERR_INVALID_ARG;
    const AtFwdPlan p = at_fwd_plan(a);
    const int64_t groups = a.B * a.Hk, quads = groups * a.Nq * group * (a.D / 4);
    if (groups * p.row_blocks * p.splits > most_workgroups(256) || (p.splits > 1 && groups * a.Nq * group > most_workgroups(kThreads)) || ceil_div(quads, kThreads) > most_workgroups(kThreads)) return MESA_ERR_UNSUPPORTED;
    if (p.ws && (!ws || !aligned16(ws) || ws_bytes < p.ws)) return MESA_ERR_WORKSPACE;
    if (a.Nk && (o.data == q.data || o.data == k.data || o.data == v.data)) return MESA_ERR_INVALID_ARG;      // other workgroups read them yet
    hipStream_t s = static_cast<hipStream_t>(stream);
    AtFwd f;
    f.s = at_shape(a, m);
    auto view = [](const mesa_attention_in &x) { return AtView{static_cast<const char *>(x.data), x.batch * 2, x.token * 2, x.head * 2}; };
    f.q = view(q);
    f.k = view(k);
    f.v = view(v);
    f.o = AtOut{static_cast<char *>(o.data), o.batch * 2, o.token * 2, o.head * 2};
    f.lse = lse;
    f.heads = uint32_t(groups);
    f.row_blocks = p.row_blocks;
    f.splits = p.splits;
    f.part_o = p.splits > 1 ? static_cast<float *>(ws) : nullptr;
    f.part_lse = p.splits > 1 ? f.part_o + size_t(p.splits) * size_t(groups) * f.s.R * size_t(a.D) : nullptr;
    const bool half = dt == MESA_F16;
    const dim3 flat(uint32_t(ceil_div(quads, kThreads)));
    if (a.Nk == 0) {
        if (half) hipLaunchKernelGGL(k_attn_nothing<_Float16>, flat, dim3(kThreads), 0, s, f, quads);
        else hipLaunchKernelGGL(k_attn_nothing<__bf16>, flat, dim3(kThreads), 0, s, f, quads);
        return launch_status();
    }
    const bool cap = a.cap > 0.0f, bias = m.slopes != nullptr;
    if (half) a.D <= 64 ? at_fwd_forms<_Float16, 64>(f, p, cap, bias, s) : at_fwd_forms<_Float16, 128>(f, p, cap, bias, s);
    else a.D <= 64 ? at_fwd_forms<__bf16, 64>(f, p, cap, bias, s) : at_fwd_forms<__bf16, 128>(f, p, cap, bias, s);
    if (const mesa_status st = launch_status()) return st;
    if (p.splits > 1) {
        const int64_t rows = groups * f.s.R;
        const bool few = p.splits > 8 && rows <= 4096;
        const dim3 grid(uint32_t(few ? rows : ceil_div(rows, a.D > 64 ? 8 : 16)));
        auto *join = half ? (few ? k_attn_join<_Float16, true> : k_attn_join<_Float16, false>) : (few ? k_attn_join<__bf16, true> : k_attn_join<__bf16, false>);
        hipLaunchKernelGGL(join, grid, dim3(kThreads), 0, s, f);
        return launch_status();
    }
    return MESA_OK;
}
