// Attention over a sequence, backward, from the forward's log-sum-exp: the weights are formed again per tile, nothing of their size reaches memory.
//
//   rows      delta_i = <dout_i, out_i>, lse in base 2; fp16: the power of two of a tile's largest |dout|
//   queries   S^T = K Q^T, dP^T = V dO^T, dS = P (dP - delta) (1 - tanh^2), dQ^T += K^T dS       a wave keeps 16 QB queries, walks the keys
//   keys      S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS                             a wave keeps 16 KB keys, walks the queries of
//                                                                                               every head that shares them
// Seven products instead of the five that a single kernel would take, and every sum in one wave's registers in a fixed order: no atomics.
//
// fp16 holds 2^-24 to 65504.  The weights enter dV's product times 2^8, and dS on the scale of the largest |dout| of its query (queries) or of the
// heads that share the key (keys), so gradients far below 1 keep their digits; the powers of two come off the sums again.
#include <algorithm>

#include "lds_attr.hpp"
#include "seq_common.hpp"

namespace seq {

namespace {

template <typename T> constexpr bool kScaled = __is_same(T, f16_t);
template <typename T> constexpr float kRaise = kScaled<T> ? 8.f : 0.f;   // weights are formed times 2^kRaise
constexpr int kNothing = -1000;   // power of two of a tile of zeros

__device__ __forceinline__ int power_of(float most) { return most > 0.f ? min(16, __builtin_amdgcn_frexp_expf(most)) : kNothing; }   // (infinite: 16)
__device__ __forceinline__ float two_to(int e) { return __builtin_amdgcn_ldexpf(1.f, e); }

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void rows_kernel(const Args p) {
    using L = Tile<T, D>;
    constexpr int E = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    __shared__ float most_of[kWaves];
    const int tid = threadIdx.x, plane = blockIdx.x / p.query_tiles, tile = blockIdx.x % p.query_tiles, b = plane / p.heads, h = plane % p.heads;
    const char *o = p.out.at + b * p.out.b + h * p.out.h, *d = p.dout.at + b * p.dout.b + h * p.dout.h;
    const int c = tid % L::CH;
    float most = 0.f;
#pragma unroll
    for (int r = tid / L::CH; r < kTile; r += kThreads / L::CH) {
        const int i = tile * kTile + r, at = min(i, p.Lq - 1);
        const float lse = p.lse[(int64_t)plane * p.Lq + at];
        const bool live = i < p.Lq && lse != -INFINITY;
        const char *xp = o + (int64_t)at * p.out.row + c * 16;
        const vec x = *reinterpret_cast<const vec *>(xp), rest = p.rest ? *reinterpret_cast<const vec *>(xp + (p.rest - p.out.at)) : vec{}, y = *reinterpret_cast<const vec *>(d + (int64_t)at * p.dout.row + c * 16);
        float delta = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            delta = __builtin_fmaf((float)x[e] + (float)rest[e], (float)y[e], delta);
            if (kScaled<T> && live) most = fmaxf(most, fabsf((float)y[e]));
        }
#pragma unroll
        for (int n = 1; n < L::CH; n *= 2) delta += __shfl_xor(delta, n);
        // a query that saw nothing, or that is not there, has no weights: 2^(score - inf) is 0 whatever the score
        if (c == 0) p.rows[((int64_t)plane * p.query_tiles + tile) * kTile + r] = live ? float2{lse * kLog2e - kRaise<T>, delta} : float2{INFINITY, 0.f};
    }
    if constexpr (kScaled<T>) {
#pragma unroll
        for (int n = 1; n < kWave; n *= 2) most = fmaxf(most, __shfl_xor(most, n));
        if (tid % kWave == 0) most_of[tid / kWave] = most;
        workgroup_sync();
        if (tid == 0) p.powers[blockIdx.x] = power_of(fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3])));
    }
}

// ---- dQ --------------------------------------------------------------------------------------------------------------------

template <typename T> constexpr int kBlocks = sizeof(T) == 2 ? 2 : 1;   // blocks of 16 queries, or keys, that a wave keeps

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void bwd_q_kernel(const Args p) {
    using L = Tile<T, D>;
    constexpr int QB = kBlocks<T>, RB = kRowBlocks<T>, NB = kTile / 16;
    extern __shared__ __align__(16) char lds[];
    __shared__ int ids[2][kTile];
    __shared__ int range[2][kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), j = lane & 15, g = lane >> 4;
    const int tiles = (p.Lq + 16 * QB * kWaves - 1) / (16 * QB * kWaves);
    int id = block_in_order();
    const int in_group = id % p.group;
    id /= p.group;
    const int tile = tiles - 1 - id % tiles, plane = id / tiles, b = plane / p.kv, kh = plane % p.kv, h = kh * p.group + in_group;
    const char *kp = p.k.at + b * p.k.b + kh * p.k.h, *vp = p.v.at + b * p.v.b + kh * p.v.h;
    const char *qp = p.q.at + b * p.q.b + h * p.q.h, *dp = p.dout.at + b * p.dout.b + h * p.dout.h;
    const float2 *stats = p.rows + ((int64_t)b * p.heads + h) * p.query_tiles * kTile;
    const int q0 = tile * 16 * QB * kWaves, qw = q0 + wave * 16 * QB;
    const int img = lds_addr(lds);

    u32x4 q[QB][L::STEPS], d[QB][L::STEPS];
    int pos[QB], mine[QB], power[QB];
    float lse[QB], delta[QB];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        const int i = min(qw + 16 * n + j, p.Lq - 1);
        L::load_row(q[n], qp, p.q.row, i, lane);
        L::load_row(d[n], dp, p.dout.row, i, lane);
        const float2 st = stats[i];
        pos[n] = i + p.off;
        mine[n] = p.documents ? p.documents[(int64_t)b * p.Lk + pos[n]] : 0;
        lse[n] = st.x, delta[n] = st.y, power[n] = 0;
        if constexpr (kScaled<T>) {
            typedef T vec __attribute__((ext_vector_type(8)));
            float most = 0.f;
#pragma unroll
            for (int s = 0; s < L::STEPS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)__builtin_bit_cast(vec, d[n][s])[e]));
            power[n] = power_of(column_max(most));
            if (power[n] == kNothing) power[n] = 0;
            lse[n] += kRaise<T> + (float)power[n];
        }
    }
    Docs dw = no_docs(), dg = no_docs();
    if (p.documents) {
        const int i = qw + lane % (16 * QB);
        dw = docs_of_wave(p.documents[(int64_t)b * p.Lk + min(i, p.Lq - 1) + p.off], true);
        if (lane == 0) range[0][wave] = dw.lo, range[1][wave] = dw.hi;
        workgroup_sync();
        dg = {range[0][0], range[1][0], false};
#pragma unroll
        for (int w = 1; w < kWaves; ++w) dg.lo = min(dg.lo, range[0][w]), dg.hi = max(dg.hi, range[1][w]);
        dg.lo = uniform(dg.lo), dg.hi = uniform(dg.hi);
    }
    const int qa = min(q0, p.Lq - 1) + p.off, qb = min(q0 + 16 * QB * kWaves, p.Lq) - 1 + p.off;
    const int wa = min(qw, p.Lq - 1) + p.off, wb = min(qw + 16 * QB, p.Lq) - 1 + p.off;
    const Marks *marks = p.marks ? p.marks + (int64_t)b * p.key_tiles : nullptr;
    auto of = [&](int t) {
        const int ka = t * kTile, kb = min(ka + kTile, p.Lk) - 1;
        bool any = near_any(p, qa, qb, ka, kb), some = near_any(p, wa, wb, ka, kb), all = near_all(p, wa, wb, ka, kb) && ka + kTile <= p.Lk;
        if (marks) {
            const Marks m = marks[t];
            const Docs dk{m.dmin, m.dmax, m.live == ~0ull};
            any |= m.prefix != 0, some |= m.prefix != 0, all |= m.prefix == ~0ull;
            if (p.documents) any &= dk.meet(dg), some &= dk.meet(dw), all &= dk.same(dw);
        }
        return (any ? 1 : 0) | (some ? 2 : 0) | (all ? 4 : 0);
    };
    int first = 0, last = p.key_tiles - 1;
    if (!p.prefix) {
        first = max(0, qa - p.window + 1) / kTile;
        last = min(last, max(-1, qb - p.dlo) >> 6);
    }
    Walk walk(first, last);

    const typename L::RowReader rows(lane);
    const typename L::ColumnReader columns(lane);
    const float slope = p.slopes ? p.slopes[h] * kLog2e : 0.f;
    f32x4 dq[QB][L::DB];
#pragma unroll
    for (int n = 0; n < QB; ++n)
#pragma unroll
        for (int db = 0; db < L::DB; ++db) dq[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto stage = [&](int t, int buf) {
        const int to = img + buf * 2 * L::BYTES;
        const char *zeros = p.documents ? p.zeros : nullptr;
        const uint64_t live = zeros ? marks[t].live : 0;
        L::stage(kp, p.k.row, t * kTile, p.Lk, live, zeros, to, wave, lane);
        L::stage(vp, p.v.row, t * kTile, p.Lk, live, zeros, to + L::BYTES, wave, lane);
        if (zeros && wave == 0) global_to_lds_4(reinterpret_cast<const char *>(p.documents + (int64_t)b * p.Lk), (unsigned)min(t * kTile + lane, p.Lk - 1) * 4, lds_addr(ids[buf]));
    };

    bool some, all, some_next, all_next;
    int t = walk.next(of, lane, some, all), buf = 0;
    if (t >= 0) stage(t, 0);
#pragma unroll 1
    while (t >= 0) {
        const int after = walk.next(of, lane, some_next, all_next);
        wait_global_loads();
        workgroup_sync();
        if (after >= 0) stage(after, buf ^ 1);
        if (some) {
            const int ki = img + buf * 2 * L::BYTES, vi = ki + L::BYTES, k0 = t * kTile;
            const uint64_t prefix = p.prefix && !all ? marks[t].prefix : 0;
#pragma unroll 1
            for (int i = 0; i < NB / RB; ++i) {
                f32x4 s[QB][RB], e[QB][RB];
#pragma unroll
                for (int n = 0; n < QB; ++n)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) s[n][rb] = e[n][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
                const int at0 = i * RB * 16 * L::ROWB;
#pragma unroll
                for (int st = 0; st < L::STEPS; ++st)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const u32x4 a = rows.read(ki + at0, rb, st), c = rows.read(vi + at0, rb, st);
#pragma unroll
                        for (int n = 0; n < QB; ++n) s[n][rb] = mma<T>(a, q[n][st], s[n][rb]), e[n][rb] = mma<T>(c, d[n][st], e[n][rb]);
                    }
                u32x4 w[QB];
#pragma unroll
                for (int n = 0; n < QB; ++n) {
                    const float from = (float)(pos[n] - k0 - 4 * g);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int at = (i * RB + rb) * 16 + 4 * g + r;
                            float by = 0.f, x = score<T, CAP>(p, s[n][rb][r], by);
                            if (p.slopes) x = __builtin_fmaf(fabsf(from - (float)((i * RB + rb) * 16 + r)), -slope, x);
                            if (!all) {
                                const int key = k0 + at, doc = p.documents ? ids[buf][at] : 0;
                                if (!(key < p.Lk && doc >= 0 && doc == mine[n] && ((prefix >> at & 1) || near_one(p, pos[n] - key)))) x = -INFINITY;
                            }
                            const float weight = __builtin_amdgcn_exp2f(x - lse[n]);
                            float ds = through_cap<T, CAP>(weight * (e[n][rb][r] - delta[n]), by);
                            if (!all) ds = weight == 0.f ? 0.f : ds;   // what is masked may meet values that are not finite
                            s[n][rb][r] = ds;
                        }
                    w[n] = pack<T>(s[n]);
                }
#pragma unroll
                for (int db = 0; db < L::DB; ++db) {
                    const u32x4 a = columns.read(ki, i, db);
#pragma unroll
                    for (int n = 0; n < QB; ++n) dq[n][db] = mma<T>(a, w[n], dq[n][db]);
                }
            }
        }
        t = after, some = some_next, all = all_next, buf ^= 1;
    }
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        settle_products(dq[n]);
        const int i = qw + 16 * n + j;
        if (i < p.Lq) L::store_row(dq[n], p.scale * two_to(power[n]), const_cast<char *>(p.dq.at) + b * p.dq.b + h * p.dq.h, p.dq.row, i, lane);
    }
}

// ---- dK, dV ----------------------------------------------------------------------------------------------------------------
//
// kPair: with 128 channels in 16 bit a wave that kept both sums of 32 keys would take more than 256 registers, and run alone on its SIMD.  Two waves share
// 32 keys instead: each forms P and dS of half of a tile's queries, the first sums dV, the second dK, and each gives the other, through LDS, the half
// that it does not sum itself.
//
// The work of a workgroup, the tiles of every head that shares its keys, is split into p.splits parts of equal length where there are few workgroups; each
// then leaves fp32 sums, which a last kernel adds in order.

template <typename T, int D> constexpr bool kPair = sizeof(T) == 2 && D == 128;
template <typename T, int D> constexpr int kKeys = 16 * kBlocks<T> * kWaves / (kPair<T, D> ? 2 : 1);   // of a workgroup

template <typename T, int D, bool CAP>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void bwd_kv_kernel(const Args p) {
    using L = Tile<T, D>;
    constexpr int KB = kBlocks<T>, RB = kRowBlocks<T>, NB = kTile / 16;
    constexpr bool PAIR = kPair<T, D>;
    extern __shared__ __align__(16) char lds[];
    __shared__ int ids[2][kTile];
    __shared__ __align__(16) float2 stats[2][kTile];
    __shared__ int range[4][kWaves];
    __shared__ __align__(16) u32x4 given[PAIR ? kWaves : 1][KB][PAIR ? kWave : 1];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), j = lane & 15, g = lane >> 4;
    const int role = PAIR ? wave & 1 : 0, group_of_keys = PAIR ? wave >> 1 : wave;
    const int tiles = (p.Lk + kKeys<T, D> - 1) / kKeys<T, D>;
    int id = block_in_order();
    const int split = id % p.splits;
    id /= p.splits;
    const int tile = id % tiles, plane = id / tiles, b = plane / p.kv, kh = plane % p.kv;
    const char *kp = p.k.at + b * p.k.b + kh * p.k.h, *vp = p.v.at + b * p.v.b + kh * p.v.h;
    const int k0 = tile * kKeys<T, D>, kw = k0 + group_of_keys * 16 * KB;
    const int img = lds_addr(lds);
    const int *documents = p.documents ? p.documents + (int64_t)b * p.Lk : nullptr;
    const Marks *marks = p.marks ? p.marks + (int64_t)b * p.key_tiles : nullptr;

    u32x4 k[KB][L::STEPS], v[KB][L::STEPS];
    int key[KB], mine[KB];
    bool always[KB];
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        const int i = min(kw + 16 * n + j, p.Lk - 1);
        L::load_row(k[n], kp, p.k.row, i, lane);
        L::load_row(v[n], vp, p.v.row, i, lane);
        key[n] = i;
        mine[n] = documents ? documents[i] : 0;
        always[n] = p.prefix && (marks[i / kTile].prefix >> (i % kTile) & 1);
    }
    Docs dw = no_docs(), dg = no_docs();
    bool prefix_any = false, prefix_some = false, prefix_all = false;
    int power = 0;
    if (marks || kScaled<T>) {
        const int i = min(kw + lane % (16 * KB), p.Lk - 1);
        if (documents) dw = docs_of_wave(documents[i], true);
        if (p.prefix) {
            const uint64_t x = __ballot(marks[i / kTile].prefix >> (i % kTile) & 1);
            prefix_some = x != 0, prefix_all = x == ~0ull;
        }
        int most = kNothing;
        if constexpr (kScaled<T>) {   // over the tiles of every head that shares these keys
            const int *of = p.powers + ((int64_t)b * p.heads + kh * p.group) * p.query_tiles;
            for (int n = tid; n < p.group * p.query_tiles; n += kThreads) most = max(most, of[n]);
            most = wave_max(most);
        }
        if (lane == 0) range[0][wave] = dw.lo, range[1][wave] = dw.hi, range[2][wave] = prefix_some, range[3][wave] = most;
        workgroup_sync();
        dg = {range[0][0], range[1][0], false};
        most = range[3][0];
        prefix_any = range[2][0] | range[2][1] | range[2][2] | range[2][3];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) dg.lo = min(dg.lo, range[0][w]), dg.hi = max(dg.hi, range[1][w]), most = max(most, range[3][w]);
        dg.lo = uniform(dg.lo), dg.hi = uniform(dg.hi);
        if (kScaled<T> && most != kNothing) power = uniform(most);
    }
    const int ka = k0, kb = min(k0 + kKeys<T, D>, p.Lk) - 1;
    const int wa = min(kw, p.Lk - 1), wb = min(kw + 16 * KB, p.Lk) - 1;
    auto of = [&](int t) {
        const int qa = t * kTile + p.off, qb = min(t * kTile + kTile, p.Lq) - 1 + p.off;
        bool any = near_any(p, qa, qb, ka, kb) || prefix_any, some = near_any(p, qa, qb, wa, wb) || prefix_some, all = near_all(p, qa, qb, wa, wb) || prefix_all;
        if (documents) {
            const Marks x = marks[qa / kTile], y = marks[min((qa + kTile - 1) / kTile, p.key_tiles - 1)];
            const Docs d{min(x.dmin, y.dmin), max(x.dmax, y.dmax), (x.live & y.live) == ~0ull};
            any &= d.meet(dg), some &= d.meet(dw), all &= d.same(dw);
        }
        return (any ? 1 : 0) | (some ? 2 : 0) | (all ? 4 : 0);
    };
    int first = 0, last = p.query_tiles - 1;
    if (!prefix_any) {
        first = max(0, ka + p.dlo - p.off) / kTile;
        last = min(last, max(-1, kb + p.window - 1 - p.off) >> 6);
    }
    const typename L::RowReader rows(lane);
    const typename L::ColumnReader columns(lane);
    f32x4 dk[KB][L::DB], dv[KB][L::DB];   // (of a pair, each wave uses dv alone: for dV the first, for dK the second)
#pragma unroll
    for (int n = 0; n < KB; ++n)
#pragma unroll
        for (int db = 0; db < L::DB; ++db) dk[n][db] = dv[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto stage = [&](int h, int t, int buf) {
        const int to = img + buf * 2 * L::BYTES;
        const char *zeros = documents ? p.zeros : nullptr;
        uint64_t live = 0;
        if (zeros) {   // of the tile's queries: their positions begin inside a tile of keys
            const int at = t * kTile + p.off, in = at % kTile;
            live = marks[at / kTile].live >> in;
            if (in) live |= marks[min(at / kTile + 1, p.key_tiles - 1)].live << (kTile - in);
        }
        L::stage(p.q.at + b * p.q.b + h * p.q.h, p.q.row, t * kTile, p.Lq, live, zeros, to, wave, lane);
        L::stage(p.dout.at + b * p.dout.b + h * p.dout.h, p.dout.row, t * kTile, p.Lq, live, zeros, to + L::BYTES, wave, lane);
        if (wave < 2) global_to_lds_4(reinterpret_cast<const char *>(p.rows + (((int64_t)b * p.heads + h) * p.query_tiles + t) * kTile), (unsigned)(wave * kWave + lane) * 4,
                                      lds_addr(stats[buf]) + wave * kWave * 4);
        if (zeros && wave == 2) global_to_lds_4(reinterpret_cast<const char *>(documents), (unsigned)min(t * kTile + lane + p.off, p.Lk - 1) * 4, lds_addr(ids[buf]));
    };

    // the heads that share these keys in turn, each one's tiles in turn: from the split's first to its last
    const int count = max(0, last - first + 1), all_tiles = p.group * count, each = (all_tiles + p.splits - 1) / p.splits;
    const int lo = min(split * each, all_tiles), hi = min(lo + each, all_tiles);
    const int head_lo = lo < hi ? lo / count : 0, head_hi = lo < hi ? (hi - 1) / count : -1;
    const int tile_lo = lo < hi ? first + lo % count : 0, tile_hi = lo < hi ? first + (hi - 1) % count : -1;
    int head = head_lo;
    Walk walk(tile_lo, head == head_hi ? tile_hi : last);
    bool some, all, some_next = false, all_next = false;
    auto next = [&](bool &s, bool &a) {
        while (true) {
            const int t = head <= head_hi ? walk.next(of, lane, s, a) : -1;
            if (t >= 0 || head >= head_hi) return t;
            ++head;
            walk = Walk(first, head == head_hi ? tile_hi : last);
        }
    };
    int t = next(some, all), buf = 0, h = kh * p.group + head;
    if (t >= 0) stage(h, t, 0);
#pragma unroll 1
    while (t >= 0) {
        const int after = next(some_next, all_next);
        wait_global_loads();
        workgroup_sync();
        if (after >= 0) stage(kh * p.group + head, after, buf ^ 1);
        const int qi = img + buf * 2 * L::BYTES, di = qi + L::BYTES, q0 = t * kTile + p.off;
        const float slope = p.slopes ? p.slopes[h] * kLog2e : 0.f, lower = two_to(-power - (int)kRaise<T>);
        // P and dS of 16 RB queries from 16 RB i on, as chunks
        auto weigh = [&](int i, u32x4 (&w)[KB], u32x4 (&x)[KB]) {
            f32x4 s[KB][RB], e[KB][RB];
#pragma unroll
            for (int n = 0; n < KB; ++n)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) s[n][rb] = e[n][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int at0 = i * RB * 16 * L::ROWB;
#pragma unroll
            for (int st = 0; st < L::STEPS; ++st)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const u32x4 a = rows.read(qi + at0, rb, st), c = rows.read(di + at0, rb, st);
#pragma unroll
                    for (int n = 0; n < KB; ++n) s[n][rb] = mma<T>(a, k[n][st], s[n][rb]), e[n][rb] = mma<T>(c, v[n][st], e[n][rb]);
                }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int at = (i * RB + rb) * 16 + 4 * g;   // of this lane's four queries
                f32x4 two[2];
                two[0] = *reinterpret_cast<const f32x4 *>(&stats[buf][at]), two[1] = *reinterpret_cast<const f32x4 *>(&stats[buf][at + 2]);
#pragma unroll
                for (int n = 0; n < KB; ++n) {
                    const float from = (float)(q0 + at - key[n]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float lse = two[r / 2][r % 2 * 2], delta = two[r / 2][r % 2 * 2 + 1];
                        float by = 0.f, y = score<T, CAP>(p, s[n][rb][r], by);
                        if (p.slopes) y = __builtin_fmaf(fabsf(from + (float)r), -slope, y);
                        if (!all) {
                            const int doc = documents ? ids[buf][at + r] : 0;
                            if (!(doc >= 0 && doc == mine[n] && (always[n] || near_one(p, q0 + at + r - key[n])))) y = -INFINITY;
                        }
                        const float weight = __builtin_amdgcn_exp2f(y - lse);
                        float ds = e[n][rb][r] - delta;
                        if constexpr (kScaled<T>) ds *= lower;
                        ds = through_cap<T, CAP>(weight * ds, by);
                        if (!all) ds = weight == 0.f ? 0.f : ds;
                        s[n][rb][r] = weight, e[n][rb][r] = ds;
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < KB; ++n) w[n] = pack<T>(s[n]), x[n] = pack<T>(e[n]);
        };
        if constexpr (PAIR) {
            static_assert(!PAIR || NB / RB == 2, "a half for each");
            u32x4 w[KB], x[KB];
            if (some) {
                weigh(role, w, x);
#pragma unroll
                for (int n = 0; n < KB; ++n) given[wave][n][lane] = role ? w[n] : x[n];
            }
            workgroup_sync();
            if (some) {
                u32x4 halves[2][KB];
#pragma unroll
                for (int n = 0; n < KB; ++n) {
                    const u32x4 own = role ? x[n] : w[n], other = given[wave ^ 1][n][lane];
                    halves[0][n] = role ? other : own, halves[1][n] = role ? own : other;
                }
                const int from = role ? qi : di;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int db = 0; db < L::DB; ++db) {
                        const u32x4 a = columns.read(from, i, db);
#pragma unroll
                        for (int n = 0; n < KB; ++n) dv[n][db] = mma<T>(a, halves[i][n], dv[n][db]);
                    }
            }
        } else if (some) {
#pragma unroll 1
            for (int i = 0; i < NB / RB; ++i) {
                u32x4 w[KB], x[KB];
                weigh(i, w, x);
#pragma unroll
                for (int db = 0; db < L::DB; ++db) {
                    const u32x4 a = columns.read(di, i, db), c = columns.read(qi, i, db);
#pragma unroll
                    for (int n = 0; n < KB; ++n) dv[n][db] = mma<T>(a, w[n], dv[n][db]), dk[n][db] = mma<T>(c, x[n], dk[n][db]);
                }
            }
        }
        t = after, h = kh * p.group + head, some = some_next, all = all_next, buf ^= 1;
    }
    // which: 0 dK, 1 dV
    auto store = [&](int which, const f32x4 *acc, float by, int i) {
        const View &to = which ? p.dv : p.dk;
        if (p.splits == 1) L::store_row(acc, by, const_cast<char *>(to.at) + b * to.b + kh * to.h, to.row, i, lane);
        else Tile<float, D>::store_row(acc, by, reinterpret_cast<char *>(p.parts + (((int64_t)split * 2 + which) * p.B * p.kv + plane) * p.Lk * D), D * 4, i, lane);
    };
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        settle_products(dk[n]);
        settle_products(dv[n]);
        const int i = kw + 16 * n + j;
        if (i < p.Lk) {
            const float by_k = p.scale * two_to(power), by_v = two_to(-(int)kRaise<T>);
            if constexpr (PAIR) {
                store(role ? 0 : 1, dv[n], role ? by_k : by_v, i);
            } else {
                store(0, dk[n], by_k, i);
                store(1, dv[n], by_v, i);
            }
        }
    }
}

// dK and dV: the splits' sums, in order; a thread per four channels.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void join_kv_kernel(const Args p, int64_t total) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= total) return;
    const int d = (int)(i % (D / 4)) * 4;
    const int64_t row = i / (D / 4), each = (int64_t)p.B * p.kv * p.Lk;   // of dK, then of dV
    f32x4 x{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < p.splits; ++s) x += *reinterpret_cast<const f32x4 *>(p.parts + ((int64_t)s * 2 * each + row) * D + d);
    const bool values = row >= each;
    const int64_t at = values ? row - each : row;
    const View &to = values ? p.dv : p.dk;
    const int plane = (int)(at / p.Lk);
    char *out = const_cast<char *>(to.at) + plane / p.kv * to.b + plane % p.kv * to.h + at % p.Lk * to.row + d * (int)sizeof(T);
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4 *>(out) = x;
    } else {
        typedef T t4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<t4 *>(out) = __builtin_convertvector(x, t4);
    }
}

template <typename T, int D, bool CAP> struct Rows {
    static hipError_t go(const Args &a, hipStream_t st) {
        const int64_t blocks = (int64_t)a.B * a.heads * a.query_tiles;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        rows_kernel<T, D><<<(unsigned)blocks, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
};
template <typename T, int D, bool CAP> struct BwdQ {
    static hipError_t go(const Args &a, hipStream_t st) {
        constexpr int lds = 4 * Tile<T, D>::BYTES, rows = 16 * kBlocks<T> * kWaves;
        static LdsAllowed allowed;
        if (hipError_t e = allow_lds(bwd_q_kernel<T, D, CAP>, lds, allowed); e != hipSuccess) return e;
        const int64_t blocks = (int64_t)a.B * a.heads * ((a.Lq + rows - 1) / rows);
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        bwd_q_kernel<T, D, CAP><<<(unsigned)blocks, kThreads, lds, st>>>(a);
        return hipGetLastError();
    }
};
template <typename T, int D, bool CAP> struct BwdKV {
    static hipError_t go(const Args &a, hipStream_t st) {
        constexpr int lds = 4 * Tile<T, D>::BYTES;
        static LdsAllowed allowed;
        if (hipError_t e = allow_lds(bwd_kv_kernel<T, D, CAP>, lds, allowed); e != hipSuccess) return e;
        const int64_t blocks = (int64_t)a.B * a.kv * ((a.Lk + kKeys<T, D> - 1) / kKeys<T, D>) * a.splits;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        bwd_kv_kernel<T, D, CAP><<<(unsigned)blocks, kThreads, lds, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
        const int64_t total = (int64_t)a.B * a.kv * a.Lk * 2 * (D / 4), joins = (total + kThreads - 1) / kThreads;
        if (!launch_holds(joins, kThreads)) return hipErrorInvalidValue;
        join_kv_kernel<T, D><<<(unsigned)joins, kThreads, 0, st>>>(a, total);
        return hipGetLastError();
    }
};
template <typename T, int D, bool CAP> struct Keys {
    static hipError_t go(int &keys) { return keys = kKeys<T, D>, hipSuccess; }
};

}  // namespace

hipError_t launch_rows(const Args &a, int dtype, int D, hipStream_t st) { return dispatch<Rows>(dtype, D, false, a, st); }
hipError_t launch_bwd_q(const Args &a, int dtype, int D, bool capped, hipStream_t st) { return dispatch<BwdQ>(dtype, D, capped, a, st); }
hipError_t launch_bwd_kv(const Args &a, int dtype, int D, bool capped, hipStream_t st) { return dispatch<BwdKV>(dtype, D, capped, a, st); }


// How many parts the work on one tile of keys is split into: until there are about kWanted workgroups, but each part is left four tiles of queries, and the parts' sums
// stay below 256 MB.
int kv_splits(const Args &a, int dtype, int D) {
    int keys = 64;
    (void)dispatch<Keys>(dtype, D, false, keys);
    constexpr int64_t kWanted = 1024;
    const int64_t units = (int64_t)a.B * a.kv * ((a.Lk + keys - 1) / keys), sums = (int64_t)a.B * a.kv * a.Lk * D * 8;
    const int64_t reach = std::min<int64_t>(a.query_tiles, ((int64_t)a.window + keys) / kTile + 2);   // tiles of one head that a tile of keys can meet
    const int64_t s = std::min({(kWanted + units - 1) / units, (int64_t)a.group * reach / 4, ((int64_t)256 << 20) / sums, (int64_t)16});
    return (int)std::max<int64_t>(1, s);
}

}  // namespace seq
