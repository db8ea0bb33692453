// Attention over a sequence, backward, from the forward's log-sum-exp: the weights are formed again per tile, nothing of their size reaches memory.
//
//   rows      delta_i = <dout_i, out_i>, lse in base 2; fp16: the powers of two of a tile's largest |dout|, and of its keys' largest sum |v|
//   queries   S^T = K Q^T, dP^T = V dO^T, dS = P (dP - delta) (1 - tanh^2), dQ^T += K^T dS       a wave keeps 16 QB queries, walks the keys
//   keys      S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS                             a wave keeps 16 KB keys, walks the queries of
//                                                                                               every head that shares them
// Seven products instead of the five that a single kernel would take, and every sum in one wave's registers in a fixed order: no atomics.
// bf16, D 128: 2 x 16 over 4 x 8192, not causal, 4.0 ms or 0.69 PFLOP/s of the five products (0.96 of the seven); 4 x 16 over 4 x 2048, causal, capped, 16 + 153 + 236 us and
// 15 for the key side's join, under the profiler's lower clock (vector instructions 49 and 43 % of the cycles, matrix ones 30 and 26 %, waves wait 30 and 37 %: neither unit is full).  The
// rows are read at the rate of memory: 100 MB in 16 us.  fp32, D 32, 2 x 4 x 3136, causal, slopes: 5 + 95 + 5 + 123 + 6 us, matrix instructions 51 to 54 % of the cycles, vector ones 25 to 28 %.
//
// fp16 holds 2^-24 to 65504.  The weights enter dV's product times 2^10, and dS on a scale that the largest |dout| of its query (queries) or of the heads that share
// the key (keys) and the largest sum |v| of the keys make: as high as it can be without passing 65504 (raise_of()), so gradients far below 1, weights of 2^-20 of a
// million keys and values of thousands keep their digits; the powers of two come off the sums again.
#include "seq_bwd.hpp"

namespace seq {

namespace {

template <typename T, int D, int CAP>
__global__ __launch_bounds__(kThreads) void rows_kernel(const Args p) {
    using L = Tile<T, D>;
    constexpr int E = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    __shared__ float most_of[kWaves];
    const int tid = threadIdx.x, c = tid % L::CH;
    float most = 0.f;
    auto power = [&](int highest) {   // of the workgroup's largest
#pragma unroll
        for (int n = 1; n < kWave; n *= 2) most = fmaxf(most, __shfl_xor(most, n));
        if (tid % kWave == 0) most_of[tid / kWave] = most;
        workgroup_sync();
        return power_of(fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3])), highest);
    };
    if constexpr (kScaled<T>) {
        const int of_queries = p.B * p.heads * p.query_tiles;
        for (int unit = (int)blockIdx.x - of_queries; unit >= 0 && unit < p.B * p.kv * p.key_tiles; unit += gridDim.x - of_queries) {   // tiles of keys
            most = 0.f;
            const int plane = unit / p.key_tiles, tile = unit % p.key_tiles, b = plane / p.kv;
            const char *v = p.v.at + b * p.v.b + plane % p.kv * p.v.h;
#pragma unroll
            for (int r = tid / L::CH; r < kTile; r += kThreads / L::CH) {
                const int i = tile * kTile + r, at = min(i, p.Lk - 1);
                const vec x = *reinterpret_cast<const vec *>(v + (int64_t)at * p.v.row + c * 16);
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) sum += fabsf((float)x[e]);
#pragma unroll
                for (int n = 1; n < L::CH; n *= 2) sum += __shfl_xor(sum, n);
                if (!p.documents || p.documents[(int64_t)b * p.Lk + at] >= 0) most = fmaxf(most, sum);
            }
            const int e = power(kMostValues);
            if (tid == 0) p.value_powers[unit] = e;
            workgroup_sync();   // (before the maxima are written again)
        }
        if ((int)blockIdx.x >= of_queries) return;
    }
    const int plane = blockIdx.x / p.query_tiles, tile = blockIdx.x % p.query_tiles, b = plane / p.heads, h = plane % p.heads;
    const char *o = p.out.at + b * p.out.b + h * p.out.h, *d = p.dout.at + b * p.dout.b + h * p.dout.h;
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
        if (c == 0) p.rows[((int64_t)plane * p.query_tiles + tile) * kTile + r] = live ? float2{p.from - lse * kLog2e + kRaise<T> + Score<T, CAP>::kQuad, delta} : float2{-INFINITY, 0.f};
    }
    if constexpr (kScaled<T>) {
        const int e = power(kMostDout);
        if (tid == 0) p.powers[blockIdx.x] = e;
    }
}

// ---- dQ --------------------------------------------------------------------------------------------------------------------

template <typename T, int D, int CAP, bool SLOPES, int QB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void bwd_q_kernel(const Args p) {
    using L = Tile<T, D>;
    constexpr int RB = kRowBlocks<T>, NB = kTile / 16;
    extern __shared__ __align__(16) char lds[];
    __shared__ __align__(16) int ids[2][kTile];
    __shared__ int range[2][kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), j = lane & 15, g = lane >> 4;
    const int tiles = (p.Lq + 16 * QB * kWaves - 1) / (16 * QB * kWaves);
    int id = block_in_order();
    const int split = id % p.q_splits;
    id /= p.q_splits;
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
    float lse[QB], delta[QB];   // (lse: what the score is added to in the weight's exponent)
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        const int i = min(qw + 16 * n + j, p.Lq - 1);
        L::load_row(q[n], qp, p.q.row, i, lane);
        L::load_row(d[n], dp, p.dout.row, i, lane);
        const float2 st = stats[i];
        pos[n] = i + p.off;
        mine[n] = p.documents ? p.documents[(int64_t)b * p.Lk + pos[n]] : 0;
        lse[n] = st.x, delta[n] = st.y, power[n] = 0;
        if (p.documents) L::clear(q[n], mine[n] >= 0), L::clear(d[n], mine[n] >= 0);
        if constexpr (kScaled<T>) {
            typedef T vec __attribute__((ext_vector_type(8)));
            float most = 0.f;
#pragma unroll
            for (int s = 0; s < L::STEPS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)__builtin_bit_cast(vec, d[n][s])[e]));
            power[n] = power_of(column_max(most), kMostDout);
            if (power[n] == kNothing) power[n] = 0;
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
    auto of = [&](int t, Marks &m) {
        const int ka = t * kTile, kb = min(ka + kTile, p.Lk) - 1;
        bool any = near_any(p, qa, qb, ka, kb), some = near_any(p, wa, wb, ka, kb), all = near_all(p, wa, wb, ka, kb) && ka + kTile <= p.Lk;
        if (marks) {
            m = marks[t];
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
    if constexpr (kScaled<T>) {
        int e = kNothing;
        for (int t = first + lane; t <= last; t += kWave) {
            Marks m;
            if (of(t, m) & 1) e = max(e, p.value_powers[((int64_t)b * p.kv + kh) * p.key_tiles + t]);
        }
        const int raise = raise_of(uniform(wave_max(e)));
#pragma unroll
        for (int n = 0; n < QB; ++n) power[n] -= raise, lse[n] -= kRaise<T> + (float)power[n];
    }
    int left = INT32_MAX, skip = 0;   // of the tiles there are, this part's
    if (p.q_splits > 1) {
        left = (Walk::count(first, last, of, lane) + p.q_splits - 1) / p.q_splits;
        skip = split * left;
    }
    Walk walk(first, last, skip);
    auto next = [&](bool &some, bool &all, Seen &marks_of) { return left-- > 0 ? walk.next(of, lane, some, all, marks_of) : -1; };

    const typename L::RowReader rows(lane);
    const typename L::ColumnReader columns(lane);
    const float slope = SLOPES ? p.slopes[h] * kLog2e : 0.f;
    f32x4 dq[QB][L::DB];
#pragma unroll
    for (int n = 0; n < QB; ++n)
#pragma unroll
        for (int db = 0; db < L::DB; ++db) dq[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto stage = [&](int t, int buf, uint64_t live) {
        const int to = img + buf * 2 * L::BYTES;
        const char *zeros = p.documents ? p.zeros : nullptr;
        L::stage(kp, p.k.row, t * kTile, p.Lk, live, zeros, to, wave, lane);
        L::stage(vp, p.v.row, t * kTile, p.Lk, live, zeros, to + L::BYTES, wave, lane);
        if (zeros && wave == 0) global_to_lds_4(reinterpret_cast<const char *>(p.documents + (int64_t)b * p.Lk), (unsigned)min(t * kTile + lane, p.Lk - 1) * 4, lds_addr(ids[buf]));
    };

    bool some, all, some_next, all_next;
    Seen here{}, ahead{};
    int t = next(some, all, here), buf = 0;
    if (t >= 0) stage(t, 0, here.live);
#pragma unroll 1
    while (t >= 0) {
        const int after = next(some_next, all_next, ahead);
        wait_global_loads();
        workgroup_sync();
        if (after >= 0) stage(after, buf ^ 1, ahead.live);
        if (some) {
            const int ki = img + buf * 2 * L::BYTES, vi = ki + L::BYTES, k0 = t * kTile;
            uint64_t seen[QB];
            bool mixed = false;   // the tile's documents are not one
            if (!all) {
                mixed = here.mixed;
#pragma unroll
                for (int n = 0; n < QB; ++n) {
                    seen[n] = bits_between(pos[n] - p.window + 1 - k0, min(pos[n] - p.dlo + 1, p.Lk) - k0) | here.prefix;
                    if (p.documents) seen[n] = mine[n] >= 0 && (mixed || mine[n] == here.doc) ? seen[n] & here.live : 0;
                    seen[n] >>= 4 * g;
                }
            }
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
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][rb][r] = Score<T, CAP>::of(p, s[n][rb][r]);
                    if (!all) {
                        const uint64_t here = seen[n] >> (i * RB * 16);
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[n][rb][r] = keep(s[n][rb][r], here, 16 * rb + r, p.masked);
                        if (mixed) {
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb) {
                                const i32x4 doc = *reinterpret_cast<const i32x4 *>(&ids[buf][16 * (i * RB + rb) + 4 * g]);
#pragma unroll
                                for (int r = 0; r < 4; ++r) s[n][rb][r] = doc[r] == mine[n] ? s[n][rb][r] : p.masked;
                            }
                        }
                    }
                    const float near = SLOPES ? (float)(pos[n] - k0 - 4 * g - i * RB * 16) : 0.f;
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float y = s[n][rb][r], add = SLOPES ? __builtin_fmaf(fabsf(near - (float)(16 * rb + r)), -slope, lse[n]) : lse[n];
                            const float weight = __builtin_amdgcn_exp2f(__builtin_fmaf(p.m, y, add));
                            s[n][rb][r] = Score<T, CAP>::through(weight * (e[n][rb][r] - delta[n]), y);
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
        t = after, some = some_next, all = all_next, here = ahead, buf ^= 1;
    }
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        settle_products(dq[n]);
        const int i = qw + 16 * n + j;
        if (i >= p.Lq) continue;
        const float by = p.scale * two_to(power[n]);
        if (p.q_splits > 1) Tile<float, D>::store_row(dq[n], by, reinterpret_cast<char *>(p.parts + (((int64_t)split * p.B * p.heads + (int64_t)b * p.heads + h) * p.Lq + i) * D), 0, 0, lane);
        else L::store_row(dq[n], by, const_cast<char *>(p.dq.at) + b * p.dq.b + h * p.dq.h, p.dq.row, i, lane);
    }
}

template <typename T, int D, int CAP> struct Rows {
    static hipError_t go(const Args &a, hipStream_t st) {
        const int64_t of_q = (int64_t)a.B * a.heads * a.query_tiles, of_k = (int64_t)a.B * a.kv * a.key_tiles;
        int64_t blocks = of_q + (kScaled<T> ? (of_k < 4096 ? of_k : 4096) : 0);   // (workgroups take several tiles of keys where there are more than sixteen to a compute unit)
        if (kScaled<T> && !launch_holds(blocks, kThreads)) blocks = of_q + 1;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        rows_kernel<T, D, CAP><<<(unsigned)blocks, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
};
template <typename T, int D, int CAP> struct BwdQ {
    template <bool SLOPES, int QB> static hipError_t launch(const Args &a, hipStream_t st) {
        constexpr int lds = 4 * Tile<T, D>::BYTES, rows = 16 * QB * kWaves;
        static LdsAllowed allowed;
        if (hipError_t e = allow_lds(bwd_q_kernel<T, D, CAP, SLOPES, QB>, lds, allowed); e != hipSuccess) return e;
        const int64_t blocks = (int64_t)a.B * a.heads * ((a.Lq + rows - 1) / rows) * a.q_splits;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        bwd_q_kernel<T, D, CAP, SLOPES, QB><<<(unsigned)blocks, kThreads, lds, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || a.q_splits == 1) return e;
        return join<T, D>(a.parts, a.q_splits, a.B, a.heads, a.Lq, a.dq, nullptr, st);
    }
    static hipError_t go(const Args &a, hipStream_t st) {
        if constexpr (sizeof(T) == 2)
            if (two_query_blocks(a, D)) return a.slopes ? launch<true, 2>(a, st) : launch<false, 2>(a, st);
        return a.slopes ? launch<true, 1>(a, st) : launch<false, 1>(a, st);
    }
};

}  // namespace

hipError_t launch_rows(const Args &a, int dtype, int D, int cap, hipStream_t st) { return dispatch<Rows>(dtype, D, cap, a, st); }
hipError_t launch_bwd_q(const Args &a, int dtype, int D, int cap, hipStream_t st) { return dispatch<BwdQ>(dtype, D, cap, a, st); }

}  // namespace seq
