// The key side of the backward pass (see seq_bwd_q.hip).
#include "seq_bwd.hpp"

namespace seq {

namespace {

bool two_key_blocks(const Args &a, int D) { return D == 128 || two_blocks(a, D, (int64_t)a.B * a.kv, a.Lk); }   // (a pair keeps two)

// kPair: with 128 channels in 16 bit a wave that kept both sums of 32 keys would take more than 256 registers, and run alone on its SIMD.  Two waves share
// 32 keys instead: each forms P and dS of half of a tile's queries, the first sums dV, the second dK, and each gives the other, through LDS, the half
// that it does not sum itself.
//
// The work of a workgroup, the tiles of every head that shares its keys, is split into p.k_splits parts of as many tiles where there are few workgroups; each
// then leaves fp32 sums, which a last kernel adds in order.

template <typename T, int D> constexpr bool kPair = sizeof(T) == 2 && D == 128;
template <typename T, int D, int KB> constexpr int kKeys = 16 * KB * kWaves / (kPair<T, D> ? 2 : 1);   // of a workgroup

template <typename T, int D, int CAP, bool SLOPES, int KB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void bwd_kv_kernel(const Args p) {
    using L = Tile<T, D>;
    constexpr int RB = kRowBlocks<T>, NB = kTile / 16;
    constexpr bool PAIR = kPair<T, D>;
    extern __shared__ __align__(16) char lds[];
    __shared__ __align__(16) int ids[2][kTile];
    __shared__ __align__(16) float2 stats[2][kTile];
    __shared__ int range[4][kWaves];
    __shared__ __align__(16) u32x4 given[PAIR ? kWaves : 1][KB][PAIR ? kWave : 1];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), j = lane & 15, g = lane >> 4;
    const int role = PAIR ? wave & 1 : 0, group_of_keys = PAIR ? wave >> 1 : wave;
    const int tiles = (p.Lk + kKeys<T, D, KB> - 1) / kKeys<T, D, KB>;
    int id = block_in_order();
    const int split = id % p.k_splits;
    id /= p.k_splits;
    const int tile = id % tiles, plane = id / tiles, b = plane / p.kv, kh = plane % p.kv;
    const char *kp = p.k.at + b * p.k.b + kh * p.k.h, *vp = p.v.at + b * p.v.b + kh * p.v.h;
    const int k0 = tile * kKeys<T, D, KB>, kw = k0 + group_of_keys * 16 * KB;
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
        if (documents) L::clear(k[n], mine[n] >= 0), L::clear(v[n], mine[n] >= 0);
        always[n] = p.prefix && (marks[i / kTile].prefix >> (i % kTile) & 1);
    }
    Docs dw = no_docs(), dg = no_docs();
    bool prefix_any = false, prefix_some = false, prefix_all = false;
    int power = 0, raise = 0;   // dS is held times 2^(raise - power)
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
    const int ka = k0, kb = min(k0 + kKeys<T, D, KB>, p.Lk) - 1;
    const int wa = min(kw, p.Lk - 1), wb = min(kw + 16 * KB, p.Lk) - 1;
    if constexpr (kScaled<T>) {   // over the keys that are seen by a query that sees these: what the window reaches from there, of their documents
        const int qa = max(ka + p.dlo, p.off), qb = min(kb + p.window, p.Lk) - 1;
        int e = kNothing, near = 0, far = p.key_tiles - 1;
        if (!p.prefix) near = max(0, qa - p.window + 1) / kTile, far = min(far, max(-1, qb - p.dlo) >> 6);
        for (int t = near + lane; t <= far; t += kWave)
            if (!documents || Docs{marks[t].dmin, marks[t].dmax, false}.meet(dg)) e = max(e, p.value_powers[(int64_t)plane * p.key_tiles + t]);
        raise = raise_of(uniform(wave_max(e)));
    }
    auto of = [&](int t, Marks &m) {   // (of a tile of queries: their positions begin inside a tile of keys)
        const int qa = t * kTile + p.off, qb = min(t * kTile + kTile, p.Lq) - 1 + p.off;
        bool any = near_any(p, qa, qb, ka, kb) || prefix_any, some = near_any(p, qa, qb, wa, wb) || prefix_some, all = near_all(p, qa, qb, wa, wb) || prefix_all;
        if (documents) {
            // (a last tile may begin inside the last keys: nothing follows them, so what is staged behind the last query, which may be padding, is zeros)
            const int at = qa / kTile, in = qa % kTile;
            const Marks x = marks[at], y = !in ? x : at + 1 < p.key_tiles ? marks[at + 1] : Marks{INT32_MAX, -1, 0, 0};
            m = Marks{min(x.dmin, y.dmin), max(x.dmax, y.dmax), in ? x.live >> in | y.live << (kTile - in) : x.live, 0};
            const Docs d{m.dmin, m.dmax, (x.live & y.live) == ~0ull};
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

    auto stage = [&](int h, int t, int buf, uint64_t live) {
        const int to = img + buf * 2 * L::BYTES;
        const char *zeros = documents ? p.zeros : nullptr;
        L::stage(p.q.at + b * p.q.b + h * p.q.h, p.q.row, t * kTile, p.Lq, live, zeros, to, wave, lane);
        L::stage(p.dout.at + b * p.dout.b + h * p.dout.h, p.dout.row, t * kTile, p.Lq, live, zeros, to + L::BYTES, wave, lane);
        if (wave < 2) global_to_lds_4(reinterpret_cast<const char *>(p.rows + (((int64_t)b * p.heads + h) * p.query_tiles + t) * kTile), (unsigned)(wave * kWave + lane) * 4,
                                      lds_addr(stats[buf]) + wave * kWave * 4);
        if (zeros && wave == 2) global_to_lds_4(reinterpret_cast<const char *>(documents), (unsigned)min(t * kTile + lane + p.off, p.Lk - 1) * 4, lds_addr(ids[buf]));
    };

    // the heads that share these keys in turn, each one's tiles in turn: of all these, this part's
    int head = 0, left = INT32_MAX, skip = 0;
    if (p.k_splits > 1) {
        const int count = Walk::count(first, last, of, lane);
        left = (p.group * count + p.k_splits - 1) / p.k_splits;
        if (count) head = split * left / count, skip = split * left % count;
    }
    Walk walk(first, last, skip);
    bool some, all, some_next = false, all_next = false;
    auto next = [&](bool &s, bool &a, Seen &marks_of) {
        while (head < p.group && left > 0) {
            const int t = walk.next(of, lane, s, a, marks_of);
            if (t >= 0) return --left, t;
            if (++head < p.group) walk = Walk(first, last);
        }
        return -1;
    };
    Seen here{}, ahead{};
    int t = next(some, all, here), buf = 0, h = kh * p.group + head;
    if (t >= 0) stage(h, t, 0, here.live);
#pragma unroll 1
    while (t >= 0) {
        const int after = next(some_next, all_next, ahead);
        wait_global_loads();
        workgroup_sync();
        if (after >= 0) stage(kh * p.group + head, after, buf ^ 1, ahead.live);
        const int qi = img + buf * 2 * L::BYTES, di = qi + L::BYTES, q0 = t * kTile + p.off;
        const float slope = SLOPES ? p.slopes[h] * kLog2e : 0.f, lower = two_to(raise - power - (int)kRaise<T>);
        uint64_t seen[KB];
        bool mixed = false;   // the tile's documents are not one (what is not live has no weights anyway)
        if (some && !all) {
            mixed = here.mixed;
#pragma unroll
            for (int n = 0; n < KB; ++n) {
                seen[n] = always[n] ? ~0ull : bits_between(key[n] + p.dlo - q0, min(key[n] + p.window, kFar) - q0);
                if (documents) seen[n] = mine[n] >= 0 && (mixed || mine[n] == here.doc) ? seen[n] : 0;
                seen[n] >>= 4 * g;
            }
        }
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
            for (int n = 0; n < KB; ++n) {
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
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int at = (i * RB + rb) * 16 + 4 * g;   // of this lane's four queries
                f32x4 two[2];
                two[0] = *reinterpret_cast<const f32x4 *>(&stats[buf][at]), two[1] = *reinterpret_cast<const f32x4 *>(&stats[buf][at + 2]);
                if constexpr (kScaled<T>) two[0][1] *= lower, two[0][3] *= lower, two[1][1] *= lower, two[1][3] *= lower;
#pragma unroll
                for (int n = 0; n < KB; ++n) {
                    const float near = SLOPES ? (float)(q0 + at - key[n]) : 0.f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float lse = two[r / 2][r % 2 * 2], delta = two[r / 2][r % 2 * 2 + 1], y = s[n][rb][r];
                        const float add = SLOPES ? __builtin_fmaf(fabsf(near + (float)r), -slope, lse) : lse;
                        const float weight = __builtin_amdgcn_exp2f(__builtin_fmaf(p.m, y, add));
                        const float ds = kScaled<T> ? __builtin_fmaf(e[n][rb][r], lower, -delta) : e[n][rb][r] - delta;
                        s[n][rb][r] = weight, e[n][rb][r] = Score<T, CAP>::through(weight * ds, y);
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
        t = after, h = kh * p.group + head, some = some_next, all = all_next, here = ahead, buf ^= 1;
    }
    // which: 0 dK, 1 dV
    auto store = [&](int which, const f32x4 *acc, float by, int i) {
        const View &to = which ? p.dv : p.dk;
        if (p.k_splits == 1) L::store_row(acc, by, const_cast<char *>(to.at) + b * to.b + kh * to.h, to.row, i, lane);
        else Tile<float, D>::store_row(acc, by, reinterpret_cast<char *>(p.parts + (((int64_t)split * 2 + which) * p.B * p.kv + plane) * p.Lk * D), D * 4, i, lane);
    };
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        settle_products(dk[n]);
        settle_products(dv[n]);
        const int i = kw + 16 * n + j;
        if (i < p.Lk) {
            const float by_k = p.scale * two_to(power - raise), by_v = two_to(-(int)(kRaise<T> + Score<T, CAP>::kQuad));
            if constexpr (PAIR) {
                store(role ? 0 : 1, dv[n], role ? by_k : by_v, i);
            } else {
                store(0, dk[n], by_k, i);
                store(1, dv[n], by_v, i);
            }
        }
    }
}

template <typename T, int D, int CAP> struct BwdKV {
    template <bool SLOPES, int KB> static hipError_t launch(const Args &a, hipStream_t st) {
        constexpr int lds = 4 * Tile<T, D>::BYTES;
        static LdsAllowed allowed;
        if (hipError_t e = allow_lds(bwd_kv_kernel<T, D, CAP, SLOPES, KB>, lds, allowed); e != hipSuccess) return e;
        const int64_t blocks = (int64_t)a.B * a.kv * ((a.Lk + kKeys<T, D, KB> - 1) / kKeys<T, D, KB>) * a.k_splits;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        bwd_kv_kernel<T, D, CAP, SLOPES, KB><<<(unsigned)blocks, kThreads, lds, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || a.k_splits == 1) return e;
        return join<T, D>(a.parts, a.k_splits, a.B, a.kv, a.Lk, a.dk, &a.dv, st);
    }
    static hipError_t go(const Args &a, hipStream_t st) {
        if constexpr (sizeof(T) == 2)
            if (two_key_blocks(a, D)) return a.slopes ? launch<true, 2>(a, st) : launch<false, 2>(a, st);
        if constexpr (!kPair<T, D>) return a.slopes ? launch<true, 1>(a, st) : launch<false, 1>(a, st);
        return hipErrorInvalidValue;   // (a pair keeps two blocks)
    }
};

}  // namespace

hipError_t launch_bwd_kv(const Args &a, int dtype, int D, int cap, hipStream_t st) { return dispatch<BwdKV>(dtype, D, cap, a, st); }

// A tile of 16-bit queries takes about 2.2 us.
int k_splits(const Args &a, int dtype, int D) {
    const int keys = dtype != NA2D_F32 && D < 128 && two_key_blocks(a, D) ? 128 : 64;
    const Work w(a, keys, a.query_tiles);
    return parts_of((int64_t)a.B * a.kv * ((a.Lk + keys - 1) / keys), w.longest * a.group, w.tiles * a.group, 2.5, (int64_t)a.B * a.kv * a.Lk * D * 8, 5.5e6);
}

}  // namespace seq
