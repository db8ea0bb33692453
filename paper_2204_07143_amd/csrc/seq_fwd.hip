// Attention over a sequence, forward: one pass over the keys with the running maximum and sum of a softmax.
//
// A wave keeps QB blocks of 16 queries as product columns, a workgroup of four waves 64 QB; per tile of 64 keys
//   S^T = K Q^T          a lane has four scores of each block of 16 keys for its query
//   P = exp2(S' - ref)   ref: the running maximum, followed only once it is left by more than kSlack (the sums are rescaled then)
//   out^T += V^T P       P is the product's other operand as it lies in the registers; V through transposing LDS reads
// Keys and values come by direct loads into two images each, the next tile on its way while one is worked on.  Tiles in which the workgroup sees
// nothing are left out, tiles in which a wave sees all take no mask.
//
// What bounds it: the SIMDs, which issue about 35 vector instructions to every 16 products of a tile.  Two images of 64 keys each take 64 KB at 128 channels in
// 16 bit, so two workgroups are on a compute unit, and a wave keeps 32 queries so that a fragment from LDS serves two products (without bank conflicts in 16 bit; in fp32, whose
// transposed reads take a word at a time, 40 % of the LDS's cycles are conflicts, behind the matrix instructions).
// bf16, D 128: 2 x 16 over 4 x 8192, not causal, 1.08 to 1.13 ms or about 1 PFLOP/s, 88 % of a library product of 8192 x 8192; 4 x 16 over 4 x 2048, causal, capped, 127 us: the cap's
// exponential and reciprocal (a quarter of the rate each) make vector instructions 52 % of the cycles, matrix instructions are 24 %, and waves wait 29 % of their time: neither unit is
// full, and two waves to a SIMD do not cover each other.  fp32, D 32, 2 x 4 x 3136, causal, slopes: 71 us, matrix instructions 45 % of the cycles and vector ones 29 %, which an fp32
// matrix instruction does not let pass beside it.
#include "lds_attr.hpp"
#include "seq_common.hpp"

namespace seq {

namespace {

// Weights reach 2^8: fp16 holds them with all digits, and their sum.  Where a row's maximum is the reference its weight is 1 and takes no rounding; elsewhere it is up to 2^8 and is
// rounded like the others.  A fixed reference instead, where a cap bounds the scores, made out 1.18 and dq 1.1 times as inexact in bf16 (causal, cap 50, L 2048), for 3 % of the time.
constexpr float kSlack = 8.f;

template <typename T, int D, int CAP, bool SLOPES, int QB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void fwd_kernel(const Args p) {
    using L = Tile<T, D>;
    constexpr int RB = kRowBlocks<T>, NB = kTile / 16;
    extern __shared__ __align__(16) char lds[];
    __shared__ __align__(16) int ids[2][kTile];
    __shared__ int range[2][kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), j = lane & 15, g = lane >> 4;
    const int tiles = (p.Lq + 16 * QB * kWaves - 1) / (16 * QB * kWaves);
    // key heads in turn, the last queries (in causal order the longest work) first, the query heads of one key head next to each other
    int id = block_in_order();
    const int split = id % p.q_splits;
    id /= p.q_splits;
    const int in_group = id % p.group;
    id /= p.group;
    const int tile = tiles - 1 - id % tiles, plane = id / tiles, b = plane / p.kv, kh = plane % p.kv, h = kh * p.group + in_group;
    const char *kp = p.k.at + b * p.k.b + kh * p.k.h, *vp = p.v.at + b * p.v.b + kh * p.v.h, *qp = p.q.at + b * p.q.b + h * p.q.h;
    const int q0 = tile * 16 * QB * kWaves, qw = q0 + wave * 16 * QB;
    const int img = lds_addr(lds);

    u32x4 q[QB][L::STEPS];
    int pos[QB], mine[QB];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        const int i = min(qw + 16 * n + j, p.Lq - 1);
        L::load_row(q[n], qp, p.q.row, i, lane);
        if (!CAP && p.m < 0.f) L::negate(q[n]);
        pos[n] = i + p.off;
        mine[n] = p.documents ? p.documents[(int64_t)b * p.Lk + pos[n]] : 0;
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
    const int wa = min(qw, p.Lq - 1) + p.off, wb = min(qw + 16 * QB, p.Lq) - 1 + p.off;   // (a wave past the end: the last query)
    const Marks *marks = p.marks ? p.marks + (int64_t)b * p.key_tiles : nullptr;
    auto of = [&](int t, Marks &m) {
        const int ka = t * kTile, kb = min(ka + kTile, p.Lk) - 1;
        bool any = near_any(p, qa, qb, ka, kb), some = near_any(p, wa, max(wa, wb), ka, kb), all = near_all(p, wa, max(wa, wb), ka, kb) && ka + kTile <= p.Lk;
        if (marks) {
            m = marks[t];
            const Docs d{m.dmin, m.dmax, m.live == ~0ull};
            any |= m.prefix != 0, some |= m.prefix != 0, all |= m.prefix == ~0ull;
            if (p.documents) any &= d.meet(dg), some &= d.meet(dw), all &= d.same(dw);
        }
        return (any ? 1 : 0) | (some ? 2 : 0) | (all ? 4 : 0);
    };
    int first = 0, last = p.key_tiles - 1;
    if (!p.prefix) {
        first = max(0, qa - p.window + 1) / kTile;
        last = min(last, max(-1, qb - p.dlo) >> 6);
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
    const float slope = SLOPES ? p.slopes[h] * kLog2e : 0.f, m = CAP ? p.m : fabsf(p.m), from = p.from;
    constexpr bool kLeast = Score<T, CAP>::kSigmoid && !SLOPES;   // the largest score is that of the least y
    constexpr float masked = kLeast ? INFINITY : -INFINITY;
    f32x4 out[QB][L::DB];
    float ref[QB], sum[QB];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        ref[n] = kLowest, sum[n] = 0.f;
#pragma unroll
        for (int db = 0; db < L::DB; ++db) out[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

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
            f32x4 s[QB][NB];
#pragma unroll
            for (int n = 0; n < QB; ++n)
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) s[n][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < L::STEPS; ++st)
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) {
                    const u32x4 a = rows.read(ki, rb, st);
#pragma unroll
                    for (int n = 0; n < QB; ++n) s[n][rb] = mma<T>(a, q[n][st], s[n][rb]);
                }
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
            u32x4 w[QB][NB / RB];
#pragma unroll
            for (int n = 0; n < QB; ++n) {
                const float near = SLOPES ? (float)(pos[n] - k0 - 4 * g) : 0.f;
#pragma unroll
                for (int rb = 0; rb < NB; ++rb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[n][rb][r] = Score<T, CAP>::of(p, s[n][rb][r]);
                        if constexpr (SLOPES) s[n][rb][r] = __builtin_fmaf(fabsf(near - (float)(16 * rb + r)), -slope, __builtin_fmaf(m, s[n][rb][r], from));
                    }
                if (!all) {
#pragma unroll
                    for (int rb = 0; rb < NB; ++rb)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][rb][r] = keep(s[n][rb][r], seen[n], 16 * rb + r, masked);
                    if (mixed) {
#pragma unroll
                        for (int rb = 0; rb < NB; ++rb) {
                            const i32x4 doc = *reinterpret_cast<const i32x4 *>(&ids[buf][16 * rb + 4 * g]);
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[n][rb][r] = doc[r] == mine[n] ? s[n][rb][r] : masked;
                        }
                    }
                }
                float most = s[n][0][0];
#pragma unroll
                for (int rb = 0; rb < NB; ++rb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) most = kLeast ? fminf(most, s[n][rb][r]) : fmaxf(most, s[n][rb][r]);
                if constexpr (!SLOPES) most = __builtin_fmaf(m, most, from);
                most = column_max(most);
                const float now = most > ref[n] + kSlack ? most : ref[n];
                if (__any(now != ref[n])) {
                    const float by = __builtin_amdgcn_exp2f(ref[n] - now);
                    sum[n] *= by;
#pragma unroll
                    for (int db = 0; db < L::DB; ++db) out[n][db] *= by;
                    ref[n] = now;
                }
#pragma unroll
                for (int rb = 0; rb < NB; ++rb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[n][rb][r] = __builtin_amdgcn_exp2f(SLOPES ? s[n][rb][r] - ref[n] : __builtin_fmaf(m, s[n][rb][r], from - ref[n]));
                        sum[n] += s[n][rb][r];
                    }
#pragma unroll
                for (int i = 0; i < NB / RB; ++i) w[n][i] = pack<T>(&s[n][i * RB]);
            }
#pragma unroll
            for (int i = 0; i < NB / RB; ++i)
#pragma unroll
                for (int db = 0; db < L::DB; ++db) {
                    const u32x4 a = columns.read(vi, i, db);
#pragma unroll
                    for (int n = 0; n < QB; ++n) out[n][db] = mma<T>(a, w[n][i], out[n][db]);
                }
        }
        t = after, some = some_next, all = all_next, here = ahead, buf ^= 1;
    }
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        settle_products(out[n]);
        const int i = qw + 16 * n + j;
        const float total = column_sum(sum[n]);
        if (i >= p.Lq) continue;
        const int64_t row = ((int64_t)b * p.heads + h) * p.Lq + i;
        if (p.q_splits > 1) {
            const int64_t all = (int64_t)p.B * p.heads * p.Lq, at = split * all + row;
            Tile<float, D>::store_row(out[n], 1.f, reinterpret_cast<char *>(p.parts + at * D), 0, 0, lane);
            if (g == 0) reinterpret_cast<float2 *>(p.parts + p.q_splits * all * D)[at] = float2{ref[n], total};
        } else {
            L::store_row(out[n], total == 0.f ? 0.f : 1.f / total, const_cast<char *>(p.out.at) + b * p.out.b + h * p.out.h, p.out.row, i, lane, p.rest ? p.rest - p.out.at : 0);
            if (p.lse && g == 0) p.lse[row] = total == 0.f ? -INFINITY : (ref[n] + __builtin_amdgcn_logf(total)) * kLn2;
        }
    }
}

// The splits of a row, in order; a thread per four channels.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void join_fwd_kernel(const Args p, int64_t total) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= total) return;
    const int d = (int)(i % (D / 4)) * 4;
    const int64_t row = i / (D / 4), all = (int64_t)p.B * p.heads * p.Lq;
    const float2 *stats = reinterpret_cast<const float2 *>(p.parts + p.q_splits * all * D) + row;
    float most = kLowest, sum = 0.f;
    for (int s = 0; s < p.q_splits; ++s) most = fmaxf(most, stats[s * all].x);
    f32x4 x{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < p.q_splits; ++s) {
        const float by = __builtin_amdgcn_exp2f(stats[s * all].x - most);
        sum = __builtin_fmaf(stats[s * all].y, by, sum);
        x += *reinterpret_cast<const f32x4 *>(p.parts + (s * all + row) * D + d) * by;
    }
    x *= sum == 0.f ? 0.f : 1.f / sum;
    const int plane = (int)(row / p.Lq);
    char *out = const_cast<char *>(p.out.at) + plane / p.heads * p.out.b + plane % p.heads * p.out.h + row % p.Lq * p.out.row + d * (int)sizeof(T);
    Tile<T, D>::store4(out, x, p.rest ? p.rest - p.out.at : 0);
    if (p.lse && d == 0) p.lse[row] = sum == 0.f ? -INFINITY : (most + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <typename T, int D, int CAP> struct Fwd {
    template <bool SLOPES, int QB> static hipError_t launch(const Args &a, hipStream_t st) {
        constexpr int lds = 4 * Tile<T, D>::BYTES, rows = 16 * QB * kWaves;
        static LdsAllowed allowed;
        if (hipError_t e = allow_lds(fwd_kernel<T, D, CAP, SLOPES, QB>, lds, allowed); e != hipSuccess) return e;
        const int64_t blocks = (int64_t)a.B * a.heads * ((a.Lq + rows - 1) / rows) * a.q_splits;
        if (!launch_holds(blocks, kThreads)) return hipErrorInvalidValue;
        fwd_kernel<T, D, CAP, SLOPES, QB><<<(unsigned)blocks, kThreads, lds, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || a.q_splits == 1) return e;
        const int64_t total = (int64_t)a.B * a.heads * a.Lq * (D / 4), joins = (total + kThreads - 1) / kThreads;
        if (!launch_holds(joins, kThreads)) return hipErrorInvalidValue;
        join_fwd_kernel<T, D><<<(unsigned)joins, kThreads, 0, st>>>(a, total);
        return hipGetLastError();
    }
    static hipError_t go(const Args &a, hipStream_t st) {
        if constexpr (sizeof(T) == 2)
            if (two_query_blocks(a, D)) return a.slopes ? launch<true, 2>(a, st) : launch<false, 2>(a, st);
        return a.slopes ? launch<true, 1>(a, st) : launch<false, 1>(a, st);
    }
};

__global__ __launch_bounds__(kThreads) void marks_kernel(const int *__restrict__ documents, const uint8_t *__restrict__ prefix, int Lk, int tiles, int total, Marks *marks, uint32_t *zeros) {
    const int lane = threadIdx.x % kWave, n = blockIdx.x * kWaves + threadIdx.x / kWave;
    if (blockIdx.x == 0 && threadIdx.x < 16) zeros[threadIdx.x] = 0;
    if (n >= total) return;
    const int b = n / tiles, t = n % tiles, at = t * kTile + lane;
    const bool there = at < Lk;
    const int64_t i = (int64_t)b * Lk + (there ? at : Lk - 1);
    const int d = documents ? documents[i] : 0;
    const bool live = there && d >= 0;
    const Docs r = docs_of_wave(d, there);
    const uint64_t l = __ballot(live), x = __ballot(live && prefix && prefix[i] != 0);
    if (lane == 0) marks[n] = Marks{r.lo, r.hi, l, x};
}

}  // namespace

hipError_t launch_marks(const Args &a, const uint8_t *prefix, Marks *marks, char *zeros, hipStream_t st) {
    const int64_t total = (int64_t)a.B * a.key_tiles;
    if (!launch_holds((total + kWaves - 1) / kWaves, kThreads)) return hipErrorInvalidValue;
    marks_kernel<<<(unsigned)((total + kWaves - 1) / kWaves), kThreads, 0, st>>>(a.documents, prefix, a.Lk, a.key_tiles, (int)total, marks, reinterpret_cast<uint32_t *>(zeros));
    return hipGetLastError();
}

// Of the forward pass and of dQ; a tile of 16-bit keys takes about 1.2 us.
int q_splits(const Args &a, int dtype, int D) {
    const int rows = dtype != NA2D_F32 && two_query_blocks(a, D) ? 128 : 64;
    const Work w(a, rows, a.key_tiles);
    return parts_of((int64_t)a.B * a.heads * ((a.Lq + rows - 1) / rows), w.longest, w.tiles, 4, (int64_t)a.B * a.heads * a.Lq * (D + 2) * 4, 2.5e6);
}

hipError_t launch_fwd(const Args &a, int dtype, int D, int cap, hipStream_t st) { return dispatch<Fwd>(dtype, D, cap, a, st); }

}  // namespace seq
