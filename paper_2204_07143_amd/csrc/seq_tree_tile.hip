// Attention of a tree of drafted tokens over a cache in 8 bits, where a key head has more than 32 rows (its query heads times the nodes) and there is enough work (plan_cache_tree()).
//
// A workgroup keeps 64 RB rows, 16 RB to a wave, and walks tiles of 64 tokens: the cache's bytes are read into registers a tile ahead, become fp16 (exactly: 0x64 in front of a
// byte, minus 1152) once for all rows on their way to LDS, and are read from there as seq_fwd.hip reads keys and values, S^T = K Q^T, O^T += V^T P.  A page's key scale multiplies
// its scores (one below zero goes the way of the masks: it turns the order of the scores); the size of its value scale goes into the weights' exponent, 2^(s + log2 |vs| - ref), so that the
// products need no scale of their own, and the sign of one below zero into the values; a row's sum takes a page's weights over |vs| again.
// Pages whose value scale is 0 have no such exponent: their tokens go into a sum of their own.  The nodes' own keys and values are the last tile of a row's work.
//
// Bound by the vector instructions (half of the cycles) and the products (a quarter), which two waves to a SIMD lay over each other in part; waves wait 27 % of their time; a quarter of the LDS's cycles
// are conflicts of the bytes' way in.  192 rows of 128
// channels fill the registers.  16 sequences to 8000 tokens, 48 nodes, 32 heads over 8, D 128, bf16: 126 us (124 with scales above 0 alone), 0.48 PFLOP/s of products, and the join 14 (64 MB of sums; 16 with a workgroup for each 8 rows); 225 in workgroups
// of 32 rows that each make fp16 of all bytes (seq_decode.hpp); 64 and 128 rows to a workgroup 168 and 163; 126 without the products' priority over another wave's softmax.
//
// The tiles of all sequences and key heads, in a row, are shared evenly by the workgroups, wherever the cuts fall: a run that has all of a row's tiles stores its result, others
// leave sums, maxima and totals, two runs a workgroup at most, that a second kernel joins in order.
#include "lds_attr.hpp"
#include "seq_decode.hpp"

namespace seq {

namespace {

constexpr int kLeastRun = 2;   // tiles of a workgroup, where there are so many
constexpr float kNothing = -100.f;   // a value scale of this power of two, or below, counts as 0

__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)seq::uniform((int)(uint32_t)x) | (uint64_t)(uint32_t)seq::uniform((int)(uint32_t)((uint64_t)x >> 32)) << 32);
}
// A lane's number that the compiler takes for a new one: what is formed from it is formed here, and not kept in registers from further up.
__device__ __forceinline__ int afresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// x 2^by, by not above 0: also where 2^by alone would be below 2^-126, and 0
__device__ __forceinline__ float lowered(float x, float by) { return x * __builtin_amdgcn_exp2f(fmaxf(by, -126.f)) * __builtin_amdgcn_exp2f(fminf(by + 126.f, 0.f)); }

// What of a sequence its rows see of the cache.
struct Span {
    int tokens, length, least, begin, tiles;   // tiles: of the cache from `begin` on, and the nodes' own
    __device__ __forceinline__ Span(const CacheArgs &p, int held) {   // held: the sequence's length as it is given
        tokens = min(max(held, 0), INT32_MAX - kNodes);
        length = (int)min((int64_t)tokens, (int64_t)p.width << p.page_log2);
        least = max(0, tokens - p.window + 1);
        begin = least / kTile;
        tiles = max(0, (length + kTile - 1) / kTile - begin) + 1;
    }
};

// The runs of the workgroups: the tiles of a sequence's units (key heads, and groups of their rows), unit after unit, sequence after sequence.
struct Schedule {
    int64_t total;
    int units, runs, held;   // held: the length of sequence `lane`
    __device__ __forceinline__ Schedule(const CacheArgs &p, int lane) : total(0), units(p.kv * p.row_groups) {
        held = lane < p.B ? p.lengths[lane] : 0;
        if (lane < p.B) total = Span(p, held).tiles;
        for (int b = lane + kWave; b < p.B; b += kWave) total += Span(p, p.lengths[b]).tiles;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) total += __shfl_xor(total, d);
        total = uniform(total * units);
        const int64_t wanted = total / kLeastRun;
        runs = wanted < 1 ? 1 : wanted < p.splits ? (int)wanted : p.splits;
    }
    __device__ __forceinline__ Span span(const CacheArgs &p, int b) const { return Span(p, b < kWave ? __builtin_amdgcn_readlane(held, b) : p.lengths[b]); }   // b: the same in all lanes
    // (in 64-bit floating point, a division of few instructions: products stay below 2^53, the quotient of the last is exact, and all that matters is that everybody cuts alike)
    __device__ __forceinline__ int64_t start(int run) const { return (int64_t)((double)total * run / runs); }
    __device__ __forceinline__ int run_of(int64_t tile) const {
        int w = (int)((double)tile * runs / (double)total);
        while (start(w + 1) <= tile) ++w;
        while (start(w) > tile) --w;
        return w;
    }
    // The sequence that has `tile`, or (tile beyond what lies before it) the tiles before sequence b.
    __device__ __forceinline__ int find(const CacheArgs &p, int64_t tile, int lane, int64_t &before) const {
        before = 0;
        for (int base = 0;; base += kWave) {
            const int64_t mine = base + lane < p.B ? (int64_t)Span(p, base ? p.lengths[base + lane] : held).tiles * units : 0;
            int64_t upto = mine;
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                const int64_t x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
            const uint64_t here = __ballot(before + upto > tile);
            if (here) {
                const int k = __builtin_ctzll(here);
                before += uniform((int64_t)__shfl(upto - mine, k));
                return base + k;
            }
            before += uniform((int64_t)__shfl(upto, kWave - 1));
        }
    }
    __device__ __forceinline__ int64_t tiles_before(const CacheArgs &p, int b, int lane) const {
        int64_t n = 0;
        for (int i = lane; i < b; i += kWave) n += Span(p, i < kWave ? held : p.lengths[i]).tiles;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) n += __shfl_xor(n, d);
        return uniform(n * units);
    }
};

// A tile's bytes of one of keys and values, on their way from the cache to LDS.
template <int D> struct TileBytes {
    static constexpr int W = D >= 64 ? 4 : 2, C = D / (4 * W), LOADS = kTile * C / kThreads;   // words of a read, reads of a row, reads of a thread
    typedef uint32_t words __attribute__((ext_vector_type(W)));
    words x[LOADS];
    __device__ static __forceinline__ int row(int i, int tid) { return (tid + i * kThreads) / C; }
    __device__ static __forceinline__ int block(int i, int wave) { return (wave * kWave + i * kThreads) / C / 16; }   // of 16 rows: a wave's read lies in one
    __device__ __forceinline__ void to_lds(int img, int tid) const {
        using L = Tile<f16_t, D>;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = row(i, tid), c = (tid + i * kThreads) % C;
#pragma unroll
            for (int k = 0; k < W / 2; ++k) {
                const uint32_t a = x[i][2 * k] ^ 0x80808080u, b = x[i][2 * k + 1] ^ 0x80808080u;
                *lds_ptr<u32x4>(img + r * L::ROWB + (((W / 2) * c + k) ^ L::swizzle(r)) * 16) = u32x4{low_pair(a), high_pair(a), low_pair(b), high_pair(b)};
            }
        }
    }
    // What this thread left there, of the pieces in `minus` (2^shift blocks of 16 rows each), with the other sign.
    __device__ __forceinline__ static void negate(int img, int tid, int wave, uint64_t minus, int shift) {
        using L = Tile<f16_t, D>;
#pragma unroll 1
        for (int i = 0; i < LOADS; ++i) {
            if (!(minus >> (block(i, wave) >> shift) & 1)) continue;
            const int r = row(i, tid), c = (tid + i * kThreads) % C;
            for (int k = 0; k < W / 2; ++k) *lds_ptr<u32x4>(img + r * L::ROWB + (((W / 2) * c + k) ^ L::swizzle(r)) * 16) ^= 0x80008000u;
        }
    }
};

template <typename T, int D, int RB, int CAP>
__global__ __launch_bounds__(kThreads, 2) void tree_tile_kernel(const CacheArgs p) {
    using L = Tile<f16_t, D>;
    using B = TileBytes<D>;
    constexpr int ROWS = 16 * RB * kWaves, STEPS = L::STEPS, DB = L::DB;
    extern __shared__ __align__(16) char lds[];
    __shared__ Tree tree;
    __shared__ Wild<D> wild;
    __shared__ int2 row_info[ROWS];   // position, and slope as bits
    __shared__ float2 aside[RB][kThreads];   // a thread's tokens whose values' scale is 0: largest score, and sum of weights beside it
    const int tid = threadIdx.x, lane = tid % kWave, wave = seq::uniform(tid / kWave), g = lane >> 4, img = lds_addr(lds);
    const Schedule schedule(p, lane);
    const int run = blockIdx.x;
    if (run >= schedule.runs) return;
    int64_t at = uniform(schedule.start(run)), left = uniform(schedule.start(run + 1)) - at, before;   // at: from here on, of the sequence's tiles
    int b = seq::uniform(schedule.find(p, at, lane, before));
    at -= before;
    const int page = 1 << p.page_log2, all_rows = p.group * p.n;
    const typename L::RowReader rows(lane);
    const typename L::ColumnReader columns(lane);
    int built = -1;
    wild.clear(tid);
#pragma unroll
    for (int n = 0; n < RB; ++n) aside[n][tid] = float2{kLowest, 0.f};

#pragma unroll 1
    for (bool begun = false; left > 0; begun = true) {
        auto span_of = [&](int b) { return RB == 3 ? Span(p, p.lengths[b]) : schedule.span(p, b); };   // (three blocks: the registers)
        Span span = span_of(b);
        while (at >= (int64_t)span.tiles * schedule.units) {
            at -= (int64_t)span.tiles * schedule.units;
            span = span_of(++b);
        }
        const int unit_id = seq::uniform((int)((double)at / span.tiles)), first = (int)(at - (int64_t)unit_id * span.tiles);
        const int count = (int)min(left, (int64_t)(span.tiles - first)), kh = unit_id / p.row_groups, row0 = unit_id % p.row_groups * ROWS + wave * 16 * RB;
        const bool whole = count == span.tiles;
        // where the cache's tiles lie, and the first one's bytes, on their way from here on
        const int cached = min(count, span.tiles - 1 - first);   // of this run
        const int pieces = page >= kTile ? 1 : kTile / page, shift = page >= kTile ? 2 : p.page_log2 - 4, chunk = kWave / pieces;   // of a tile: pages, and 16-token blocks to one
        int unit = -1;                // of one of the next 64 pieces: its page, and of that
        float ks = 0.f, lv = 0.f;   // the keys' scale, the size of the values' in base 2, kNothing for 0
        uint64_t minus = 0;         // those whose values' scale is below zero
        auto look_up = [&](int tile) {
            const int size = kTile / pieces;
            const int64_t token = (int64_t)tile * kTile + (int64_t)size * lane;
            const bool seen = token < span.length && token + size > span.least;
            const int id = p.table[(int64_t)b * p.width + (seen ? token >> p.page_log2 : 0)];
            unit = seen && (unsigned)id < (unsigned)p.pages ? id : -1;
            const int64_t u = (int64_t)max(unit, 0) * p.kv + kh;
            const float k = p.ks[u], scale = p.vs[u];
            ks = unit < 0 ? 0.f : k, lv = unit < 0 ? 0.f : fmaxf(__builtin_amdgcn_logf(fabsf(scale)), kNothing);
            minus = __ballot(unit >= 0 && scale < 0.f);
        };
        auto lane_of = [](float x, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), l)); };
        B keys, values;
        auto load = [&](int t) {   // the run's tile t; its blocks have been looked up
            const int t0 = (span.begin + first + t) * kTile, tid = RB == 3 ? afresh(threadIdx.x) : (int)threadIdx.x;
#pragma unroll
            for (int i = 0; i < B::LOADS; ++i) {
                const int u = __builtin_amdgcn_readlane(unit, (t & (chunk - 1)) * pieces + (B::block(i, wave) >> shift));
                const int64_t cell = (((int64_t)max(u, 0) * p.kv + kh) * page + ((t0 + B::row(i, tid)) & (page - 1))) * D + (tid + i * kThreads) % B::C * (4 * B::W);
                keys.x[i] = *reinterpret_cast<const typename B::words *>(p.k + cell);
                values.x[i] = *reinterpret_cast<const typename B::words *>(p.v + cell);
            }
        };
        if (cached > 0) {
            look_up(span.begin + first);
            load(0);
        }
        workgroup_sync();   // (what the run before reads of LDS)
        if (b != built) {
            tree.build(p.parents + (int64_t)b * p.n, p.n, RB == 3 ? afresh(threadIdx.x) : tid);   // (afresh: the registers)
            built = b;
            workgroup_sync();
        }

        // rows as fp16 on a power of two of their own, with the scale's sign
        const int lane_q = afresh(threadIdx.x) % kWave;
        u32x4 q[RB][STEPS];
        float c[RB], ref[RB], sum[RB];
        f32x4 out[RB][DB];
#pragma unroll
        for (int n = 0; n < RB; ++n) {
            const int row = min(row0 + 16 * n + (lane_q & 15), all_rows - 1), h = kh * p.group + row / p.n, i = row % p.n;
            const char *q_at = p.a.at + b * p.a.b + h * p.a.h + (int64_t)i * p.a.row + 16 * (lane_q >> 4);
            if (lane_q < 16) row_info[wave * 16 * RB + 16 * n + lane_q] = int2{span.tokens + tree.depth[i], p.slopes ? (int)__float_as_uint(p.slopes[h] * kLog2e) : 0};   // (of this wave alone)
            typedef T vec __attribute__((ext_vector_type(8)));
            float most = 0.f;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                q[n][s] = *reinterpret_cast<const u32x4 *>(q_at + 64 * s);
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)__builtin_bit_cast(vec, q[n][s])[e]));
            }
            most = column_max(most);
            const int power = most > 0.f && most < INFINITY ? __builtin_amdgcn_frexp_expf(most) : 0;
            c[n] = __builtin_amdgcn_ldexpf(fabsf(p.c), power);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                f16x8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (f16_t)__builtin_amdgcn_ldexpf((float)__builtin_bit_cast(vec, q[n][s])[e], -power);
                q[n][s] = __builtin_bit_cast(u32x4, y) ^ (p.c < 0.f ? 0x80008000u : 0u);
            }
            ref[n] = kLowest, sum[n] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) out[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // Of two blocks of 16 keys s by + plus, scores in base 2 (with log2 vs), as weights over the row's reference, and their sum over vs.  by is not negative.
        auto weigh = [&](int n, f32x4 (&s)[2], const float (&by)[2], const float (&plus)[2], const float (&inv)[2]) {
            float most[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) most[i] = __builtin_fmaf(fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3])), by[i], plus[i]);
            most[0] = fmaxf(most[0], most[1]);
            if (__any(most[0] > ref[n] + kSlack)) {
                most[0] = column_max(most[0]);
                const float now = most[0] > ref[n] + kSlack ? most[0] : ref[n], down = __builtin_amdgcn_exp2f(ref[n] - now);
                sum[n] *= down;
#pragma unroll
                for (int db = 0; db < DB; ++db) out[n][db] *= down;
                ref[n] = now;
            }
            float part[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float less = plus[i] - ref[n];
#pragma unroll
                for (int r = 0; r < 4; ++r) s[i][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][r], by[i], less));
                part[i] = (s[i][0] + s[i][1]) + (s[i][2] + s[i][3]);
            }
            sum[n] = __builtin_fmaf(part[1], inv[1], __builtin_fmaf(part[0], inv[0], sum[n]));
        };
        constexpr float kOnes[2] = {1.f, 1.f}, kZeros[2] = {0.f, 0.f};
        auto capped = [&](float x) {
            if constexpr (CAP == kTanhCap) return 0.5f * p.cap * tanhf(0.5f * kLn2 * x);
            else if constexpr (CAP == kSigmoidCap) return __builtin_fmaf(-p.cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x)), 0.5f * p.cap);
            else return x;
        };

        // ---- the cache's tiles
#pragma unroll 1
        for (int t = 0; t < cached; ++t) {
            const int ki = img + (t & 1) * 2 * L::BYTES, vi = ki + L::BYTES, t0 = (span.begin + first + t) * kTile, slot = (t & (chunk - 1)) * pieces;
            const int mine = RB == 3 ? afresh(threadIdx.x) : tid;   // (the registers)
            keys.to_lds(ki, mine);
            values.to_lds(vi, mine);
            const uint64_t here = ((1ull << pieces) - 1) << slot;   // the tile's pieces
            if (minus & here) values.negate(vi, mine, wave, minus >> slot, shift);
            uint64_t there = 0;
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
                if (__builtin_amdgcn_readlane(unit, slot + (rb >> shift)) >= 0) there |= 0xffffull << 16 * rb;
            // Values that are 0 add to a row's sum alone, and have no scale whose exponent their weights could take: into the thread's own sum, by scores formed once more.
            if (const uint64_t zero = __ballot(lv == kNothing) & here) {
                uint64_t apart = 0;
#pragma unroll
                for (int rb = 0; rb < 4; ++rb)
                    if (zero >> (slot + (rb >> shift)) & 1) apart |= 0xffffull << 16 * rb;
                there &= ~apart;
                workgroup_sync();
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int n = 0; n < RB; ++n) {
                        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                        for (int st = 0; st < STEPS; ++st)
#pragma unroll
                            for (int i = 0; i < 2; ++i) s[i] = mma<f16_t>(rows.read(ki + half * 32 * L::ROWB, i, st), q[n][st], s[i]);
                        settle_products(s);
                        const int lane = afresh(threadIdx.x) % kWave, g = lane >> 4;
                        const int2 info = row_info[wave * 16 * RB + 16 * n + (lane & 15)];
                        const float near = (float)(info.x - t0 - 32 * half - 4 * g), slope = __uint_as_float((uint32_t)info.y);
                        const uint64_t seen = (bits_between(info.x - p.window + 1 - t0, span.length - t0) & apart) >> (32 * half + 4 * g);
                        float2 &mine = aside[n][wave * kWave + lane];
                        const float2 old = mine;
                        float now = old.x;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float by = c[n] * lane_of(ks, slot + ((2 * half + i) >> shift));
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                s[i][r] = keep(__builtin_fmaf(near - (float)(16 * i + r), -slope, capped(s[i][r] * by)), seen, 16 * i + r, -INFINITY);
                                now = fmaxf(now, s[i][r]);
                            }
                        }
                        float all_of = old.y * __builtin_amdgcn_exp2f(old.x - now);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r) all_of += __builtin_amdgcn_exp2f(s[i][r] - now);
                        mine = float2{now, all_of};
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            const bool known = ((t + 1) & (chunk - 1)) != 0;   // where the next tile lies: else that is looked up when this one's scales are not needed any more
            if (t + 1 < cached && known) load(t + 1);
            workgroup_sync();
            // every row sees all of it, and no scale turns the order of its scores
            const bool all = there == ~0ull && t0 + kTile <= span.length && span.tokens + p.n - 1 - t0 < p.window && !(__ballot(ks < 0.f) & here);
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const int kh_at = ki + half * 32 * L::ROWB;
                float k2[2], l2[2], o2[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int from = slot + ((2 * half + i) >> shift);
                    k2[i] = lane_of(ks, from), l2[i] = lane_of(lv, from), o2[i] = __builtin_amdgcn_exp2f(-l2[i]);
                }
                // reads of LDS on their way ahead of the products that take them: all of a half's, or where the registers are full the next, or with a cap none of the keys
                constexpr int AHEAD = RB < 3 ? STEPS : CAP ? 0 : 1, VAHEAD = RB < 3 ? DB : 2;
                u32x4 a[AHEAD + 1][2], v[VAHEAD];
                auto read_keys = [&](int st) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) a[st % (AHEAD + 1)][i] = rows.read(kh_at, i, st);
                };
                auto read_values = [&](int db) { v[db % VAHEAD] = columns.read(vi + half * 32 * L::ROWB, 0, db); };
#pragma unroll
                for (int st = 0; st < AHEAD; ++st) read_keys(st);
                __builtin_amdgcn_sched_barrier(0);
                f32x4 s[RB][2];
#pragma unroll
                for (int n = 0; n < RB; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    if (st + AHEAD < STEPS) read_keys(st + AHEAD);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int n = 0; n < RB; ++n) s[n][i] = mma<f16_t>(a[st % (AHEAD + 1)][i], q[n][st], s[n][i]);
                    if constexpr (RB == 3) __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
#pragma unroll
                for (int db = 0; db < VAHEAD; ++db) read_values(db);
                __builtin_amdgcn_sched_barrier(0);
                u32x4 w[RB];
#pragma unroll
                for (int n = 0; n < RB; ++n) {
                    float by[2], plus[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) by[i] = c[n] * k2[i], plus[i] = l2[i];
                    if constexpr (CAP) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[n][i][r] = capped(s[n][i][r] * by[i]);
                            by[i] = 1.f;
                        }
                    }
                    if (p.slopes || !all) {
                        const int2 info = row_info[wave * 16 * RB + 16 * n + (lane & 15)];
                        const float near = (float)(info.x - t0 - 32 * half - 4 * g), slope = __uint_as_float((uint32_t)info.y);
                        const uint64_t seen = (bits_between(info.x - p.window + 1 - t0, span.length - t0) & there) >> (32 * half + 4 * g);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const float x = __builtin_fmaf(near - (float)(16 * i + r), -slope, __builtin_fmaf(s[n][i][r], by[i], plus[i]));
                                s[n][i][r] = keep(x, seen, 16 * i + r, -INFINITY);
                            }
                            by[i] = 1.f, plus[i] = 0.f;
                        }
                    }
                    weigh(n, s[n], by, plus, o2);
                    w[n] = pack<f16_t>(s[n]);
                }
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
#pragma unroll
                    for (int n = 0; n < RB; ++n) out[n][db] = mma<f16_t>(v[db % VAHEAD], w[n], out[n][db]);
                    if (db + VAHEAD < DB) read_values(db + VAHEAD);
                    if constexpr (RB == 3) __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
            }
            if (t + 1 < cached && !known) {
                look_up(span.begin + first + t + 1);
                load(t + 1);
            }
        }

        // ---- the nodes' own, products in the type of q.  In bfloat16 weights are the sum of two of them, 2^-17 off at most: no less exact than the cache's, in fp16.
        if (first + count == span.tiles) {
            using N = Tile<T, D>;
            const int tid = afresh(threadIdx.x), lane = tid % kWave, j = lane & 15, g = lane >> 4;
            const int ki = img + (cached & 1) * 2 * L::BYTES, vi = ki + L::BYTES;
#pragma unroll
            for (int i = 0; i < N::LOADS; ++i) {
                const int id = tid + i * kThreads, r = id / N::CH, ch = id % N::CH, node = min(r, p.n - 1);
                const bool live = r < p.n && tree.above[node];   // (what is no node may be anything)
                u32x4 x = *reinterpret_cast<const u32x4 *>(p.tk.at + b * p.tk.b + kh * p.tk.h + (int64_t)node * p.tk.row + ch * 16);
                u32x4 y = *reinterpret_cast<const u32x4 *>(p.tv.at + b * p.tv.b + kh * p.tv.h + (int64_t)node * p.tv.row + ch * 16);
                x = live ? x : u32x4{0, 0, 0, 0}, y = live ? y : u32x4{0, 0, 0, 0};
                const int place = r * N::ROWB + (ch ^ N::swizzle(r)) * 16;
                *lds_ptr<u32x4>(ki + place) = x;
                *lds_ptr<u32x4>(vi + place) = y;
            }
#pragma unroll 1
            for (int id = tid; id < kNodes * N::CH; id += kThreads) {   // (this thread's own, once more: the registers)
                const int r = id / N::CH, ch = id % N::CH, place = vi + r * N::ROWB + (ch ^ N::swizzle(r)) * 16;
                u32x4 y = *lds_ptr<u32x4>(place);
                if (wild.template take<T>(y, 4, r, 8 * ch)) *lds_ptr<u32x4>(place) = y;
            }
            workgroup_sync();
#pragma unroll
            for (int n = 0; n < RB; ++n) {
                const int row = min(row0 + 16 * n + j, all_rows - 1), h = kh * p.group + row / p.n, i = row % p.n, depth = tree.depth[i];
                const char *q_at = p.a.at + b * p.a.b + h * p.a.h + (int64_t)i * p.a.row + 16 * g;
                const float slope = p.slopes ? p.slopes[h] * kLog2e : 0.f;
                u32x4 f[STEPS];
#pragma unroll
                for (int st = 0; st < STEPS; ++st) f[st] = *reinterpret_cast<const u32x4 *>(q_at + 64 * st);
#pragma unroll 1
                for (int half = 0; half < (p.n > 32 ? 2 : 1); ++half) {
                    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (int st = 0; st < STEPS; ++st)
#pragma unroll
                        for (int k = 0; k < 2; ++k) s[k] = mma<T>(rows.read(ki + half * 32 * L::ROWB, k, st), f[st], s[k]);
                    settle_products(s);
                    const uint64_t seen = tree.above[i] >> (32 * half + 4 * g);
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int far = depth - tree.depth[32 * half + 16 * k + 4 * g + r];
                            const float x = __builtin_fmaf((float)far, -slope, capped(s[k][r] * p.c));
                            s[k][r] = (seen >> (16 * k + r) & 1) && far < p.window ? x : -INFINITY;
                        }
                    weigh(n, s, kOnes, kZeros, kOnes);
                    const u32x4 w = pack<T>(s);
                    u32x4 rest{};
                    if constexpr (__is_same(T, bf16_t)) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) rest[e] = pack_remainders(w[e], s[e / 2][e % 2 * 2], s[e / 2][e % 2 * 2 + 1]);
                    }
#pragma unroll
                    for (int db = 0; db < DB; ++db) {
                        const u32x4 a = columns.read(vi + half * 32 * L::ROWB, 0, db);
                        out[n][db] = mma<T>(a, w, out[n][db]);
                        if constexpr (__is_same(T, bf16_t)) out[n][db] = mma<T>(a, rest, out[n][db]);
                    }
                    settle_products(out[n]);
                }
            }
        }

        // ---- this run's rows
        const int lane = afresh(threadIdx.x) % kWave, j = lane & 15, g = lane >> 4;
        const int place = 2 * run + begun;
        float *parts = p.part + (int64_t)place * ROWS * D, *stats = p.part + (int64_t)p.splits * 2 * ROWS * D + (int64_t)place * ROWS * 2;
#pragma unroll
        for (int n = 0; n < RB; ++n) {
            settle_products(out[n]);
            const int row = row0 + 16 * n + j, in_unit = wave * 16 * RB + 16 * n + j;
            const float2 rest = aside[n][wave * kWave + lane];
            if (__any(rest.y != 0.f)) {   // both under the larger reference
                const float now = fmaxf(ref[n], column_max(rest.x)), down = __builtin_amdgcn_exp2f(ref[n] - now);
                sum[n] = __builtin_fmaf(sum[n], down, lowered(rest.y, rest.x - now));
#pragma unroll
                for (int db = 0; db < DB; ++db) out[n][db] *= down;
                ref[n] = now, aside[n][wave * kWave + lane] = float2{kLowest, 0.f};
            }
            float total = column_sum(sum[n]);
            if (row >= all_rows) continue;
            const bool node = tree.above[row % p.n] != 0;
            if (wild.any) {
                const uint64_t seen = tree.seen(row % p.n, p.window);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[n][db][r] = wild.of(out[n][db][r], 16 * db + 4 * g + r, seen);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (!node) total = 0.f;   // whatever its query is
            if (whole) {
                const int h = kh * p.group + row / p.n;
                const float by = total == 0.f ? 0.f : 1.f / total;
                if (!node) {
#pragma unroll
                    for (int db = 0; db < DB; ++db) out[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
                Tile<T, D>::store_row(out[n], by, const_cast<char *>(p.b.at) + b * p.b.b + h * p.b.h, p.b.row, row % p.n, lane);
            } else {
                if (!node) {
#pragma unroll
                    for (int db = 0; db < DB; ++db) out[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
                Tile<float, D>::store_row(out[n], 1.f, reinterpret_cast<char *>(parts + (int64_t)in_unit * D), 0, 0, lane);
                if (g == 0) reinterpret_cast<float2 *>(stats)[in_unit] = float2{node ? ref[n] : kLowest, total};
            }
        }
        if (wild.any) {
            workgroup_sync();
            wild.clear(afresh(threadIdx.x));
        }
        at += count, left -= count;
    }
}

// The runs of a row that several have, in order: a thread per four channels, of several rows (finding a unit's runs takes longer than a row's sums).
template <int D, int RB> struct Joined {
    static constexpr int ROWS = 16 * RB * kWaves, COLS = D / 4, EACH = kThreads / COLS, TIMES = RB, BLOCKS = ROWS / EACH / TIMES;   // of a unit
    static_assert(BLOCKS * EACH * TIMES == ROWS, "rows of a unit");
};
template <typename T, int D, int RB>
__global__ __launch_bounds__(kThreads) void tree_join_kernel(const CacheArgs p) {
    using J = Joined<D, RB>;
    constexpr int ROWS = J::ROWS;
    const int lane = threadIdx.x % kWave, col = threadIdx.x % J::COLS;
    const int unit = (int)(blockIdx.x / J::BLOCKS) % (p.kv * p.row_groups), b = (int)(blockIdx.x / J::BLOCKS) / (p.kv * p.row_groups);
    const Schedule schedule(p, lane);
    const int tiles = schedule.span(p, b).tiles;
    const int64_t first = schedule.tiles_before(p, b, lane) + (int64_t)unit * tiles;
    const int from = seq::uniform(schedule.run_of(first)), to = seq::uniform(schedule.run_of(first + tiles - 1));
    if (from == to) return;
    const int begun = seq::uniform((int)(schedule.start(from) < first));   // the first run had another row's work before
    const int kh = unit / p.row_groups;
#pragma unroll 1
    for (int i = 0; i < J::TIMES; ++i) {
        const int in_unit = ((int)(blockIdx.x % J::BLOCKS) * J::TIMES + i) * J::EACH + threadIdx.x / J::COLS, row = unit % p.row_groups * ROWS + in_unit;
        if (row >= p.group * p.n) return;
        const float2 *stats = reinterpret_cast<const float2 *>(p.part + (int64_t)p.splits * 2 * ROWS * D) + in_unit;
        float m = kLowest, sum = 0.f;
        f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int run = from; run <= to; ++run) {
            const int64_t place = 2 * run + (run == from ? begun : 0);
            const float2 st = stats[place * ROWS];
            const f32x4 y = *reinterpret_cast<const f32x4 *>(p.part + (place * ROWS + in_unit) * D + col * 4);
            const float now = fmaxf(m, st.x), old = __builtin_amdgcn_exp2f(m - now), by = __builtin_amdgcn_exp2f(st.x - now);
            sum = lowered(sum, m - now) + lowered(st.y, st.x - now), x = x * old + y * by, m = now;
        }
        const int h = kh * p.group + row / p.n;
        Tile<T, D>::store4(const_cast<char *>(p.b.at) + b * p.b.b + h * p.b.h + (int64_t)(row % p.n) * p.b.row + col * 4 * (int)sizeof(T), x * (sum == 0.f ? 0.f : 1.f / sum));
    }
}

template <typename T, int D, int CAP> struct TreeTile {
    template <int RB> static hipError_t launch(const CacheArgs &a, hipStream_t st) {
        constexpr int lds = 4 * Tile<f16_t, D>::BYTES;
        static LdsAllowed allowed;
        if (hipError_t e = allow_lds(tree_tile_kernel<T, D, RB, CAP>, lds, allowed); e != hipSuccess) return e;
        tree_tile_kernel<T, D, RB, CAP><<<(unsigned)a.splits, kThreads, lds, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        const int64_t joins = (int64_t)a.B * a.kv * a.row_groups * Joined<D, RB>::BLOCKS;
        if (!launch_holds(joins, kThreads)) return hipErrorInvalidValue;
        tree_join_kernel<T, D, RB><<<(unsigned)joins, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    static hipError_t go(const CacheArgs &a, hipStream_t st) {
        const int rb = tree_row_blocks(a, D);
        if constexpr (D < 128 || CAP != kTanhCap)
            if (rb == 3) return launch<3>(a, st);
        return rb == 1 ? launch<1>(a, st) : launch<2>(a, st);
    }
};

}  // namespace

// Blocks of 16 rows to a wave: those for which rows' work, and what a tile takes besides, is least.
int tree_row_blocks(const CacheArgs &a, int D) {
    int best = 1;
    double least = 0;
    for (int rb = 1; rb <= (D < 128 || !a.tanh ? 3 : 2); ++rb) {   // (the library's tanh and three blocks of 128 channels do not fit the registers)
        const int groups = (a.group * a.n + 64 * rb - 1) / (64 * rb);
        const double time = groups * (rb + 0.6);
        if (rb == 1 || time < least) best = rb, least = time;
    }
    return best;
}
// Two workgroups to each compute unit, fewer where the table has less work for them.
void plan_tree_tiles(CacheArgs &a, int64_t longest, int D) {
    const int rows = 64 * tree_row_blocks(a, D);
    a.row_groups = (a.group * a.n + rows - 1) / rows;
    const int64_t reach = longest < (int64_t)a.window + kTile ? longest : (int64_t)a.window + kTile;
    const double tiles = (double)a.B * a.kv * a.row_groups * ((reach + kTile - 1) / kTile + 1), wanted = tiles / kLeastRun;
    a.splits = wanted < 1 ? 1 : wanted < 512 ? (int)wanted : 512;
}
size_t tree_tile_bytes(const CacheArgs &a, int D) { return (size_t)a.splits * 2 * 64 * tree_row_blocks(a, D) * (D + 2) * sizeof(float); }

hipError_t launch_tree_tiles(const CacheArgs &a, int dtype, int D, int cap, hipStream_t st) {
#define SEQ_D(T, N) (cap == kNoCap ? TreeTile<T, N, kNoCap>::go(a, st) : cap == kSigmoidCap ? TreeTile<T, N, kSigmoidCap>::go(a, st) : TreeTile<T, N, kTanhCap>::go(a, st))
#define SEQ_T(T) (D == 32 ? SEQ_D(T, 32) : D == 64 ? SEQ_D(T, 64) : SEQ_D(T, 128))
    return dtype == NA2D_F16 ? SEQ_T(f16_t) : SEQ_T(bf16_t);
#undef SEQ_T
#undef SEQ_D
}

}  // namespace seq
