// Attention of a few new tokens over a cache in 8 bits.
//
// The rows of a key head, its query heads times the new tokens, are columns of the products, 16 to a block; tokens come in steps of 32.  A wave
// takes every fourth step of its workgroup's range, straight from memory into registers, the next step's keys on their way from the moment that
// one's are used, and its values likewise:
//   S^T = K Q^T     a byte b enters as fp16: (b ^ 0x80) behind the byte 0x64 is 1152 + b, exactly; the page's scale multiplies the sums
//   P = exp2(S' - ref), rounded to fp16
//   O^T += vs V^T P  a lane holds D / 16 channels of its eight tokens; product block db takes channel db of each lane, so no value changes lanes
// The four waves' parts are joined through LDS.  Few sequences: their ranges are split over workgroups, and a second kernel joins the splits in order.
//
// Bound by memory where there is much to read: 64 sequences of up to 16000 tokens, 32 heads over 8, D 128, capped, 1.25 GB in 231 us with the join, 5.4 of the 5.7 TB/s that a
// large read reaches.  Short ranges are bound by what follows on each other: about 4 us to the first step and behind the last, 0.85 us a step of a wave (1.25 with 32 rows), two launches.
// 16 sequences with a window of 2048 and 5 tokens each, 16 heads over 2: 15 + 4 us (reads two steps ahead 16, 48 rows to a workgroup 18, 256 tokens a split 15).
#pragma once

#include "seq_cache.hpp"

namespace seq {

namespace {

constexpr int kStep = 32;
constexpr float kSlack = 8.f;

__device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }
__device__ __forceinline__ uint32_t minus1152(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) - f16x2{(f16_t)1152.f, (f16_t)1152.f}); }
// bytes 0, 1 and bytes 2, 3 of four (each ^ 0x80) as fp16
__device__ __forceinline__ uint32_t low_pair(uint32_t x) { return minus1152(perm(0x64646464u, x, 0x04010400u)); }
__device__ __forceinline__ uint32_t high_pair(uint32_t x) { return minus1152(perm(0x64646464u, x, 0x04030402u)); }

template <int D> struct Shape {
    static constexpr int STEPS = D / 32;     // products over the head vector
    static constexpr int DB = D / 16;        // channels of a lane's values, blocks of 16 channels
};

// A step's bytes: two blocks of 16 keys, lane (j, g) 8 bytes of row j for each product step; of the values, channels DB j .. of the tokens 4 g + e of both blocks.
// STREAM: the bytes are read once in the call, and need not stay in the caches (64 sequences of 9000 tokens, 8 x 128: 254 us / 243; where row groups read them again, 40 rows: 24.5 / 25.9)
template <bool STREAM, typename W> __device__ __forceinline__ W read(const int8_t *at) {
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const W *>(at));
    else return *reinterpret_cast<const W *>(at);
}
typedef uint32_t w2 __attribute__((ext_vector_type(2)));

template <int D, bool STREAM> struct Keys {
    uint32_t k[2][2 * (D / 32)];
    __device__ static __forceinline__ unsigned offset(int lane) { return (unsigned)((lane & 15) * D + (lane >> 4) * (D >= 64 ? 16 : 8)); }
    __device__ __forceinline__ void load(int i, const int8_t *block, unsigned of) {
        if constexpr (D >= 64) {   // 16 bytes: two product steps
#pragma unroll
            for (int u = 0; u < D / 64; ++u) {
                const u32x4 x = read<STREAM, u32x4>(block + of + u * 64);
#pragma unroll
                for (int e = 0; e < 4; ++e) k[i][4 * u + e] = x[e];
            }
        } else {
            const w2 x = read<STREAM, w2>(block + of);
            k[i][0] = x[0], k[i][1] = x[1];
        }
    }
    // of block i for product step s
    __device__ __forceinline__ u32x4 get(int i, int s) const {
        const uint32_t x = k[i][2 * s] ^ 0x80808080u, y = k[i][2 * s + 1] ^ 0x80808080u;
        return u32x4{low_pair(x), high_pair(x), low_pair(y), high_pair(y)};
    }
};
template <int D, bool STREAM> struct Values {
    uint32_t v[8][D >= 64 ? D / 64 : 1];
    __device__ static __forceinline__ unsigned offset(int lane) { return (unsigned)((lane >> 4) * 4 * D + (lane & 15) * (D / 16)); }
    __device__ __forceinline__ void load(int i, const int8_t *block, unsigned of) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int8_t *at = block + of + e * D;
            if constexpr (D == 128) {
                const w2 x = read<STREAM, w2>(at);
                v[4 * i + e][0] = x[0], v[4 * i + e][1] = x[1];
            } else if constexpr (D == 64) {
                v[4 * i + e][0] = read<STREAM, uint32_t>(at);
            } else {
                v[4 * i + e][0] = read<STREAM, uint16_t>(at);
            }
        }
    }
    // channel db of the eight tokens
    __device__ __forceinline__ u32x4 get(int db) const {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = minus1152((perm(v[2 * i + 1][db / 4], v[2 * i][db / 4], 0x0c000c00u | (uint32_t)(db % 4) | (uint32_t)(db % 4 + 4) << 16) ^ 0x00800080u) | 0x64006400u);
        return r;
    }
};

// ---- a tree of nodes behind the cache ---------------------------------------------------------------------------------------

constexpr int kNodes = 64;   // at most: a node's ancestors are bits of a word

// The nodes of a sequence: of each itself and its ancestors (0: no node), and how many it has above it.
struct Tree {
    uint64_t above[kNodes];
    int depth[kNodes];
    // By the first wave, a node to a lane: after six rounds a lane has looked 64 nodes up.
    __device__ __forceinline__ void build(const int *parents, int n, int tid) {
        if (tid >= kWave) return;
        int at = tid < n ? parents[tid] : -2;
        bool bad = at != -1 && (at < 0 || at >= tid);
        at = bad ? -1 : at;
        uint64_t mine = 1ull << tid;
#pragma unroll
        for (int round = 0; round < 6; ++round) {
            const int from = at < 0 ? tid : at;
            const uint64_t theirs = (uint64_t)(uint32_t)__shfl((int)(uint32_t)mine, from) | (uint64_t)(uint32_t)__shfl((int)(uint32_t)(mine >> 32), from) << 32;
            const bool their_bad = __shfl((int)bad, from);
            const int next = __shfl(at, from);
            if (at >= 0) mine |= theirs, bad |= their_bad, at = next;
        }
        above[tid] = bad ? 0 : mine;
        depth[tid] = __builtin_popcountll(mine) - 1;
    }
    // the nodes that node i sees
    __device__ __forceinline__ uint64_t seen(int i, int window) const {
        uint64_t all = above[i];
        if (depth[i] >= window)
            for (uint64_t left = all; left; left &= left - 1) {
                const int k = __builtin_ctzll(left);
                if (depth[i] - depth[k] >= window) all &= ~(1ull << k);
            }
        return all;
    }
};

// Values of nodes that are infinite or no numbers, which would reach the rows that do not see them as 0 times them.  Products have 0 in their place; for each channel the nodes
// with such a value are bits, and rows that see one get what it is.
template <int D> struct Wild {
    uint64_t up[D], down[D];   // infinite; no numbers: both
    int any;
    __device__ __forceinline__ void clear(int tid) {
        for (int d = tid; d < D; d += kThreads) up[d] = down[d] = 0;
        if (tid == 0) any = 0;
    }
    // w: the node's values from `channel` on, two to a word; true where it is changed
    template <typename T, class Words> __device__ __forceinline__ bool take(Words &w, int count, int node, int channel) {
        constexpr uint32_t kStep = __is_same(T, f16_t) ? 0x04000400u : 0x00800080u;   // of the exponent
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < count; ++i) bad |= ((w[i] & 0x7fff7fffu) + kStep) & 0x80008000u;
        if (!bad) return false;
        any = 1;
#pragma unroll
        for (int i = 0; i < count; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t x = w[i] >> 16 * half;
                if (!(((x & 0x7fffu) + (kStep & 0xffffu)) & 0x8000u)) continue;
                const bool number = !(x & 0x7fffu & ~(0x8000u - (kStep & 0xffffu))), minus = x & 0x8000u;
                if (!number || !minus) atomicOr((unsigned long long *)&up[channel + 2 * i + half], 1ull << node);
                if (!number || minus) atomicOr((unsigned long long *)&down[channel + 2 * i + half], 1ull << node);
                w[i] &= 0xffffu << 16 * (1 - half);
            }
        return true;
    }
    __device__ __forceinline__ float of(float x, int channel, uint64_t seen) const {
        const bool plus = up[channel] & seen, minus = down[channel] & seen;
        return plus && minus ? NAN : plus ? INFINITY : minus ? -INFINITY : x;
    }
};

// The nodes' own part of a row's attention, 16 keys to a wave, products in the type of q.  In bfloat16 weights are the sum of two of them, 2^-17 off at most: no less exact than
// the cache's, in fp16.
template <typename T, int D, int RT, int CAP>
__device__ __forceinline__ void attend_nodes(const CacheArgs &p, const Tree &tree, Wild<D> &wild, int b, int kh, int row0, int wave, int lane, const float (&slope)[RT], f32x4 (&out)[RT][D / 16], float (&ref)[RT],
                                             float (&sum)[RT]) {
    constexpr int STEPS = D / 32, DB = D / 16;
    const int j = lane & 15, g = lane >> 4, all_rows = p.group * p.n, key = min(16 * wave + j, p.n - 1);
    if (16 * wave >= p.n) return;
    u32x4 k[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) k[s] = *reinterpret_cast<const u32x4 *>(p.tk.at + b * p.tk.b + kh * p.tk.h + (int64_t)key * p.tk.row + (32 * s + 8 * g) * 2);
    uint32_t v[4][DB / 2];   // channels DB j .. of the keys 4 g + e; zeros of what is no node, which may be anything
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int at = 16 * wave + 4 * g + e;
        const bool there = at < p.n && tree.above[at];
        const uint32_t *from = reinterpret_cast<const uint32_t *>(p.tv.at + b * p.tv.b + kh * p.tv.h + (int64_t)min(at, p.n - 1) * p.tv.row + DB * j * 2);
#pragma unroll
        for (int i = 0; i < DB / 2; ++i) v[e][i] = there ? from[i] : 0u;
        wild.template take<T>(v[e], DB / 2, at, DB * j);
    }
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        const int row = min(row0 + 16 * n + j, all_rows - 1), h = kh * p.group + row / p.n, i = row % p.n;
        const char *at = p.a.at + b * p.a.b + h * p.a.h + (int64_t)i * p.a.row;
        f32x4 products[1] = {{0.f, 0.f, 0.f, 0.f}}, &s = products[0];
#pragma unroll
        for (int st = 0; st < STEPS; ++st) s = mma<T>(k[st], *reinterpret_cast<const u32x4 *>(at + (32 * st + 8 * g) * 2), s);
        settle_products(products);
        const uint64_t seen = tree.above[i] >> (16 * wave + 4 * g);
        float most = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float x = s[r] * p.c;
            if constexpr (CAP == kTanhCap) x = 0.5f * p.cap * tanhf(0.5f * kLn2 * x);
            else if constexpr (CAP == kSigmoidCap) x = __builtin_fmaf(-p.cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x)), 0.5f * p.cap);
            const int far = tree.depth[i] - tree.depth[min(16 * wave + 4 * g + r, kNodes - 1)];
            x = __builtin_fmaf((float)far, -slope[n], x);
            s[r] = (seen >> r & 1) && far < p.window ? x : -INFINITY;
            most = fmaxf(most, s[r]);
        }
        most = column_max(most);
        ref[n] = fmaxf(most, kLowest);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] - ref[n]);
            sum[n] += s[r];
        }
        typedef T t2 __attribute__((ext_vector_type(2)));
        typedef float f2 __attribute__((ext_vector_type(2)));
        uint32_t w[2], rest[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{s[2 * e], s[2 * e + 1]}, t2));
            if constexpr (__is_same(T, bf16_t)) rest[e] = pack_remainders(w[e], s[2 * e], s[2 * e + 1]);
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const uint32_t sel = db % 2 ? 0x07060302u : 0x05040100u;
            const uint32_t a0 = perm(v[1][db / 2], v[0][db / 2], sel), a1 = perm(v[3][db / 2], v[2][db / 2], sel);
            out[n][db] = mfma_16x16x16<T>(a0, a1, w[0], w[1], out[n][db]);
            if constexpr (__is_same(T, bf16_t)) out[n][db] = mfma_16x16x16<T>(a0, a1, rest[0], rest[1], out[n][db]);
        }
    }
}

// TREE: the rows are nodes of a tree (p.parents) that stand behind the cache, at its length plus their depth, and the last part of a row's work is the nodes' own.
template <typename T, int D, int RT, int CAP, bool PAGE16, bool TREE>
__global__ __launch_bounds__(kThreads, RT == 1 ? 3 : 2) void decode_kernel(const CacheArgs p) {
    using S = Shape<D>;
    constexpr int ROWS = 16 * RT;
    __shared__ __align__(16) float parts[kWaves][16][D + 4];
    __shared__ float refs[kWaves][ROWS], sums[kWaves][ROWS];
    __shared__ __align__(16) char tree_at[TREE ? sizeof(Tree) : 16];
    __shared__ __align__(16) char wild_at[TREE ? sizeof(Wild<D>) : 16];
    Tree &tree = *reinterpret_cast<Tree *>(tree_at);
    Wild<D> &wild = *reinterpret_cast<Wild<D> *>(wild_at);
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), j = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int split = id % p.splits;
    id /= p.splits;
    const int rg = id % p.row_groups;
    id /= p.row_groups;
    const int kh = id % p.kv, b = id / p.kv, page = PAGE16 ? 16 : 1 << p.page_log2;
    const int all_rows = p.group * p.n, row0 = rg * ROWS;
    const int64_t most_tokens = (int64_t)p.width << p.page_log2;
    const int tokens = TREE ? min(max(p.lengths[b], 0), INT32_MAX - kNodes) : max(p.lengths[b], 0), length = (int)min((int64_t)tokens, most_tokens);
    const int first_query = TREE ? tokens : tokens - p.n, ranges = TREE ? p.splits - 1 : p.splits;
    if constexpr (TREE) {
        tree.build(p.parents + (int64_t)b * p.n, p.n, tid);
        wild.clear(tid);
        workgroup_sync();
    }

    // rows as fp16 on a power of two of their own
    u32x4 q[RT][S::STEPS];
    int pos[RT];
    float c[RT], slope[RT];
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        const int row = min(row0 + 16 * n + j, all_rows - 1), h = kh * p.group + row / p.n, i = row % p.n;
        const char *at = p.a.at + b * p.a.b + h * p.a.h + (int64_t)i * p.a.row;
        pos[n] = first_query + (TREE ? tree.depth[i] : i);
        slope[n] = p.slopes ? p.slopes[h] * kLog2e : 0.f;
        typedef T vec __attribute__((ext_vector_type(8)));
        vec x[S::STEPS];
        float most = 0.f;
#pragma unroll
        for (int s = 0; s < S::STEPS; ++s) {
            const int channel = D >= 64 ? s / 2 * 64 + g * 16 + s % 2 * 8 : g * 8;
            x[s] = *reinterpret_cast<const vec *>(at + channel * (int)sizeof(T));
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)x[s][e]));
        }
        most = column_max(most);
        const int power = most > 0.f && most < INFINITY ? __builtin_amdgcn_frexp_expf(most) : 0;
        c[n] = __builtin_amdgcn_ldexpf(p.c, power);   // (bfloat16's power may be 128: 2^128 alone is infinite)
#pragma unroll
        for (int s = 0; s < S::STEPS; ++s) {
            f16x8 y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (f16_t)__builtin_amdgcn_ldexpf((float)x[s][e], -power);
            q[n][s] = __builtin_bit_cast(u32x4, y);
        }
    }

    // the range that any row sees, in steps, and this workgroup's part of it
    const int least = max(0, first_query - p.window + 1), begin = least / kStep, end = (length + kStep - 1) / kStep;   // least: the first position that is seen
    const int each = max(0, (end - begin + ranges - 1) / ranges), from = begin + split * each, to = min(end, from + each);

    f32x4 out[RT][S::DB];
    float ref[RT], sum[RT];
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        ref[n] = kLowest, sum[n] = 0.f;
#pragma unroll
        for (int db = 0; db < S::DB; ++db) out[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // A lane looks up one of the wave's next 64 steps: its pages (two where they are of 16 tokens) and their scales.  Where there is none it reads the first
    // entry, or the first page's scales, and takes nothing from them: without branches the reads are on their way together.  Of a step's two pages one may hold
    // no token that is seen: its entry and its scale may be anything (a weight of 0 times a scale that is NaN would be NaN), and it is none.
    if constexpr (TREE)
        if (split == ranges) attend_nodes<T, D, RT, CAP>(p, tree, wild, b, kh, row0, wave, lane, slope, out, ref, sum);
    constexpr int PAGES = PAGE16 ? 2 : 1;
    int unit[PAGES];
    float ks[PAGES], vs[PAGES];
    auto look_up = [&](int step) {
#pragma unroll
        for (int i = 0; i < PAGES; ++i) {
            const int64_t token = (int64_t)step * kStep + 16 * i;
            const bool seen = step < to && token < length && (!PAGE16 || token + 16 > least);   // (what is seen is in the table: length is)
            const int page_id = p.table[(int64_t)b * p.width + (seen ? token >> (PAGE16 ? 4 : p.page_log2) : 0)];
            unit[i] = seen && (unsigned)page_id < (unsigned)p.pages ? page_id : -1;
        }
#pragma unroll
        for (int i = 0; i < PAGES; ++i) {
            const int64_t u = (int64_t)max(unit[i], 0) * p.kv + kh;
            const float k = p.ks[u], v = p.vs[u];
            ks[i] = unit[i] < 0 ? 0.f : k, vs[i] = unit[i] < 0 ? 0.f : v;
        }
    };
    auto cell_of = [&](int step, int slot, int i) {   // in bytes; of what is no page: of page 0
        const int u = __builtin_amdgcn_readlane(unit[i % PAGES], slot);
        return (((int64_t)max(u, 0) * p.kv + kh) * page + ((step * kStep + 16 * i) & (page - 1))) * D;
    };
    auto scale_of = [&](const float (&x)[PAGES], int slot, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x[i % PAGES]), slot)); };

    const unsigned key_at = Keys<D, RT == 1>::offset(lane), value_at = Values<D, RT == 1>::offset(lane);
#pragma unroll 1
    for (int base = from + wave; base < to; base += kWave * kWaves) {
        look_up(base + lane * kWaves);
        const int steps = min(kWave, (to - base + kWaves - 1) / kWaves);
        Keys<D, RT == 1> keys;
        Values<D, RT == 1> values;
#pragma unroll
        for (int i = 0; i < 2; ++i) keys.load(i, p.k + cell_of(base, 0, i), key_at);
        asm volatile("" ::: "memory");   // (keys first: they are waited for first)
#pragma unroll
        for (int i = 0; i < 2; ++i) values.load(i, p.v + cell_of(base, 0, i), value_at);
#pragma unroll 1
        for (int at = 0; at < steps; ++at) {
            const int step = base + at * kWaves, t0 = step * kStep;
            f32x4 s[RT][2];
#pragma unroll
            for (int n = 0; n < RT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) s[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < S::STEPS; ++st)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x4 a = keys.get(i, st);
#pragma unroll
                    for (int n = 0; n < RT; ++n) s[n][i] = mma<f16_t>(a, q[n][st], s[n][i]);
                }
            // The next keys, while this step's weights and values are worked on.  Without a branch: behind one, the compiler would wait for the values, which are
            // read last, before it takes the keys.  Behind the last step all lanes read one place of the step that they have.
            const bool more = at + 1 < steps;
            const int slot = more ? at + 1 : at, ahead = base + slot * kWaves;
            const unsigned in_block = more ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i < 2; ++i) keys.load(i, p.k + cell_of(ahead, slot, i), key_at & in_block);
            const bool there[2] = {__builtin_amdgcn_readlane(unit[0], at) >= 0, __builtin_amdgcn_readlane(unit[PAGES - 1], at) >= 0};
            // every row sees all of it
            const bool all = there[0] && there[1] && (TREE ? t0 + kStep <= length : t0 + kStep - 1 <= first_query) && first_query + p.n - 1 - t0 < p.window;
            u32x4 w[RT];
#pragma unroll
            for (int n = 0; n < RT; ++n) {
                float most = -INFINITY;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float by = c[n] * scale_of(ks, at, i);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float x = s[n][i][r] * by;
                        if constexpr (CAP == kTanhCap) x = 0.5f * p.cap * tanhf(0.5f * kLn2 * x);
                        else if constexpr (CAP == kSigmoidCap) x = __builtin_fmaf(-p.cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x)), 0.5f * p.cap);
                        s[n][i][r] = x;
                    }
                }
                if (p.slopes) {
                    const float near = (float)(pos[n] - t0 - 4 * g);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][i][r] = __builtin_fmaf(near - (float)(16 * i + r), -slope[n], s[n][i][r]);
                }
                if (!all) {
                    uint64_t seen = bits_between(pos[n] - p.window + 1 - t0, (TREE ? length : pos[n] + 1) - t0);
                    seen &= (there[0] ? 0xffffull : 0ull) | (there[1] ? 0xffff0000ull : 0ull);
                    seen >>= 4 * g;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][i][r] = keep(s[n][i][r], seen, 16 * i + r, -INFINITY);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) most = fmaxf(most, s[n][i][r]);
                most = column_max(most);
                const float now = most > ref[n] + kSlack ? most : ref[n];
                if (__any(now != ref[n])) {
                    const float by = __builtin_amdgcn_exp2f(ref[n] - now);
                    sum[n] *= by;
#pragma unroll
                    for (int db = 0; db < S::DB; ++db) out[n][db] *= by;
                    ref[n] = now;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[n][i][r] = __builtin_amdgcn_exp2f(s[n][i][r] - ref[n]);
                        sum[n] += s[n][i][r];
                    }
                w[n] = pack<f16_t>(s[n]);
            }
            const float v0 = scale_of(vs, at, 0), v1 = scale_of(vs, at, 1);
            if constexpr (PAGE16) {   // the two blocks have scales of their own
#pragma unroll
                for (int db = 0; db < S::DB; ++db) {
                    u32x4 a = values.get(db);
                    asm volatile("" : "+v"(a));
#pragma unroll
                    for (int n = 0; n < RT; ++n) {
                        const f32x4 zero{0.f, 0.f, 0.f, 0.f};
                        const f32x4 x = mfma_16x16x16<f16_t>(a[0], a[1], w[n][0], w[n][1], zero), y = mfma_16x16x16<f16_t>(a[2], a[3], w[n][2], w[n][3], zero);
#pragma unroll
                        for (int r = 0; r < 4; ++r) out[n][db][r] = __builtin_fmaf(y[r], v1, __builtin_fmaf(x[r], v0, out[n][db][r]));
                        asm volatile("" : "+v"(out[n][db]));   // (in turn: all the products' sums at once would not fit the registers)
                    }
                }
            } else {
#pragma unroll
                for (int db = 0; db < S::DB; ++db) {
                    u32x4 a = values.get(db);
                    asm volatile("" : "+v"(a));
#pragma unroll
                    for (int n = 0; n < RT; ++n) {
                        const f32x4 x = mma<f16_t>(a, w[n], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r) out[n][db][r] = __builtin_fmaf(x[r], v0, out[n][db][r]);
                        asm volatile("" : "+v"(out[n][db]));
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) values.load(i, p.v + cell_of(ahead, slot, i), value_at & in_block);
        }
    }

    // the four waves' parts, then this workgroup's
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        settle_products(out[n]);
        if constexpr (TREE) {
            if (!tree.above[min(row0 + 16 * n + j, all_rows - 1) % p.n]) {   // no node, whatever its query is
                ref[n] = kLowest, sum[n] = 0.f;
#pragma unroll
                for (int db = 0; db < S::DB; ++db) out[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        const float total = column_sum(sum[n]);
        if (g == 0) refs[wave][16 * n + j] = ref[n], sums[wave][16 * n + j] = total;
    }
    const int64_t unit_rows = (int64_t)ROWS, item = (((int64_t)b * p.kv + kh) * p.row_groups + rg) * p.splits + split;
    const int64_t items = (int64_t)p.B * p.kv * p.row_groups * p.splits;
    float *part = p.part + item * unit_rows * D, *stats = p.part + items * unit_rows * D + item * unit_rows * 2;
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        workgroup_sync();   // (also before parts are written again)
        float most = refs[0][16 * n + j];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) most = fmaxf(most, refs[w][16 * n + j]);
        const float by = __builtin_amdgcn_exp2f(ref[n] - most);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int db = 0; db < S::DB; ++db) parts[wave][j][S::DB * (4 * g + r) + db] = out[n][db][r] * by;
        workgroup_sync();
        for (int i = tid; i < 16 * D / 8; i += kThreads) {
            const int r = i / (D / 8), d = i % (D / 8) * 8, row = row0 + 16 * n + r;
            if (row >= all_rows) continue;
            float m = refs[0][16 * n + r], total = 0.f;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) m = fmaxf(m, refs[w][16 * n + r]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) total += sums[w][16 * n + r] * __builtin_amdgcn_exp2f(refs[w][16 * n + r] - m);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = parts[0][r][d + e] + parts[1][r][d + e] + parts[2][r][d + e] + parts[3][r][d + e];
            if constexpr (TREE)
                if (wild.any) {
                    const uint64_t seen = tree.seen(row % p.n, p.window);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = wild.of(x[e], d + e, seen);
                }
            if (p.splits == 1) {
                const float by_sum = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= by_sum;
                const int h = kh * p.group + row / p.n;
                store_vec32<T, 8>(const_cast<char *>(p.b.at) + b * p.b.b + h * p.b.h + (int64_t)(row % p.n) * p.b.row + d * (int)sizeof(T), x);
            } else {
                store_vec32<float, 8>(part + (16 * n + r) * D + d, x);
                if (d == 0) stats[2 * (16 * n + r)] = m, stats[2 * (16 * n + r) + 1] = total;
            }
        }
    }
}

// The splits of a row: a workgroup per row, a thread per four channels of every kThreads * 4 / D-th split, then those in order.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const CacheArgs p, int rows_each) {
    constexpr int COLS = D / 4, PARTS = kThreads / COLS;
    __shared__ __align__(16) f32x4 sums[PARTS][COLS];
    __shared__ float2 stat[PARTS];
    const int all_rows = p.group * p.n, col = threadIdx.x % COLS, part = threadIdx.x / COLS;
    const int row = (int)(blockIdx.x % all_rows), plane = (int)(blockIdx.x / all_rows), b = plane / p.kv, kh = plane % p.kv;
    const int64_t items = (int64_t)p.B * p.kv * p.row_groups * p.splits, first = (((int64_t)plane * p.row_groups + row / rows_each) * p.splits) * rows_each + row % rows_each;
    const float2 *stats = reinterpret_cast<const float2 *>(p.part + items * rows_each * D) + first;
    float m = kLowest, sum = 0.f;
    f32x4 x{0.f, 0.f, 0.f, 0.f};
    for (int s = part; s < p.splits; s += PARTS) {
        const float2 st = stats[s * rows_each];
        const f32x4 y = *reinterpret_cast<const f32x4 *>(p.part + (first + (int64_t)s * rows_each) * D + col * 4);
        const float now = fmaxf(m, st.x), old = __builtin_amdgcn_exp2f(m - now), by = __builtin_amdgcn_exp2f(st.x - now);
        m = now, sum = sum * old + st.y * by, x = x * old + y * by;
    }
    sums[part][col] = x;
    if (col == 0) stat[part] = float2{m, sum};
    workgroup_sync();
    if (part) return;
    for (int s = 1; s < PARTS && s < p.splits; ++s) m = fmaxf(m, stat[s].x);
    sum = 0.f, x = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < PARTS && s < p.splits; ++s) {
        const float by = __builtin_amdgcn_exp2f(stat[s].x - m);
        sum += stat[s].y * by;
        x += sums[s][col] * by;
    }
    const int h = kh * p.group + row / p.n;
    Tile<T, D>::store4(const_cast<char *>(p.b.at) + b * p.b.b + h * p.b.h + (int64_t)(row % p.n) * p.b.row + col * 4 * (int)sizeof(T), x * (sum == 0.f ? 0.f : 1.f / sum));
}

inline int rows_each(const CacheArgs &a) { return a.group * a.n > 16 ? 32 : 16; }

}  // namespace

}  // namespace seq
