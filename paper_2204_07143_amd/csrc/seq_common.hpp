// What the kernels of the attention over token sequences share: their arguments, the tiles of 64 tokens that they walk and stage, and the
// fragments that the matrix instructions take.
//
// A head vector of D elements is CH = D sizeof(T) / 16 chunks of 16 bytes.  The 16 x 16 products of na2d_mfma.hpp take one chunk per lane of
// each operand: lane (j = lane % 16, g = lane / 16) holds chunk 4 s + g of row j for step s, and of the sums column j, rows 4 g + r.  In fp32 a
// chunk is four instructions of depth 4 (element e of the lanes' chunks).  Since a lane's four sums of a block of 16 rows are, rounded, the
// chunk (half a chunk in 16 bit) that a product over those rows takes, the weights go from one product to the next in registers.
#pragma once

#include <initializer_list>

#include "na2d_mfma.hpp"
#include "seq.h"

namespace seq {

using namespace na2d;

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;        // tokens staged at a time
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kFar = 1 << 30;    // a window without end
constexpr float kLowest = -1.7e38f;   // start of a running maximum: below every finite score, and not infinite

// A tile of 64 tokens as the masks see it: the range of its documents (of the tokens that are not padding; empty if there are none), and per
// token whether it is there at all and whether it is marked as prefix.
struct Marks {
    int dmin, dmax;
    uint64_t live, prefix;
};

struct View {   // one tensor: byte strides of batch and head, bytes from row to row
    const char *at;
    int64_t b, h;
    int row;
};

struct Args {
    View q, k, v, out, dout, dq, dk, dv;
    char *rest;            // strides of out
    float *lse;
    const float *slopes;
    const int *documents;
    const Marks *marks;    // of every 64 keys, [B, key_tiles]; null: neither documents nor prefix
    const char *zeros;     // 64 bytes of zeros, where marks are
    float2 *rows;          // backward: (lse in base 2, delta) of every query, [B * heads, query_tiles * 64]
    int *powers;           // backward, fp16: per tile of 64 queries the power of two of its largest |dout|, [B * heads, query_tiles], and
    int *value_powers;     // per tile of 64 keys that of its values' largest sum of magnitudes, [B * kv, key_tiles]
    float *parts;          // where work is split: each part's fp32 sums.  queries: [q_splits, B * heads, Lq, D], in the forward pass with float2 (maximum, sum)
                           // [q_splits, B * heads, Lq] behind them; keys: of dK and dV, [k_splits, 2, B * kv, Lk, D]
    int q_splits, k_splits;   // parts that the work on one tile of queries, or of keys, is split into
    int B, heads, kv, group, Lq, Lk, off;   // off: Lk - Lq
    int key_tiles, query_tiles;
    int causal, window;    // window: kFar where there is none
    int prefix, packed;    // marks hold prefix bits, documents
    int dlo;               // smallest distance that the order and the window allow; the largest is window - 1
    float scale;
    float c;               // capped: 2 scale log2(e) / cap
    float m, from;         // a score in base 2 is m y + from (see Score)
    float masked;          // the y of what is masked
};

// ---- products --------------------------------------------------------------------------------------------------------------

template <typename T> __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return mfma_16x16x32<T>(a, b, c);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
}
template <typename T> constexpr int kRowBlocks = sizeof(T) == 2 ? 2 : 1;   // blocks of 16 rows that one chunk of weights spans

// the sums of kRowBlocks blocks as a chunk, rounded to the type (nearest even)
template <typename T> __device__ __forceinline__ u32x4 pack(const f32x4 *s) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(u32x4, s[0]);
    } else {
        typedef T t2 __attribute__((ext_vector_type(2)));
        typedef float f2 __attribute__((ext_vector_type(2)));
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{s[i / 2][i % 2 * 2], s[i / 2][i % 2 * 2 + 1]}, t2));
        return r;
    }
}

// ---- tiles in LDS ----------------------------------------------------------------------------------------------------------
//
// 64 rows of CH chunks, as direct loads leave them (lane l of a load writes 16 bytes at 16 l), chunk c of row r in place c ^ swizzle(r).

template <typename T, int D> struct Tile {
    static constexpr int CH = D * (int)sizeof(T) / 16, ROWB = CH * 16, BYTES = kTile * ROWB;
    static constexpr int STEPS = CH / 4;                        // products over the head vector
    static constexpr int DB = D / 16;                           // blocks of 16 channels
    static constexpr int LOADS = kTile * CH / kThreads;         // of 16 bytes, per thread and image

    // Of the rows r (r0 .. r3 its low bits).  What is read at once is to lie in different banks of 256 bytes: of a row fragment the chunks g of rows 0 .. 3 and
    // 12 .. 15 with the chunks g + 1 of rows 4 .. 11; of a transposed one, pairs of chunks of eight rows in turn.
    __device__ static __forceinline__ int swizzle(int r) {
        const int r0 = r & 1, r1 = r >> 1 & 1, r2 = r >> 2 & 1, r3 = r >> 3 & 1;
        if constexpr (CH >= 16) return (r2 ^ r3) << 3 | r1 << 2 | r0 << 1 | r3;
        else if constexpr (CH == 8) return r1 << 2 | (r2 ^ r3) << 1 | r3;
        else return (r2 ^ r3) << 1 | r3;
    }

    // Rows first .. first + 63 of a plane into the image at `img`; a row past the end is the last one once more, where `zeros` are given, one that is not live is zeros.
    __device__ static __forceinline__ void stage(const char *plane, int pitch, int first, int rows, uint64_t live, const char *zeros, int img, int wave, int lane) {
        static_assert(CH <= kWave, "a row is at most one load");
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = wave + i * kWaves, r = at * (kWave / CH) + lane / CH, c = (lane % CH) ^ swizzle(r);
            const int row = first + r < rows ? first + r : rows - 1;
            const unsigned off = (unsigned)(row * pitch + c * 16);
            if (zeros) {
                const char *g = live >> r & 1 ? plane + off : zeros;
                global_to_lds_16(g, img + at * kWave * 16);
            } else {
                global_to_lds_16(plane, off, img + at * kWave * 16);
            }
        }
    }

    // Row fragments: lane (j, g) reads chunk 4 s + g of row 16 rb + j.
    struct RowReader {
        int at;
        __device__ __forceinline__ RowReader(int lane) : at((lane & 15) * ROWB + ((lane >> 4) ^ swizzle(lane & 15)) * 16) {}
        __device__ __forceinline__ u32x4 read(int img, int rb, int s) const { return *lds_ptr<u32x4>((at ^ (s * 64)) + img + rb * 16 * ROWB); }
    };

    // Transposed fragments: for channels 16 db .. + 15 (the product's rows) a chunk of the positions that pack() has in a lane's chunk of step t.
    struct ColumnReader {
        int at[sizeof(T) == 2 ? 1 : 4];
        __device__ __forceinline__ ColumnReader(int lane) {
            const int j = lane & 15, g = lane >> 4;
            if constexpr (sizeof(T) == 2) {
                const int r = 4 * g + (j >> 2);
                at[0] = r * ROWB + (((j >> 1) & 1) ^ swizzle(r)) * 16 + (j & 1) * 8;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) at[e] = (4 * g + e) * ROWB + ((j >> 2) ^ swizzle(4 * g + e)) * 16 + (j & 3) * 4;
            }
        }
        __device__ __forceinline__ u32x4 read(int img, int t, int db) const {
            if constexpr (sizeof(T) == 2) {
                const int a = (at[0] ^ (db * 32)) + img + t * 32 * ROWB;
                const u32x2 x = lds_read_tr16(a), y = lds_read_tr16(a + 16 * ROWB);
                return u32x4{x.x, x.y, y.x, y.y};
            } else {
                u32x4 r;
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = *lds_ptr<uint32_t>((at[e] ^ (db * 64)) + img + t * 16 * ROWB);
                return r;
            }
        }
    };

    // This lane's chunks of row `row` straight from memory: the other operand of products with row fragments.
    __device__ static __forceinline__ void load_row(u32x4 (&f)[STEPS], const char *plane, int pitch, int row, int lane) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) f[s] = *reinterpret_cast<const u32x4 *>(plane + (int64_t)row * pitch + (4 * s + (lane >> 4)) * 16);
    }
    __device__ static __forceinline__ void negate(u32x4 (&f)[STEPS]) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) f[s] ^= sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
    }
    // zeros in place of a token that is not live
    __device__ static __forceinline__ void clear(u32x4 (&f)[STEPS], bool live) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) f[s] &= live ? ~0u : 0u;
    }
    // Four channels as they are stored.  rest: where what the rounding took goes, as an offset; 0: nowhere
    __device__ static __forceinline__ void store4(char *to, f32x4 x, int64_t rest = 0) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4 *>(to) = x;
        } else {
            typedef T t4 __attribute__((ext_vector_type(4)));
            const t4 y = __builtin_convertvector(x, t4);
            *reinterpret_cast<t4 *>(to) = y;
            if (rest) *reinterpret_cast<t4 *>(to + rest) = __builtin_convertvector(x - __builtin_convertvector(y, f32x4), t4);
        }
    }
    // Sums with channels as rows, [DB] blocks, column `row` of a tensor: four channels of each block.
    __device__ static __forceinline__ void store_row(const f32x4 *acc, float by, char *plane, int pitch, int row, int lane, int64_t rest = 0) {
#pragma unroll
        for (int db = 0; db < DB; ++db) store4(plane + (int64_t)row * pitch + (16 * db + 4 * (lane >> 4)) * (int)sizeof(T), acc[db] * by, rest);
    }
};

// ---- masks -----------------------------------------------------------------------------------------------------------------

// Queries at positions qa .. qb against keys ka .. kb: any pair, or every pair, that order and window allow.
__device__ __forceinline__ bool near_any(const Args &p, int qa, int qb, int ka, int kb) { return qb - ka >= p.dlo && qa - kb < p.window; }
__device__ __forceinline__ bool near_all(const Args &p, int qa, int qb, int ka, int kb) { return qa - kb >= p.dlo && qb - ka < p.window; }

// Bits lo .. hi - 1 of 64, whatever lo and hi.
__device__ __forceinline__ uint64_t bits_between(int lo, int hi) {
    lo = max(0, min(lo, 64)), hi = max(0, min(hi, 64));
    const uint64_t from = lo < 64 ? ~0ull << lo : 0ull, to = hi < 64 ? ~(~0ull << hi) : ~0ull;
    return from & to;
}
// A column's 64 rows of a tile as a mask: this lane's rows 16 rb + 4 g + r are bits 16 rb + r of mask >> 4 g.  Two instructions an element.
__device__ __forceinline__ float keep(float y, uint64_t lane_mask, int bit, float masked) {
    const int word = bit < 32 ? (int)(uint32_t)lane_mask : (int)(uint32_t)(lane_mask >> 32);
    const uint32_t on = (uint32_t)(word << (31 - bit % 32) >> 31);
    return __uint_as_float((__float_as_uint(y) & on) | (__float_as_uint(masked) & ~on));
}

// A range of documents; every token of it being live as well.
struct Docs {
    int lo, hi;
    bool all;
    __device__ __forceinline__ bool meet(const Docs &o) const { return lo <= o.hi && o.lo <= hi; }
    __device__ __forceinline__ bool same(const Docs &o) const { return all && o.all && lo == hi && o.lo == o.hi && lo == o.lo; }
};
__device__ __forceinline__ Docs no_docs() { return {0, 0, true}; }
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) x = min(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) x = max(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// of the wave's tokens; `there` false: no token in this lane
__device__ __forceinline__ Docs docs_of_wave(int d, bool there) {
    const bool live = there && d >= 0;
    Docs r{uniform(wave_min(live ? d : INT32_MAX)), uniform(wave_max(live ? d : -1)), __ballot(there && d < 0) == 0};
    return r;
}

// What of a tile's marks the masks take.
struct Seen {
    int doc;               // the tile's document, if it is one
    bool mixed;            // it is not
    uint64_t live, prefix;
};

// Walks the tiles first .. last that `of` says something about: a lane looks at one tile, 64 at a time.  of(tile, marks) gives bits: 1 any pair of the
// workgroup's is seen, 2 any pair of this wave's, 4 every pair of this wave's.  The first bit must not differ between waves.  The lane keeps its tile's marks:
// read from memory when their tile's turn comes, they would be waited for behind the loads of another tile.
struct Walk {
    uint64_t todo, mine, whole, mixed;
    int doc;
    uint64_t live, prefix;
    int base, last, skip;   // skip: how many of them to leave out before the first
    __device__ __forceinline__ Walk(int first, int last_, int skip_ = 0) : todo(0), mine(0), whole(0), mixed(0), doc(0), live(0), prefix(0), base(first - kWave), last(last_), skip(skip_) {}
    template <class F> __device__ __forceinline__ int next(F of, int lane, bool &is_mine, bool &is_whole, Seen &seen) {
        while (!todo) {
            base += kWave;
            if (base > last) return -1;
            Marks m{0, 0, 0, 0};
            const int bits = base + lane <= last ? of(base + lane, m) : 0;
            doc = m.dmin, live = m.live, prefix = m.prefix;
            todo = __ballot(bits & 1);
            mine = __ballot(bits & 2);
            whole = __ballot(bits & 4);
            mixed = __ballot(m.dmin != m.dmax);
            const int n = __builtin_popcountll(todo), out = min(skip, n);
            skip -= out;
            if (out == n) todo = 0;
            else for (int i = 0; i < out; ++i) todo &= todo - 1;
        }
        const int i = __builtin_ctzll(todo);
        todo &= todo - 1;
        is_mine = mine >> i & 1;
        is_whole = whole >> i & 1;
        seen = {__builtin_amdgcn_readlane(doc, i), (bool)(mixed >> i & 1), lane64(live, i), lane64(prefix, i)};
        return base + i;
    }
    __device__ static __forceinline__ uint64_t lane64(uint64_t x, int i) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, i) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), i) << 32;
    }
    // how many there are
    template <class F> __device__ static __forceinline__ int count(int first, int last, F of, int lane) {
        int n = 0;
        for (int base = first; base <= last; base += kWave) {
            Marks m;
            n += __builtin_popcountll(__ballot(base + lane <= last ? of(base + lane, m) & 1 : 0));
        }
        return n;
    }
};

// blockIdx in an order in which what follows each other runs on the same XCD (consecutive workgroups go to the eight in turn, each has an L2 of its own)
__device__ __forceinline__ int block_in_order() {
    const int n = gridDim.x, each = n / 8, rest = n % 8, x = blockIdx.x % 8;
    return x * each + min(x, rest) + blockIdx.x / 8;
}

// ---- scores ----------------------------------------------------------------------------------------------------------------
//
// A score in base 2 is m y + from (args.m, args.from), less slope |distance|:
//   no cap   y = <q, k>, m = scale log2(e)
//   kSigmoid with z = scale <q, k> / cap and y = 1 / (1 + e^2z): tanh z = 1 - 2 y, so m = -2 cap log2(e), from = cap log2(e), and the score's derivative by
//            the product, 1 - tanh^2, is 4 y (1 - y).  A score of 0 is then off by up to 4 x 2^-24 of the cap, another by up to 8 x 2^-24 = 2^-21 (2^-24 of y for the sum, 2^-23
//            each for the exponential and the reciprocal, y counting twice; the exponent and the score once each);
//   kTanh    takes the library's tanh for y, m = cap log2(e): off by 2^-21 or so of the score itself.  More instructions, so only where the other form is not enough: fp16, 4 x 16 over
//            4 x 2048, D 128, causal, forward 110 us with the sigmoid and 137 with the tanh, backward 371 and 440; 8 x 8192, D 64, 147 and 200, 445 and 571.
// What is masked has a y that gives weights of 0 and, where 1 - tanh^2 is formed from it, something finite.
enum CapForm { kNoCap = 0, kSigmoidCap = 1, kTanhCap = 2 };
// The weights are rounded by half a step of their type, 2^-11 of them in fp16 and 2^-8 in bf16.  2^-21 of the cap is no more than that up to 2^10 in fp16, and half of it
// at 2^12, the largest that is accepted in 16 bit, in bf16.  fp32 always takes the tanh.
inline int cap_form(int weights, float cap) { return cap == 0.f ? kNoCap : weights == NA2D_F32 || (weights == NA2D_F16 && cap > 1024.f) ? kTanhCap : kSigmoidCap; }

template <typename T, int CAP> struct Score {
    static constexpr bool kSigmoid = CAP == kSigmoidCap;
    __device__ static __forceinline__ float of(const Args &p, float s) {
        if constexpr (!CAP) return s;
        else if constexpr (kSigmoid) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * p.c));
        else return tanhf(s * (0.5f * kLn2 * p.c));
    }
    // 1 - tanh^2, over 4 in 16 bit: the weights beside it are formed times 2^kQuad
    static constexpr float kQuad = kSigmoid ? 2.f : 0.f;
    __device__ static __forceinline__ float through(float ds, float y) {
        if constexpr (!CAP) return ds;
        else if constexpr (kSigmoid) return ds * __builtin_fmaf(-y, y, y);
        else return ds * __builtin_fmaf(-y, y, 1.f);
    }
};

// ---- host ------------------------------------------------------------------------------------------------------------------

hipError_t launch_marks(const Args &a, const uint8_t *prefix, Marks *marks, char *zeros, hipStream_t st);
hipError_t launch_fwd(const Args &a, int dtype, int D, int cap, hipStream_t st);   // cap: a CapForm
hipError_t launch_rows(const Args &a, int dtype, int D, int cap, hipStream_t st);
hipError_t launch_bwd_q(const Args &a, int dtype, int D, int cap, hipStream_t st);
hipError_t launch_bwd_kv(const Args &a, int dtype, int D, int cap, hipStream_t st);
int q_splits(const Args &a, int dtype, int D);
int k_splits(const Args &a, int dtype, int D);

// How many parts the work on a tile of queries, or of keys, is split into: the number for which an estimate in units of a tile's time is least.  `units`
// workgroups have `longest` tiles at most, `tiles` on average, and what takes two more before them.  Two workgroups to a compute unit get all it does (four do not
// more).  A join takes `join` tiles, and one for each `each` bytes of the `sums` that every part leaves; they stay below 256 MB.
// Against a fixed number of workgroups (512 to 1024 in all), forward / backward in us: 4 x 12 x 512 fp16, D 64, causal 20.4 / 50 -> 12.6 / 40; 1 x 4 x 8192 fp16, D 64,
// capped 139 / 358 -> 116 / 320; 2 x 8 over 2 x 777 bf16, D 128, 25.5 / 72 -> 19.2 / 62; 2 x 8 x 1500 of 5 documents 22.9 / 59 -> 15.4 / 40; the furthest the other way 4 x 4 x 3136 fp16,
// D 32, not causal 79 / 197 -> 78 / 205 and 1 x 16 x 2048 bf16, D 64 37 / 112 -> 38 / 118, where a round of workgroups does not come out even.
inline int parts_of(int64_t units, double longest, double tiles, double join, int64_t sums, double each) {
    int best = 1;
    double least = 0;
    for (int s = 1; s == 1 || (s <= 32 && s * 4 <= longest && s * sums <= (int64_t)256 << 20); ++s) {
        const double one = longest / s + 2, all = (double)units * (tiles + 2 * s) / 512, time = (one > all ? one : all) + (s > 1 ? join + (double)s * sums / each : 0);
        if (s == 1 || time < least) best = s, least = time;
    }
    return best;
}
// The tiles that a workgroup has at most, and on average, of `all`, with tiles of `rows` of its own: what the window reaches, where no prefix reaches further; half of
// them where there are documents (with a prefix on average only: it is for prompts, which end where the documents do); on average what lies before the middle
// of the queries in causal order.
struct Work {
    double longest, tiles;
    Work(const Args &a, int rows, int all) {
        const int64_t reach = ((int64_t)a.window + rows) / kTile + 2;
        longest = a.prefix || reach > all ? all : (double)reach;
        if (a.packed && !a.prefix) longest = longest > 2 ? longest / 2 : longest;
        tiles = longest * (a.causal && reach > all && a.Lq <= a.Lk ? 1 - 0.5 * a.Lq / a.Lk : 1.0) * (a.packed ? 0.5 : 1.0);
    }
};

// 16 bit: two blocks of 16 queries, or keys, to a wave (a fragment from LDS then serves two products) where that leaves two workgroups to each compute unit; but up
// to 64 channels in causal order, where the work of workgroups differs, one, and the larger number of them.  Forward, us for one / two: 2 x 16 over 4 x 8192, D 128, not
// causal 1462 / 1128; 4 x 16 over 4 x 2048, D 128, capped, causal 143 / 124; 4 x 16 x 2048, D 64, not causal 118 / 108, causal 71 / 79; D 32 76 / 71 and 58 / 70;
// 3 x 6 x 1571, D 64, 234 workgroups of two, 39.2 / 41.5.  Key side, a backward pass: D 64, not causal 308 / 287, causal 226 / 236, capped too 290 / 318.  Long rows are even:
// 16 x 8192, D 64, causal, forward 213 / 230, backward 627 / 606.
inline bool two_blocks(const Args &a, int D, int64_t planes, int rows) { return (D == 128 || !a.causal) && planes * ((rows + 127) / 128) >= 512; }
inline bool two_query_blocks(const Args &a, int D) { return two_blocks(a, D, (int64_t)a.B * a.heads, a.Lq); }

// L<T, D, cap>::go(...) of a type, head dim and form of the cap (one that cap_form() gives for the type)
template <typename T, int D, template <typename, int, int> class L, typename... A> hipError_t dispatch_cap(int cap, A &&...a) {
    if (cap == kNoCap) return L<T, D, kNoCap>::go(a...);
    if constexpr (sizeof(T) == 2)
        if (cap == kSigmoidCap) return L<T, D, kSigmoidCap>::go(a...);
    if constexpr (!__is_same(T, bf16_t)) return L<T, D, kTanhCap>::go(a...);
    return hipErrorInvalidValue;
}
template <template <typename, int, int> class L, typename... A> hipError_t dispatch(int dtype, int D, int cap, A &&...a) {
#define SEQ_T(T) (D == 32 ? dispatch_cap<T, 32, L>(cap, a...) : D == 64 ? dispatch_cap<T, 64, L>(cap, a...) : dispatch_cap<T, 128, L>(cap, a...))
    return dtype == NA2D_F32 ? SEQ_T(float) : dtype == NA2D_F16 ? SEQ_T(f16_t) : SEQ_T(bf16_t);
#undef SEQ_T
}

}  // namespace seq
