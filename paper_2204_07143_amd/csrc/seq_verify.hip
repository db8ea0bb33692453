// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
//   p = softmax(logits / T);  a token is drawn by u: the lowest t with p_0 + .. + p_t > u
//   tree: at each node a token is drawn from its p, and the walk goes on at the child that has it
//   line with the draft's q: token x is accepted if u q(x) < p(x), else one is drawn from max(p - q, 0)
//
// The answers are whole numbers that sums over a long row decide, so all of it is in 64 bits: in fp32, with 2^-24 of error in each of 131072 partial sums, one draw in a hundred would
// be another token.  Rows are read in parts of a few thousand logits, a wave each, that leave maximum and sum.  Tree: the last workgroup of a row finds the part in which its
// draw falls, and reads that part once more to find the token; the last row of a sequence walks.  Line: a second launch finds where the line ends, takes the parts' sums of
// max(p - q, 0) there, and its last workgroup draws from them.
//
// The floor is reading the logits once; an element's 14 instructions in 64 bits and about as many others are 60 % of the cycles, and at the end of a row comes the latency of the last workgroup.  16 x 48 rows of 131072,
// bf16: 90 us (2.2 TB/s) and 4.6 for the tickets' zeros; 130 with the library's exponential and rows' draws in launches of their own.  24 lines of 8 in fp32, 50021: 22 + 16; one of 6 in fp16,
// 32000: 5 + 11, dependent reads.
#include "seq_verify.hpp"

namespace seq {

namespace {

constexpr int kChunks = 4;   // of 16 bytes that a lane reads at a time

// A row's logits in aligned chunks of 16 bytes, element 0 somewhere in the first; -inf for what lies outside the row, and for what is no number.
template <typename T> struct Row {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    const char *base;
    int shift, V;   // shift: elements of the first chunk in front of the row
    __device__ __forceinline__ Row(const char *at, int V_) : base(reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(at) & ~(uintptr_t)15)), shift((int)((uintptr_t)at & 15) / (int)sizeof(T)), V(V_) {}
    __device__ __forceinline__ int first(int chunk) const { return chunk * E - shift; }
    __device__ __forceinline__ vec read(int chunk) const {
        const int at = first(chunk);
        vec x;
        if (at >= 0 && at + E <= V) {
            x = *reinterpret_cast<const vec *>(base + (int64_t)chunk * 16);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = at + e >= 0 && at + e < V ? reinterpret_cast<const T *>(base + (int64_t)chunk * 16)[e] : (T)-INFINITY;
        }
        return x;
    }
    static constexpr float kTop = sizeof(T) == 4 ? 0x1.fffffep127f : __is_same(T, f16_t) ? 65504.f : 0x1.fep127f;   // the largest finite value
    __device__ static __forceinline__ float value(T x) {
        return fminf(fmaxf((float)x, -INFINITY), kTop);   // (the larger of a NaN and another is the other)
    }
    __device__ __forceinline__ T raw(int token) const { return token >= 0 && token < V ? reinterpret_cast<const T *>(base)[shift + token] : (T)-INFINITY; }
    __device__ __forceinline__ float at(int token) const { return value(reinterpret_cast<const T *>(base)[shift + token]); }
};

// The bits of 2^(k / 32), less k 2^47: with n 2^47 added, n = k modulo 32, they are those of 2^(n / 32)
__device__ const uint64_t kRoots[32] = {
    0x3ff0000000000000, 0x3fefd9b0d3158574, 0x3fefb5586cf9890f, 0x3fef9301d0125b51, 0x3fef72b83c7d517b, 0x3fef54873168b9aa,
    0x3fef387a6e756238, 0x3fef1e9df51fdee1, 0x3fef06fe0a31b715, 0x3feef1a7373aa9cb, 0x3feedea64c123422, 0x3feece086061892d,
    0x3feebfdad5362a27, 0x3feeb42b569d4f82, 0x3feeab07dd485429, 0x3feea47eb03a5585, 0x3feea09e667f3bcd, 0x3fee9f75e8ec5f74,
    0x3feea11473eb0187, 0x3feea589994cce13, 0x3feeace5422aa0db, 0x3feeb737b0cdc5e5, 0x3feec49182a3f090, 0x3feed503b23e255d,
    0x3feee89f995ad3ad, 0x3feeff76f2fb5e47, 0x3fef199bdd85529c, 0x3fef3720dcef9069, 0x3fef5818dcfba487, 0x3fef7c97337b9b5f,
    0x3fefa4afa2a490da, 0x3fefd0765b6e4540};

// e^((x - most) / T) in 64 bits, 0 where x is -inf or no number: a table of roots and a short polynomial, as P. T. P. Tang has it (Table-driven implementation of the exponential function in
// IEEE floating-point arithmetic, ACM Transactions on Mathematical Software 15, 1989); the number added to round is 1.5 2^52, whose last place is 1.  With y = 32 (x - most) log2(e) / T, n the whole number next to it and f = y - n:
// 2^(n / 32) from a table and the exponent, 2^(f / 32) as its Taylor polynomial of degree 5, off by (ln 2 / 64)^6 / 720 < 2^-48; y's own rounding is 2^-53 of it.  y is held at
// 32 times -1023, where the exponent's bits, and with them the weight, are 0 (down from 2^-1022 weights are no longer exact).  14 instructions in 64 bits an
// element; the table's entries lie in different banks of the LDS.
struct Weights {
    double by;                // 32 log2(e) / T
    const uint64_t *roots;    // in LDS
    __device__ __forceinline__ double operator()(float x, double most) const {
        constexpr double kWhole = 0x1.8p52;
        const double y = fmax(((double)x - most) * by, -32736.0), m = y + kWhole, f = y - (m - kWhole);
        const double r = __builtin_fma(f, __builtin_fma(f, __builtin_fma(f, __builtin_fma(f, __builtin_fma(f, 0x1.5d87fe78a6731p-35, 0x1.3b2ab6fba4e77p-27), 0x1.c6b08d704a0c0p-20), 0x1.ebfbdff82c58fp-13), 0x1.62e42fefa39efp-6), 1.0);
        const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, m);
        const uint2 root = reinterpret_cast<const uint2 *>(roots)[n & 31];
        const uint64_t whole = (uint64_t)(root.y + ((uint32_t)n << 15)) << 32 | root.x;
        return r * __builtin_bit_cast(double, whole);
    }
};

struct Temperature {
    bool greedy;
    Weights weight;
    __device__ __forceinline__ Temperature(const VerifyArgs &p, int b, const uint64_t *roots) {
        const float t = p.temperatures ? p.temperatures[b] : 1.f;
        greedy = !(t > 0.f);
        // (an infinite T makes all weights 1, but those of -inf)
        weight = {greedy ? 0.0 : fmax(32 * 1.4426950408889634074 / (double)t, 1e-290), roots};
    }
};
__device__ __forceinline__ void load_roots(uint64_t *roots) {
    if (threadIdx.x < 32) roots[threadIdx.x] = kRoots[threadIdx.x];
}
__device__ __forceinline__ double number(float u) { return u >= 1.f ? 1.0 - 0x1p-24 : u > 0.f ? (double)u : 0.0; }

__device__ __forceinline__ double shuffle(double x, int from) { return __shfl(x, from); }
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ double wave_scan(double x, int lane) {   // sums up to this lane
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const double y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// A part's statistics, by a wave.  A lane keeps a maximum and a sum of its own over the blocks, the next block's reads on their way while one is worked on.
template <typename T, int BLOCKS> __device__ __forceinline__ PartStats part_stats(const Row<T> &r, int part, const Temperature &t, int lane) {
    using R = Row<T>;
    constexpr int U = kChunks;
    typename R::vec raw[U], next[U];
    const int chunk = part * (kWave * U * BLOCKS) + lane;
    if (r.first(chunk - lane) >= r.V) return {0.0, -INFINITY, INT32_MAX};   // (parts are counted for the worst alignment)
#pragma unroll
    for (int j = 0; j < U; ++j) raw[j] = r.read(chunk + j * kWave);
    float most = -INFINITY;
    double sum = 0.0;
    int first = INT32_MAX;
#pragma unroll 1
    for (int block = 0; block < BLOCKS; ++block) {
        if (block + 1 < BLOCKS) {
#pragma unroll
            for (int j = 0; j < U; ++j) next[j] = r.read(chunk + ((block + 1) * U + j) * kWave);
        }
        float now = most;
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < R::E; ++e) now = fmaxf(now, R::value(raw[j][e]));
        if (__any(now == R::kTop)) {
#pragma unroll
            for (int j = 0; j < U; ++j)
#pragma unroll
                for (int e = 0; e < R::E; ++e)
                    if ((float)raw[j][e] == INFINITY) raw[j][e] = (T)R::kTop;
        }
        if (t.greedy) {
            if (now > most) {
#pragma unroll
                for (int j = U - 1; j >= 0; --j)
#pragma unroll
                    for (int e = R::E - 1; e >= 0; --e) first = (float)raw[j][e] == now ? r.first(chunk + (block * U + j) * kWave) + e : first;
            }
        } else {
            const double from = now;
            sum *= t.weight(most, from);   // (0 while there is none)
#pragma unroll
            for (int j = 0; j < U; ++j) {
#pragma unroll
                for (int e = 0; e < R::E; ++e) sum += t.weight((float)raw[j][e], from);   // (a NaN weighs nothing)
                asm volatile("" : "+v"(sum));   // (a chunk after the other: the registers)
            }
        }
        most = now;
        if (block + 1 < BLOCKS) {
#pragma unroll
            for (int j = 0; j < U; ++j) raw[j] = next[j];
        }
    }
    const float all = wave_max(most);
    if (t.greedy) return {0.0, all, wave_min(most == all ? first : INT32_MAX)};
    return {wave_sum(sum * t.weight(most, all)), all, 0};
}

// What one workgroup leaves for another of the same launch: stores that go through to memory and loads that come from there, whichever compute unit's caches lie between
// (instead of fences, which write back and invalidate whole caches: 12288 of them took 450 us).
template <typename V> __device__ __forceinline__ void leave(V *to, V x) { __hip_atomic_store(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V> __device__ __forceinline__ V take(const V *from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void leave(PartStats *to, const PartStats &x) {
    leave(&to->sum, x.sum);
    leave(reinterpret_cast<uint64_t *>(&to->most), (uint64_t)__float_as_uint(x.most) | (uint64_t)(uint32_t)x.at << 32);
}
__device__ __forceinline__ PartStats take(const PartStats *from) {
    const double sum = take(&from->sum);
    const uint64_t rest = take(reinterpret_cast<const uint64_t *>(&from->most));
    return {sum, __uint_as_float((uint32_t)rest), (int)(uint32_t)(rest >> 32)};
}

// Counts the workgroups that came here, each after what it leaves; true in all threads of the last of `all`.  Whoever is last, the work it does is the same.
__device__ __forceinline__ bool last_of(int *ticket, int all) {
    __shared__ int mine;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // a wave's stores have arrived
    workgroup_sync();
    if (threadIdx.x == 0) {
        mine = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    workgroup_sync();
    return mine == all - 1;
}

// A row's maximum, where it is first, and the sum of its weights, from its parts: by LANES lanes.  SAME: the parts were left in this launch.
template <int LANES, bool SAME> struct RowStats {
    float most;
    int at;
    double sum;
    double mine;   // what this lane's first part has of the sum
    __device__ __forceinline__ RowStats(const PartStats *s, int parts, const Temperature &t, int lane) : most(-INFINITY), at(INT32_MAX), sum(0.0), mine(0.0) {
        PartStats first{0.0, -INFINITY, INT32_MAX};
        if (lane < parts) first = get(s + lane);
        most = first.most;
        for (int k = lane + LANES; k < parts; k += LANES) most = fmaxf(most, get(s + k).most);
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        if (t.greedy) {
            if (first.most == most) at = first.at;
            for (int k = lane + LANES; k < parts; k += LANES) {
                const PartStats x = get(s + k);
                if (x.most == most) at = min(at, x.at);
            }
#pragma unroll
            for (int d = 1; d < LANES; d *= 2) at = min(at, __shfl_xor(at, d));
            if (most == -INFINITY) at = -1;
        } else if (most > -INFINITY) {
            sum = mine = share(first, t);
            for (int k = lane + LANES; k < parts; k += LANES) sum += share(get(s + k), t);
        }
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
    }
    __device__ static __forceinline__ PartStats get(const PartStats *s) { return SAME ? take(s) : *s; }
    __device__ __forceinline__ double share(const PartStats &x, const Temperature &t) const { return x.sum * t.weight(x.most, most); }
};

// The part in which the running sum of `of`(part) passes `target`, and the sum before it: by a wave.  Where none does (rounding), the last that has any; -1: none has.
template <class F> __device__ __forceinline__ int find_part(F of, int parts, double target, int lane, double &before) {
    double run = 0.0;
    int last = -1;
    before = 0.0;
    for (int base = 0; base < parts; base += kWave) {
        const double w = base + lane < parts ? of(base + lane) : 0.0, to = run + wave_scan(w, lane);
        const uint64_t there = __ballot(w > 0.0), passed = there & __ballot(to > target);
        const double ahead = __shfl_up(to, 1);
        if (there) {
            const int k = passed ? __builtin_ctzll(passed) : 63 - __builtin_clzll(there);
            last = base + k;
            const double x = shuffle(ahead, k);
            before = k ? x : run;
        }
        if (passed) break;
        run = shuffle(to, kWave - 1);
    }
    return last;
}

// The token of part `part` at which the running sum passes target, before + what the part has up to it: by a workgroup, all threads of which get it.  weights(chunk, w) gives a chunk's
// weights, weights(token) one.  A thread sums U chunks; those of the thread in which it happens are then looked at one by one, an element to a lane.
template <typename T, int U, class Weigh> __device__ __forceinline__ int find_token(const Row<T> &r, int part, double before, double target, const Weigh &weights) {
    constexpr int E = Row<T>::E;
    static_assert(U * E <= kWave, "an element to a lane");
    __shared__ double totals[kWaves], ahead_of[kWaves];
    __shared__ int found[kWaves], lasts[kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < U; ++j) {
        double w[E];
        weights((part * kThreads + tid) * U + j, w);
#pragma unroll
        for (int e = 0; e < E; ++e) sum += w[e];
        asm volatile("" : "+v"(sum));   // (a chunk after the other: the registers)
    }
    const double to = wave_scan(sum, lane);
    if (lane == kWave - 1) totals[wave] = to;
    workgroup_sync();
    double ahead = before;
    for (int k = 0; k < wave; ++k) ahead += totals[k];
    const uint64_t there = __ballot(sum > 0.0), passed = there & __ballot(ahead + to > target);
    const int who = passed ? __builtin_ctzll(passed) : there ? 63 - __builtin_clzll(there) : 0;
    const double up_to = shuffle(to, max(who - 1, 0));
    if (lane == 0) found[wave] = passed ? tid + who : -1, lasts[wave] = there ? tid + who : -1, ahead_of[wave] = who ? ahead + up_to : ahead;
    workgroup_sync();
    int best = -1;
    for (int k = kWaves - 1; k >= 0; --k)
        if (found[k] >= 0) best = found[k];
    if (best < 0)   // (rounding: none does; the last that has any)
        for (int k = 0; k < kWaves; ++k)
            if (lasts[k] >= 0) best = lasts[k];
    if (best < 0) return -1;
    const int token = r.first((part * kThreads + best) * U) + lane;
    const double w = lane < U * E && token >= 0 && token < r.V ? weights(token) : 0.0, run = ahead_of[best / kWave] + wave_scan(w, lane);
    const uint64_t some = __ballot(w > 0.0), over = some & __ballot(run > target);
    return some ? token - lane + (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some)) : -1;
}

// A row's weights
template <typename T> struct Plain {
    const Row<T> &r;
    double most;
    const Weights &weight;
    __device__ __forceinline__ void operator()(int chunk, double (&w)[Row<T>::E]) const {
        const auto x = r.read(chunk);
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e) w[e] = weight(Row<T>::value(x[e]), most);
    }
    __device__ __forceinline__ double operator()(int token) const { return weight(r.at(token), most); }
};

// Zeros: the tickets of a tree's rows and sequences.
__global__ __launch_bounds__(kThreads) void tickets_kernel(int *tickets, int count) {
    const int at = blockIdx.x * kThreads + threadIdx.x;
    if (at < count) tickets[(int64_t)at * kTicket] = 0;
}

// Tree: from node 0 on, by a wave, a node to a lane.
__device__ __forceinline__ void walk(const VerifyArgs &p, int b, int lane) {
    const int64_t at = (int64_t)b * p.n + lane;
    const bool there = lane < p.n;
    const int parent = !there ? -2 : p.parents ? p.parents[at] : lane - 1, token = there ? p.tokens[at] : -1, drawn = there ? take(p.drawn + at) : -1;
    int node = 0, count = 0, mine = -1, next = -1;
    for (int step = 0; step < p.n; ++step) {
        if (lane == step) mine = node;
        count = step + 1;
        next = __shfl(drawn, node);
        const uint64_t child = __ballot(next >= 0 && parent == node && lane > node && token == next);
        if (!child) break;
        node = __builtin_ctzll(child);
    }
    if (there) p.path[at] = mine;
    if (lane == 0) p.counts[b] = count, p.next[b] = next;
}

// Tree: a wave to a part.  A row's last workgroup draws its token, a sequence's last row walks.
template <typename T, int U>
__global__ __launch_bounds__(kThreads) void tree_kernel(const VerifyArgs p) {
    using R = Row<T>;
    __shared__ uint64_t roots[32];
    __shared__ double shared[3];
    __shared__ int shared_part;
    load_roots(roots);
    const int tid = threadIdx.x, lane = tid % kWave, groups = (p.parts + kWaves - 1) / kWaves, part = (int)(blockIdx.x % (unsigned)groups) * kWaves + uniform(tid / kWave);
    const int row = (int)(blockIdx.x / (unsigned)groups), b = row / p.n, i = row % p.n;
    PartStats *stats = p.stats + (int64_t)row * p.parts;
    const R r(p.logits + b * p.batch + i * p.row, p.V);
    const Temperature t(p, b, roots);
    workgroup_sync();
    if (part < p.parts) {
        const PartStats s = part_stats<T, U>(r, part, t, lane);
        if (lane == 0) leave(stats + part, s);
    }
    if (!last_of(p.tickets + (int64_t)row * kTicket, groups)) return;
    if (tid < kWave) {
        const RowStats<kWave, true> s(stats, p.parts, t, lane);
        double before = 0.0, target = 0.0;
        int part = t.greedy ? s.at : -1;
        if (!t.greedy) {
            target = number(p.uniforms[row]) * s.sum;
            part = find_part([&](int k) { return k == lane ? s.mine : s.share(take(stats + k), t); }, p.parts, target, lane, before);
        }
        if (lane == 0) shared[0] = before, shared[1] = target, shared[2] = s.most, shared_part = part;
    }
    workgroup_sync();
    int token = shared_part;
    if (!t.greedy && token >= 0) {
        const double most = shared[2];
        token = find_token<T, U>(r, token, shared[0], shared[1], Plain<T>{r, most, t.weight});
    }
    if (tid == 0) leave(p.drawn + row, token);
    if (last_of(p.tickets + ((int64_t)p.B * p.n + b) * kTicket, p.n) && tid < kWave) walk(p, b, lane);
}

// Line: a part of a row of the target, or of the draft.
template <typename T, int U>
__global__ __launch_bounds__(kThreads) void stats_kernel(const VerifyArgs p) {
    __shared__ uint64_t roots[32];
    load_roots(roots);
    const int lane = threadIdx.x % kWave, groups = (p.parts + kWaves - 1) / kWaves, part = (int)(blockIdx.x % (unsigned)groups) * kWaves + uniform(threadIdx.x / kWave);
    int row = (int)(blockIdx.x / (unsigned)groups);
    PartStats *to = p.stats + (int64_t)row * p.parts + part;
    const bool of_draft = row >= p.B * p.n;
    if (of_draft) row -= p.B * p.n;
    const int rows = of_draft ? p.n - 1 : p.n, b = row / rows, i = row % rows;
    const Row<T> r(of_draft ? p.draft + b * p.draft_batch + i * p.draft_row : p.logits + b * p.batch + i * p.row, p.V);
    const Temperature t(p, b, roots);
    workgroup_sync();
    if (part >= p.parts) return;
    const PartStats s = part_stats<T, U>(r, part, t, lane);
    if (lane == 0) {
        *to = s;
        if (!of_draft && i == 0 && part == 0) p.tickets[(int64_t)b * kTicket] = 0;
    }
}

// What is left of p less q.  Not in one instruction with the product that p comes from: that would leave the product's rounding where p and q are one.
__device__ __forceinline__ double left_of(double p, double q) {
#pragma clang fp contract(off)
    return fmax(p - q, 0.0);
}

// p, less q where a token was refused, of a chunk of the row that a line ends at
template <typename T> struct Rest {
    Row<T> r, d;
    double most, most_d, over, over_d;   // over, over_d: 1 over the sums; over_d 0: nothing is taken off
    Weights weight;
    __device__ __forceinline__ void operator()(int chunk, double (&w)[Row<T>::E]) const {
        const auto x = r.read(chunk);
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e) w[e] = weight(Row<T>::value(x[e]), most) * over;
        if (over_d == 0.0) return;
        typename Row<T>::vec y;
        if (r.shift == d.shift) {
            y = d.read(chunk);
        } else {
#pragma unroll
            for (int e = 0; e < Row<T>::E; ++e) y[e] = d.raw(r.first(chunk) + e);
        }
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e) w[e] = left_of(w[e], weight(Row<T>::value(y[e]), most_d) * over_d);
    }
    __device__ __forceinline__ double operator()(int token) const {
        const double w = weight(r.at(token), most) * over;
        return over_d == 0.0 ? w : left_of(w, weight(d.at(token), most_d) * over_d);
    }
};

// Line: a workgroup to a part of what the next token is drawn from.  Each finds for itself where the line ends, LANES lanes to a row; then the parts' sums; a sequence's last
// workgroup draws.
template <typename T, int U, int LANES>
__global__ __launch_bounds__(kThreads) void line_kernel(const VerifyArgs p) {
    constexpr int E = Row<T>::E;
    __shared__ uint64_t roots[32];
    __shared__ double sums[kWaves], drawn[3], over[64], over_d[64];
    __shared__ float most[64], most_d[64];
    __shared__ int at[64], taken[64], found;   // taken: 1 accepted, 0 refused, -1: no token
    load_roots(roots);
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, b = (int)(blockIdx.x / (unsigned)p.parts), part = (int)(blockIdx.x % (unsigned)p.parts);
    const PartStats *target = p.stats + (int64_t)b * p.n * p.parts, *draft = p.stats + ((int64_t)p.B * p.n + (int64_t)b * (p.n - 1)) * p.parts;
    const Temperature t(p, b, roots);
    workgroup_sync();
    for (int i0 = 0; i0 < p.n; i0 += kThreads / LANES) {
        const int i = min(i0 + tid / LANES, p.n - 1), j = max(min(i, p.n - 2), 0);   // the row, and the draft's
        const bool last_row = i == p.n - 1;
        const int x = last_row ? -1 : p.tokens[(int64_t)b * p.n + i + 1];
        const bool token = (unsigned)x < (unsigned)p.V;
        const double u = number(p.uniforms[(int64_t)b * (p.n + 1) + i]);
        const float xp = token ? Row<T>(p.logits + b * p.batch + i * p.row, p.V).at(x) : -INFINITY, xq = token ? Row<T>(p.draft + b * p.draft_batch + j * p.draft_row, p.V).at(x) : -INFINITY;
        const RowStats<LANES, false> s(target + (int64_t)i * p.parts, p.parts, t, tid % LANES), q(draft + (int64_t)j * p.parts, last_row ? 0 : p.parts, t, tid % LANES);
        if (tid % LANES == 0) {
            // A row's sum differs with its alignment, by less than 2^-43 of it: on either side up to 330 additions of positive numbers (2^24 tokens in fp32), and a few weights in the place
            // of one.  Rows that are one have one sum, so that nothing is left of p less q; q of other rows this near is off by no more than by that rounding.
            const double sum_d = q.most == s.most && fabs(q.sum - s.sum) <= 0x1p-42 * s.sum ? s.sum : q.sum;
            const double os = s.sum > 0.0 ? 1.0 / s.sum : 0.0, oq = sum_d > 0.0 ? 1.0 / sum_d : 0.0;
            most[i] = s.most, most_d[i] = q.most, over[i] = os, over_d[i] = oq, at[i] = s.at;
            const double px = s.sum > 0.0 ? t.weight(xp, s.most) * os : 0.0, qx = sum_d > 0.0 ? t.weight(xq, q.most) * oq : 0.0;
            taken[i] = !token ? -1 : t.greedy ? x == s.at : u * qx < px;
        }
    }
    workgroup_sync();
    const uint64_t ends = __ballot(lane >= p.n - 1 || taken[lane] != 1);
    const int last = __builtin_ctzll(ends);
    if (part == 0) {
        if (tid < p.n) p.path[(int64_t)b * p.n + tid] = tid <= last ? tid : -1;
        if (tid == 0) {
            p.counts[b] = last + 1;
            if (t.greedy) p.next[b] = at[last];
        }
    }
    if (t.greedy) return;
    const bool refused = taken[last] == 0;
    Rest<T> rest{Row<T>(p.logits + b * p.batch + last * p.row, p.V), Row<T>(refused ? p.draft + b * p.draft_batch + last * p.draft_row : p.logits, p.V), (double)most[last],
                 (double)most_d[last], over[last], refused ? over_d[last] : 0.0, t.weight};
    double *parts = p.rest + (int64_t)b * p.parts;
    double sum = 0.0;
    if (rest.over > 0.0)
#pragma unroll
        for (int j = 0; j < U; ++j) {
            double w[E];
            rest(part * kThreads * U + j * kThreads + tid, w);
#pragma unroll
            for (int e = 0; e < E; ++e) sum += w[e];
        }
    sum = wave_sum(sum);
    if (lane == 0) sums[wave] = sum;
    workgroup_sync();
    if (tid == 0) leave(parts + part, (sums[0] + sums[1]) + (sums[2] + sums[3]));
    if (!last_of(p.tickets + (int64_t)b * kTicket, p.parts)) return;
    if (tid < kWave) {
        const double mine = lane < p.parts ? take(parts + lane) : 0.0;
        double all = mine, before;
        for (int k = lane + kWave; k < p.parts; k += kWave) all += take(parts + k);
        all = wave_sum(all);
        const bool left = all > 0.0;   // else p and q are one
        const PartStats *stats = target + (int64_t)last * p.parts;
        const double to = number(p.uniforms[(int64_t)b * (p.n + 1) + p.n]) * (left ? all : rest.over > 0.0 ? 1.0 : 0.0);
        const int k = find_part([&](int k) { return left ? k == lane ? mine : take(parts + k) : rest.over > 0.0 ? stats[k].sum * t.weight(stats[k].most, rest.most) * rest.over : 0.0; }, p.parts, to, lane, before);
        if (lane == 0) found = k, drawn[0] = before, drawn[1] = to, drawn[2] = left ? rest.over_d : 0.0;
    }
    workgroup_sync();
    rest.over_d = drawn[2];
    const int token = found < 0 ? -1 : find_token<T, U>(rest.r, found, drawn[0], drawn[1], rest);
    if (tid == 0) p.next[b] = token;
}

template <typename T, int U> hipError_t verify(const VerifyArgs &a, hipStream_t st) {
    const int groups = (a.parts + kWaves - 1) / kWaves;
    if (a.drafted) {
        stats_kernel<T, U><<<(unsigned)((int64_t)a.B * (2 * a.n - 1) * groups), kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        auto *kernel = a.n <= 4 ? line_kernel<T, U, 64> : a.n <= 8 ? line_kernel<T, U, 32> : line_kernel<T, U, 16>;   // all rows at once, up to 16
        kernel<<<(unsigned)(a.B * a.parts), kThreads, 0, st>>>(a);
    } else {
        const int tickets = a.B * (a.n + 1);
        tickets_kernel<<<(tickets + kThreads - 1) / kThreads, kThreads, 0, st>>>(a.tickets, tickets);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        tree_kernel<T, U><<<(unsigned)((int64_t)a.B * a.n * groups), kThreads, 0, st>>>(a);
    }
    return hipGetLastError();
}
template <typename T> hipError_t verify(const VerifyArgs &a, hipStream_t st) { return a.blocks == 1 ? verify<T, 1>(a, st) : verify<T, 4>(a, st); }

}  // namespace

// Parts of four blocks (two: 98 us for 90 at 16 x 48 rows of 131072, bf16; eight: 106), or of one where that leaves compute units without work (24 lines of 8 in fp32, 50021: 4 us less).  A
// part is kThreads chunks for each of its blocks.
void plan_verify(VerifyArgs &a, int dtype) {
    static_assert(kThreads == kWave * kChunks, "a workgroup that looks for a token in a part gives each thread `blocks` chunks");
    const int E = dtype == NA2D_F32 ? 4 : 8;
    const int64_t chunks = ((int64_t)a.V + 2 * (E - 1)) / E, rows = (int64_t)a.B * (a.drafted ? 2 * a.n - 1 : a.n);
    const auto parts = [&](int blocks) { return (chunks + (int64_t)kThreads * blocks - 1) / ((int64_t)kThreads * blocks); };
    a.blocks = rows * parts(4) < 8192 ? 1 : 4;
    a.parts = (int)parts(a.blocks);
}
hipError_t launch_verify(const VerifyArgs &a, int dtype, hipStream_t st) {
    return dtype == NA2D_F32 ? verify<float>(a, st) : dtype == NA2D_F16 ? verify<f16_t>(a, st) : verify<bf16_t>(a, st);
}

}  // namespace seq
