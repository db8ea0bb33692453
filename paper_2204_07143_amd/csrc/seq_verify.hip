// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
//   p = softmax(logits / T);  a token is drawn by u: the lowest t with p_0 + .. + p_t > u
//   tree: at each node a token is drawn from its p, and the walk goes on at the child that has it
//   line with the draft's q: token x is accepted if u q(x) < p(x), else one is drawn from max(p - q, 0)
//
// The answers are whole numbers that sums over a long row decide, so all of it is in 64 bits: in fp32, with 2^-24 of error in each of 131072 partial sums, one draw in a hundred would
// be another token.  Rows are read in parts of a few thousand logits, a workgroup each, that leave maximum and sum; a second launch finds the part in which a draw falls,
// and reads that part once more to find the token (tree: at every node at once; line: the parts' sums of max(p - q, 0) first); a last one walks.
#include "seq_verify.hpp"

namespace seq {

namespace {

constexpr float kMost = 3.402823466e38f;

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
    __device__ static __forceinline__ float value(T x) {
        const float y = (float)x;
        return y != y ? -INFINITY : fminf(y, kMost);
    }
    __device__ __forceinline__ float at(int token) const { return value(reinterpret_cast<const T *>(base)[shift + token]); }
};

// e^((x - most) / T), 0 of -inf
__device__ __forceinline__ double weight(float x, float most, double by) { return x == -INFINITY ? 0.0 : exp(((double)x - (double)most) * by); }

struct Temperature {
    bool greedy;
    double by;
    __device__ __forceinline__ Temperature(const VerifyArgs &p, int b) {
        const float t = p.temperatures ? p.temperatures[b] : 1.f;
        greedy = !(t > 0.f);
        by = greedy ? 0.0 : 1.0 / (double)t;
    }
};
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

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void stats_kernel(const VerifyArgs p) {
    using R = Row<T>;
    __shared__ double sums[kWaves];
    __shared__ float mosts[kWaves];
    __shared__ int firsts[kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int part = (int)(blockIdx.x % (unsigned)p.parts);
    int64_t row = blockIdx.x / (unsigned)p.parts;
    PartStats *to = p.stats + row * p.parts + part;
    const bool of_draft = row >= (int64_t)p.B * p.n;
    if (of_draft) row -= (int64_t)p.B * p.n;
    const int rows = of_draft ? p.n - 1 : p.n, b = (int)(row / rows), i = (int)(row % rows);
    const R r(of_draft ? p.draft + b * p.draft_batch + i * p.draft_row : p.logits + b * p.batch + i * p.row, p.V);
    const Temperature t(p, b);
    typename R::vec raw[U];
#pragma unroll
    for (int j = 0; j < U; ++j) raw[j] = r.read(part * kThreads * U + j * kThreads + tid);
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < R::E; ++e) most = fmaxf(most, R::value(raw[j][e]));
    most = wave_max(most);
    if (lane == 0) mosts[wave] = most;
    workgroup_sync();
    most = fmaxf(fmaxf(mosts[0], mosts[1]), fmaxf(mosts[2], mosts[3]));
    double sum = 0.0;
    int first = INT32_MAX;
    if (t.greedy) {
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < R::E; ++e)
                if (R::value(raw[j][e]) == most) first = min(first, r.first(part * kThreads * U + j * kThreads + tid) + e);
        first = wave_min(first);
        if (lane == 0) firsts[wave] = first;
    } else {
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < R::E; ++e) sum += weight(R::value(raw[j][e]), most, t.by);
        sum = wave_sum(sum);
        if (lane == 0) sums[wave] = sum;
    }
    workgroup_sync();
    if (tid == 0) *to = t.greedy ? PartStats{0.0, most, min(min(firsts[0], firsts[1]), min(firsts[2], firsts[3]))} : PartStats{(sums[0] + sums[1]) + (sums[2] + sums[3]), most, 0};
}

// A row's maximum, where it is first, and the sum of its weights, from its parts: by a wave.
struct RowStats {
    float most;
    int at;
    double sum;
    __device__ __forceinline__ RowStats(const PartStats *s, int parts, const Temperature &t, int lane) : most(-INFINITY), at(INT32_MAX), sum(0.0) {
        for (int k = lane; k < parts; k += kWave) most = fmaxf(most, s[k].most);
        most = wave_max(most);
        if (t.greedy) {
            for (int k = lane; k < parts; k += kWave)
                if (s[k].most == most) at = min(at, s[k].at);
            at = most == -INFINITY ? -1 : wave_min(at);
        } else {
            for (int k = lane; k < parts; k += kWave) sum += s[k].sum * weight(s[k].most, most, t.by);
            sum = wave_sum(sum);
        }
    }
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

// The token of part `part` at which the running sum of `of`(token, the chunk's element) passes target: by a workgroup, all threads of which get it.  read(chunk): prepares a
// chunk; of(e): the weight of its element e.
template <typename T, int U, class Read> __device__ __forceinline__ int find_token(const Row<T> &r, int part, double before, double target, Read weights) {
    constexpr int E = Row<T>::E;
    __shared__ double totals[kWaves];
    __shared__ int found[kWaves], lasts[kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, chunk = (part * kThreads + tid) * U;
    double w[U][E], sum = 0.0;
#pragma unroll
    for (int j = 0; j < U; ++j) {
        weights(chunk + j, w[j]);
#pragma unroll
        for (int e = 0; e < E; ++e) sum += w[j][e];
    }
    const double to = wave_scan(sum, lane);
    if (lane == kWave - 1) totals[wave] = to;
    workgroup_sync();
    double ahead = before;
    for (int k = 0; k < wave; ++k) ahead += totals[k];
    const double mine = __shfl_up(to, 1);
    double run = lane ? ahead + mine : ahead;
    int token = -1, last = -1;
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            run += w[j][e];
            if (w[j][e] > 0.0) {
                last = r.first(chunk + j) + e;
                if (token < 0 && run > target) token = last;
            }
        }
    const uint64_t passed = __ballot(token >= 0), there = __ballot(last >= 0);
    const int first_token = __shfl(token, passed ? __builtin_ctzll(passed) : 0), last_token = __shfl(last, there ? 63 - __builtin_clzll(there) : 0);
    if (lane == 0) found[wave] = passed ? first_token : -1, lasts[wave] = there ? last_token : -1;
    workgroup_sync();
    int best = -1, end = -1;
    for (int k = kWaves - 1; k >= 0; --k) {
        if (found[k] >= 0) best = found[k];
        if (end < 0) end = lasts[k];
    }
    return best >= 0 ? best : end;
}

// Tree: the token drawn at each node, a workgroup each.
template <typename T, int U>
__global__ __launch_bounds__(kThreads) void draw_kernel(const VerifyArgs p) {
    __shared__ double shared[3];
    __shared__ int shared_part;
    const int tid = threadIdx.x, lane = tid % kWave, b = (int)(blockIdx.x / (unsigned)p.n), i = (int)(blockIdx.x % (unsigned)p.n);
    const PartStats *stats = p.stats + (int64_t)blockIdx.x * p.parts;
    const Temperature t(p, b);
    if (tid < kWave) {
        const RowStats s(stats, p.parts, t, lane);
        double before = 0.0, target = 0.0;
        int part = t.greedy ? s.at : -1;
        if (!t.greedy) {
            target = number(p.uniforms[blockIdx.x]) * s.sum;
            part = find_part([&](int k) { return stats[k].sum * weight(stats[k].most, s.most, t.by); }, p.parts, target, lane, before);
        }
        if (lane == 0) shared[0] = before, shared[1] = target, shared[2] = s.most, shared_part = part;
    }
    workgroup_sync();
    int token = shared_part;
    if (!t.greedy && token >= 0) {
        const Row<T> r(p.logits + b * p.batch + i * p.row, p.V);
        const float most = (float)shared[2];
        token = find_token<T, U>(r, token, shared[0], shared[1], [&](int chunk, double (&w)[Row<T>::E]) {
            const auto x = r.read(chunk);
#pragma unroll
            for (int e = 0; e < Row<T>::E; ++e) w[e] = weight(Row<T>::value(x[e]), most, t.by);
        });
    }
    if (tid == 0) p.drawn[blockIdx.x] = token;
}

// Tree: from node 0 on, a wave to a sequence, a node to a lane.
__global__ __launch_bounds__(kWave) void walk_kernel(const VerifyArgs p) {
    const int lane = threadIdx.x, b = blockIdx.x;
    const int64_t at = (int64_t)b * p.n + lane;
    const bool there = lane < p.n;
    const int parent = !there ? -2 : p.parents ? p.parents[at] : lane - 1, token = there ? p.tokens[at] : -1, drawn = there ? p.drawn[at] : -1;
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

// Line: how many of a sequence's nodes are accepted, and how the next token is drawn, by a wave; every wave that asks comes to the same answer.
template <typename T> struct Line {
    int last;          // the node that the line ends at
    bool residual;     // a token was refused there
    __device__ __forceinline__ Line(const VerifyArgs &p, const PartStats *target, const PartStats *draft, int b, const Temperature &t, int lane) : last(p.n - 1), residual(false) {
        for (int i = 0; i < p.n - 1; ++i) {
            const int x = p.tokens[(int64_t)b * p.n + i + 1];
            if ((unsigned)x >= (unsigned)p.V) {
                last = i;
                return;
            }
            const RowStats s(target + (int64_t)i * p.parts, p.parts, t, lane);
            bool taken = x == s.at;
            if (!t.greedy) {
                const RowStats q(draft + (int64_t)i * p.parts, p.parts, t, lane);
                const double px = s.sum > 0.0 ? weight(Row<T>(p.logits + b * p.batch + i * p.row, p.V).at(x), s.most, t.by) / s.sum : 0.0;
                const double qx = q.sum > 0.0 ? weight(Row<T>(p.draft + b * p.draft_batch + i * p.draft_row, p.V).at(x), q.most, t.by) / q.sum : 0.0;
                taken = number(p.uniforms[(int64_t)b * (p.n + 1) + i]) * qx < px;
            }
            if (!taken) {
                last = i, residual = true;
                return;
            }
        }
    }
};

// p and max(p - q, 0) of a chunk of the row that a line ends at
template <typename T> struct Rest {
    Row<T> r, d;
    float most, most_d;
    double over, over_d, by;   // over_d 0: nothing is taken off
    __device__ __forceinline__ void operator()(int chunk, double (&w)[Row<T>::E]) const {
        const auto x = r.read(chunk);
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e) w[e] = weight(Row<T>::value(x[e]), most, by) * over;
        if (over_d == 0.0) return;
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e) {
            const int token = r.first(chunk) + e;
            if (token >= 0 && token < r.V) w[e] = fmax(w[e] - weight(d.at(token), most_d, by) * over_d, 0.0);
        }
    }
};

// Line: the parts' sums of what the next token is drawn from (part 0 leaves path and count).  A workgroup to a part.
template <typename T, int U, bool LOCATE>
__global__ __launch_bounds__(kThreads) void line_kernel(const VerifyArgs p) {
    constexpr int E = Row<T>::E;
    __shared__ double shared[6], sums[kWaves];
    __shared__ int state[2];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, b = LOCATE ? (int)blockIdx.x : (int)(blockIdx.x / (unsigned)p.parts), part = LOCATE ? 0 : (int)(blockIdx.x % (unsigned)p.parts);
    const PartStats *target = p.stats + (int64_t)b * p.n * p.parts, *draft = p.stats + ((int64_t)p.B * p.n + (int64_t)b * (p.n - 1)) * p.parts;
    const Temperature t(p, b);
    if (tid < kWave) {
        const Line<T> line(p, target, draft, b, t, lane);
        const RowStats s(target + (int64_t)line.last * p.parts, p.parts, t, lane);
        double most_d = 0.0, over_d = 0.0;
        if (line.residual && !t.greedy) {
            const RowStats q(draft + (int64_t)line.last * p.parts, p.parts, t, lane);
            most_d = q.most, over_d = q.sum > 0.0 ? 1.0 / q.sum : 0.0;
        }
        if (lane == 0) {
            state[0] = line.last, state[1] = t.greedy ? s.at : 0;
            shared[0] = s.most, shared[1] = s.sum > 0.0 ? 1.0 / s.sum : 0.0, shared[2] = most_d, shared[3] = over_d;
        }
    }
    workgroup_sync();
    const int last = state[0];
    if (!LOCATE && part == 0) {
        for (int i = tid; i < p.n; i += kThreads) p.path[(int64_t)b * p.n + i] = i <= last ? i : -1;
        if (tid == 0) p.counts[b] = last + 1;
    }
    if (t.greedy) {
        if (LOCATE && tid == 0) p.next[b] = state[1];
        return;
    }
    Rest<T> rest{Row<T>(p.logits + b * p.batch + last * p.row, p.V), Row<T>(p.n > 1 ? p.draft + b * p.draft_batch + min(last, p.n - 2) * p.draft_row : p.logits, p.V), (float)shared[0], (float)shared[2], shared[1],
                 shared[3], t.by};
    if constexpr (!LOCATE) {
        double sum = 0.0;
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
        if (tid == 0) p.rest[(int64_t)b * p.parts + part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    } else {
        if (tid < kWave) {
            const double *parts = p.rest + (int64_t)b * p.parts;
            double all = 0.0, before;
            for (int k = lane; k < p.parts; k += kWave) all += parts[k];
            all = wave_sum(all);
            const bool left = all > 0.0;   // else p and q are one
            const PartStats *stats = target + (int64_t)last * p.parts;
            const float most = (float)shared[0];
            const double over = shared[1], u = number(p.uniforms[(int64_t)b * (p.n + 1) + p.n]), to = u * (left ? all : over > 0.0 ? 1.0 : 0.0);
            const int found = find_part([&](int k) { return left ? parts[k] : stats[k].sum * weight(stats[k].most, most, t.by) * over; }, p.parts, to, lane, before);
            if (lane == 0) state[1] = found, shared[4] = before, shared[5] = to, shared[3] = left ? shared[3] : 0.0;
        }
        workgroup_sync();
        rest.over_d = shared[3];
        const int token = state[1] < 0 ? -1 : find_token<T, U>(rest.r, state[1], shared[4], shared[5], rest);
        if (tid == 0) p.next[b] = token;
    }
}

template <typename T, int U> hipError_t verify(const VerifyArgs &a, hipStream_t st) {
    const int64_t rows = (int64_t)a.B * (a.drafted ? 2 * a.n - 1 : a.n);
    stats_kernel<T, U><<<(unsigned)(rows * a.parts), kThreads, 0, st>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (a.drafted) {
        line_kernel<T, U, false><<<(unsigned)(a.B * a.parts), kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        line_kernel<T, U, true><<<(unsigned)a.B, kThreads, 0, st>>>(a);
    } else {
        draw_kernel<T, U><<<(unsigned)(a.B * a.n), kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        walk_kernel<<<(unsigned)a.B, kWave, 0, st>>>(a);
    }
    return hipGetLastError();
}
template <typename T> hipError_t verify(const VerifyArgs &a, hipStream_t st) { return a.unroll == 1 ? verify<T, 1>(a, st) : verify<T, 4>(a, st); }

}  // namespace

// Parts of 4 chunks a thread, or of one where that leaves compute units without work.
void plan_verify(VerifyArgs &a, int dtype) {
    const int E = dtype == NA2D_F32 ? 4 : 8;
    const int64_t chunks = ((int64_t)a.V + 2 * (E - 1)) / E, rows = (int64_t)a.B * (a.drafted ? 2 * a.n - 1 : a.n);
    const auto parts = [&](int unroll) { return (chunks + (int64_t)kThreads * unroll - 1) / ((int64_t)kThreads * unroll); };
    a.unroll = rows * parts(4) < 512 ? 1 : 4;
    a.parts = (int)parts(a.unroll);
}
hipError_t launch_verify(const VerifyArgs &a, int dtype, hipStream_t st) {
    return dtype == NA2D_F32 ? verify<float>(a, st) : dtype == NA2D_F16 ? verify<f16_t>(a, st) : verify<bf16_t>(a, st);
}

}  // namespace seq
