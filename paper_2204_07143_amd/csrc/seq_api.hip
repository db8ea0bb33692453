// C ABI of the attention over token sequences and of its cache: argument validation (host only, before any HIP call) and dispatch.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "seq_cache.hpp"
#include "seq_verify.hpp"

namespace seq {
namespace {

int elem(int dtype) { return dtype == NA2D_F32 ? 4 : 2; }
bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
int from_hip(hipError_t e) {
    if (e == hipSuccess) return NA2D_OK;
    (void)hipGetLastError();   // leave no stale error behind for the caller's next HIP call
    return NA2D_ERR_LAUNCH;
}
// strides of a tensor [B, heads, rows, D]: whole multiples of 16 bytes, none negative, a plane below 2^31 bytes, an offset to any plane below 2^60 bytes; of one
// that is written, no two rows in the same place: in order of size, each stride reaches over all that the smaller ones span
int check_strides(const seq_strides &s, int64_t B, int64_t heads, int64_t rows, int64_t D, int e, bool written) {
    for (int64_t x : {s.batch, s.head, s.row}) {
        if (x < 0 || x > ((int64_t)1 << 45)) return NA2D_ERR_SHAPE;
        if (x * e % 16) return NA2D_ERR_ALIGN;
    }
    if (rows > 1 && s.row > (int64_t)INT32_MAX / e / (rows - 1)) return NA2D_ERR_SHAPE;   // (first: the product below would pass 64 bits)
    if (((rows - 1) * s.row + D) * e > (int64_t)INT32_MAX || B > ((int64_t)1 << 24) || heads > ((int64_t)1 << 16)) return NA2D_ERR_SHAPE;
    if ((double)(B - 1) * s.batch + (double)(heads - 1) * s.head > 0x1p58) return NA2D_ERR_SHAPE;
    if (!written) return NA2D_OK;
    struct Dim { int64_t stride, last; } dims[3] = {{s.batch, B - 1}, {s.head, heads - 1}, {s.row, rows - 1}};
    std::sort(dims, dims + 3, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    int64_t span = D;
    for (const Dim &d : dims) {
        if (d.last && d.stride < span) return NA2D_ERR_ALIAS;
        span += d.last * d.stride;
    }
    return NA2D_OK;
}
View view(const void *at, const seq_strides &s, int e) { return {static_cast<const char *>(at), s.batch * e, s.head * e, (int)(s.row * e)}; }

constexpr double kLog2eExact = 1.4426950408889634;
// what <q, k> is multiplied by: to a score in base 2, or to the exponent of e^2z
float base2(float scale, float cap) { return cap > 0.f ? (float)(2.0 * kLog2eExact * scale / cap) : (float)(kLog2eExact * scale); }

int common(int B, int heads, int kv, int D, int dtype, float scale, float cap, int window) {
    if (dtype != NA2D_F32 && dtype != NA2D_F16 && dtype != NA2D_BF16) return NA2D_ERR_DTYPE;
    if (B <= 0 || heads <= 0 || kv <= 0 || heads % kv) return NA2D_ERR_SHAPE;
    if (D != 32 && D != 64 && D != 128) return NA2D_ERR_HEAD_DIM;
    // (a cap's scores are off by up to 2^-21 of it in 16 bit, see cap_form(): at 2^12 that is half of what bf16 weights are rounded by)
    if (cap != 0.f && (cap < 0x1p-20f || (dtype != NA2D_F32 && cap > 4096.f))) return NA2D_ERR_SHAPE;
    if (!std::isfinite(scale) || !std::isfinite(cap) || cap < 0.f || window < 0 || window > kFar) return NA2D_ERR_SHAPE;
    if (!std::isfinite(base2(scale, cap))) return NA2D_ERR_SHAPE;   // (infinite, it would make NaN of products that are 0)
    return NA2D_OK;
}

int validate(const seq_problem *p, bool backward) {
    if (!p) return NA2D_ERR_NULL;
    if (int e = common(p->B, p->heads, p->kv_heads, p->D, p->dtype, p->scale, p->softcap, p->window)) return e;
    if (p->Lq <= 0 || p->Lk <= 0 || p->Lq > 1 << 24 || p->Lk > 1 << 24 || (p->causal != 0 && p->causal != 1)) return NA2D_ERR_SHAPE;
    const int e = elem(p->dtype);
    const auto of_queries = [&](const seq_strides &s, bool written) { return check_strides(s, p->B, p->heads, p->Lq, p->D, e, written); };
    const auto of_keys = [&](const seq_strides &s, bool written) { return check_strides(s, p->B, p->kv_heads, p->Lk, p->D, e, written); };
    for (int r : {of_queries(p->q, false), of_keys(p->k, false), of_keys(p->v, false), of_queries(p->out, true)})
        if (r) return r;
    if (backward)
        for (int r : {of_queries(p->dout, false), of_queries(p->dq, true), of_keys(p->dk, true), of_keys(p->dv, true)})
            if (r) return r;
    // every launch of the passes (the smallest tiles: 64 rows) holds its workgroups
    const int64_t q_tiles = ((int64_t)p->Lq + kTile - 1) / kTile, k_tiles = ((int64_t)p->Lk + kTile - 1) / kTile;
    const int64_t of_q = (int64_t)p->B * p->heads * q_tiles, of_k = (int64_t)p->B * p->kv_heads * k_tiles;
    if (!launch_holds(of_q, kThreads) || !launch_holds(of_k, kThreads) || (backward && p->dtype == NA2D_F16 && !launch_holds(of_q + 1, kThreads))) return NA2D_ERR_SHAPE;
    return NA2D_OK;
}

Args args(const seq_problem *p, const float *slopes, const int32_t *documents, bool packed, bool prefix) {
    Args a{};
    a.slopes = slopes, a.documents = documents;
    a.B = p->B, a.heads = p->heads, a.kv = p->kv_heads, a.group = p->heads / p->kv_heads, a.Lq = p->Lq, a.Lk = p->Lk, a.off = p->Lk - p->Lq;
    a.key_tiles = (p->Lk + kTile - 1) / kTile, a.query_tiles = (p->Lq + kTile - 1) / kTile;
    a.causal = p->causal, a.window = p->window ? p->window : kFar;
    a.dlo = p->causal ? 0 : 1 - a.window;
    a.scale = p->scale;
    if (p->softcap > 0.f) {
        const bool sigmoid = cap_form(p->dtype, p->softcap) == kSigmoidCap;
        a.c = base2(p->scale, p->softcap);
        a.m = (float)((sigmoid ? -2.0 : 1.0) * kLog2eExact * p->softcap), a.from = sigmoid ? (float)(kLog2eExact * p->softcap) : 0.f;
        a.masked = sigmoid ? 1e18f : -1e18f;   // its square is finite, and its weight 0 for every cap from 2^-20 on
    } else {
        a.m = p->scale == 0.f ? 1e-37f : base2(p->scale, 0.f);   // (0 times what is masked would be no number)
        a.masked = a.m > 0.f ? -INFINITY : INFINITY;
    }
    a.packed = packed, a.prefix = prefix;
    a.q_splits = q_splits(a, p->dtype, p->D), a.k_splits = k_splits(a, p->dtype, p->D);
    return a;
}

// The workspace: zeros, the marks of the keys' tiles, and for a backward pass the rows' statistics, the tiles' powers of two and the splits' sums.
struct Space {
    int64_t marks, rows, powers, value_powers, parts, bytes;
    Space(const Args &a, int D, bool marked, bool backward) {
        const int64_t queries = (int64_t)a.B * a.heads * a.query_tiles;
        auto up = [](int64_t x) { return (x + 63) / 64 * 64; };
        marks = marked ? 64 : 0;
        rows = marked ? up(marks + (int64_t)sizeof(Marks) * a.B * a.key_tiles) : 0;
        powers = up(rows + (backward ? (int64_t)sizeof(float2) * queries * kTile : 0));
        value_powers = up(powers + (backward ? (int64_t)sizeof(int) * queries : 0));
        parts = up(value_powers + (backward ? (int64_t)sizeof(int) * a.B * a.kv * a.key_tiles : 0));
        const int64_t of_q = a.q_splits > 1 ? (int64_t)sizeof(float) * a.q_splits * a.B * a.heads * a.Lq * (backward ? D : D + 2) : 0;
        const int64_t of_k = backward && a.k_splits > 1 ? (int64_t)sizeof(float) * a.k_splits * 2 * a.B * a.kv * a.Lk * D : 0;
        bytes = parts + (of_q > of_k ? of_q : of_k);   // (one after the other)
    }
};

#define SEQ_REQUIRE(ptr)                            \
    do {                                            \
        if (!(ptr)) return NA2D_ERR_NULL;           \
        if (misaligned(ptr)) return NA2D_ERR_ALIGN; \
    } while (0)

// slopes, documents, prefix: aligned to their elements; documents need a position for every query
int check_marks(const seq_problem *p, const float *slopes, const int32_t *documents) {
    if (((uintptr_t)slopes | (uintptr_t)documents) & 3u) return NA2D_ERR_ALIGN;
    return documents && p->Lq > p->Lk ? NA2D_ERR_SHAPE : NA2D_OK;
}
int prepare(Args &a, const Space &s, const uint8_t *prefix, void *workspace, size_t bytes, hipStream_t st) {
    if (s.bytes && (!workspace || misaligned(workspace) || bytes < (size_t)s.bytes)) return NA2D_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    a.parts = reinterpret_cast<float *>(ws + s.parts);
    if (s.marks) {
        a.marks = reinterpret_cast<const Marks *>(ws + s.marks);
        a.zeros = ws;
        return from_hip(launch_marks(a, prefix, reinterpret_cast<Marks *>(ws + s.marks), ws, st));
    }
    return NA2D_OK;
}

int cache_validate(const seq_cache_problem *p, int call) {
    if (!p) return NA2D_ERR_NULL;
    if (call != SEQ_CACHE_APPEND && call != SEQ_CACHE_GATHER && call != SEQ_CACHE_ATTENTION) return NA2D_ERR_SHAPE;
    if (int e = common(p->B, p->heads, p->kv_heads, p->D, p->dtype, p->scale, p->softcap, p->window)) return e;
    if (call == SEQ_CACHE_ATTENTION && p->dtype == NA2D_F32) return NA2D_ERR_DTYPE;
    if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128) return NA2D_ERR_SHAPE;
    if (p->pages <= 0 || p->table_width <= 0 || p->n <= 0 || p->n > 1 << 24 || (int64_t)p->table_width * p->page > kFar) return NA2D_ERR_SHAPE;
    const int heads = call == SEQ_CACHE_ATTENTION ? p->heads : p->kv_heads, e = elem(p->dtype);
    if (int r = check_strides(p->q, p->B, heads, p->n, p->D, e, call == SEQ_CACHE_GATHER)) return r;
    if (int r = check_strides(p->out, p->B, heads, p->n, p->D, e, call != SEQ_CACHE_APPEND)) return r;
    if (call == SEQ_CACHE_ATTENTION && (int64_t)p->heads / p->kv_heads * p->n > 1 << 24) return NA2D_ERR_SHAPE;
    return NA2D_OK;
}
CacheArgs cache_args(const seq_cache_problem *p) {
    CacheArgs a{};
    a.B = p->B, a.heads = p->heads, a.kv = p->kv_heads, a.group = p->heads / p->kv_heads, a.pages = p->pages, a.width = p->table_width, a.n = p->n;
    a.page_log2 = p->page == 16 ? 4 : p->page == 32 ? 5 : p->page == 64 ? 6 : 7;
    a.window = p->window ? p->window : kFar;
    a.c = base2(p->scale, p->softcap);
    a.cap = (float)(2.0 * kLog2eExact * p->softcap);
    plan_cache_attention(a, (int64_t)p->table_width * p->page);
    return a;
}
// attention of a tree: the nodes' own keys and values beside the call's
int tree_validate(const seq_cache_problem *p, const seq_strides *k, const seq_strides *v) {
    if (int e = cache_validate(p, SEQ_CACHE_ATTENTION)) return e;
    if (p->n > 64) return NA2D_ERR_SHAPE;
    if (!k != !v) return NA2D_ERR_NULL;
    for (const seq_strides *s : {k, v})
        if (s)
            if (int r = check_strides(*s, p->B, p->kv_heads, p->n, p->D, elem(p->dtype), false)) return r;
    return NA2D_OK;
}
CacheArgs tree_args(const seq_cache_problem *p) {
    CacheArgs a = cache_args(p);
    if (!p->window) a.window = INT32_MAX;   // (nodes stand as far as a length says, whatever the table holds)
    a.tanh = cap_form(NA2D_F16, p->softcap) == kTanhCap;
    plan_cache_tree(a, (int64_t)p->table_width * p->page, p->D);
    return a;
}

int verify_validate(const seq_verify_problem *p) {
    if (!p) return NA2D_ERR_NULL;
    if (p->dtype != NA2D_F32 && p->dtype != NA2D_F16 && p->dtype != NA2D_BF16) return NA2D_ERR_DTYPE;
    if (p->B <= 0 || p->B > 1 << 24 || p->n <= 0 || p->n > 64 || p->V <= 0 || p->V > 1 << 24 || (p->drafted != 0 && p->drafted != 1)) return NA2D_ERR_SHAPE;
    for (int64_t s : {p->batch, p->row, p->draft_batch, p->draft_row})
        if (s < 0 || s > (int64_t)1 << 45) return NA2D_ERR_SHAPE;
    if ((double)(p->B - 1) * p->batch > 0x1p58 || (double)(p->B - 1) * p->draft_batch > 0x1p58) return NA2D_ERR_SHAPE;
    VerifyArgs a{};
    a.B = p->B, a.n = p->n, a.V = p->V, a.drafted = p->drafted;
    plan_verify(a, p->dtype);
    return launch_holds((int64_t)p->B * (2 * p->n) * a.parts, kThreads) ? NA2D_OK : NA2D_ERR_SHAPE;
}
VerifyArgs verify_args(const seq_verify_problem *p) {
    VerifyArgs a{};
    const int e = elem(p->dtype);
    a.B = p->B, a.n = p->n, a.V = p->V, a.drafted = p->drafted;
    a.batch = p->batch * e, a.row = p->row * e, a.draft_batch = p->draft_batch * e, a.draft_row = p->draft_row * e;
    plan_verify(a, p->dtype);
    return a;
}
// The workspace: the parts' statistics, then the parts' rests or the tokens drawn, then tickets.
struct VerifySpace {
    int64_t behind, tickets, bytes;
    VerifySpace(const VerifyArgs &a) {
        behind = (int64_t)sizeof(PartStats) * a.B * (a.drafted ? 2 * a.n - 1 : a.n) * a.parts;
        tickets = behind + (a.drafted ? (int64_t)sizeof(double) * a.B * a.parts : (int64_t)sizeof(int) * a.B * a.n);
        bytes = tickets + (int64_t)sizeof(int) * kTicket * a.B * (a.drafted ? 1 : a.n + 1);
    }
};

bool odd4(std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return true;
    return false;
}

// pairs 0: no rotation, where that is allowed
int check_rotation(const seq_rotation &r, int D, int dtype, bool none_allowed, bool normed) {
    if (r.pairs < 0 || r.pairs % 8 || 2 * (int64_t)r.pairs > D || (!r.pairs && !none_allowed)) return NA2D_ERR_SHAPE;
    if (r.interleaved != 0 && r.interleaved != 1) return NA2D_ERR_SHAPE;
    if (r.pairs) {
        if (r.axes < 1 || r.axes > 4) return NA2D_ERR_SHAPE;
        int64_t sum = 0;
        for (int a = 0; a < r.axes; ++a) {
            if (r.sections[a] < 1) return NA2D_ERR_SHAPE;
            sum += r.sections[a];
        }
        if (sum != r.pairs) return NA2D_ERR_SHAPE;
    }
    if (normed) {
        if (r.weight_dtype != NA2D_F32 && r.weight_dtype != dtype) return NA2D_ERR_DTYPE;
        if (!(r.eps > 0.f) || !std::isfinite(r.eps)) return NA2D_ERR_SHAPE;
    }
    return NA2D_OK;
}
Rotation rotation(const seq_rotation &r, const int32_t *positions, int64_t batch, const float *freqs, const void *weight) {
    Rotation x{};
    x.positions = positions, x.batch = batch, x.freqs = freqs, x.weight = weight;
    x.pairs = r.pairs, x.axes = r.axes, x.interleaved = r.interleaved, x.weight32 = r.weight_dtype == NA2D_F32, x.eps = r.eps;
    for (int a = 0, at = 0; a < 3; ++a) x.ends[a] = at += a < r.axes ? r.sections[a] : 0;
    return x;
}

int rotary_validate(const seq_rotary_problem *p, bool backward) {
    if (!p) return NA2D_ERR_NULL;
    if (p->dtype != NA2D_F32 && p->dtype != NA2D_F16 && p->dtype != NA2D_BF16) return NA2D_ERR_DTYPE;
    if (p->B <= 0 || p->heads <= 0 || p->kv_heads < 0 || p->L <= 0 || (int64_t)p->B * p->L > INT32_MAX || (p->shared != 0 && p->shared != 1)) return NA2D_ERR_SHAPE;
    if (p->D != 16 && p->D != 32 && p->D != 64 && p->D != 128) return NA2D_ERR_HEAD_DIM;
    if (int e = check_rotation(p->rotation, p->D, p->dtype, false, false)) return e;
    const int e = elem(p->dtype);
    struct { const seq_strides &s; int heads; bool written, backward; } all[] = {{p->q, p->heads, false, false}, {p->q_out, p->heads, !backward, false}, {p->dq, p->heads, true, true},
        {p->k, p->kv_heads, false, false}, {p->k_out, p->kv_heads, !backward, false}, {p->dk, p->kv_heads, true, true}};
    for (const auto &x : all)
        if (x.heads && (backward || !x.backward))
            if (int r = check_strides(x.s, p->B, x.heads, p->L, p->D, e, x.written)) return r;
    return NA2D_OK;
}
RotaryArgs rotary_args(const seq_rotary_problem *p, const int32_t *positions, const float *freqs, bool backward) {
    RotaryArgs a{};
    a.r = rotation(p->rotation, positions, p->shared ? 0 : (int64_t)p->rotation.axes * p->L, freqs, nullptr);
    a.tokens = (int64_t)p->B * p->L, a.L = p->L, a.sides = p->kv_heads ? 2 : 1;
    a.side[0].heads = p->heads, a.side[1].heads = p->kv_heads;
    plan_rotary(a, p->dtype, p->D, backward);
    return a;
}
bool misaligned_weight(const void *w, const seq_rotation &r) { return reinterpret_cast<uintptr_t>(w) & (r.weight_dtype == NA2D_F32 ? 3u : 1u); }

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" {

int seq_validate_problem(const seq_problem *p, int backward) { return validate(p, backward != 0); }

size_t seq_attention_workspace_bytes(const seq_problem *p, int marked, int backward) {
    if (validate(p, backward != 0) != NA2D_OK) return 0;
    int64_t most = 0;
    for (int marks = 0; marks < (marked ? 4 : 1); ++marks) {   // documents, a prefix, or both: the largest
        const int64_t n = Space(args(p, nullptr, nullptr, marks & 1, marks & 2), p->D, marked != 0, backward != 0).bytes;
        most = n > most ? n : most;
    }
    return (size_t)most;
}

int seq_attention_fwd(const seq_problem *p, const void *q, const void *k, const void *v, const float *slopes, const int32_t *documents, const uint8_t *prefix,
                      void *out, float *lse, void *rest, void *workspace, size_t workspace_bytes, void *stream) {
    if (int e = validate(p, false)) return e;
    SEQ_REQUIRE(q); SEQ_REQUIRE(k); SEQ_REQUIRE(v); SEQ_REQUIRE(out);
    if (odd4({lse}) || misaligned(rest)) return NA2D_ERR_ALIGN;
    if (int e = check_marks(p, slopes, documents)) return e;
    for (const void *i : {q, k, v})
        if (out == i || (rest && rest == i)) return NA2D_ERR_ALIAS;
    if (rest == out) return NA2D_ERR_ALIAS;
    if (rest && p->dtype == NA2D_F32) return NA2D_ERR_DTYPE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int e = elem(p->dtype);
    Args a = args(p, slopes, documents, documents != nullptr, prefix != nullptr);
    a.q = view(q, p->q, e), a.k = view(k, p->k, e), a.v = view(v, p->v, e), a.out = view(out, p->out, e), a.lse = lse, a.rest = static_cast<char *>(rest);
    if (int r = prepare(a, Space(a, p->D, documents || prefix, false), prefix, workspace, workspace_bytes, st)) return r;
    return from_hip(launch_fwd(a, p->dtype, p->D, cap_form(p->dtype, p->softcap), st));
}

int seq_attention_bwd(const seq_problem *p, const void *q, const void *k, const void *v, const float *slopes, const int32_t *documents, const uint8_t *prefix,
                      const void *out, const float *lse, const void *rest, const void *dout, void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes, void *stream) {
    if (int e = validate(p, true)) return e;
    SEQ_REQUIRE(q); SEQ_REQUIRE(k); SEQ_REQUIRE(v); SEQ_REQUIRE(out); SEQ_REQUIRE(dout); SEQ_REQUIRE(dq); SEQ_REQUIRE(dk); SEQ_REQUIRE(dv);
    if (!lse) return NA2D_ERR_NULL;
    if (odd4({lse}) || misaligned(rest)) return NA2D_ERR_ALIGN;
    if (int e = check_marks(p, slopes, documents)) return e;
    if (rest && p->dtype == NA2D_F32) return NA2D_ERR_DTYPE;
    for (const void *o : {dq, dk, dv})
        for (const void *i : {q, k, v, out, dout, rest, (const void *)lse})
            if (o == i) return NA2D_ERR_ALIAS;
    if (dq == dk || dq == dv || dk == dv) return NA2D_ERR_ALIAS;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int e = elem(p->dtype);
    Args a = args(p, slopes, documents, documents != nullptr, prefix != nullptr);
    a.q = view(q, p->q, e), a.k = view(k, p->k, e), a.v = view(v, p->v, e), a.out = view(out, p->out, e), a.lse = const_cast<float *>(lse), a.rest = const_cast<char *>(static_cast<const char *>(rest));
    a.dout = view(dout, p->dout, e), a.dq = view(dq, p->dq, e), a.dk = view(dk, p->dk, e), a.dv = view(dv, p->dv, e);
    const Space s(a, p->D, documents || prefix, true);
    if (int r = prepare(a, s, prefix, workspace, workspace_bytes, st)) return r;
    a.rows = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + s.rows);
    a.powers = reinterpret_cast<int *>(static_cast<char *>(workspace) + s.powers);
    a.value_powers = reinterpret_cast<int *>(static_cast<char *>(workspace) + s.value_powers);
    const int cap = cap_form(p->dtype, p->softcap);
    if (int r = from_hip(launch_rows(a, p->dtype, p->D, cap, st))) return r;
    if (int r = from_hip(launch_bwd_q(a, p->dtype, p->D, cap, st))) return r;
    return from_hip(launch_bwd_kv(a, p->dtype, p->D, cap, st));
}

int seq_rotary_validate(const seq_rotary_problem *p, int backward) { return rotary_validate(p, backward != 0); }

int seq_rotary_fwd(const seq_rotary_problem *p, const void *q, const void *k, const int32_t *positions, const float *freqs, const void *q_weight, const void *k_weight,
                   void *q_out, void *k_out, void *stream) {
    if (int e = rotary_validate(p, false)) return e;
    if (!positions || !freqs) return NA2D_ERR_NULL;
    if (int e = check_rotation(p->rotation, p->D, p->dtype, false, q_weight || k_weight)) return e;
    if (odd4({positions, freqs}) || misaligned_weight(q_weight, p->rotation) || misaligned_weight(k_weight, p->rotation)) return NA2D_ERR_ALIGN;
    SEQ_REQUIRE(q); SEQ_REQUIRE(q_out);
    if (p->kv_heads) { SEQ_REQUIRE(k); SEQ_REQUIRE(k_out); }
    else if (k || k_out || k_weight) return NA2D_ERR_SHAPE;
    for (const void *o : {q_out, k_out})
        for (const void *i : {q, k, (const void *)positions, (const void *)freqs, q_weight, k_weight})
            if (o && o == i) return NA2D_ERR_ALIAS;
    if (q_out == k_out) return NA2D_ERR_ALIAS;
    const int e = elem(p->dtype);
    RotaryArgs a = rotary_args(p, positions, freqs, false);
    a.side[0].x = view(q, p->q, e), a.side[0].z = view(q_out, p->q_out, e), a.side[0].weight = q_weight;
    a.side[1].x = view(k, p->k, e), a.side[1].z = view(k_out, p->k_out, e), a.side[1].weight = k_weight;
    return from_hip(launch_rotary(a, p->dtype, p->D, static_cast<hipStream_t>(stream)));
}

size_t seq_rotary_bwd_workspace_bytes(const seq_rotary_problem *p) {
    if (rotary_validate(p, true) != NA2D_OK) return 0;
    const RotaryArgs a = rotary_args(p, nullptr, nullptr, true);
    return sizeof(float) * (size_t)(a.side[0].blocks + a.side[1].blocks) * p->D;
}

int seq_rotary_bwd(const seq_rotary_problem *p, const void *q, const void *k, const int32_t *positions, const float *freqs, const void *q_weight, const void *k_weight,
                   const void *dq_out, const void *dk_out, void *dq, void *dk, void *dq_weight, void *dk_weight, void *workspace, size_t workspace_bytes, void *stream) {
    if (int e = rotary_validate(p, true)) return e;
    if (!positions || !freqs) return NA2D_ERR_NULL;
    if (int e = check_rotation(p->rotation, p->D, p->dtype, false, q_weight || k_weight)) return e;
    if (odd4({positions, freqs}) || misaligned_weight(q_weight, p->rotation) || misaligned_weight(k_weight, p->rotation) || misaligned_weight(dq_weight, p->rotation) ||
        misaligned_weight(dk_weight, p->rotation))
        return NA2D_ERR_ALIGN;
    if (q_weight) { SEQ_REQUIRE(q); if (!dq_weight) return NA2D_ERR_NULL; }
    if (k_weight) { SEQ_REQUIRE(k); if (!dk_weight) return NA2D_ERR_NULL; }
    SEQ_REQUIRE(dq_out); SEQ_REQUIRE(dq);
    if (p->kv_heads) { SEQ_REQUIRE(dk_out); SEQ_REQUIRE(dk); }
    else if (k || dk_out || dk || k_weight) return NA2D_ERR_SHAPE;
    const void *outs[] = {dq, dk, dq_weight, dk_weight};
    for (int i = 0; i < 4; ++i) {
        for (const void *x : {q, k, (const void *)positions, (const void *)freqs, q_weight, k_weight, dq_out, dk_out})
            if (outs[i] && outs[i] == x) return NA2D_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (outs[i] && outs[i] == outs[j]) return NA2D_ERR_ALIAS;
    }
    const size_t need = q_weight || k_weight ? seq_rotary_bwd_workspace_bytes(p) : 0;
    if (need && (!workspace || misaligned(workspace) || workspace_bytes < need)) return NA2D_ERR_WORKSPACE;
    const int e = elem(p->dtype);
    RotaryArgs a = rotary_args(p, positions, freqs, true);
    a.side[0].x = view(q, p->q, e), a.side[0].z = view(dq_out, p->q_out, e), a.side[0].dx = view(dq, p->dq, e);
    a.side[1].x = view(k, p->k, e), a.side[1].z = view(dk_out, p->k_out, e), a.side[1].dx = view(dk, p->dk, e);
    a.side[0].weight = q_weight, a.side[0].weight_grad = dq_weight, a.side[1].weight = k_weight, a.side[1].weight_grad = dk_weight;
    a.side[0].parts = static_cast<float *>(workspace), a.side[1].parts = a.side[0].parts + (need ? (int64_t)a.side[0].blocks * p->D : 0);
    return from_hip(launch_rotary_bwd(a, p->dtype, p->D, static_cast<hipStream_t>(stream)));
}

int seq_cache_validate(const seq_cache_problem *p, int call) { return cache_validate(p, call); }

int seq_cache_append(const seq_cache_problem *p, const void *k, const void *v, const int32_t *table, const int32_t *lengths, const int32_t *counts,
                     int8_t *k_pages, int8_t *v_pages, float *k_scales, float *v_scales, void *stream) {
    if (int e = cache_validate(p, SEQ_CACHE_APPEND)) return e;
    SEQ_REQUIRE(k); SEQ_REQUIRE(v); SEQ_REQUIRE(k_pages); SEQ_REQUIRE(v_pages);
    if (!table || !lengths || !k_scales || !v_scales) return NA2D_ERR_NULL;
    if (odd4({table, lengths, counts, k_scales, v_scales})) return NA2D_ERR_ALIGN;
    if (k_pages == v_pages || k_scales == v_scales) return NA2D_ERR_ALIAS;
    CacheArgs a = cache_args(p);
    const int e = elem(p->dtype);
    a.a = view(k, p->q, e), a.b = view(v, p->out, e), a.k = k_pages, a.v = v_pages, a.ks = k_scales, a.vs = v_scales;
    a.table = table, a.lengths = lengths, a.extra = counts;
    return from_hip(launch_append(a, p->dtype, p->D, static_cast<hipStream_t>(stream)));
}

int seq_cache_append_rows(const seq_cache_problem *p, const seq_rotation *r, int32_t given, const void *k, const void *v, const int32_t *rows, const int32_t *positions, int shared,
                          const float *freqs, const void *weight, const int32_t *table, const int32_t *lengths, const int32_t *counts, int8_t *k_pages, int8_t *v_pages,
                          float *k_scales, float *v_scales, void *stream) {
    if (!p) return NA2D_ERR_NULL;
    if (given <= 0 || given > 1 << 24 || p->n > 1 << 24 || (!rows && p->n > given) || (shared != 0 && shared != 1)) return NA2D_ERR_SHAPE;
    seq_cache_problem of_given = *p;
    of_given.n = given;
    if (p->n <= 0) return NA2D_ERR_SHAPE;
    if (int e = cache_validate(&of_given, SEQ_CACHE_APPEND)) return e;
    if (r) {
        if (int e = check_rotation(*r, p->D, p->dtype, true, weight != nullptr)) return e;
        if (r->pairs && !freqs) return NA2D_ERR_NULL;
        if (r->pairs && !positions && r->axes != 1) return NA2D_ERR_SHAPE;
        if (misaligned_weight(weight, *r)) return NA2D_ERR_ALIGN;
    } else if (weight || positions || freqs) {
        return NA2D_ERR_NULL;
    }
    SEQ_REQUIRE(k); SEQ_REQUIRE(v); SEQ_REQUIRE(k_pages); SEQ_REQUIRE(v_pages);
    if (!table || !lengths || !k_scales || !v_scales) return NA2D_ERR_NULL;
    if (odd4({table, lengths, counts, rows, positions, freqs, k_scales, v_scales})) return NA2D_ERR_ALIGN;
    if (k_pages == v_pages || k_scales == v_scales) return NA2D_ERR_ALIAS;
    RowsArgs a{};
    a.c = cache_args(p);
    const int e = elem(p->dtype);
    a.c.a = view(k, p->q, e), a.c.b = view(v, p->out, e), a.c.k = k_pages, a.c.v = v_pages, a.c.ks = k_scales, a.c.vs = v_scales;
    a.c.table = table, a.c.lengths = lengths, a.c.extra = counts;
    a.rows = rows, a.given = given;
    if (r) a.r = rotation(*r, positions, shared ? 0 : (int64_t)r->axes * given, freqs, weight);
    return from_hip(launch_append_rows(a, p->dtype, p->D, static_cast<hipStream_t>(stream)));
}

int seq_cache_gather(const seq_cache_problem *p, const int8_t *k_pages, const int8_t *v_pages, const float *k_scales, const float *v_scales, const int32_t *table,
                     const int32_t *lengths, const int32_t *first, void *k, void *v, void *stream) {
    if (int e = cache_validate(p, SEQ_CACHE_GATHER)) return e;
    SEQ_REQUIRE(k); SEQ_REQUIRE(v); SEQ_REQUIRE(k_pages); SEQ_REQUIRE(v_pages);
    if (!table || !lengths || !first || !k_scales || !v_scales) return NA2D_ERR_NULL;
    if (odd4({table, lengths, first, k_scales, v_scales})) return NA2D_ERR_ALIGN;
    if (k == v) return NA2D_ERR_ALIAS;
    CacheArgs a = cache_args(p);
    const int e = elem(p->dtype);
    a.a = view(k, p->q, e), a.b = view(v, p->out, e), a.k = const_cast<int8_t *>(k_pages), a.v = const_cast<int8_t *>(v_pages);
    a.ks = const_cast<float *>(k_scales), a.vs = const_cast<float *>(v_scales), a.table = table, a.lengths = lengths, a.extra = first;
    return from_hip(launch_gather(a, p->dtype, p->D, static_cast<hipStream_t>(stream)));
}

size_t seq_cache_attention_workspace_bytes(const seq_cache_problem *p) {
    return cache_validate(p, SEQ_CACHE_ATTENTION) == NA2D_OK ? cache_attention_bytes(cache_args(p), p->D) : 0;
}

int seq_cache_attention(const seq_cache_problem *p, const void *q, const int8_t *k_pages, const int8_t *v_pages, const float *k_scales, const float *v_scales,
                        const int32_t *table, const int32_t *lengths, const float *slopes, void *out, void *workspace, size_t workspace_bytes, void *stream) {
    if (int e = cache_validate(p, SEQ_CACHE_ATTENTION)) return e;
    SEQ_REQUIRE(q); SEQ_REQUIRE(out); SEQ_REQUIRE(k_pages); SEQ_REQUIRE(v_pages);
    if (!table || !lengths || !k_scales || !v_scales) return NA2D_ERR_NULL;
    if (odd4({table, lengths, slopes, k_scales, v_scales})) return NA2D_ERR_ALIGN;
    if (out == q) return NA2D_ERR_ALIAS;
    CacheArgs a = cache_args(p);
    const size_t need = cache_attention_bytes(a, p->D);
    if (need && (!workspace || misaligned(workspace) || workspace_bytes < need)) return NA2D_ERR_WORKSPACE;
    const int e = elem(p->dtype);
    a.a = view(q, p->q, e), a.b = view(out, p->out, e), a.k = const_cast<int8_t *>(k_pages), a.v = const_cast<int8_t *>(v_pages);
    a.ks = const_cast<float *>(k_scales), a.vs = const_cast<float *>(v_scales), a.table = table, a.lengths = lengths, a.slopes = slopes;
    a.part = static_cast<float *>(workspace);
    return from_hip(launch_cache_attention(a, p->dtype, p->D, cap_form(NA2D_F16, p->softcap), static_cast<hipStream_t>(stream)));
}

size_t seq_cache_tree_attention_workspace_bytes(const seq_cache_problem *p) {
    return tree_validate(p, nullptr, nullptr) == NA2D_OK ? cache_tree_bytes(tree_args(p), p->D) : 0;
}

int seq_cache_tree_attention(const seq_cache_problem *p, const seq_strides *k_strides, const seq_strides *v_strides, const void *q, const void *k, const void *v, const int32_t *parents,
                             const int8_t *k_pages, const int8_t *v_pages, const float *k_scales, const float *v_scales, const int32_t *table, const int32_t *lengths, const float *slopes,
                             void *out, void *workspace, size_t workspace_bytes, void *stream) {
    if (int e = tree_validate(p, k_strides, v_strides)) return e;
    SEQ_REQUIRE(q); SEQ_REQUIRE(k); SEQ_REQUIRE(v); SEQ_REQUIRE(out); SEQ_REQUIRE(k_pages); SEQ_REQUIRE(v_pages);
    if (!k_strides || !parents || !table || !lengths || !k_scales || !v_scales) return NA2D_ERR_NULL;
    if (odd4({parents, table, lengths, slopes, k_scales, v_scales})) return NA2D_ERR_ALIGN;
    if (out == q || out == k || out == v) return NA2D_ERR_ALIAS;
    CacheArgs a = tree_args(p);
    if (!workspace || misaligned(workspace) || workspace_bytes < cache_tree_bytes(a, p->D)) return NA2D_ERR_WORKSPACE;
    const int e = elem(p->dtype);
    a.a = view(q, p->q, e), a.b = view(out, p->out, e), a.tk = view(k, *k_strides, e), a.tv = view(v, *v_strides, e), a.parents = parents;
    a.k = const_cast<int8_t *>(k_pages), a.v = const_cast<int8_t *>(v_pages), a.ks = const_cast<float *>(k_scales), a.vs = const_cast<float *>(v_scales);
    a.table = table, a.lengths = lengths, a.slopes = slopes;
    a.part = static_cast<float *>(workspace);
    return from_hip(launch_cache_tree(a, p->dtype, p->D, cap_form(NA2D_F16, p->softcap), static_cast<hipStream_t>(stream)));
}

int seq_verify_validate(const seq_verify_problem *p) { return verify_validate(p); }

size_t seq_verify_workspace_bytes(const seq_verify_problem *p) {
    if (verify_validate(p) != NA2D_OK) return 0;
    return (size_t)VerifySpace(verify_args(p)).bytes;
}

int seq_verify(const seq_verify_problem *p, const void *logits, const void *draft, const int32_t *tokens, const int32_t *parents, const float *uniforms, const float *temperatures,
               int32_t *path, int32_t *counts, int32_t *next, void *workspace, size_t workspace_bytes, void *stream) {
    if (int e = verify_validate(p)) return e;
    if (!logits || !tokens || !uniforms || !path || !counts || !next || (p->drafted && p->n > 1 && !draft)) return NA2D_ERR_NULL;
    if (p->drafted ? parents != nullptr : draft != nullptr) return NA2D_ERR_SHAPE;
    const uintptr_t element = (uintptr_t)elem(p->dtype) - 1;
    if (((uintptr_t)logits | (uintptr_t)draft) & element || odd4({tokens, parents, uniforms, temperatures, path, counts, next})) return NA2D_ERR_ALIGN;
    const int32_t *outs[] = {path, counts, next};
    for (int i = 0; i < 3; ++i) {
        for (const void *x : {logits, draft, (const void *)tokens, (const void *)parents, (const void *)uniforms, (const void *)temperatures})
            if ((const void *)outs[i] == x) return NA2D_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (outs[i] == outs[j]) return NA2D_ERR_ALIAS;
    }
    if (!workspace || misaligned(workspace) || workspace_bytes < seq_verify_workspace_bytes(p)) return NA2D_ERR_WORKSPACE;
    VerifyArgs a = verify_args(p);
    a.logits = static_cast<const char *>(logits), a.draft = static_cast<const char *>(draft), a.tokens = tokens, a.parents = parents, a.uniforms = uniforms, a.temperatures = temperatures;
    a.path = path, a.counts = counts, a.next = next;
    a.stats = static_cast<PartStats *>(workspace);
    const VerifySpace space(a);
    char *ws = static_cast<char *>(workspace);
    a.drawn = reinterpret_cast<int *>(ws + space.behind), a.rest = reinterpret_cast<double *>(ws + space.behind), a.tickets = reinterpret_cast<int *>(ws + space.tickets);
    return from_hip(launch_verify(a, p->dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
