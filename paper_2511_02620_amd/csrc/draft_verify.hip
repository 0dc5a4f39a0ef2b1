// Verification of drafted tokens: which of them stand under the target's probabilities, and the token that follows them.
// Formulas at the entry points in difr.h.
//
// What is decided here are whole numbers: u q < p, and the first token whose cumulative weight passes u of the whole, among 150,000
// weights many of which are 1e-7 and less.  Sums good to 2^-24 would choose another token in one row of some hundreds, so weights are
// formed and summed in 64 bits throughout: 2^((x - m) log2(e) / T), good to 2^-50, relative to the largest logit m of what is summed.
// fp64 multiply-adds run at the rate of fp32 ones here.
//
// A row is cut into cells of 2048 entries, a wave's work: statistics of all cells first (largest logit, sum of weights), from which rows
// are normalised and drafts accepted or not; then, for a draft that fell, the sums of max(p - q, 0) by cells; then the cell where the sum
// passes u of the whole is formed once more, entry by entry.  No sum depends on the order in which workgroups run.
#include "difr_host.hpp"
#include "draft_verify.hpp"

namespace difr {

constexpr int kCell = 2048;

// log2(e) / T; a temperature beyond 2^100 counts as that (what is left of logits that differ by less than 1e20 is a uniform row either
// way, and a masked entry stays masked).
__device__ __forceinline__ double exponent_factor(float T) { return 1.44269504088896340736 / (double)fminf(T, 0x1p100f); }

struct Weight {
    double m, c, least;  // reference, log2(e) / T, and the least difference that is told from what is below it (a weight of 2^-1000)
    __device__ __forceinline__ Weight(float top, double factor) : m((double)top), c(factor), least(-1000.0 / factor) {}
    // 2^((x - m) c): the whole part of the exponent goes into the exponent field, the rest, within 1/2 of 0, through a polynomial
    // (Chebyshev interpolation of 2^f / 2^f in degree 10: relative error 3.2e-16)
    __device__ __forceinline__ double operator()(float x) const
    {
        double d = (double)x - m;
        d = d > least ? d : least;
        const double t = __builtin_fma(d, c, 0x1.8p52), n = t - 0x1.8p52, f = __builtin_fma(d, c, -n);
        double p = 0x1.e6063f7217bc6p-28;
        p = __builtin_fma(p, f, 0x1.b675bca4eeebbp-24);
        p = __builtin_fma(p, f, 0x1.62bfd47773353p-20);
        p = __builtin_fma(p, f, 0x1.ffcb54062e698p-17);
        p = __builtin_fma(p, f, 0x1.430913096fd9fp-13);
        p = __builtin_fma(p, f, 0x1.5d87fe9d7a584p-10);
        p = __builtin_fma(p, f, 0x1.3b2ab6fba1ddap-7);
        p = __builtin_fma(p, f, 0x1.c6b08d703ce49p-5);
        p = __builtin_fma(p, f, 0x1.ebfbdff82c598p-3);
        p = __builtin_fma(p, f, 0x1.62e42fefa3a19p-1);
        p = __builtin_fma(p, f, 1.0);
        // (the low half of t is the whole part; with what is shifted out of the field it is at least -1000)
        return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
    }
};
constexpr double kNothing = 0x1p-900;  // a weight below this is a masked entry's

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_top(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// Of a cell: its largest logit (NaN: it holds a NaN or +inf; -inf: no finite logit) and the sum of its weights relative to that.
struct CellStats {
    double *sum;
    float *top;
};
struct Workspace {
    CellStats target, draft;  // by row and cell
    double *rest;             // [B][cells]: sums of max(p - q, 0) where a draft fell
    struct Stop *stop;        // [B]
};
// Where a sequence stops.
struct Stop {
    double rho;             // S_p / S_q: weights of the draft in units of the target's
    double p_sum;           // S_p, relative to p_top
    double p_factor, q_factor;
    float p_top, q_top;
    int32_t place;          // row of the sequence where it stops
    int32_t kind;           // 0: from p, 1: from max(p - q, 0), 2: from p without the drafted token, 3: no token can be drawn
};

static int64_t cells_of(int64_t V) { return (V + kCell - 1) / kCell; }

// Entries of a cell that a lane has: vectors of 16 bytes, 64 lanes apart.
template <int DT>
struct Cell {
    static constexpr int E = Elem<DT>::kPerVec, kVectors = kCell / (64 * E);
    static __device__ __forceinline__ void load(const typename Elem<DT>::type *row, int64_t first, int64_t V, int lane, u32x4 q[kVectors])
    {
#pragma unroll
        for (int i = 0; i < kVectors; ++i) {
            const int64_t at = first + (i * 64 + lane) * E;
            constexpr uint32_t kMasked = DT == 0 ? 0xFF80FF80u : 0xFF800000u;
            q[i] = at < V ? load_vector<DT>(row, at, V) : u32x4{kMasked, kMasked, kMasked, kMasked};
        }
    }
};

template <int DT>
__global__ __launch_bounds__(kBlock) void cell_stats_kernel(const void *logits, int64_t rows, int64_t V, int64_t ld, float T, const float *Ts,
                                                            CellStats out, int64_t cells)
{
    typedef typename Elem<DT>::type elem;
    constexpr int E = Elem<DT>::kPerVec;
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (id >= rows * cells) return;
    const int64_t row = id / cells, cell = id - row * cells;
    u32x4 q[Cell<DT>::kVectors];
    Cell<DT>::load(reinterpret_cast<const elem *>(logits) + row * ld, cell * kCell, V, lane, q);
    float top = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < Cell<DT>::kVectors; ++i) {
        float x[E];
        unpack_vector<DT>(q[i], x);
#pragma unroll
        for (int j = 0; j < E; j += 2) {
            top = fmaxf(top, fmaxf(x[j], x[j + 1]));
            bad |= __builtin_isunordered(x[j], x[j + 1]);
        }
    }
    top = wave_top(top);
    double sum = 0.0;
    if (__any(bad) || top == INFINITY) {
        top = NAN;
    } else if (top > -INFINITY) {
        const Weight w(top, exponent_factor(Ts ? Ts[row] : T));
#pragma unroll
        for (int i = 0; i < Cell<DT>::kVectors; ++i) {
            float x[E];
            unpack_vector<DT>(q[i], x);
#pragma unroll
            for (int j = 0; j < E; ++j) sum += w(x[j]);
        }
        sum = wave_sum64(sum);
    }
    if (lane == 0) {
        out.sum[id] = sum;
        out.top[id] = top;
    }
}

// A whole row from its cells, by one wave: NaN as `top` where it cannot be scored.
struct RowStats {
    float top;
    double sum, factor;
    __device__ __forceinline__ bool good() const { return sum > 0.0; }
};
__device__ RowStats row_stats(const CellStats &s, int64_t row, int64_t cells, float T, int lane)
{
    float top = -INFINITY;
    bool bad = !(T > 0.0f && T < INFINITY);
    for (int64_t c = lane; c < cells; c += 64) {
        const float t = s.top[row * cells + c];
        bad |= t != t;
        top = fmaxf(top, t);
    }
    top = wave_top(top);
    RowStats r{NAN, 0.0, 1.0};
    if (__any(bad) || top == -INFINITY) return r;
    r.top = top;
    r.factor = exponent_factor(T);
    const Weight w(top, r.factor);
    double sum = 0.0;
    for (int64_t c = lane; c < cells; c += 64) {
        const float t = s.top[row * cells + c];
        if (t > -INFINITY) sum += s.sum[row * cells + c] * w(t);
    }
    r.sum = wave_sum64(sum);
    return r;
}

template <int DT>
__device__ __forceinline__ float logit_at(const void *logits, int64_t row, int64_t ld, int64_t v)
{
    return Elem<DT>::to_float(reinterpret_cast<const typename Elem<DT>::type *>(logits)[row * ld + v]);
}

// The rows of a sequence: the first, and the number of drafted tokens.  Offsets that run backwards or past D are held inside.
struct Span {
    int64_t first_draft, drafts;
    __device__ __forceinline__ Span(const DraftBatch &b, int64_t s)
    {
        const int64_t lo = b.offsets[s], hi = b.offsets[s + 1];
        first_draft = lo < 0 ? 0 : lo > b.D ? b.D : lo;
        const int64_t end = hi > b.D ? b.D : hi;
        drafts = end > first_draft ? end - first_draft : 0;
    }
};

__device__ __forceinline__ float row_temperature(const DraftBatch &b, int64_t row) { return b.temperatures ? b.temperatures[row] : b.temperature; }
__device__ __forceinline__ float draft_temperature(const DraftChain &c, int64_t k)
{
    return c.temperatures ? c.temperatures[k] : c.temperature;
}

// One wave a sequence: which drafts stand, and from what the next token is drawn.
template <int DT>
__global__ __launch_bounds__(64) void draft_decide_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int64_t cells)
{
    const int64_t s = blockIdx.x;
    const int lane = threadIdx.x;
    const Span span(b, s);
    const int64_t row0 = span.first_draft + s;
    Stop stop{};
    bool outside = false;
    int64_t i = 0;
    for (;; ++i) {
        const int64_t row = row0 + i, k = span.first_draft + i;
        const RowStats p = row_stats(ws.target, row, cells, row_temperature(b, row), lane);
        stop.p_top = p.top, stop.p_sum = p.sum, stop.p_factor = p.factor;
        if (!p.good()) {
            stop.kind = 3;
            break;
        }
        if (i == span.drafts) break;
        const int32_t t = b.tokens[k];
        const bool inside = t >= 0 && t < b.V;
        double q = 1.0;
        RowStats qs{};
        if (c.draft) {
            qs = row_stats(ws.draft, k, cells, draft_temperature(c, k), lane);
            if (!qs.good()) {
                stop.kind = 3;
                break;
            }
            q = inside ? Weight(qs.top, qs.factor)(logit_at<DT>(c.draft, k, c.ld, t)) / qs.sum : 0.0;
        }
        const Weight w(p.top, p.factor);
        const double e = inside ? w(logit_at<DT>(b.logits, row, b.ld, t)) : 0.0;
        if (!(e > kNothing && (double)c.accept_u[k] * q < e / p.sum)) {
            stop.kind = c.draft ? 1 : inside ? 2 : 0;
            if (c.draft) stop.rho = p.sum / qs.sum, stop.q_top = qs.top, stop.q_factor = qs.factor;
            outside = !inside;
            break;
        }
        if (lane == 0) {
            o.tokens[row] = t;
            if (o.logp) o.logp[row] = (float)log(e / p.sum);
            o.flags[row] = (uint8_t)kFlagMatch;
        }
    }
    stop.place = (int32_t)i;
    if (lane == 0) {
        o.accepted[s] = (int32_t)i;
        ws.stop[s] = stop;
    }
    for (int64_t j = i + lane; j <= span.drafts; j += 64) {
        o.tokens[row0 + j] = -1;
        if (o.logp) o.logp[row0 + j] = j == i ? NAN : 0.0f;
        o.flags[row0 + j] = j > i ? 0 : stop.kind == 3 ? (uint8_t)kFlagNonfinite : outside ? (uint8_t)kFlagInvalidClaim : 0;
    }
}

// Sums of max(p - q, 0) over the cells of the rows where a draft fell, in units of p's weights.
template <int DT>
__global__ __launch_bounds__(kBlock) void draft_rest_kernel(DraftBatch b, DraftChain c, Workspace ws, int64_t cells)
{
    typedef typename Elem<DT>::type elem;
    constexpr int E = Elem<DT>::kPerVec;
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (id >= b.B * cells) return;
    const int64_t s = id / cells, cell = id - s * cells;
    const Stop stop = ws.stop[s];
    if (stop.kind != 1) return;
    const int64_t k = Span(b, s).first_draft + stop.place, row = k + s;
    u32x4 x[Cell<DT>::kVectors], y[Cell<DT>::kVectors];
    Cell<DT>::load(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell * kCell, b.V, lane, x);
    Cell<DT>::load(reinterpret_cast<const elem *>(c.draft) + k * c.ld, cell * kCell, b.V, lane, y);
    const Weight wp(stop.p_top, stop.p_factor), wq(stop.q_top, stop.q_factor);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < Cell<DT>::kVectors; ++i) {
        float xs[E], ys[E];
        unpack_vector<DT>(x[i], xs);
        unpack_vector<DT>(y[i], ys);
#pragma unroll
        for (int j = 0; j < E; ++j) sum += fmax(__builtin_fma(-stop.rho, wq(ys[j]), wp(xs[j])), 0.0);
    }
    sum = wave_sum64(sum);
    if (lane == 0) ws.rest[id] = sum;
}

// Inclusive prefix sum over a wave's lanes.
__device__ __forceinline__ double wave_prefix(double v, int lane)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// The first of `n` numbers, none negative, at which their running sum exceeds `level` (the last that is above kNothing where none does; -1 where
// none is), and the sum before it.  get(i) gives number i; one wave.
template <class F>
__device__ int64_t first_above(int64_t n, double level, int lane, double *before, F &&get)
{
    double base = 0.0, last_before = 0.0;
    int64_t last = -1;
    for (int64_t i0 = 0; i0 < n; i0 += 64) {
        const double v = i0 + lane < n ? get(i0 + lane) : 0.0;
        const double c = base + wave_prefix(v, lane);
        const uint64_t some = __ballot(v > kNothing), over = __ballot(v > kNothing && c > level);
        if (over) {
            const int l = __builtin_ctzll(over);
            *before = __shfl(c - v, l);
            return i0 + l;
        }
        if (some) {
            const int l = 63 - __builtin_clzll(some);
            last = i0 + l;
            last_before = __shfl(c - v, l);
        }
        base = __shfl(c, 63);
    }
    *before = last_before;
    return last;
}

// The token whose cumulative weight is the first above u of the whole, by one wave.  cell_sum(c): sum of the weights of cell c; weight(v):
// weight of entry v.  -1 where the whole is not above `nothing`.
template <class C, class W>
__device__ int64_t draw_token(int64_t V, int64_t cells, float u, double nothing, int lane, C &&cell_sum, W &&weight)
{
    double total = 0.0;
    for (int64_t c = lane; c < cells; c += 64) total += cell_sum(c);
    total = wave_sum64(total);
    if (!(total > nothing)) return -1;
    double before;
    const double level = (double)(u > 0.0f ? u : 0.0f) * total;
    const int64_t cell = first_above(cells, level, lane, &before, cell_sum);
    if (cell < 0) return -1;
    const int64_t first = cell * kCell, n = V - first < kCell ? V - first : kCell;
    double unused;
    const int64_t at = first_above(n, level - before, lane, &unused, [&](int64_t i) { return weight(first + i); });
    return at < 0 ? -1 : first + at;
}

// One wave a sequence: the token that follows the drafts that stand.
template <int DT>
__global__ __launch_bounds__(64) void draft_draw_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int64_t cells)
{
    const int64_t s = blockIdx.x;
    const int lane = threadIdx.x;
    const Stop stop = ws.stop[s];
    if (stop.kind == 3) return;
    const int64_t k = Span(b, s).first_draft + stop.place, row = k + s;
    const Weight wp(stop.p_top, stop.p_factor);
    auto p = [&](int64_t v) { return wp(logit_at<DT>(b.logits, row, b.ld, v)); };
    auto p_cell = [&](int64_t cell) {
        const float top = ws.target.top[row * cells + cell];
        return top > -INFINITY ? ws.target.sum[row * cells + cell] * wp(top) : 0.0;
    };
    int64_t t = -1;
    if (stop.kind == 1) {
        const Weight wq(stop.q_top, stop.q_factor);
        t = draw_token(b.V, cells, c.sample_u[s], 0x1p-40 * stop.p_sum, lane, [&](int64_t cell) { return ws.rest[s * cells + cell]; },
                 [&](int64_t v) { return fmax(__builtin_fma(-stop.rho, wq(logit_at<DT>(c.draft, k, c.ld, v)), p(v)), 0.0); });
    } else if (stop.kind == 2) {
        // the cell of the drafted token is summed without it
        const int32_t out = b.tokens[k];
        const int64_t its = out / kCell;
        double rest = 0.0;
        for (int64_t v = its * kCell + lane; v < b.V && v < (its + 1) * kCell; v += 64) rest += v == out ? 0.0 : p(v);
        rest = wave_sum64(rest);
        t = draw_token(b.V, cells, c.sample_u[s], 0.0, lane, [&](int64_t cell) { return cell == its ? rest : p_cell(cell); },
                 [&](int64_t v) { return v == out ? 0.0 : p(v); });
    }
    if (t < 0) t = draw_token(b.V, cells, c.sample_u[s], 0.0, lane, p_cell, p);  // (also where nothing is left of p - q)
    if (lane == 0) {
        o.tokens[row] = (int32_t)t;
        if (o.logp) o.logp[row] = (float)log(p(t) / stop.p_sum);
    }
}

// One wave a sequence: the path that the drawn tokens take through its tree.
template <int DT>
__global__ __launch_bounds__(64) void tree_walk_kernel(DraftBatch b, DraftTree tree, DraftOutputs o, Workspace ws, int64_t cells)
{
    const int64_t s = blockIdx.x;
    const int lane = threadIdx.x;
    const Span span(b, s);
    const int64_t row0 = span.first_draft + s;
    int64_t node = -1, n = 0;
    bool drawn = true;
    for (;; ++n) {
        const int64_t row = row0 + node + 1;
        const RowStats p = row_stats(ws.target, row, cells, row_temperature(b, row), lane);
        if (!p.good()) {
            drawn = false;
            break;
        }
        const Weight w(p.top, p.factor);
        auto weight = [&](int64_t v) { return w(logit_at<DT>(b.logits, row, b.ld, v)); };
        const int64_t t = draw_token(b.V, cells, tree.sample_u[row], 0.0, lane,
                               [&](int64_t cell) {
                                   const float top = ws.target.top[row * cells + cell];
                                   return top > -INFINITY ? ws.target.sum[row * cells + cell] * w(top) : 0.0;
                               },
                               weight);
        // the first child that holds it
        int64_t child = -1;
        for (int64_t j0 = node + 1; j0 < span.drafts && child < 0; j0 += 64) {
            const int64_t j = j0 + lane;
            bool fits = false;
            if (j < span.drafts) fits = (tree.parents ? tree.parents[span.first_draft + j] : j - 1) == node && b.tokens[span.first_draft + j] == t;
            const uint64_t which = __ballot(fits);
            if (which) child = j0 + __builtin_ctzll(which);
        }
        if (lane == 0) {
            o.tokens[row0 + n] = (int32_t)t;
            o.nodes[row0 + n] = (int32_t)child;
            if (o.logp) o.logp[row0 + n] = (float)log(weight(t) / p.sum);
            o.flags[row0 + n] = child >= 0 ? (uint8_t)kFlagMatch : 0;
        }
        if (child < 0) break;
        node = child;
    }
    // what lies behind the last drawn token
    if (lane == 0) o.accepted[s] = (int32_t)n;
    for (int64_t j = n + (drawn ? 1 : 0) + lane; j <= span.drafts; j += 64) {
        o.tokens[row0 + j] = -1;
        o.nodes[row0 + j] = -1;
        if (o.logp) o.logp[row0 + j] = j == n ? NAN : 0.0f;
        o.flags[row0 + j] = j == n ? (uint8_t)kFlagNonfinite : 0;
    }
}

bool draft_shape(int64_t B, int64_t D, int64_t V)
{
    const int64_t most = ((int64_t)1 << 26) - 64;  // cells: a wave each, and their threads are counted in 32 bits
    return (D + B) <= most / cells_of(V > 0 ? V : 1);
}

static size_t carve(Workspace *w, void *base, int64_t B, int64_t D, int64_t V, bool draft)
{
    const int64_t cells = cells_of(V), R = D + B;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *p = base ? (char *)base + at : nullptr;
        at += (bytes + 63) / 64 * 64;
        return p;
    };
    Workspace ws{};
    ws.target = CellStats{(double *)take(R * cells * 8), (float *)take(R * cells * 4)};
    if (draft) ws.draft = CellStats{(double *)take(D * cells * 8), (float *)take(D * cells * 4)};
    if (draft) ws.rest = (double *)take(B * cells * 8);
    ws.stop = (Stop *)take(B * sizeof(Stop));
    if (w) *w = ws;
    return at;
}

size_t draft_workspace_bytes(int64_t B, int64_t D, int64_t V, bool draft) { return carve(nullptr, nullptr, B, D, V, draft); }

static dim3 by_waves(int64_t waves) { return dim3((unsigned)((waves + kWaves - 1) / kWaves)); }
static int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

template <int DT>
static void run_chain(const DraftBatch &b, const DraftChain &c, const DraftOutputs &o, const Workspace &ws, hipStream_t stream)
{
    const int64_t cells = cells_of(b.V), R = b.D + b.B;
    cell_stats_kernel<DT><<<by_waves(R * cells), dim3(kBlock), 0, stream>>>(b.logits, R, b.V, b.ld, b.temperature, b.temperatures, ws.target, cells);
    if (c.draft && b.D)
        cell_stats_kernel<DT><<<by_waves(b.D * cells), dim3(kBlock), 0, stream>>>(c.draft, b.D, b.V, c.ld, c.temperature, c.temperatures, ws.draft, cells);
    draft_decide_kernel<DT><<<dim3((unsigned)b.B), dim3(64), 0, stream>>>(b, c, o, ws, cells);
    if (c.draft && b.D) draft_rest_kernel<DT><<<by_waves(b.B * cells), dim3(kBlock), 0, stream>>>(b, c, ws, cells);
    draft_draw_kernel<DT><<<dim3((unsigned)b.B), dim3(64), 0, stream>>>(b, c, o, ws, cells);
}

int launch_draft_verify(const DraftBatch &b, const DraftChain &c, const DraftOutputs &o, void *workspace, hipStream_t stream)
{
    Workspace ws;
    carve(&ws, workspace, b.B, b.D, b.V, c.draft != nullptr);
    b.dtype == 0 ? run_chain<0>(b, c, o, ws, stream) : run_chain<1>(b, c, o, ws, stream);
    return launched();
}

template <int DT>
static void run_tree(const DraftBatch &b, const DraftTree &t, const DraftOutputs &o, const Workspace &ws, hipStream_t stream)
{
    const int64_t cells = cells_of(b.V), R = b.D + b.B;
    cell_stats_kernel<DT><<<by_waves(R * cells), dim3(kBlock), 0, stream>>>(b.logits, R, b.V, b.ld, b.temperature, b.temperatures, ws.target, cells);
    tree_walk_kernel<DT><<<dim3((unsigned)b.B), dim3(64), 0, stream>>>(b, t, o, ws, cells);
}

int launch_tree_verify(const DraftBatch &b, const DraftTree &t, const DraftOutputs &o, void *workspace, hipStream_t stream)
{
    Workspace ws;
    carve(&ws, workspace, b.B, b.D, b.V, false);
    b.dtype == 0 ? run_tree<0>(b, t, o, ws, stream) : run_tree<1>(b, t, o, ws, stream);
    return launched();
}

}  // namespace difr
