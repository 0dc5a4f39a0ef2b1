// Verification of drafted tokens: which of them stand under the target's probabilities, and the token that follows them.
// Formulas at the entry points in difr.h.
//
// What is decided here are whole numbers: u q < p, and the first token whose cumulative weight passes u of the whole, among 150,000
// weights many of which are 1e-7 and less.  Sums good to 2^-24 would choose another token in one row of some hundreds, so weights are
// formed and summed in 64 bits throughout: 2^((x - m) log2(e) / T), good to 2^-50, relative to the largest logit m of what is summed.
// fp64 multiply-adds run at the rate of fp32 ones here; a weight is some 20 instructions, which is what bounds large batches (a pass over
// a row of 151,936 logits is 0.075 us of the whole device, reading it 0.045).
//
// A row is cut into cells of 1024 entries, a wave's work: statistics of all cells first (largest logit, sum of weights), from which rows
// are normalised and drafts accepted or not; then, for a draft that fell, the sums of max(p - q, 0) by cells; then the cell where the sum
// passes u of the whole is formed once more, entry by entry.  No sum depends on the order in which workgroups run.
//
// Small batches: the statistics of all rows at once.  Large ones level by level, so that rows behind a draft that fell are not read:
// a launch for the rows with number k of all sequences that have come there, then one that says which go on.
#include "difr_host.hpp"
#include "draft_verify.hpp"

namespace difr {

constexpr int kCell = 1024;

// log2(e) / T; a temperature beyond 2^100 counts as that (what is left of logits that differ by less than 1e20 is a uniform row either
// way, and a masked entry stays masked).
__device__ __forceinline__ double exponent_factor(float T) { return 1.44269504088896340736 / (double)fminf(T, 0x1p100f); }

struct Weight {
    double m, c, least;  // reference, log2(e) / T, and the least difference that is told from what is below it (a weight of 2^-1000)
    __device__ __forceinline__ Weight(float top, double factor) : m((double)top), c(factor), least(-1000.0 / factor) {}
    // 2^((x - m) c): the whole part of the exponent goes into the exponent field, the rest, within 1/2 of 0, through a polynomial
    // (Chebyshev interpolation of 2^f in degree 10: relative error 3.2e-16)
    __device__ __forceinline__ double at(float x) const
    {
        double d = (double)x - m;
        d = __builtin_fmax(d, least);
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

// Sums and maxima over a wave (lane 63 has them; the caller's value is lane 63's, for all lanes) by moves between lanes of the vector unit.
template <int CTRL, int ROWS>
__device__ __forceinline__ double from_lane(double v)  // 0 where there is none
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xF, true);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xF, true);
    return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double last_lane(double v)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63), __builtin_amdgcn_readlane(__double2loint(v), 63));
}
// Inclusive prefix sums over the lanes.
__device__ __forceinline__ double wave_prefix(double v)
{
    v += from_lane<0x111, 0xF>(v);  // the lane before
    v += from_lane<0x112, 0xF>(v);  // two before
    v += from_lane<0x114, 0xF>(v);
    v += from_lane<0x118, 0xF>(v);
    v += from_lane<0x142, 0xA>(v);  // the last lane of the 16 before, into the second and fourth 16
    v += from_lane<0x143, 0xC>(v);  // lane 31, into the upper half
    return v;
}
__device__ __forceinline__ double wave_sum64(double v) { return last_lane(wave_prefix(v)); }
__device__ __forceinline__ float wave_top(float v)
{
    auto step = [&](auto CTRL, auto ROWS) {
        const int i = __float_as_int(v);
        v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(i, i, decltype(CTRL)::value, decltype(ROWS)::value, 0xF, false)));
    };
    step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xF>());
    step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xF>());
    step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xF>());
    step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xF>());
    step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xA>());
    step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xC>());
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Of a cell: its largest logit (NaN: it holds a NaN or +inf; -inf: no finite logit) and the sum of its weights relative to that.
struct CellStats {
    double *sum;
    float *top;
};
// Where a sequence stops.
struct Stop {
    double rho;             // S_p / S_q: weights of the draft in units of the target's
    double p_sum;           // S_p, relative to p_top
    double p_factor, q_factor;
    float p_top, q_top;
    int32_t place;          // row of the sequence where it stops
    int32_t kind;
};
enum { kFromTarget, kFromRest, kWithoutDraft, kNoToken };
struct Workspace {
    CellStats target, draft;  // by row and cell
    double *rest;             // [B][cells]: sums of max(p - q, 0) where a draft fell
    Stop *stop;               // [B]
    int32_t *at;              // [B]: the row that a sequence has come to (of a tree: the node, and -1 is the root), kDone where it has stopped
    int32_t *depth;           // [B]: trees: tokens accepted so far
};
constexpr int32_t kDone = -2;

static int64_t cells_of(int64_t V) { return (V + kCell - 1) / kCell; }

// Entries of a cell that a lane has: vectors of 16 bytes, 64 lanes apart.
template <int DT>
struct Cell {
    static constexpr int E = Elem<DT>::kPerVec, kVectors = kCell / (64 * E);
    u32x4 q[kVectors];
    __device__ __forceinline__ Cell(const typename Elem<DT>::type *row, int64_t first, int64_t V, int lane)
    {
        if (first + kCell <= V) {
#pragma unroll
            for (int i = 0; i < kVectors; ++i) q[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any *>(row + first + (i * 64 + lane) * E));
            return;
        }
#pragma unroll
        for (int i = 0; i < kVectors; ++i) {
            const int64_t at = first + (i * 64 + lane) * E;
            constexpr uint32_t kMasked = DT == 0 ? 0xFF80FF80u : 0xFF800000u;
            q[i] = at < V ? load_vector<DT>(row, at, V) : u32x4{kMasked, kMasked, kMasked, kMasked};
        }
    }
};

template <int DT>
__device__ __forceinline__ void cell_stats(const typename Elem<DT>::type *row, int64_t cell, int64_t V, float T, const CellStats &out, int64_t id, int lane)
{
    constexpr int E = Elem<DT>::kPerVec;
    const Cell<DT> c(row, cell * kCell, V, lane);
    float top = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < Cell<DT>::kVectors; ++i) {
        float x[E];
        unpack_vector<DT>(c.q[i], x);
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
        const Weight w(top, exponent_factor(T));
        double part[2] = {0.0, 0.0};
#pragma unroll
        for (int i = 0; i < Cell<DT>::kVectors; ++i) {
            float x[E];
            unpack_vector<DT>(c.q[i], x);
#pragma unroll
            for (int j = 0; j < E; ++j) part[j & 1] += w.at(x[j]);
        }
        sum = wave_sum64(part[0] + part[1]);
    }
    if (lane == 0) {
        out.sum[id] = sum;
        out.top[id] = top;
    }
}

__device__ __forceinline__ float row_temperature(const DraftBatch &b, int64_t row) { return b.temperatures ? b.temperatures[row] : b.temperature; }
__device__ __forceinline__ float draft_temperature(const DraftChain &c, int64_t k) { return c.temperatures ? c.temperatures[k] : c.temperature; }

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

// Statistics of all cells: of the target's rows, then of the draft's.  A wave a cell.
template <int DT>
__global__ __launch_bounds__(kBlock) void all_stats_kernel(DraftBatch b, DraftChain c, Workspace ws, uint32_t cells, uint32_t total)
{
    typedef typename Elem<DT>::type elem;
    const uint32_t id = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= total) return;
    const uint32_t row = id / cells, cell = id - row * cells, R = (uint32_t)(b.D + b.B);
    const int lane = threadIdx.x & 63;
    if (row < R)
        cell_stats<DT>(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell, b.V, row_temperature(b, row), ws.target, id, lane);
    else
        cell_stats<DT>(reinterpret_cast<const elem *>(c.draft) + (row - R) * c.ld, cell, b.V, draft_temperature(c, row - R), ws.draft,
                       id - (int64_t)R * cells, lane);
}

// Statistics of the rows that the sequences have come to, the target's and the draft's; LAST: of all rows from there on.
template <int DT, bool LAST>
__global__ __launch_bounds__(kBlock) void level_stats_kernel(DraftBatch b, DraftChain c, Workspace ws, int level, uint32_t cells, uint32_t total)
{
    typedef typename Elem<DT>::type elem;
    const uint32_t id = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= total) return;
    const uint32_t both = c.draft ? 2 : 1, s = id / (cells * both), of_draft = (id - s * cells * both) / cells, cell = id % cells;
    if (level && ws.at[s] != level) return;
    const Span span(b, s);
    const int lane = threadIdx.x & 63;
    for (int64_t i = level; i <= (LAST ? span.drafts : level); ++i) {
        const int64_t k = span.first_draft + i, row = k + s;
        if (!of_draft)
            cell_stats<DT>(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell, b.V, row_temperature(b, row), ws.target, row * cells + cell, lane);
        else if (i < span.drafts)
            cell_stats<DT>(reinterpret_cast<const elem *>(c.draft) + k * c.ld, cell, b.V, draft_temperature(c, k), ws.draft, k * cells + cell, lane);
    }
}
template <int DT>
__global__ __launch_bounds__(kBlock) void node_stats_kernel(DraftBatch b, Workspace ws, bool first, uint32_t cells, uint32_t total)
{
    typedef typename Elem<DT>::type elem;
    const uint32_t id = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= total) return;
    const uint32_t s = id / cells, cell = id - s * cells;
    const int32_t node = first ? -1 : ws.at[s];
    if (node == kDone) return;
    const int64_t row = Span(b, s).first_draft + s + node + 1;
    cell_stats<DT>(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell, b.V, row_temperature(b, row), ws.target, row * cells + cell, threadIdx.x & 63);
}

// A whole row from its cells, by 16 lanes: sum 0 where it cannot be scored.
struct RowStats {
    float top;
    double sum, factor;
};
__device__ __forceinline__ RowStats row_stats(const CellStats &s, int64_t row, int64_t cells, float T, int lane16)
{
    float top = -INFINITY;
    bool bad = !(T > 0.0f && T < INFINITY);
    const float *tops = s.top + row * cells;
    const double *sums = s.sum + row * cells;
    constexpr int kHeld = 10;  // of the first cells are loaded at once: 160 of them
    float t[kHeld];
    double v[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int64_t c = lane16 + 16 * i;
        t[i] = c < cells ? tops[c] : -INFINITY;
        v[i] = c < cells ? sums[c] : 0.0;
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        bad |= t[i] != t[i];
        top = fmaxf(top, t[i]);
    }
    for (int64_t c = lane16 + 16 * kHeld; c < cells; c += 16) {
        bad |= tops[c] != tops[c];
        top = fmaxf(top, tops[c]);
    }
    int any = bad;
#pragma unroll
    for (int o = 8; o; o >>= 1) {
        top = fmaxf(top, __shfl_xor(top, o));
        any |= __shfl_xor(any, o);
    }
    RowStats r{NAN, 0.0, 1.0};
    if (any || top == -INFINITY) return r;
    r.top = top;
    r.factor = exponent_factor(T);
    const Weight w(top, r.factor);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (t[i] > -INFINITY) sum += v[i] * w.at(t[i]);
    for (int64_t c = lane16 + 16 * kHeld; c < cells; c += 16)
        if (tops[c] > -INFINITY) sum += sums[c] * w.at(tops[c]);
#pragma unroll
    for (int o = 8; o; o >>= 1) sum += __shfl_xor(sum, o);
    r.sum = sum;
    return r;
}

template <int DT>
__device__ __forceinline__ float logit_at(const void *logits, int64_t row, int64_t ld, int64_t v)
{
    return Elem<DT>::to_float(reinterpret_cast<const typename Elem<DT>::type *>(logits)[row * ld + v]);
}

// Which drafts of a sequence stand, by a workgroup: from row `from` on, whose statistics are there up to row `to` (or the last).  The first
// eight groups of 16 lanes have a row of the target each, the others the draft's of the same number.  False where rows behind `to` are needed;
// else `stop` says where the sequence stops.  `write`: outputs too.
struct DecideLds {
    float top[16];
    double sum[16], factor[16], weight[16];  // weight: the drafted token's
    Stop stop;
    int go;
};
template <int DT>
__device__ bool decide_drafts(const DraftBatch &b, const DraftChain &c, const DraftOutputs &o, const Workspace &ws, int64_t s, const Span &span, int64_t cells,
                       int64_t from, int64_t to, bool write, DecideLds &lds, Stop &stop, int64_t &reached)
{
    const int tid = threadIdx.x, group = tid >> 4, lane16 = tid & 15;
    const int64_t row0 = span.first_draft + s, last = to < span.drafts ? to : span.drafts;
    for (int64_t base = from;; base += 8) {
        const int64_t i = base + (group & 7), k = span.first_draft + i;
        const bool of_draft = group >= 8;
        if (i <= last && (!of_draft || (c.draft && i < span.drafts))) {
            const int32_t t = i < span.drafts ? b.tokens[k] : -1;
            const bool inside = t >= 0 && t < b.V;
            const float x = !inside ? -INFINITY : of_draft ? logit_at<DT>(c.draft, k, c.ld, t) : logit_at<DT>(b.logits, row0 + i, b.ld, t);
            const RowStats r = of_draft ? row_stats(ws.draft, k, cells, draft_temperature(c, k), lane16)
                                        : row_stats(ws.target, row0 + i, cells, row_temperature(b, row0 + i), lane16);
            if (lane16 == 0) {
                lds.top[group] = r.top, lds.sum[group] = r.sum, lds.factor[group] = r.factor;
                lds.weight[group] = inside && r.sum > 0.0 ? Weight(r.top, r.factor).at(x) : 0.0;
            }
        }
        __syncthreads();
        if (tid == 0) {
            lds.go = -1;
            for (int g = 0; g < 8 && base + g <= last && lds.go < 0; ++g) {
                const int64_t at = base + g, kk = span.first_draft + at;
                Stop &st = lds.stop;
                st.place = (int32_t)at;
                st.p_top = lds.top[g], st.p_sum = lds.sum[g], st.p_factor = lds.factor[g];
                st.q_top = 0.0f, st.q_factor = 1.0, st.rho = 0.0;
                if (!(lds.sum[g] > 0.0) || (at < span.drafts && c.draft && !(lds.sum[8 + g] > 0.0))) {
                    st.kind = kNoToken;
                    lds.go = 0;
                } else if (at == span.drafts) {
                    st.kind = kFromTarget;
                    lds.go = 0;
                } else {
                    const int32_t t = b.tokens[kk];
                    const bool inside = t >= 0 && t < b.V;
                    const double q = c.draft ? lds.weight[8 + g] / lds.sum[8 + g] : inside ? 1.0 : 0.0, e = lds.weight[g];
                    if (e > kNothing && (double)c.accept_u[kk] * q < e / lds.sum[g]) {
                        if (write) {
                            o.tokens[row0 + at] = t;
                            if (o.logp) o.logp[row0 + at] = (float)log(e / lds.sum[g]);
                            o.flags[row0 + at] = (uint8_t)kFlagMatch;
                        }
                    } else {
                        st.kind = c.draft ? kFromRest : inside ? kWithoutDraft : kFromTarget;
                        if (c.draft) st.rho = lds.sum[g] / lds.sum[8 + g], st.q_top = lds.top[8 + g], st.q_factor = lds.factor[8 + g];
                        lds.go = inside ? 0 : 1;
                    }
                }
            }
        }
        __syncthreads();
        const int go = lds.go;
        if (go >= 0) {
            stop = lds.stop;
            if (write) {
                if (tid == 0) o.accepted[s] = stop.place;
                for (int64_t j = stop.place + tid; j <= span.drafts; j += kBlock) {
                    const bool here = j == stop.place;
                    if (!here || stop.kind == kNoToken) {  // (the drawn token is written when it is drawn)
                        o.tokens[row0 + j] = -1;
                        if (o.logp) o.logp[row0 + j] = here ? NAN : 0.0f;
                    }
                    o.flags[row0 + j] = !here ? 0 : stop.kind == kNoToken ? (uint8_t)kFlagNonfinite : go == 1 ? (uint8_t)kFlagInvalidClaim : 0;
                }
            }
            return true;
        }
        if (base + 8 > last) {
            reached = last + 1;
            return false;
        }
    }
}

// Large batches: after level `level` (LAST: after all), a workgroup a sequence.
template <int DT, bool LAST>
__global__ __launch_bounds__(kBlock) void draft_decide_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int level, int64_t cells)
{
    __shared__ DecideLds lds;
    const int64_t s = blockIdx.x;
    if (level && ws.at[s] != level) return;
    const Span span(b, s);
    Stop stop;
    int64_t reached = 0;
    const bool stops = decide_drafts<DT>(b, c, o, ws, s, span, cells, level, LAST ? span.drafts : level, true, lds, stop, reached);
    if (threadIdx.x == 0) {
        ws.at[s] = stops ? kDone : (int32_t)reached;
        if (stops) ws.stop[s] = stop;
    }
}

// Sums of max(p - q, 0) over the cells of the rows where a draft fell, in units of p's weights.  DECIDE (small batches): the workgroup finds out by
// itself where that is; `spread` workgroups share the cells of a sequence.
template <int DT, bool DECIDE>
__global__ __launch_bounds__(kBlock) void draft_rest_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int64_t cells, int spread)
{
    typedef typename Elem<DT>::type elem;
    constexpr int E = Elem<DT>::kPerVec;
    __shared__ DecideLds lds;
    const int64_t s = blockIdx.x / (unsigned)spread;
    const int share = (int)(blockIdx.x - s * spread), lane = threadIdx.x & 63;
    const Span span(b, s);
    Stop stop;
    if constexpr (DECIDE) {
        int64_t unused;
        decide_drafts<DT>(b, c, o, ws, s, span, cells, 0, span.drafts, share == 0, lds, stop, unused);
        if (share == 0 && threadIdx.x == 0) ws.stop[s] = stop;
    } else {
        stop = ws.stop[s];
    }
    if (stop.kind != kFromRest) return;
    const int64_t k = span.first_draft + stop.place, row = k + s;
    const Weight wp(stop.p_top, stop.p_factor), wq(stop.q_top, stop.q_factor);
    for (int64_t cell = share * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); cell < cells; cell += spread * kWaves) {
        const Cell<DT> x(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell * kCell, b.V, lane);
        const Cell<DT> y(reinterpret_cast<const elem *>(c.draft) + k * c.ld, cell * kCell, b.V, lane);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < Cell<DT>::kVectors; ++i) {
            float xs[E], ys[E];
            unpack_vector<DT>(x.q[i], xs);
            unpack_vector<DT>(y.q[i], ys);
#pragma unroll
            for (int j = 0; j < E; ++j) sum += __builtin_fmax(__builtin_fma(-stop.rho, wq.at(ys[j]), wp.at(xs[j])), 0.0);
        }
        sum = wave_sum64(sum);
        if (lane == 0) ws.rest[s * cells + cell] = sum;
    }
}

// Of numbers that the threads of a workgroup have, PER each in order, none negative: the first at which their running sum, begun at `base`,
// exceeds `level`, else the last above kNothing, else -1; the sum before it, and the sum of all.
struct PickLds {
    double wave[kWaves], before;
    int first, last;
};
template <int PER>
__device__ __forceinline__ int pick(const double (&v)[PER], double base, double level, PickLds &lds, double &before, double &end)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    double own = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) own += v[j];
    const double prefix = wave_prefix(own);
    __syncthreads();  // (the last call's are read)
    if (lane == 63) lds.wave[wave] = prefix;
    if (tid == 0) lds.first = 1 << 30, lds.last = -1;
    __syncthreads();
    double start = base;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) start += w < wave ? lds.wave[w] : 0.0;
    end = base;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) end += lds.wave[w];
    double c = start + (prefix - own);
    int mine = 1 << 30, some = -1;
    double mine_before = 0.0, some_before = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (v[j] > kNothing) {
            some = tid * PER + j;
            some_before = c;
            if (c + v[j] > level && mine == 1 << 30) {
                mine = some;
                mine_before = c;
            }
        }
        c += v[j];
    }
    const uint64_t over = __ballot(mine < 1 << 30), any = __ballot(some >= 0);
    if (over && lane == __builtin_ctzll(over)) atomicMin(&lds.first, mine);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&lds.last, some);
    __syncthreads();
    const int at = lds.first < 1 << 30 ? lds.first : lds.last;
    if (at >= 0 && at / PER == tid) lds.before = mine == at ? mine_before : some_before;
    __syncthreads();
    before = lds.before;
    return at;
}

// The token whose cumulative weight is the first above u of the whole, by a workgroup.  cell_sum(c): sum of the weights of cell c; weight(v):
// weight of entry v.  -1 where the whole is not above `nothing`.
template <class C, class W>
__device__ int64_t draw_token(int64_t V, int64_t cells, float u, double nothing, PickLds &lds, C &&cell_sum, W &&weight)
{
    const int tid = threadIdx.x;
    double total = 0.0, before, end;
    double v[1] = {0.0};
    for (int64_t c0 = 0; c0 < cells; c0 += kBlock) {
        v[0] = c0 + tid < cells ? cell_sum(c0 + tid) : 0.0;
        pick(v, total, INFINITY, lds, before, end);
        total = end;
    }
    if (!(total > nothing)) return -1;
    const double level = (double)(u > 0.0f ? u : 0.0f) * total;
    double base = 0.0, found_before = 0.0;
    int64_t cell = -1;
    for (int64_t c0 = 0; c0 < cells; c0 += kBlock) {
        if (cells > kBlock) v[0] = c0 + tid < cells ? cell_sum(c0 + tid) : 0.0;
        const int at = pick(v, base, level, lds, before, end);
        if (at >= 0) cell = c0 + at, found_before = before;
        if (end > level) break;
        base = end;
    }
    if (cell < 0) return -1;
    constexpr int PER = kCell / kBlock;
    const int64_t first = cell * kCell + tid * PER;
    double w[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) w[j] = first + j < V ? weight(first + j) : 0.0;
    const int at = pick(w, 0.0, level - found_before, lds, before, end);
    return at < 0 ? -1 : cell * kCell + at;
}

// A workgroup a sequence: the token that follows the drafts that stand.  DECIDE: finds out by itself where that is (drafts without a distribution).
template <int DT, bool DECIDE>
__global__ __launch_bounds__(kBlock) void draft_draw_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int64_t cells)
{
    __shared__ PickLds lds;
    __shared__ DecideLds decision;
    const int64_t s = blockIdx.x;
    const Span span(b, s);
    Stop stop;
    if constexpr (DECIDE) {
        int64_t unused;
        decide_drafts<DT>(b, c, o, ws, s, span, cells, 0, span.drafts, true, decision, stop, unused);
    } else {
        stop = ws.stop[s];
    }
    if (stop.kind == kNoToken) return;
    const int64_t k = span.first_draft + stop.place, row = k + s;
    const Weight wp(stop.p_top, stop.p_factor);
    auto p = [&](int64_t v) { return wp.at(logit_at<DT>(b.logits, row, b.ld, v)); };
    auto p_cell = [&](int64_t cell) {
        const float top = ws.target.top[row * cells + cell];
        return top > -INFINITY ? ws.target.sum[row * cells + cell] * wp.at(top) : 0.0;
    };
    const float u = c.sample_u[s];
    int64_t t = -1;
    if (stop.kind == kFromRest) {
        const Weight wq(stop.q_top, stop.q_factor);
        t = draw_token(b.V, cells, u, 0x1p-40 * stop.p_sum, lds, [&](int64_t cell) { return ws.rest[s * cells + cell]; },
                       [&](int64_t v) { return __builtin_fmax(__builtin_fma(-stop.rho, wq.at(logit_at<DT>(c.draft, k, c.ld, v)), p(v)), 0.0); });
    } else if (stop.kind == kWithoutDraft) {
        // the cell of the drafted token is summed without it
        const int32_t out = b.tokens[k];
        const int64_t its = out / kCell;
        constexpr int PER = kCell / kBlock;
        double w[PER], before, rest;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int64_t v = its * kCell + threadIdx.x * PER + j;
            w[j] = v < b.V && v != out ? p(v) : 0.0;
        }
        pick(w, 0.0, INFINITY, lds, before, rest);
        t = draw_token(b.V, cells, u, 0.0, lds, [&](int64_t cell) { return cell == its ? rest : p_cell(cell); },
                       [&](int64_t v) { return v == out ? 0.0 : p(v); });
    }
    if (t < 0) t = draw_token(b.V, cells, u, 0.0, lds, p_cell, p);  // (also where nothing is left of p - q)
    if (threadIdx.x == 0) {
        o.tokens[row] = (int32_t)t;
        if (o.logp) o.logp[row] = (float)log(p(t) / stop.p_sum);
    }
}

// A workgroup a sequence: the path that the drawn tokens take through its tree.  ONE: a single step, from where the sequence is (large batches, level by
// level); else to the end.
template <int DT, bool ONE>
__global__ __launch_bounds__(kBlock) void tree_walk_kernel(DraftBatch b, DraftTree tree, DraftOutputs o, Workspace ws, bool first, int64_t cells)
{
    __shared__ PickLds lds;
    __shared__ int lds_child;
    const int64_t s = blockIdx.x;
    const int tid = threadIdx.x;
    const Span span(b, s);
    const int64_t row0 = span.first_draft + s;
    int64_t node = -1, n = 0;
    if (!first) {
        node = ws.at[s];
        if (node == kDone) return;
        n = ws.depth[s];
    }
    bool drawn = true;
    for (;; ++n) {
        const int64_t row = row0 + node + 1;
        const RowStats p = row_stats(ws.target, row, cells, row_temperature(b, row), tid & 15);  // (by each 16 lanes)
        if (!(p.sum > 0.0)) {
            drawn = false;
            break;
        }
        const Weight w(p.top, p.factor);
        auto weight = [&](int64_t v) { return w.at(logit_at<DT>(b.logits, row, b.ld, v)); };
        const int64_t t = draw_token(b.V, cells, tree.sample_u[row], 0.0, lds,
                                     [&](int64_t cell) {
                                         const float top = ws.target.top[row * cells + cell];
                                         return top > -INFINITY ? ws.target.sum[row * cells + cell] * w.at(top) : 0.0;
                                     },
                                     weight);
        // the first child that holds it
        if (tid == 0) lds_child = 1 << 30;
        __syncthreads();
        for (int64_t j = node + 1 + tid; j < span.drafts; j += kBlock)
            if ((tree.parents ? tree.parents[span.first_draft + j] : j - 1) == node && b.tokens[span.first_draft + j] == t) {
                atomicMin(&lds_child, (int)j);
                break;
            }
        __syncthreads();
        const int child = lds_child;
        __syncthreads();
        const bool fits = child < 1 << 30;
        if (tid == 0) {
            o.tokens[row0 + n] = (int32_t)t;
            o.nodes[row0 + n] = fits ? child : -1;
            if (o.logp) o.logp[row0 + n] = (float)log(weight(t) / p.sum);
            o.flags[row0 + n] = fits ? (uint8_t)kFlagMatch : 0;
        }
        if (!fits) break;
        node = child;
        if constexpr (ONE) {
            if (tid == 0) ws.at[s] = (int32_t)node, ws.depth[s] = (int32_t)n + 1;
            return;
        }
    }
    // what lies behind the last drawn token
    if (tid == 0) {
        o.accepted[s] = (int32_t)n;
        if (ONE) ws.at[s] = kDone;
    }
    for (int64_t j = n + (drawn ? 1 : 0) + tid; j <= span.drafts; j += kBlock) {
        o.tokens[row0 + j] = -1;
        o.nodes[row0 + j] = -1;
        if (o.logp) o.logp[row0 + j] = j == n ? NAN : 0.0f;
        o.flags[row0 + j] = j == n ? (uint8_t)kFlagNonfinite : 0;
    }
}

// Trees that have not ended after the levels that were launched: statistics of all rows that may still come.
template <int DT>
__global__ __launch_bounds__(kBlock) void tree_tail_stats_kernel(DraftBatch b, Workspace ws, uint32_t cells, uint32_t total)
{
    typedef typename Elem<DT>::type elem;
    const uint32_t id = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= total) return;
    const uint32_t s = id / cells, cell = id - s * cells;
    const int32_t node = ws.at[s];
    if (node == kDone) return;
    const Span span(b, s);
    for (int64_t j = node; j < span.drafts; ++j) {  // (only nodes behind this one can follow it)
        const int64_t row = span.first_draft + s + j + 1;
        cell_stats<DT>(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell, b.V, row_temperature(b, row), ws.target, row * cells + cell, threadIdx.x & 63);
    }
}

bool draft_shape(int64_t B, int64_t D, int64_t V)
{
    const int64_t most = ((int64_t)1 << 26) - 64;  // cells: a wave each, and their threads are counted in 32 bits
    return 2 * (D + B) <= most / cells_of(V > 0 ? V : 1);
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
    ws.at = (int32_t *)take(B * 4);
    ws.depth = (int32_t *)take(B * 4);
    if (w) *w = ws;
    return at;
}

size_t draft_workspace_bytes(int64_t B, int64_t D, int64_t V, bool draft) { return carve(nullptr, nullptr, B, D, V, draft); }

static dim3 by_waves(int64_t waves) { return dim3((unsigned)((waves + kWaves - 1) / kWaves)); }
static int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

// Entries of a level from which on a batch is taken level by level: a level is 8 us then, and its two launches 5.
constexpr int64_t kLevelEntries = 8 << 20;
constexpr int64_t kLevels = 12;
// Entries of all rows from which on trees are taken level by level, and levels: what goes deeper has the rows behind formed at once.
constexpr int64_t kTreeEntries = 32 << 20;
constexpr int kTreeLevels = 6;

template <int DT>
static void run_chain(const DraftBatch &b, const DraftChain &c, const DraftOutputs &o, const Workspace &ws, hipStream_t stream)
{
    const int64_t cells = cells_of(b.V), R = b.D + b.B, both = c.draft ? 2 : 1;
    const dim3 each((unsigned)b.B), block(kBlock);
    const int64_t levels = (b.D + b.B - 1) / b.B;  // rows with drafts of the longest sequence, if they are alike
    if (b.B * b.V * both >= kLevelEntries && levels > 1) {
        const int64_t total = b.B * cells * both;
        int level = 0;
        for (; level < levels && level < kLevels; ++level) {
            level_stats_kernel<DT, false><<<by_waves(total), block, 0, stream>>>(b, c, ws, level, (uint32_t)cells, (uint32_t)total);
            draft_decide_kernel<DT, false><<<each, block, 0, stream>>>(b, c, o, ws, level, cells);
        }
        level_stats_kernel<DT, true><<<by_waves(total), block, 0, stream>>>(b, c, ws, level, (uint32_t)cells, (uint32_t)total);
        draft_decide_kernel<DT, true><<<each, block, 0, stream>>>(b, c, o, ws, level, cells);
        const int64_t spread = (cells + kWaves - 1) / kWaves;
        if (c.draft) draft_rest_kernel<DT, false><<<dim3((unsigned)(b.B * spread)), block, 0, stream>>>(b, c, o, ws, cells, (int)spread);
        draft_draw_kernel<DT, false><<<each, block, 0, stream>>>(b, c, o, ws, cells);
        return;
    }
    const int64_t total = (R + (c.draft ? b.D : 0)) * cells;
    all_stats_kernel<DT><<<by_waves(total), block, 0, stream>>>(b, c, ws, (uint32_t)cells, (uint32_t)total);
    if (!c.draft) {
        draft_draw_kernel<DT, true><<<each, block, 0, stream>>>(b, c, o, ws, cells);
        return;
    }
    // as many workgroups to a sequence as fill the device, a cell at least to each wave
    const int64_t most = (cells + kWaves - 1) / kWaves, fill = (1024 + b.B - 1) / b.B, spread = most < fill ? most : fill;
    draft_rest_kernel<DT, true><<<dim3((unsigned)(b.B * spread)), block, 0, stream>>>(b, c, o, ws, cells, (int)spread);
    draft_draw_kernel<DT, false><<<each, block, 0, stream>>>(b, c, o, ws, cells);
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
    const int64_t cells = cells_of(b.V), R = b.D + b.B, total = b.B * cells;
    const dim3 each((unsigned)b.B), block(kBlock);
    // few rows are all formed at once; of many only those on the paths, level by level
    if (R * b.V < kTreeEntries) {
        const DraftChain none{};
        all_stats_kernel<DT><<<by_waves(R * cells), block, 0, stream>>>(b, none, ws, (uint32_t)cells, (uint32_t)(R * cells));
        tree_walk_kernel<DT, false><<<each, block, 0, stream>>>(b, t, o, ws, true, cells);
        return;
    }
    const int64_t nodes = (b.D + b.B - 1) / b.B;
    const int levels = (int)(nodes < kTreeLevels ? nodes + 1 : kTreeLevels);
    for (int level = 0; level < levels; ++level) {
        node_stats_kernel<DT><<<by_waves(total), block, 0, stream>>>(b, ws, level == 0, (uint32_t)cells, (uint32_t)total);
        tree_walk_kernel<DT, true><<<each, block, 0, stream>>>(b, t, o, ws, level == 0, cells);
    }
    tree_tail_stats_kernel<DT><<<by_waves(total), block, 0, stream>>>(b, ws, (uint32_t)cells, (uint32_t)total);
    tree_walk_kernel<DT, false><<<each, block, 0, stream>>>(b, t, o, ws, false, cells);
}

int launch_tree_verify(const DraftBatch &b, const DraftTree &t, const DraftOutputs &o, void *workspace, hipStream_t stream)
{
    Workspace ws;
    carve(&ws, workspace, b.B, b.D, b.V, false);
    b.dtype == 0 ? run_tree<0>(b, t, o, ws, stream) : run_tree<1>(b, t, o, ws, stream);
    return launched();
}

}  // namespace difr
