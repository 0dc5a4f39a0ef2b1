// Verification of drafted tokens: which of them stand under the target's probabilities, and the token that follows them.
// Formulas at the entry points in difr.h.
//
// What is decided here are whole numbers: u q < p, and the first token whose cumulative weight passes u of the whole, among 150,000
// weights many of which are 1e-7 and less.  Sums good to 2^-24 would choose another token in one row of some hundreds (18 of 6000 rows of 151,936
// random logits), so weights are formed and summed in 64 bits throughout: 2^((x - m) log2(e) / T), good to 2^-44, relative to the largest logit m of what is summed.
// fp64 multiply-adds run at nearly the rate of fp32 ones here (2.3 and 1.8 ns an instruction and SIMD); a weight is some 20 instructions, which
// is what bounds large batches: 512 rows of 151,936 bf16 logits 60 us, of which reading them is 22.
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

// The least difference of logits that is told from what is below it: a weight of 2^-1000.
__device__ __forceinline__ double least_of(float T) { return (double)fminf(T, 0x1p100f) * (-1000.0 / 1.44269504088896340736); }

struct Weight {
    double m, c, least;  // reference, log2(e) / T, least difference
    __device__ __forceinline__ Weight(float top, double factor, double least_) : m((double)top), c(factor), least(least_) {}
    // 2^((x - m) c): the whole part of the exponent goes into the exponent field, the rest, within 1/2 of 0, through a polynomial
    // (degree 9, constant 1, the least largest relative error, found by least squares reweighted with their errors: 1.53e-14 as it is evaluated.
    // The exponent itself is off by 1.7e-16 of it.)
    __device__ __forceinline__ double at(float x) const { return power(__builtin_fmax((double)x - m, least), c); }
    __device__ __forceinline__ double drawable(float x) const;  // 0 for a masked entry
    static __device__ __forceinline__ double power(double d, double c)  // 2^(d c), |d c| <= 1000
    {
        const double t = __builtin_fma(d, c, 0x1.8p52), n = t - 0x1.8p52, f = __builtin_fma(d, c, -n);
        double p = 0x1.b3de2fdc6e28ep-24;
        p = __builtin_fma(p, f, 0x1.63e696d581a8cp-20);
        p = __builtin_fma(p, f, 0x1.ffce2fc397054p-17);
        p = __builtin_fma(p, f, 0x1.430897f2caaa0p-13);
        p = __builtin_fma(p, f, 0x1.5d87fd9386f2bp-10);
        p = __builtin_fma(p, f, 0x1.3b2ab724125d3p-7);
        p = __builtin_fma(p, f, 0x1.c6b08d70c8822p-5);
        p = __builtin_fma(p, f, 0x1.ebfbdff81be03p-3);
        p = __builtin_fma(p, f, 0x1.62e42fefa37d1p-1);
        p = __builtin_fma(p, f, 1.0);
        // (the low half of t is the whole part; with what is shifted out of the field it is at least -1000)
        return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
    }
};
// A sum relative to reference `from`, made relative to this one: by the root of the factor, twice, which reaches 2^-2000 (sums are below 2^600).
// A weight and the two factors are 4.6e-14 off together, and 7e-15 more by the exponents of weights down to 2^-60: 2^-44.
__device__ __forceinline__ double moved_to(double sum, float from, float to, double factor, double least)
{
    const double d = 0.5 * ((double)from - (double)to), r = Weight::power(__builtin_fmax(d, least), factor);
    return sum * r * r;
}
constexpr double kNothing = 0x1p-998;  // a weight up to this is a masked entry's, which is 2^-1000

__device__ __forceinline__ double Weight::drawable(float x) const
{
    const double w = at(x);
    return w > kNothing ? w : 0.0;
}
// ln of the probability of logit x, of a row whose weights have this sum.
__device__ __forceinline__ double log_probability(float x, const Weight &of, double sum)
{
    return ((double)x - of.m) * of.c * 0.693147180559945309417 - log(sum);
}

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

// Of a cell: the sum of its weights relative to a reference logit (its largest, or 0), which is NaN where it holds a NaN or +inf, -inf where
// it has no finite logit.  The cells of a row are padded to whole lines, and a workgroup writes whole halves of them.
struct __attribute__((aligned(16))) CellStats {
    double sum;
    float top, unused;
};
// Where a sequence stops.
struct Stop {
    double rho;             // S_p / S_q: weights of the draft in units of the target's
    double p_sum;           // S_p, relative to p_top
    float p_T, q_T;
    float p_top, q_top;
    int32_t place;          // row of the sequence where it stops
    int32_t kind;
};
enum { kFromTarget, kFromRest, kWithoutDraft, kNoToken };
struct Workspace {
    CellStats *target, *draft;  // by row and cell, `cells` of each row and what pads them
    float *p_logit, *q_logit; // [D + B], [D]: the drafted token's, where rows are taken level by level
    double *rest;             // [B][cells]: sums of max(p - q, 0) where a draft fell
    Stop *stop;               // [B]
    int32_t *at;              // [B]: the row that a sequence has come to (of a tree: the node, and -1 is the root), kDone where it has stopped
    int32_t *depth;           // [B]: trees: tokens accepted so far
};
constexpr int32_t kDone = -2;
constexpr int kMany = 2;  // cells of a wave in large batches: what a row needs is formed once for them, and more is in flight

constexpr int kCellLine = 16;  // cells of a row are padded to a multiple of this
__host__ __device__ inline int64_t padded_cells(int64_t cells) { return (cells + kCellLine - 1) / kCellLine * kCellLine; }
static int64_t cells_of(int64_t V) { return (V + kCell - 1) / kCell; }

// Entries of a cell that a lane has: vectors of 16 bytes, 64 lanes apart.
template <int DT>
struct Cell {
    static constexpr int E = Elem<DT>::kPerVec, kVectors = kCell / (64 * E);
    u32x4 q[kVectors];
    __device__ __forceinline__ void load(const typename Elem<DT>::type *row, int64_t first, int64_t V, int lane)
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

// Entries whose exponent (x log2(e) / T) is within 400 of 0 need no reference: their powers and sums are far from the ends of fp64.
constexpr double kPlain = 400.0;

// Statistics of 4 CELLS cells of a row from `cell0` on, CELLS of them a wave's, which are all read before the first is summed.  `out`: the row's.
// Where all entries are plain the reference is 0, which saves the search for the largest one and three instructions an entry; a cell with masked entries,
// infinities, NaN or large exponents is taken relative to its largest logit.
template <int DT, int CELLS>
__device__ __forceinline__ void cell_stats(const typename Elem<DT>::type *row, uint32_t cell0, uint32_t cells, int64_t V, float T, CellStats *out,
                                           CellStats *lds)
{
    constexpr int E = Elem<DT>::kPerVec;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t cell = cell0 + wave * CELLS;
    Cell<DT> c[CELLS];
#pragma unroll
    for (int k = 0; k < CELLS; ++k) c[k].load(row, (int64_t)(cell + k < cells ? cell + k : cells - 1) * kCell, V, lane);
    const double factor = exponent_factor(T);
    const float plain = (float)(least_of(T) * (-kPlain / 1000.0));  // (a temperature that is none: the row is not scored)
#pragma unroll
    for (int k = 0; k < CELLS; ++k) {
        float most = 0.0f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < Cell<DT>::kVectors; ++i) {
            float x[E];
            unpack_vector<DT>(c[k].q[i], x);
#pragma unroll
            for (int j = 0; j < E; j += 2) {
                most = fmaxf(most, fmaxf(fabsf(x[j]), fabsf(x[j + 1])));
                bad |= __builtin_isunordered(x[j], x[j + 1]);
            }
        }
        float top = 0.0f;
        double sum = 0.0;
        if (!__any(bad || !(most < plain))) {
            double part[2] = {0.0, 0.0};
#pragma unroll
            for (int i = 0; i < Cell<DT>::kVectors; ++i) {
                float x[E];
                unpack_vector<DT>(c[k].q[i], x);
#pragma unroll
                for (int j = 0; j < E; ++j) part[j & 1] += Weight::power((double)x[j], factor);
            }
            sum = wave_sum64(part[0] + part[1]);
        } else {
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < Cell<DT>::kVectors; ++i) {
                float x[E];
                unpack_vector<DT>(c[k].q[i], x);
#pragma unroll
                for (int j = 0; j < E; ++j) top = fmaxf(top, x[j]);
            }
            top = wave_top(top);
            if (__any(bad) || top == INFINITY) {
                top = NAN;
            } else if (top > -INFINITY) {
                const Weight w(top, factor, least_of(T));
#pragma unroll
                for (int i = 0; i < Cell<DT>::kVectors; ++i) {
                    float x[E];
                    unpack_vector<DT>(c[k].q[i], x);
#pragma unroll 1
                    for (int j = 0; j < E; ++j) sum += w.at(x[j]);
                }
                sum = wave_sum64(sum);
            }
        }
        if (lane == 0) lds[wave * CELLS + k] = CellStats{sum, top, 0.0f};
    }
    __syncthreads();
    if (threadIdx.x < kWaves * CELLS && cell0 + threadIdx.x < padded_cells(cells)) out[cell0 + threadIdx.x] = lds[threadIdx.x];
    __syncthreads();
}

constexpr float kBelowOne = 0x1.fffffep-1f;  // what larger random numbers count as

// (The value itself in a register: left to itself the compiler puts it in memory of the thread's, to choose between two addresses.)
__device__ __forceinline__ float temperature_of(const float *Ts, float T, int64_t row)
{
    asm("" : "+v"(T));
    return Ts ? Ts[row] : T;
}
__device__ __forceinline__ float row_temperature(const DraftBatch &b, int64_t row) { return temperature_of(b.temperatures, b.temperature, row); }

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

// Statistics of all cells: of the target's rows, then of the draft's.  A workgroup 4 CELLS cells of a row, of which there are `groups` such.
template <int DT, int CELLS>
__global__ __launch_bounds__(kBlock) void all_stats_kernel(DraftBatch b, DraftChain c, Workspace ws, uint32_t cells, uint32_t groups)
{
    typedef typename Elem<DT>::type elem;
    __shared__ CellStats lds[kWaves * CELLS];
    const uint32_t row = blockIdx.x / groups, cell = (blockIdx.x - row * groups) * (kWaves * CELLS), R = (uint32_t)(b.D + b.B);
    const bool of_draft = row >= R;
    const int64_t at = of_draft ? row - R : row;
    const elem *const p = of_draft ? reinterpret_cast<const elem *>(c.draft) + at * c.ld : reinterpret_cast<const elem *>(b.logits) + at * b.ld;
    const float T = temperature_of(of_draft ? c.temperatures : b.temperatures, of_draft ? c.temperature : b.temperature, at);
    cell_stats<DT, CELLS>(p, cell, cells, b.V, T, (of_draft ? ws.draft : ws.target) + at * padded_cells(cells), lds);
}

// Statistics of the rows that the sequences have come to, the target's and the draft's; LAST: of all rows from there on.
template <int DT, bool LAST>
__global__ __launch_bounds__(kBlock) void level_stats_kernel(DraftBatch b, DraftChain c, Workspace ws, int level, uint32_t cells, uint32_t groups)
{
    typedef typename Elem<DT>::type elem;
    __shared__ CellStats lds[kWaves * kMany];
    const uint32_t both = c.draft ? 2 : 1, r = blockIdx.x / groups, s = r / both, cell = (blockIdx.x - r * groups) * (kWaves * kMany);
    const bool of_draft = r - s * both != 0;
    if (level && ws.at[s] != level) return;
    const Span span(b, s);
    for (int64_t i = level; i <= (LAST ? span.drafts : level); ++i) {
        if (of_draft && i >= span.drafts) break;
        const int64_t k = span.first_draft + i, at = of_draft ? k : k + s;
        const elem *const p = of_draft ? reinterpret_cast<const elem *>(c.draft) + at * c.ld : reinterpret_cast<const elem *>(b.logits) + at * b.ld;
        const float T = temperature_of(of_draft ? c.temperatures : b.temperatures, of_draft ? c.temperature : b.temperature, at);
        cell_stats<DT, kMany>(p, cell, cells, b.V, T, (of_draft ? ws.draft : ws.target) + at * padded_cells(cells), lds);
        // the drafted token's logit, while its page is at hand
        const int32_t t = i < span.drafts ? b.tokens[k] : -1;
        if (t >= 0 && t < b.V && (uint32_t)t / kCell - cell < kWaves * kMany && threadIdx.x == 0)
            (of_draft ? ws.q_logit : ws.p_logit)[at] = Elem<DT>::to_float(p[t]);
    }
}
// The same for trees; LAST: of all rows that may still come.
template <int DT, bool LAST>
__global__ __launch_bounds__(kBlock) void node_stats_kernel(DraftBatch b, Workspace ws, bool first, uint32_t cells, uint32_t groups)
{
    typedef typename Elem<DT>::type elem;
    __shared__ CellStats lds[kWaves * kMany];
    const uint32_t s = blockIdx.x / groups, cell = (blockIdx.x - s * groups) * (kWaves * kMany);
    const int32_t node = first ? -1 : ws.at[s];
    if (node == kDone) return;
    const Span span(b, s);
    for (int64_t j = node; j < (LAST ? span.drafts : node + 1); ++j) {  // (only nodes behind this one can follow it)
        const int64_t row = span.first_draft + s + j + 1;
        cell_stats<DT, kMany>(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell, cells, b.V, row_temperature(b, row),
                              ws.target + row * padded_cells(cells), lds);
    }
}

// A whole row from its cells, by a wave: sum 0 where it cannot be scored.
struct RowStats {
    float top;
    double sum, factor;
};
__device__ __forceinline__ RowStats row_stats(const CellStats *stats, int64_t row, int64_t cells, float T, int lane)
{
    float top = -INFINITY;
    bool bad = !(T > 0.0f && T < INFINITY);
    const CellStats *const of = stats + row * padded_cells(cells);
    constexpr int kHeld = 3;  // of the first cells are loaded at once: 192 of them
    CellStats held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int64_t c = lane + 64 * i;
        held[i] = CellStats{0.0, -INFINITY, 0.0f};
        if (c < cells) held[i] = of[c];
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        bad |= held[i].top != held[i].top;
        top = fmaxf(top, held[i].top);
    }
    for (int64_t c = lane + 64 * kHeld; c < cells; c += 64) {
        bad |= of[c].top != of[c].top;
        top = fmaxf(top, of[c].top);
    }
    top = wave_top(top);
    RowStats r{NAN, 0.0, 1.0};
    if (__any(bad) || top == -INFINITY) return r;
    r.top = top;
    r.factor = exponent_factor(T);
    const double least = least_of(T);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (held[i].top > -INFINITY) sum += moved_to(held[i].sum, held[i].top, top, r.factor, least);
    for (int64_t c = lane + 64 * kHeld; c < cells; c += 64)
        if (of[c].top > -INFINITY) sum += moved_to(of[c].sum, of[c].top, top, r.factor, least);
    r.sum = wave_sum64(sum);
    return r;
}

template <int DT>
__device__ __forceinline__ float logit_at(const void *logits, int64_t row, int64_t ld, int64_t v)
{
    return Elem<DT>::to_float(reinterpret_cast<const typename Elem<DT>::type *>(logits)[row * ld + v]);
}

// Which drafts of a sequence stand, by a workgroup of WAVES waves: from row `from` on, whose statistics are there up to row `to` (or the last).
// A wave has a row of the target, another the draft's of the same number; then lanes 0, 1, ... of the first wave a row each.  False where
// rows behind `to` are needed; else lds.stop says where the sequence stops.  `write`: outputs too.
template <int WAVES>
struct DecideLds {
    float top[WAVES], T[WAVES], u[WAVES];
    double sum[WAVES], weight[WAVES];  // weight: the drafted token's
    int32_t token[WAVES];
    Stop stop;
    int go;
};
template <int DT, int WAVES, bool LEVELS>
__device__ __forceinline__ bool decide_drafts(const DraftBatch &b, const DraftChain &c, const DraftOutputs &o, const Workspace &ws, int64_t s,
                                              const Span &span, int64_t cells, int64_t from, int64_t to, bool write, DecideLds<WAVES> &lds, int64_t &reached)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rows = c.draft ? WAVES / 2 : WAVES;  // of a round
    const int64_t row0 = span.first_draft + s, last = to < span.drafts ? to : span.drafts;
    const bool of_draft = wave >= rows;
    const CellStats *const mine = of_draft ? ws.draft : ws.target;
    for (int64_t base = from;; base += rows) {
        const int64_t i = base + (of_draft ? wave - rows : wave), k = span.first_draft + i, row = of_draft ? k : row0 + i;
        if (i <= last && (!of_draft || i < span.drafts)) {
            const int32_t t = i < span.drafts ? b.tokens[k] : -1;
            const float u = i < span.drafts ? c.accept_u[k] : 0.0f;
            const bool inside = t >= 0 && t < b.V;
            const float x = !inside  ? -INFINITY
                            : LEVELS ? (of_draft ? ws.q_logit : ws.p_logit)[row]
                                     : logit_at<DT>(of_draft ? c.draft : b.logits, row, of_draft ? c.ld : b.ld, t);
            const float T = temperature_of(of_draft ? c.temperatures : b.temperatures, of_draft ? c.temperature : b.temperature, row);
            const RowStats r = row_stats(mine, row, cells, T, lane);
            if (lane == 0) {
                lds.top[wave] = r.top, lds.sum[wave] = r.sum, lds.T[wave] = T;
                lds.weight[wave] = inside && r.sum > 0.0 ? Weight(r.top, r.factor, least_of(T)).at(x) : 0.0;
                lds.token[wave] = inside ? t : -1, lds.u[wave] = u;
            }
        }
        __syncthreads();
        if (wave == 0) {
            const int g = lane < rows ? lane : 0, d = c.draft ? rows + g : g;
            const int64_t at = base + g;
            const bool own = lane < rows && at <= last;
            const int32_t t = lds.token[g];
            const double ps = lds.sum[g], qs = lds.sum[d], p = lds.weight[g] / ps;
            const bool scored = ps > 0.0 && (at >= span.drafts || !c.draft || qs > 0.0);
            const double q = c.draft ? lds.weight[d] / qs : t >= 0 ? 1.0 : 0.0;
            const double u = lds.u[g] > kBelowOne ? kBelowOne : lds.u[g];  // (a NaN accepts nothing)
            const bool stands = own && scored && at < span.drafts && lds.weight[g] > kNothing && u * q < p;
            const uint64_t stops = __ballot(own && !stands);
            const int first = stops ? __builtin_ctzll(stops) : 64;
            if (lane == 0) lds.go = first < 64 ? 1 : 0;
            if (stands && lane < first && write) {
                o.tokens[row0 + at] = t;
                if (o.logp) o.logp[row0 + at] = (float)log(p);
                o.flags[row0 + at] = (uint8_t)kFlagMatch;
            }
            if (lane == first) {
                Stop &st = lds.stop;
                st.place = (int32_t)at;
                st.p_top = lds.top[g], st.p_sum = ps, st.p_T = lds.T[g];
                st.kind = !scored ? kNoToken : at == span.drafts ? kFromTarget : c.draft ? kFromRest : t >= 0 ? kWithoutDraft : kFromTarget;
                const bool rest = st.kind == kFromRest;
                st.rho = rest ? ps / qs : 0.0, st.q_top = rest ? lds.top[d] : 0.0f, st.q_T = rest ? lds.T[d] : 1.0f;
                if (write) {
                    o.accepted[s] = (int32_t)at;
                    o.flags[row0 + at] = !scored ? (uint8_t)kFlagNonfinite : at < span.drafts && t < 0 ? (uint8_t)kFlagInvalidClaim : 0;
                    if (!scored) {  // (else the drawn token is written when it is drawn)
                        o.tokens[row0 + at] = -1;
                        if (o.logp) o.logp[row0 + at] = NAN;
                    }
                }
            }
        }
        __syncthreads();
        if (lds.go) {
            if (write)
                for (int64_t j = lds.stop.place + 1 + tid; j <= span.drafts; j += WAVES * 64) {
                    o.tokens[row0 + j] = -1;
                    if (o.logp) o.logp[row0 + j] = 0.0f;
                    o.flags[row0 + j] = 0;
                }
            return true;
        }
        if (base + rows > last) {
            reached = last + 1;
            return false;
        }
        __syncthreads();
    }
}

// Large batches: after level `level`, by two waves a sequence; LAST: after all.
template <int DT, bool LAST>
__global__ __launch_bounds__(128) void draft_decide_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int level, int64_t cells)
{
    __shared__ DecideLds<2> lds;
    const int64_t s = blockIdx.x;
    if (level && ws.at[s] != level) return;
    const Span span(b, s);
    int64_t reached = 0;
    const bool stops = decide_drafts<DT, 2, true>(b, c, o, ws, s, span, cells, level, LAST ? span.drafts : level, true, lds, reached);
    if (threadIdx.x == 0) {
        ws.at[s] = stops ? kDone : (int32_t)reached;
        if (stops) ws.stop[s] = lds.stop;
    }
}

// Sums of max(p - q, 0) over the cells of the rows where a draft fell, in units of p's weights.  DECIDE (small batches): the workgroup finds out by
// itself where that is; `spread` workgroups share the cells of a sequence.
template <int DT, bool DECIDE>
__global__ __launch_bounds__(DECIDE ? 1024 : kBlock) void draft_rest_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int64_t cells, int spread)
{
    typedef typename Elem<DT>::type elem;
    constexpr int E = Elem<DT>::kPerVec;
    constexpr int WAVES = DECIDE ? 16 : kWaves, CELLS = DECIDE ? 1 : kMany;
    __shared__ DecideLds<16> lds;
    __shared__ double lds_sum[WAVES * CELLS];
    const int64_t s = blockIdx.x / (unsigned)spread;
    const int share = (int)(blockIdx.x - s * spread), lane = threadIdx.x & 63;
    const Span span(b, s);
    int64_t unused;
    if (DECIDE) decide_drafts<DT, 16, false>(b, c, o, ws, s, span, cells, 0, span.drafts, share == 0, lds, unused);
    if (DECIDE && share == 0 && threadIdx.x == 0) ws.stop[s] = lds.stop;
    const Stop stop = DECIDE ? lds.stop : ws.stop[s];
    if (stop.kind != kFromRest) return;
    const int64_t k = span.first_draft + stop.place, row = k + s;
    const Weight wp(stop.p_top, exponent_factor(stop.p_T), least_of(stop.p_T)), wq(stop.q_top, exponent_factor(stop.q_T), least_of(stop.q_T));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t cell0 = (int64_t)share * (WAVES * CELLS); cell0 < cells; cell0 += (int64_t)spread * (WAVES * CELLS)) {
        for (int n = 0; n < CELLS; ++n) {
            const int64_t cell = cell0 + wave * CELLS + n;
            double sum = 0.0;
            if (cell < cells) {
                Cell<DT> x, y;
                x.load(reinterpret_cast<const elem *>(b.logits) + row * b.ld, cell * kCell, b.V, lane);
                y.load(reinterpret_cast<const elem *>(c.draft) + k * c.ld, cell * kCell, b.V, lane);
#pragma unroll
                for (int i = 0; i < Cell<DT>::kVectors; ++i) {
                    float xs[E], ys[E];
                    unpack_vector<DT>(x.q[i], xs);
                    unpack_vector<DT>(y.q[i], ys);
#pragma unroll
                    for (int j = 0; j < E; ++j) sum += __builtin_fmax(__builtin_fma(-stop.rho, wq.at(ys[j]), wp.at(xs[j])), 0.0);
                }
                sum = wave_sum64(sum);
            }
            if (lane == 0) lds_sum[wave * CELLS + n] = sum;
        }
        __syncthreads();
        if (threadIdx.x < WAVES * CELLS && cell0 + threadIdx.x < padded_cells(cells)) ws.rest[s * padded_cells(cells) + cell0 + threadIdx.x] = lds_sum[threadIdx.x];
        __syncthreads();
    }
}

// Of numbers that the threads of a workgroup have, PER each in order, none negative: the first above 0 at which their running sum, begun at
// `base`, exceeds level(end), else the last above 0, else -1; `end` is the sum of all.  Of the number: the sum before it, it, its thread's tag.
struct Picked {
    int at;
    double before, value, end;
    float tag;
};
struct PickLds {
    double wave[kWaves];
    Picked found;
    int first, last;
};
template <int PER, class L>
__device__ __forceinline__ Picked pick(const double (&v)[PER], float tag, double base, L &&level_of, PickLds &lds)
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
    double end = base;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) end += lds.wave[w];
    const double level = level_of(end);
    double c = start + (prefix - own);
    int mine = 1 << 30, some = -1;
    double mine_before = 0.0, some_before = 0.0, mine_value = 0.0, some_value = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (v[j] > 0.0) {
            some = tid * PER + j;
            some_before = c, some_value = v[j];
            if (c + v[j] > level && mine == 1 << 30) {
                mine = some;
                mine_before = c, mine_value = v[j];
            }
        }
        c += v[j];
    }
    const uint64_t over = __ballot(mine < 1 << 30), any = __ballot(some >= 0);
    if (over && lane == __builtin_ctzll(over)) atomicMin(&lds.first, mine);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&lds.last, some);
    __syncthreads();
    const int at = lds.first < 1 << 30 ? lds.first : lds.last;
    if (at >= 0 && at / PER == tid) {
        const bool crosses = mine == at;
        lds.found.before = crosses ? mine_before : some_before, lds.found.value = crosses ? mine_value : some_value, lds.found.tag = tag;
    }
    __syncthreads();
    return Picked{at, lds.found.before, lds.found.value, end, lds.found.tag};
}

// The token whose cumulative weight is the first above u of the whole, by a workgroup.  cell_sum(c, reference): the sum of the weights of cell c, 0 where
// it holds none that can be drawn, and what they are relative to; weight(v, reference): that of entry v, in a unit of the cell's own, 0 where it cannot
// be drawn.  A cell whose sum is not 0 holds an entry whose weight is not, so a token is found (u is below 1, so some sum exceeds the level)
// unless the whole is not above `nothing`: then -1.
template <class C, class W>
__device__ __forceinline__ int64_t draw_token(int64_t V, int64_t cells, float u, double nothing, PickLds &lds, C &&cell_sum, W &&weight)
{
    const int tid = threadIdx.x;
    const double share = (double)(u > 0.0f ? fminf(u, kBelowOne) : 0.0f);
    const bool at_once = cells <= kBlock;  // (their sum is known when they are searched)
    double total = 0.0;
    if (!at_once) {
        double sum = 0.0;
        float unused;
        for (int64_t c = tid; c < cells; c += kBlock) sum += cell_sum(c, unused);
        const double v[1] = {sum};
        total = pick(v, 0.0f, 0.0, [](double) { return 0.0; }, lds).end;
    }
    double base = 0.0, level = 0.0;
    Picked in{-1, 0.0, 1.0, 0.0, 0.0f};
    int64_t cell = -1;
    for (int64_t c0 = 0; c0 < cells; c0 += kBlock) {
        float reference = 0.0f;
        const double v[1] = {c0 + tid < cells ? cell_sum(c0 + tid, reference) : 0.0};
        const Picked got = pick(v, reference, base, [&](double sum) { return share * (at_once ? sum : total); }, lds);
        if (at_once) total = got.end;
        level = share * total;
        base = got.end;
        if (got.at < 0) continue;
        cell = c0 + got.at, in = got;
        if (base > level) break;
    }
    if (cell < 0 || !(total > nothing)) return -1;
    constexpr int PER = kCell / kBlock;
    const int64_t first = cell * kCell + tid * PER;
    double w[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) w[j] = first + j < V ? weight(first + j, in.tag) : 0.0;
    // (the sum before the cell is rounded and may lie above the level by that: then the first entry it is)
    const double rest = __builtin_fmax(level - in.before, 0.0) / in.value;
    return cell * kCell + pick(w, 0.0f, 0.0, [&](double sum) { return rest * sum; }, lds).at;
}

// A workgroup a sequence: the token that follows the drafts that stand.  DECIDE: finds out by itself where that is (drafts without a distribution).
template <int DT, bool DECIDE>
__global__ __launch_bounds__(kBlock) void draft_draw_kernel(DraftBatch b, DraftChain c, DraftOutputs o, Workspace ws, int64_t cells)
{
    __shared__ PickLds lds;
    __shared__ DecideLds<kWaves> decision;
    const int64_t s = blockIdx.x;
    const Span span(b, s);
    int64_t unused;
    if (DECIDE) decide_drafts<DT, kWaves, false>(b, c, o, ws, s, span, cells, 0, span.drafts, true, decision, unused);
    const Stop stop = DECIDE ? decision.stop : ws.stop[s];
    if (stop.kind == kNoToken) return;
    const int64_t k = span.first_draft + stop.place, row = k + s;
    const Weight wp(stop.p_top, exponent_factor(stop.p_T), least_of(stop.p_T)), wq(stop.q_top, exponent_factor(stop.q_T), least_of(stop.q_T));
    auto x = [&](int64_t v) { return logit_at<DT>(b.logits, row, b.ld, v); };
    const CellStats *const stats = ws.target + row * padded_cells(cells);
    // the cell of a draft without a distribution is summed without it
    int64_t out = -1, its = -1;
    double rest = 0.0;
    if (stop.kind == kWithoutDraft) {
        out = b.tokens[k];
        its = out / kCell;
        constexpr int PER = kCell / kBlock;
        const Weight of_cell(stats[its].top, wp.c, wp.least);
        double w[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int64_t v = its * kCell + threadIdx.x * PER + j;
            w[j] = v < b.V && v != out ? of_cell.drawable(x(v)) : 0.0;
        }
        rest = pick(w, 0.0f, 0.0, [](double) { return 0.0; }, lds).end;
    }
    const float u = c.sample_u[s];
    int64_t t = -1;
    for (bool from_rest = stop.kind == kFromRest;; from_rest = false) {
        t = draw_token(b.V, cells, u, from_rest || its >= 0 ? 0x1p-40 * stop.p_sum : 0.0, lds,
                       [&](int64_t cell, float &reference) {
                           if (from_rest) {
                               // (1024 weights of more than 2^-980 in all are not all up to kNothing)
                               const double sum = ws.rest[s * padded_cells(cells) + cell];
                               return sum > 0x1p-980 ? sum : 0.0;
                           }
                           const CellStats of = stats[cell];
                           reference = of.top;
                           return of.top > -INFINITY ? moved_to(cell == its ? rest : of.sum, of.top, stop.p_top, wp.c, wp.least) : 0.0;
                       },
                       [&](int64_t v, float reference) {
                           if (from_rest) {
                               const double r = __builtin_fma(-stop.rho, wq.at(logit_at<DT>(c.draft, k, c.ld, v)), wp.at(x(v)));
                               return r > kNothing ? r : 0.0;
                           }
                           return v == out ? 0.0 : Weight(reference, wp.c, wp.least).drawable(x(v));
                       });
        // where nothing is left: p, and the drafted token with it
        if (t >= 0 || (!from_rest && its < 0)) break;
        its = out = -1;
    }
    if (threadIdx.x == 0) {
        o.tokens[row] = (int32_t)t;
        if (o.logp) o.logp[row] = (float)log_probability(x(t), wp, stop.p_sum);
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
        const RowStats p = row_stats(ws.target, row, cells, row_temperature(b, row), tid & 63);  // (by each wave)
        if (!(p.sum > 0.0)) {
            drawn = false;
            break;
        }
        const Weight w(p.top, p.factor, least_of(row_temperature(b, row)));
        auto x = [&](int64_t v) { return logit_at<DT>(b.logits, row, b.ld, v); };
        const int64_t t = draw_token(b.V, cells, tree.sample_u[row], 0.0, lds,
                                     [&](int64_t cell, float &reference) {
                                         const CellStats of = ws.target[row * padded_cells(cells) + cell];
                                         reference = of.top;
                                         return of.top > -INFINITY ? moved_to(of.sum, of.top, p.top, w.c, w.least) : 0.0;
                                     },
                                     [&](int64_t v, float reference) { return Weight(reference, w.c, w.least).drawable(x(v)); });
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
            if (o.logp) o.logp[row0 + n] = (float)log_probability(x(t), w, p.sum);
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

bool draft_shape(int64_t B, int64_t D, int64_t V)
{
    const int64_t most = ((int64_t)1 << 26) - 64;  // cells: a wave each, and their threads are counted in 32 bits
    return 2 * (D + B) <= most / padded_cells(cells_of(V > 0 ? V : 1));
}

static size_t carve(Workspace *w, void *base, int64_t B, int64_t D, int64_t V, bool draft)
{
    const int64_t cells = padded_cells(cells_of(V)), R = D + B;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *p = base ? (char *)base + at : nullptr;
        at += (bytes + 127) / 128 * 128;
        return p;
    };
    Workspace ws{};
    ws.target = (CellStats *)take(R * cells * sizeof(CellStats));
    if (draft) ws.draft = (CellStats *)take(D * cells * sizeof(CellStats));
    ws.p_logit = (float *)take(R * 4);
    if (draft) ws.q_logit = (float *)take(D * 4);
    if (draft) ws.rest = (double *)take(B * cells * 8);
    ws.stop = (Stop *)take(B * sizeof(Stop));
    ws.at = (int32_t *)take(B * 4);
    ws.depth = (int32_t *)take(B * 4);
    if (w) *w = ws;
    return at;
}

size_t draft_workspace_bytes(int64_t B, int64_t D, int64_t V, bool draft) { return carve(nullptr, nullptr, B, D, V, draft); }

static int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

// Entries of a level, target's and draft's, from which on a batch is taken level by level.  All rows at once / level by level, us a call:
// 48, 96, 128, 160, 256 sequences of 5 drafts, 128,256 bf16 (12, 24, 31, 39, 63 << 20 entries a level): 86 / 117, 142 / 154, 167 / 171,
// 222 / 199, 314 / 267; 128 and 256 of 7, 151,936 (37, 74 << 20): 232 / 219, 449 / 329; 128 of 3 (37 << 20): 127 / 137.
constexpr int64_t kLevelEntries = 40 << 20;
constexpr int64_t kLevels = 12;
// Entries of all rows from which on trees are taken level by level, and levels: what goes deeper has the rows behind formed at once.
// All rows at once / level by level, us a call, bf16: 64 trees of widths 2, 1, 128,251 (39 << 20 entries) 50 / 64; 8 of widths 4, 2, 2, 1,
// 151,936 (52 << 20) 65 / 74; 8, 16, 64 of widths 4, 3, 2, 1, 128,251 (64, 127, 509 << 20) 77 / 74, 125 / 75, 421 / 90.
constexpr int64_t kTreeEntries = 60 << 20;
constexpr int kTreeLevels = 6;
constexpr int64_t kManyCells = 16384;  // from which on waves take kMany

template <int DT>
static void run_all_stats(const DraftBatch &b, const DraftChain &c, const Workspace &ws, int64_t cells, hipStream_t stream)
{
    const int64_t rows = b.D + b.B + (c.draft ? b.D : 0), many = (cells + kWaves * kMany - 1) / (kWaves * kMany), one = (cells + kWaves - 1) / kWaves;
    if (rows * cells >= kManyCells)
        all_stats_kernel<DT, kMany><<<dim3((unsigned)(rows * many)), dim3(kBlock), 0, stream>>>(b, c, ws, (uint32_t)cells, (uint32_t)many);
    else
        all_stats_kernel<DT, 1><<<dim3((unsigned)(rows * one)), dim3(kBlock), 0, stream>>>(b, c, ws, (uint32_t)cells, (uint32_t)one);
}

template <int DT>
static void run_chain(const DraftBatch &b, const DraftChain &c, const DraftOutputs &o, const Workspace &ws, hipStream_t stream)
{
    const int64_t cells = cells_of(b.V), both = c.draft ? 2 : 1, groups = (cells + kWaves * kMany - 1) / (kWaves * kMany);
    const dim3 each((unsigned)b.B), block(kBlock);
    const int64_t levels = (b.D + b.B - 1) / b.B;  // rows with drafts of the longest sequence, if they are alike (what longer
                                                       // ones have behind is formed at once, behind their stop too)
    if (b.B * b.V * both >= kLevelEntries && levels > 1) {
        const dim3 rows((unsigned)(b.B * both * groups));
        int level = 0;
        for (; level < levels && level < kLevels; ++level) {
            level_stats_kernel<DT, false><<<rows, block, 0, stream>>>(b, c, ws, level, (uint32_t)cells, (uint32_t)groups);
            draft_decide_kernel<DT, false><<<each, dim3(128), 0, stream>>>(b, c, o, ws, level, cells);
        }
        level_stats_kernel<DT, true><<<rows, block, 0, stream>>>(b, c, ws, level, (uint32_t)cells, (uint32_t)groups);
        draft_decide_kernel<DT, true><<<each, dim3(128), 0, stream>>>(b, c, o, ws, level, cells);
        if (c.draft) draft_rest_kernel<DT, false><<<dim3((unsigned)(b.B * groups)), block, 0, stream>>>(b, c, o, ws, cells, (int)groups);
        draft_draw_kernel<DT, false><<<each, block, 0, stream>>>(b, c, o, ws, cells);
        return;
    }
    run_all_stats<DT>(b, c, ws, cells, stream);
    if (!c.draft) {
        draft_draw_kernel<DT, true><<<each, block, 0, stream>>>(b, c, o, ws, cells);
        return;
    }
    // as many workgroups to a sequence as fill the device, a cell at least to each wave
    const int64_t most = (cells + 15) / 16, fill = (256 + b.B - 1) / b.B, spread = most < fill ? most : fill;
    draft_rest_kernel<DT, true><<<dim3((unsigned)(b.B * spread)), dim3(1024), 0, stream>>>(b, c, o, ws, cells, (int)spread);
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
    const int64_t cells = cells_of(b.V), groups = (cells + kWaves * kMany - 1) / (kWaves * kMany);
    const dim3 rows((unsigned)(b.B * groups));
    const dim3 each((unsigned)b.B), block(kBlock);
    // few rows are all formed at once; of many only those on the paths, level by level
    if ((b.D + b.B) * b.V < kTreeEntries) {
        run_all_stats<DT>(b, DraftChain{}, ws, cells, stream);
        tree_walk_kernel<DT, false><<<each, block, 0, stream>>>(b, t, o, ws, true, cells);
        return;
    }
    const int64_t nodes = (b.D + b.B - 1) / b.B;
    const int levels = (int)(nodes < kTreeLevels ? nodes + 1 : kTreeLevels);
    for (int level = 0; level < levels; ++level) {
        node_stats_kernel<DT, false><<<rows, block, 0, stream>>>(b, ws, level == 0, (uint32_t)cells, (uint32_t)groups);
        tree_walk_kernel<DT, true><<<each, block, 0, stream>>>(b, t, o, ws, level == 0, cells);
    }
    node_stats_kernel<DT, true><<<rows, block, 0, stream>>>(b, ws, false, (uint32_t)cells, (uint32_t)groups);
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
