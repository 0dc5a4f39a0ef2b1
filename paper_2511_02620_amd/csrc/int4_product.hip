// out[n][v] = sum_k h[n][k] w[v][k] for a head w in 4-bit integers with group scales: the few hidden states that are decoded together.
//
// What bounds it is reading the codes once, so everything else has to hide behind that: a compute unit gets some 10 bytes of codes a
// cycle.  A code goes to the matrix cores as the fp16 number code - zero: masked into the fraction of 1024 (or, from bits 4 ... 7, 16 times
// itself), which takes an instruction for two codes, and an addition (or multiply-add) of two more, all of them exact.  Hidden states are scaled by a
// power of two that brings their row's largest magnitude between 2^15 and 2^16, and go there as one fp16 number (bf16 states: exact down to 2^-32 of that
// magnitude) or three (fp32 states); what is cut off is below 2^-39 of it.  A group's sum of exact products is accumulated in fp32 and scaled in
// fp32; the row's power of two comes off at the end.
#include "difr_host.hpp"
#include "int4.hpp"
#include "softmax_row.hpp"

namespace difr {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint16_t u16_any __attribute__((aligned(1)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

struct Int4Product {
    const void *h;
    int64_t N, d, ldh;
    Int4Matrix m;
    void *out;
    int64_t ld;
    int f32_out;
    int passes, per_pass;   // of the blocks of 16 rows of the head that a wave has, `per_pass` at a time
    const uint8_t *image;   // hidden states as the matrix instructions want them (int4_image_kernel), or null
    const uint32_t *tops;   // with the image: the largest magnitudes of its rows, by which they are scaled
};

constexpr int kSlab = 256;                     // elements of a row that a step takes
constexpr int kHiddenBytes = 122 * 1024;       // of LDS for hidden states that stay there

// Eight codes as fp16 numbers code - zero, two at a time: 0 4 1 5 2 6 3 7.  Hidden states are put in that order.  (Masks and 1024 in registers: one
// instruction takes one constant of another kind.)
struct CodeBits {
    uint32_t low = 0x000F000Fu, high = 0x00F000F0u, one = 0x64006400u;
    __device__ __forceinline__ CodeBits() { asm("" : "+v"(low), "+v"(high), "+v"(one)); }
    __device__ __forceinline__ f16x8 of(uint32_t w, f16x2 less) const  // less: -(1024 + zero), twice
    {
        const f16x2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f}, less64 = less + f16x2{(_Float16)960.0f, (_Float16)960.0f};
        auto pair = [](uint32_t bits) { return __builtin_bit_cast(f16x2, bits); };
        const uint32_t up = w >> 8;
        const f16x2 a = pair((w & low) | one) + less, b = __builtin_elementwise_fma(pair((w & high) | one), sixteenth, less64);
        const f16x2 c = pair((up & low) | one) + less, d = __builtin_elementwise_fma(pair((up & high) | one), sixteenth, less64);
        return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    }
};

// A block of 16 rows and a slab as a wave fetches it: neighbouring lanes neighbouring bytes (the caches are asked for each run of lanes apart; a lane
// a row of its own took four times the requests, and those were what the time went to).  Codes: lane l 16 bytes l % 8 of rows l / 8 and 8 + l / 8.
// Scales and zero points: lanes 4 r ... 4 r + 3 those of row r.
struct Int4Fetched {
    u32x4 w[2];
    uint32_t s, z;
};
constexpr int kCodePitch = kSlab / 2 + 16;  // bytes of a row of codes in LDS: 16 rows spread over the banks

// The same as the matrix instructions take it.  Lane (kg, v), v = lane % 16, has of row v the codes of the slots 8 kg ... of each step of 32:
// of every group the kg-th quarter.
template <int G>
struct Int4Slab {
    static constexpr int kGroups = kSlab / G;
    uint32_t w[8];                    // by steps
    uint32_t s[G == 32 ? 4 : 2];      // of the groups of each half, as they are stored
    uint32_t z[2];
    template <int GS>
    __device__ __forceinline__ float scale() const  // of group GS
    {
        if constexpr (G == 128)
            return __uint_as_float((uint32_t)s[GS] << 16);
        else
            return __uint_as_float(GS % 2 ? s[GS / 2] & 0xFFFF0000u : s[GS / 2] << 16);
    }
    template <int GS>
    __device__ __forceinline__ f16x2 less() const  // -(1024 + zero point) of group GS, twice
    {
        const uint32_t zero = G == 128 ? z[GS % 2] : G == 64 ? z[GS / 2 % 2] >> (8 * (GS % 2)) & 0xFFu : z[GS / 4 % 2] >> (8 * (GS % 4)) & 0xFFu;
        return __builtin_bit_cast(f16x2, (zero << 16 | zero) + 0xE400E400u);
    }
};

// Eight elements of a row of at least eight, zeros from element d on: there the row's last eight are loaded and moved down.  (In two steps, so that no
// branch stands between loads.)
template <int HT>
struct EightStates {
    static constexpr int E = Elem<HT>::kPerVec;
    u32x4 q[8 / E];
    int down;
    __device__ __forceinline__ void fetch(const typename Elem<HT>::type *p, int64_t at, int64_t d)
    {
        const int64_t from = at + 8 <= d ? at : d - 8;
        down = at - from < 8 ? (int)(at - from) : 8;
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) q[i] = *reinterpret_cast<const u32x4_any *>(p + from + i * E);
    }
    // The largest magnitude among the row's elements that were loaded, as the bits of an fp32 number (of a NaN above those of an infinity).
    __device__ __forceinline__ uint32_t largest() const
    {
        if constexpr (HT == 0) {
            auto magnitudes = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu); };
            const u16x2 top = __builtin_elementwise_max(__builtin_elementwise_max(magnitudes(q[0].x), magnitudes(q[0].y)),
                                                        __builtin_elementwise_max(magnitudes(q[0].z), magnitudes(q[0].w)));
            return (uint32_t)max(top.x, top.y) << 16;
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, q[i / 4][i % 4] & 0x7FFFFFFFu);
            return top;
        }
    }
    __device__ __forceinline__ void values(float (&e)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) unpack_vector<HT>(q[i], e + i * E);
        if (down) {
#pragma unroll
            for (int step = 8; step; step >>= 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float behind = j + step < 8 ? e[j + step] : 0.0f;
                    e[j] = down & step ? behind : e[j];
                }
            }
        }
    }
};
// Over the lanes of half a wave, whose last has it: by moves between lanes of the vector unit.
__device__ __forceinline__ uint32_t largest_of_32(uint32_t top)
{
    auto step = [&](auto CTRL, auto ROWS) {
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp((int)top, (int)top, decltype(CTRL)::value, decltype(ROWS)::value, 0xF, false));
    };
    step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xF>());  // the lane before
    step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xF>());
    step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xF>());
    step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xF>());
    step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xA>());  // the last lane of the 16 before, into the second and fourth 16
    return top;
}
// The exponent of the power of two that brings a row's largest magnitude between 2^15 and 2^16.
__device__ __forceinline__ int shift_of(uint32_t top) { return 16 - __builtin_amdgcn_frexp_expf(__uint_as_float(top)); }

// Eight elements, scaled, in the order of the codes, as the matrix instructions want them: one fp16 number each, or three whose sum they are.  Cut, not
// rounded: what is next to 2^16 stays below it.  (What is no finite number stays so, or gives NaN.)
template <int HT>
struct Eight {
    static constexpr int P = HT == 0 ? 1 : 3;
    u32x4 part[P];
    __device__ __forceinline__ Eight(float (&e)[8], int shift)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = ldexpf(e[j], shift);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            uint32_t pair[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const auto h = __builtin_amdgcn_cvt_pkrtz(e[j], e[j + 4]);
                pair[j] = __builtin_bit_cast(uint32_t, h);
                e[j] -= (float)h.x, e[j + 4] -= (float)h.y;
            }
            part[p] = u32x4{pair[0], pair[1], pair[2], pair[3]};
        }
    }
};

// The step of a half slab (128 elements) in which the eight elements `piece` of it are multiplied, and the quarter of the lanes that has them.
template <int G>
__device__ __forceinline__ void step_of(int piece, int &j, int &kg)
{
    if constexpr (G == 128)
        kg = piece >> 2, j = piece & 3;
    else if constexpr (G == 64)
        kg = piece >> 1 & 3, j = (piece >> 3) * 2 + (piece & 1);
    else
        kg = piece & 3, j = piece >> 2;
}
template <int G>
__device__ __forceinline__ int piece_of(int j, int kg)
{
    return G == 128 ? kg * 4 + j : G == 64 ? (j >> 1) * 8 + kg * 2 + (j & 1) : j * 4 + kg;
}

// Batches of more than 16 hidden states, whose fragments are the same for every workgroup and do not fit its LDS: an image of them in
// global memory.  For each slab, tile of 16 states and part, 8 fragments of 64 lanes of 16 bytes.  (40 rows of 4096, bf16: 2.2 to 4.3 us.)
constexpr int kFragment = 1024;
constexpr int kTopBytes = 1024 * 4;  // of the workspace: the largest magnitudes of the rows of a launch; then the image

// A workgroup a row, whose largest magnitude it finds first; it keeps what it has read of up to 8192 elements.
constexpr int kImageThreads = 512, kImageHeld = 2;
template <int HT, int G>
__global__ __launch_bounds__(kImageThreads) void int4_image_kernel(const typename Elem<HT>::type *h, int64_t N, int64_t d, int64_t ldh, int slabs,
                                                                   int tiles, uint8_t *image, uint32_t *tops)
{
    constexpr int P = Eight<HT>::P, F = P * 8;
    __shared__ uint32_t lds_top[kImageThreads / 32];
    const int first = threadIdx.x, row = blockIdx.x, n = row & 15;
    const typename Elem<HT>::type *const from = h + (row < N ? row : N - 1) * ldh;  // (what is made of rows behind is not stored)
    uint8_t *const to = image + (int64_t)(row >> 4) * (F * kFragment) + n * 16;
    const int pieces = slabs * 32;
    EightStates<HT> held[kImageHeld];
#pragma unroll
    for (int i = 0; i < kImageHeld; ++i) held[i].fetch(from, (int64_t)(first + i * kImageThreads) * 8, d);
    uint32_t top = 0;
    for (int piece = first + kImageHeld * kImageThreads; piece < pieces; piece += kImageThreads) {
        EightStates<HT> more;
        more.fetch(from, (int64_t)piece * 8, d);
        top = max(top, more.largest());
    }
#pragma unroll
    for (int i = 0; i < kImageHeld; ++i) top = max(top, held[i].largest());
    top = largest_of_32(top);
    if (threadIdx.x % 32 == 31) lds_top[threadIdx.x / 32] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kImageThreads / 32; ++w) top = max(top, lds_top[w]);
    const int shift = shift_of(top);
    if (first == 0) tops[row] = top;
    auto put = [&](int piece, const EightStates<HT> &states) __attribute__((always_inline)) {
        float e[8];
        states.values(e);
        const Eight<HT> x(e, shift);
        int j, kg;
        step_of<G>(piece & 15, j, kg);
        uint8_t *const at = to + (int64_t)(piece >> 5) * tiles * (F * kFragment) + (((piece >> 4 & 1) * 4 + j) * kFragment + kg * 256);
#pragma unroll
        for (int p = 0; p < P; ++p) *reinterpret_cast<u32x4 *>(at + p * 8 * kFragment) = x.part[p];
    };
#pragma unroll
    for (int i = 0; i < kImageHeld; ++i)
        if (first + i * kImageThreads < pieces) put(first + i * kImageThreads, held[i]);
    for (int piece = first + kImageHeld * kImageThreads; piece < pieces; piece += kImageThreads) {
        EightStates<HT> more;
        more.fetch(from, (int64_t)piece * 8, d);
        put(piece, more);
    }
}

// Hidden states in P parts; NT tiles of 16 of them from the image, a step ahead (RESIDENT: up to 16, converted by each workgroup and kept in
// LDS); KS slabs at once, each with its share of the waves (small heads, whose blocks are fewer than waves); RB blocks of 16 rows of
// the head to a wave at a time; D steps of codes in flight, in registers.  What bounds it, and steps of its making (those with the
// codes as bf16 numbers 16 + code), us: one bf16 row by 151,936 x 4096, 59 to 60 (5.4 TB/s; 1.05 instructions a cycle and unit): a lane fetching a
// row of its own 81, whole lines dealt by LDS 67, 16 waves instead of 8 64.  40 rows by 128,256 x 4096, 98: 0.49 vector instructions a cycle and
// unit, matrix cores busy in 25 % of the cycles, LDS reads between them, in two waves a SIMD that overlap little; RB = 1 with 16 waves 112 / 103 (spills), 4 and 3
// blocks spilt too.  17 rows by 50,257 x 2000, 25: RB = 1 with 16 waves, against 29 with RB = 2 and 8.
template <int HT, bool RESIDENT, int NT, int KS, int G, bool ZEROS, int RB, int D, int W, bool PAST>
__global__ __launch_bounds__(W * 64, 1) void int4_product_kernel(Int4Product a)
{
    constexpr int kProductWaves = W, kProductThreads = W * 64;
    constexpr int P = Eight<HT>::P, kGroups = kSlab / G, F = P * 8;
    constexpr int kSteps = G / 32;     // matrix instructions of a group
    constexpr int kStage = KS * NT * F * kFragment, kPieces = kStage / 16 / kProductThreads;
    constexpr int kTeams = kProductWaves / KS;
    static_assert(RESIDENT ? NT == 1 : kPieces * 16 * kProductThreads == kStage, "one tile stays; all threads fetch the image");
    __shared__ __attribute__((aligned(16))) uint8_t lds[RESIDENT ? kHiddenBytes : 2 * kStage];
    __shared__ __attribute__((aligned(16))) uint8_t lds_code[kProductWaves][RB * 16 * kCodePitch];  // a wave's own
    __shared__ uint32_t lds_top[NT * 16];                                                           // rows' largest magnitudes
    static_assert(KS == 1 || RB * NT * kFragment <= RB * 16 * kCodePitch, "a wave's share of the sums fits where its codes were");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int v = lane & 15, kg = lane >> 4;
    const int ks = wave % KS, team = wave / KS;                    // which slab of a step, which blocks
    const int64_t n0 = (int64_t)blockIdx.y * (16 * NT);
    const int rows_here = a.N - n0 < 16 * NT ? (int)(a.N - n0) : 16 * NT;
    const int64_t blocks = (a.m.V + 15) / 16;
    const int64_t block0 = blocks * blockIdx.x / gridDim.x, block1 = blocks * (blockIdx.x + 1) / gridDim.x;
    const int mine = (int)(block1 - block0);
    const int nslab = (int)((a.m.K + kSlab - 1) / kSlab), per = (nslab + KS - 1) / KS, total = a.passes * per;
    const bool odd = a.m.K % kSlab != 0;                           // the last slab is half a slab
    const int live_groups = (int)((a.d + G - 1) / G);              // what lies behind does not count

    auto barrier = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // ---- hidden states that stay: rows of K elements (and 16 bytes, to spread a fragment over the banks) of each part
    const int hpitch = nslab * (kSlab * 2) + 16, plane = rows_here * hpitch;
    // A slab of a row to half a wave at a time: from the first to the last for the magnitudes, and back again.
    constexpr int kHalves = kProductThreads / 32;
    EightStates<HT> states;
    const int all = rows_here * nslab, lane_piece = lane & 31;
    const uint32_t part = 65536u / nslab + 1;                      // id / nslab = id part / 2^16: of ids up to 244, which fit the LDS
    auto row_of = [&](int id) { return (int)((uint32_t)id * part >> 16); };
    auto fetch_states = [&](int at) __attribute__((always_inline)) {
        const int id = min(at + (tid >> 5), all - 1), row = row_of(id);
        states.fetch(reinterpret_cast<const typename Elem<HT>::type *>(a.h) + (n0 + row) * a.ldh, (id - row * nslab) * kSlab + lane_piece * 8, a.d);
    };
    auto put_states = [&]() __attribute__((always_inline)) {
        barrier();  // (lds_top is 0)
        int at = 0;
        for (;; fetch_states(at += kHalves)) {
            const uint32_t top = largest_of_32(states.largest());
            if (lane_piece == 31) atomicMax(&lds_top[row_of(min(at + (tid >> 5), all - 1))], top);
            if (at + kHalves >= all) break;
        }
        barrier();
        for (;; fetch_states(at -= kHalves)) {
            const int id = at + (tid >> 5), row = row_of(id);
            if (id < all) {
                float e[8];
                states.values(e);
                const Eight<HT> x(e, shift_of(lds_top[row]));
#pragma unroll
                for (int p = 0; p < P; ++p)
                    *reinterpret_cast<u32x4 *>(lds + p * plane + row * hpitch + (id - row * nslab) * (kSlab * 2) + lane_piece * 16) = x.part[p];
            }
            if (at == 0) break;
        }
    };
    // ---- or come from the image, a step ahead: global memory -> registers -> LDS
    u32x4 x[RESIDENT ? 1 : kPieces];
    const uint8_t *const image = RESIDENT ? nullptr : a.image + (int64_t)blockIdx.y * (NT * F * kFragment);
    const int64_t image_slab = (int64_t)gridDim.y * (NT * F * kFragment);
    auto fetch_hidden = [&](int step) __attribute__((always_inline)) {
        if constexpr (!RESIDENT)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int id = i * kProductThreads + tid, s = id / (NT * F * 64), at = id - s * (NT * F * 64);
                const int sl = step * KS + s < nslab ? step * KS + s : nslab - 1;
                x[i] = *reinterpret_cast<const u32x4 *>(image + sl * image_slab + at * 16);
            }
    };
    auto put_hidden = [&](int stage) __attribute__((always_inline)) {
        if constexpr (!RESIDENT)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) *reinterpret_cast<u32x4 *>(lds + stage * kStage + (i * kProductThreads + tid) * 16) = x[i];
    };
    // fragment of step j of a half slab
    auto hidden = [&](int stage, int sl, int t, int p, int seg, int j) __attribute__((always_inline)) {
        if constexpr (RESIDENT)
            return *reinterpret_cast<const f16x8 *>(lds + p * plane + (v < rows_here ? v : 0) * hpitch + (sl * 32 + seg * 16 + piece_of<G>(j, kg)) * 16);
        else
            return *reinterpret_cast<const f16x8 *>(lds + stage * kStage + ((ks * NT + t) * F + p * 8 + seg * 4 + j) * kFragment + lane * 16);
    };
    // ---- the head: registers, D steps ahead.  Rows of the workgroup by 32-bit offsets from its first.
    Int4Fetched slab[D][RB];
    const int pitch = (int)(a.m.K / 2), groups = (int)(a.m.K / G);
    const int64_t row0 = block0 * 16;
    const int row_end = (int)((block1 * 16 < a.m.V ? block1 * 16 : a.m.V) - row0);
    const uint8_t *const codes = a.m.codes + row0 * pitch, *const scales = reinterpret_cast<const uint8_t *>(a.m.scales + row0 * groups);
    const uint8_t *const zeros = ZEROS ? a.m.zeros + row0 * groups : nullptr;
    auto first_block = [&](int pass) { return (pass * kTeams + team) * a.per_pass; };
    int f_pass = 0, f_step = 0;
    uint32_t at_code[RB][2], at_group[RB];
    // (rows that are not there: the last one again, from the caches)
    auto aim = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int r = (first_block(f_pass) + min(b, a.per_pass - 1)) * 16;
            at_code[b][0] = (uint32_t)min(r + (lane >> 3), row_end - 1) * (uint32_t)pitch;
            at_code[b][1] = (uint32_t)min(r + 8 + (lane >> 3), row_end - 1) * (uint32_t)pitch;
            at_group[b] = (uint32_t)min(r + (lane >> 2), row_end - 1) * (uint32_t)groups;
        }
    };
    aim();
    // No branches around loads: the waits for them are counted.
    auto fetch_head = [&](Int4Fetched (&to)[RB]) __attribute__((always_inline)) {
        const int ask = f_step * KS + ks, sl = ask < nslab ? ask : nslab - 1;
        const bool half = odd && sl + 1 == nslab;  // the first half again in the second's place
        const uint8_t *const c0 = codes + sl * (kSlab / 2), *const s0 = scales + sl * (kGroups * 2), *const z0 = ZEROS ? zeros + sl * kGroups : nullptr;
        const uint32_t part = lane & (half ? 3 : 7), own = lane & (G == 32 ? (half ? 1 : 3) : (half ? 0 : 1)), zown = lane & (half ? 0 : 1);
#pragma unroll
        for (int b = 0; b < RB; ++b) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 *const from = reinterpret_cast<const u32x4 *>(c0 + (at_code[b][i] + part * 16));
                if constexpr (PAST)
                    to[b].w[i] = __builtin_nontemporal_load(from);
                else
                    to[b].w[i] = *from;
            }
            if constexpr (G == 128) {
                to[b].s = *reinterpret_cast<const u16_any *>(s0 + (2 * at_group[b] + own * 2));
                if constexpr (ZEROS) to[b].z = *(z0 + (at_group[b] + zown));
            } else {
                to[b].s = *reinterpret_cast<const u32_any *>(s0 + (2 * at_group[b] + own * 4));
                if constexpr (ZEROS && G == 64) to[b].z = *reinterpret_cast<const u16_any *>(z0 + (at_group[b] + zown * 2));
                if constexpr (ZEROS && G == 32) to[b].z = *reinterpret_cast<const u32_any *>(z0 + (at_group[b] + zown * 4));
            }
        }
        if (++f_step == per) {
            f_step = 0;
            if (f_pass + 1 < a.passes) ++f_pass;
            aim();
        }
    };
    // From the fetching lanes to the multiplying ones: codes by way of LDS (a wave's operations on it keep their order), the rest from lane 4 v.
    uint8_t *const my_code = lds_code[wave];
    auto deal = [&](const Int4Fetched (&from)[RB], Int4Slab<G> (&to)[RB]) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<u32x4 *>(my_code + (b * 16 + i * 8 + (lane >> 3)) * kCodePitch + (lane & 7) * 16) = from[b].w[i];
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        static_for<RB>([&](auto B) __attribute__((always_inline)) {
            constexpr int b = decltype(B)::value;
            const uint8_t *const c = my_code + (b * 16 + v) * kCodePitch;
            static_for<2>([&](auto SEG) __attribute__((always_inline)) {
                constexpr int seg = decltype(SEG)::value;
                if constexpr (G == 128) {
                    const u32x4 q = *reinterpret_cast<const u32x4 *>(c + seg * 64 + kg * 16);
                    to[b].w[seg * 4] = q.x, to[b].w[seg * 4 + 1] = q.y, to[b].w[seg * 4 + 2] = q.z, to[b].w[seg * 4 + 3] = q.w;
                } else if constexpr (G == 64) {
                    static_for<2>([&](auto J) __attribute__((always_inline)) {
                        constexpr int j = decltype(J)::value;
                        const u32x2 q = *reinterpret_cast<const u32x2 *>(c + seg * 64 + j * 32 + kg * 8);
                        to[b].w[seg * 4 + 2 * j] = q.x, to[b].w[seg * 4 + 2 * j + 1] = q.y;
                    });
                } else {
                    static_for<4>([&](auto J) __attribute__((always_inline)) {
                        constexpr int j = decltype(J)::value;
                        to[b].w[seg * 4 + j] = *reinterpret_cast<const uint32_t *>(c + seg * 64 + j * 16 + kg * 4);
                    });
                }
            });
            static_for<(G == 32 ? 4 : 2)>([&](auto I) __attribute__((always_inline)) {
                constexpr int i = decltype(I)::value;
                to[b].s[i] = __builtin_amdgcn_ds_bpermute(v * 16 + i * 4, from[b].s);
                if constexpr (ZEROS && i < 2) to[b].z[i] = __builtin_amdgcn_ds_bpermute(v * 16 + i * 4, from[b].z);
            });
        });
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    };

    const CodeBits code_values;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 acc[RB][NT];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[b][t] = zero;

    int pass = 0, step = 0;
    auto multiply = [&](const Int4Slab<G> (&w)[RB], int stage) __attribute__((always_inline)) {
        const int sl = step * KS + ks;
        if (sl >= nslab || first_block(pass) >= mine) return;
        // groups of the slab that count (none of the second half of half a slab, whose codes are the first's again and whose states are 0)
        const int live = sl + 1 == nslab ? live_groups - sl * kGroups : kGroups;
        static_for<2>([&](auto SEG) __attribute__((always_inline)) {
            constexpr int seg = decltype(SEG)::value;
            f32x4 part[RB][NT];
            static_for<4>([&](auto J) __attribute__((always_inline)) {
                constexpr int j = decltype(J)::value, g = j / kSteps, js = j % kSteps, gs = seg * (128 / G) + g;  // step of the half, group, step of it
                f16x8 f[NT][P];
                static_for<NT * P>([&](auto I) __attribute__((always_inline)) {
                    constexpr int t = decltype(I)::value / P, p = decltype(I)::value % P;
                    f[t][p] = hidden(stage, sl, t, p, seg, j);
                });
                static_for<RB>([&](auto B) __attribute__((always_inline)) {
                    constexpr int b = decltype(B)::value;
                    f16x2 less = {(_Float16)-1032.0f, (_Float16)-1032.0f};
                    if constexpr (ZEROS) less = w[b].template less<gs>();
                    const f16x8 c = code_values.of(w[b].w[seg * 4 + j], less);
                    static_for<NT * P>([&](auto I) __attribute__((always_inline)) {
                        constexpr int t = decltype(I)::value / P, p = decltype(I)::value % P;
                        part[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[t][p], c, js == 0 && p == 0 ? zero : part[b][t], 0, 0, 0);
                    });
                    if constexpr (js + 1 == kSteps) {
                        const float scale = gs < live ? w[b].template scale<gs>() : 0.0f;
                        static_for<NT>([&](auto TT) __attribute__((always_inline)) {
                            constexpr int t = decltype(TT)::value;
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[b][t][r] = __builtin_fmaf(scale, part[b][t][r], acc[b][t][r]);
                        });
                    }
                });
            });
        });
    };

    // Lane (kg, v): rows 4 kg ... 4 kg + 3 of a tile of hidden states, row v of the block.
    auto store = [&]() __attribute__((always_inline)) {
        static_for<RB>([&](auto B) __attribute__((always_inline)) {
            constexpr int b = decltype(B)::value;
            const int r = (first_block(pass) + b) * 16 + v;
            const bool in_pass = b < a.per_pass && first_block(pass) + b < mine;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = t * 16 + kg * 4 + i;
                    const float sum = ldexpf(acc[b][t][i], -shift_of(lds_top[n]));
                    if (in_pass && r < row_end && n < rows_here) {
                        if (a.f32_out)
                            reinterpret_cast<float *>(a.out)[(n0 + n) * a.ld + row0 + r] = sum;
                        else
                            store_element<0>(reinterpret_cast<uint16_t *>(a.out) + (n0 + n) * a.ld + row0 + r, sum);
                    }
                    acc[b][t][i] = 0.0f;
                }
        });
    };
    // The shares of a team's waves are added up, in the order of their slabs.
    auto join = [&]() __attribute__((always_inline)) {
        auto share = [&](int w, int b, int t) { return reinterpret_cast<f32x4 *>(lds_code[w]) + (b * NT + t) * 64 + lane; };
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t) *share(wave, b, t) = acc[b][t];
        barrier();
        if (ks == 0)
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 1; i < KS; ++i) acc[b][t] += *share(wave + i, b, t);
        barrier();
    };

    // Loads go out in the order of the loop below, from the start on, and stay in it: waits count what has gone out since.
    if constexpr (RESIDENT) {
        fetch_states(0);
        if (tid < 16) lds_top[tid] = 0;
    } else if (tid < NT * 16) {
        lds_top[tid] = a.tops[n0 + tid];
    }
    fetch_hidden(0);
    static_for<D>([&](auto U) __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        fetch_head(slab[decltype(U)::value]);
    });
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (RESIDENT) put_states();
    put_hidden(0);
    int n_put = per > 1 ? 1 : 0;  // the next step to put in LDS
    fetch_hidden(n_put);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (RESIDENT) barrier();
    for (int at0 = 0; at0 < total; at0 += D) {  // (whole rounds of D: the steps past the end have no blocks)
        static_for<D>([&](auto U) __attribute__((always_inline)) {
            constexpr int u = decltype(U)::value;
            const int at = at0 + u;
            if constexpr (!RESIDENT) barrier();  // the step's hidden states are in LDS, and nobody reads those before them any more
            Int4Slab<G> w[RB];
            deal(slab[u], w);
            __builtin_amdgcn_sched_barrier(0);
            fetch_head(slab[u]);
            __builtin_amdgcn_sched_barrier(0);
            multiply(w, at & 1);
            if (++step == per) {
                if constexpr (KS > 1) join();
                if (ks == 0) store();
                if constexpr (KS > 1)
#pragma unroll
                    for (int b = 0; b < RB; ++b)
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[b][t] = zero;
                step = 0;
                ++pass;
            }
            put_hidden((at + 1) & 1);
            n_put = n_put + 1 < per ? n_put + 1 : 0;
            fetch_hidden(n_put);
            __builtin_amdgcn_sched_barrier(0);
        });
    }
}

// Heads of fewer blocks of 16 rows than the waves of the device: the slabs of a row are shared (by a rule on the head alone, so that a row's
// sums do not depend on the rows beside it).
static bool shared_slabs(int64_t V) { return (V + 15) / 16 < 1024; }
// Whether N hidden states stay in LDS.
static bool resident(int64_t N, int64_t K, int parts)
{
    const int64_t slabs = (K + kSlab - 1) / kSlab;
    return N <= 16 && N * parts * (slabs * kSlab * 2 + 16) <= kHiddenBytes;
}

template <int HT, bool RESIDENT, int NT, int KS, int RB, int D, int W>
static void run_product(Int4Product a, hipStream_t stream)
{
    constexpr int kTeams = W / KS;
    const int64_t blocks = (a.m.V + 15) / 16, grid = blocks < 256 ? blocks : 256;
    const int64_t most = (blocks + grid - 1) / grid, each = (most + kTeams - 1) / kTeams;  // blocks of a workgroup, of a team
    a.passes = (int)((each + RB - 1) / RB);
    a.per_pass = (int)((each + a.passes - 1) / a.passes);
    const unsigned tiles = (unsigned)((a.N + 16 * NT - 1) / (16 * NT));
    auto run = [&](auto G) {
        constexpr int group = decltype(G)::value;
        if constexpr (!RESIDENT)
            int4_image_kernel<HT, group><<<dim3(tiles * NT * 16), dim3(kImageThreads), 0, stream>>>(
                (const typename Elem<HT>::type *)a.h, a.N, a.d, a.ldh, (int)((a.m.K + kSlab - 1) / kSlab), (int)(tiles * NT),
                const_cast<uint8_t *>(a.image), const_cast<uint32_t *>(a.tops));
        auto go = [&](auto ZEROS, auto PAST) {
            int4_product_kernel<HT, RESIDENT, NT, KS, group, decltype(ZEROS)::value, RB, D, W, decltype(PAST)::value>
                <<<dim3((unsigned)grid, tiles), dim3(W * 64), 0, stream>>>(a);
        };
        // a matrix larger than the 256 MB Infinity Cache is read past it (with D = 4 for 3, 151,936 x 4096 64 -> 58 us; 50,257 x 2000, which fits,
        // lost: 29 -> 32)
        if (KS == 1 && a.m.V * a.m.K / 2 > (int64_t)256 << 20)
            a.m.zeros ? go(std::true_type(), std::bool_constant<KS == 1>()) : go(std::false_type(), std::bool_constant<KS == 1>());
        else
            a.m.zeros ? go(std::true_type(), std::false_type()) : go(std::false_type(), std::false_type());
    };
    a.m.group == 32 ? run(std::integral_constant<int, 32>()) : a.m.group == 64 ? run(std::integral_constant<int, 64>()) : run(std::integral_constant<int, 128>());
}

constexpr int kShortRows = 8;  // hidden states of a pass over the head

// Rows of fewer than eight elements, whose hidden states do not fill 16 bytes: a thread a row of the head.
template <int HT>
__global__ __launch_bounds__(kBlock) void int4_short_kernel(Int4Product a)
{
    const int64_t v = (int64_t)blockIdx.x * kBlock + threadIdx.x, n0 = (int64_t)blockIdx.y * kShortRows;
    if (v >= a.m.V) return;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(a.m.codes + v * (a.m.K / 2));
    const int64_t g = v * (a.m.K / a.m.group);
    const float s = __uint_as_float((uint32_t)a.m.scales[g] << 16), z = a.m.zeros ? (float)a.m.zeros[g] : 8.0f;
    for (int64_t n = n0; n < n0 + kShortRows && n < a.N; ++n) {
        const typename Elem<HT>::type *row = reinterpret_cast<const typename Elem<HT>::type *>(a.h) + n * a.ldh;
        float sum = 0.0f;
        // (a weight is exact in fp32)
        for (int k = 0; k < (int)a.d; ++k) sum = __builtin_fmaf(s * ((float)(w >> (4 * k) & 15u) - z), Elem<HT>::to_float(row[k]), sum);
        if (a.f32_out)
            reinterpret_cast<float *>(a.out)[n * a.ld + v] = sum;
        else
            store_element<0>(reinterpret_cast<uint16_t *>(a.out) + n * a.ld + v, sum);
    }
}

// Rows of hidden states whose image is made at once, and tiles of them that it holds.
static int64_t image_rows(int64_t N) { return N < 1024 ? (N + 63) / 64 * 64 : 1024; }

size_t int4_product_workspace_bytes(int64_t N, int64_t d, int dtype)
{
    const int64_t K = (d + kInt4Slab - 1) / kInt4Slab * kInt4Slab;
    const int parts = dtype == 0 ? 1 : 3;
    if (d < 8 || resident(N, K, parts)) return 0;
    return (size_t)(kTopBytes + image_rows(N) / 16 * ((K + kSlab - 1) / kSlab) * (parts * 8) * kFragment);
}

int launch_int4_product(const void *h, int h_dtype, int64_t N, int64_t d, int64_t ldh, const Int4Matrix &m, void *out, int dtype, int64_t ld,
                        void *workspace, hipStream_t stream)
{
    const int64_t most = 1024;  // rows of hidden states of a launch
    const bool stay = resident(N, m.K, h_dtype == 0 ? 1 : 3), shared = shared_slabs(m.V);
    for (int64_t n = 0; n < N; n += most) {
        const Int4Product a{(const char *)h + n * ldh * (h_dtype == 0 ? 2 : 4), N - n < most ? N - n : most, d, ldh, m,
                            (char *)out + n * ld * (dtype == 0 ? 2 : 4), ld, dtype != 0, 0, 0, stay || !workspace ? nullptr : (const uint8_t *)workspace + kTopBytes, (const uint32_t *)workspace};
        if (d < 8) {
            const dim3 grid((unsigned)((m.V + kBlock - 1) / kBlock), (unsigned)((a.N + kShortRows - 1) / kShortRows));
            if (h_dtype == 0)
                int4_short_kernel<0><<<grid, dim3(kBlock), 0, stream>>>(a);
            else
                int4_short_kernel<1><<<grid, dim3(kBlock), 0, stream>>>(a);
        } else if (h_dtype == 0) {
            if (stay)
                shared ? run_product<0, true, 1, 4, 1, 3, 16>(a, stream) : run_product<0, true, 1, 1, 1, 4, 16>(a, stream);
            else if (shared)
                run_product<0, false, 1, 4, 1, 2, 8>(a, stream);
            else
                a.N <= 32 ? run_product<0, false, 2, 1, 1, 2, 16>(a, stream) : a.N <= 48 ? run_product<0, false, 3, 1, 2, 2, 8>(a, stream) : run_product<0, false, 4, 1, 2, 1, 8>(a, stream);
        } else {
            if (stay)
                shared ? run_product<1, true, 1, 2, 1, 3, 16>(a, stream) : run_product<1, true, 1, 1, 1, 3, 16>(a, stream);
            else if (shared)
                run_product<1, false, 1, 2, 1, 2, 8>(a, stream);
            else
                a.N <= 16 ? run_product<1, false, 1, 1, 4, 1, 8>(a, stream) : run_product<1, false, 2, 1, 3, 1, 8>(a, stream);
        }
    }
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace difr
