// The product of two matrices in microscaled 4-bit floating point, out[n][v] = sum_k a[n][k] b[v][k]: hidden states by an LM head.
// Elements stay as they are stored until the matrix cores take them, 32 with their scale at a time; accumulation is in fp32.
#include "difr_host.hpp"
#include "softmax_row.hpp"
#include "token_loss.hpp"

namespace difr {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Mx4Product {
    const uint8_t *a, *as;  // [N][K / 2] codes and [N][K / 32] scales of the hidden states
    const uint8_t *b, *bs;  // [V] of the head
    int64_t N, V, K;
    void *out;
    int64_t ld;
    const uint8_t *ta, *tb;  // the scales by tiles and slabs (mx4_tile_scales_kernel)
};

constexpr int kMxTile = 256;       // rows of either matrix that a workgroup multiplies
constexpr int kMxSlabBytes = 128;  // of a row, staged through LDS per step: 256 elements

// How the product is cut: token blocks of kMxTile rows of a, times `splits` contiguous ranges of tiles of kMxTile rows of b.
struct Mx4Plan {
    int n_tb, n_vt, splits;
};

// The 32 codes of a lane's fragment, 4 bits each, in four dwords, and nothing above them: the instruction reads the lower half only for this type.
__device__ __forceinline__ i32x8 fp4_operand(i32x4 v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// acc += a b for fragments of 32 x 64 elements; byte STEP of the two scale registers is the scale of the lane's 32.
template <int STEP>
__device__ __forceinline__ f32x16 fp4_mfma(i32x4 a, i32x4 b, f32x16 acc, int scale_a, int scale_b)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(a), fp4_operand(b), acc, 4, 4, STEP, scale_a, STEP, scale_b);
}

// The scales of a matrix in the order the product's tiles want them: for each tile of 256 rows and each slab of 256 elements, 8 bytes a
// row, those of the slab's even blocks and then those of its odd ones.  A lane of the product has the even or the odd ones, and one
// 4-byte read serves it for four steps; a tile's share of a slab is 2 KB without gaps, where the rows themselves would have to be
// gathered 8 bytes at a time.  Rows and blocks that are not there get 0.  One workgroup 32 rows and 16 slabs: rows are read 128 bytes at
// a time, turned in LDS, and written 256 bytes at a time.
constexpr int kScaleRows = 32, kScaleSlabs = 16;
__global__ __launch_bounds__(kBlock) void mx4_tile_scales_kernel(const uint8_t *a, int64_t N, const uint8_t *b, int64_t V, int64_t K, int n_tb,
                                                                 uint8_t *out)
{
    __shared__ uint32_t lds[kScaleRows][2 * kScaleSlabs + 1];
    const int tile = blockIdx.x / (kMxTile / kScaleRows), row0 = blockIdx.x % (kMxTile / kScaleRows) * kScaleRows, slab0 = blockIdx.y * kScaleSlabs;
    const int nk = (int)((K + 255) / 256), words = (int)(K / 128);  // slabs, and 4-byte words of scales of a row
    const bool is_a = tile < n_tb;
    const int64_t first = (int64_t)(is_a ? tile : tile - n_tb) * kMxTile + row0, rows = is_a ? N : V;
    const uint32_t *m = reinterpret_cast<const uint32_t *>(is_a ? a : b);
#pragma unroll
    for (int i = 0; i < kScaleRows * 2 * kScaleSlabs / kBlock; ++i) {
        const int e = threadIdx.x + i * kBlock, r = e / (2 * kScaleSlabs), w = e % (2 * kScaleSlabs), word = 2 * slab0 + w;
        lds[r][w] = first + r < rows && word < words ? m[(first + r) * words + word] : 0u;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kScaleRows * kScaleSlabs / kBlock; ++i) {
        const int e = threadIdx.x + i * kBlock, r = e % kScaleRows, k = e / kScaleRows;
        if (slab0 + k >= nk) continue;
        const uint32_t lo = lds[r][2 * k], hi = lds[r][2 * k + 1];
        const uint2 w = {__builtin_amdgcn_perm(hi, lo, 0x06040200u), __builtin_amdgcn_perm(hi, lo, 0x07050301u)};
        *reinterpret_cast<uint2 *>(out + (((int64_t)tile * nk + slab0 + k) * kMxTile + row0 + r) * 8) = w;
    }
}

// One 32 x 32 block of accumulators.  This lane's are of one row of the output, columns 8 (r / 4) + (r % 4) + 4 lh of the block; lanes l
// and l + 32 have the same row and four columns each in turn.
template <bool AGPR>
__device__ __forceinline__ void fetch_block(const f32x16 acc, float x[16])
{
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        if constexpr (AGPR)
            asm("v_accvgpr_read_b32 %0, %1" : "=v"(x[r]) : "a"(acc[r]));
        else
            x[r] = acc[r];
    }
}
// In bf16 they trade, so that each has eight in a row: q[h] holds columns 16 h + 8 lh ... + 7.
template <bool AGPR>
__device__ __forceinline__ void pack_block(const f32x16 acc, u32x4 q[2])
{
    float x[16];
    fetch_block<AGPR>(acc, x);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float *y = x + 8 * h;
        const auto s0 = __builtin_amdgcn_permlane32_swap(pack_bf16(y[0], y[1]), pack_bf16(y[4], y[5]), false, false);
        const auto s1 = __builtin_amdgcn_permlane32_swap(pack_bf16(y[2], y[3]), pack_bf16(y[6], y[7]), false, false);
        q[h] = u32x4{s0[0], s1[0], s0[1], s1[1]};
    }
}

// When the 16 copies of a slab go out, spaced as in the fused LM head: after every second matrix instruction of the 32 of the fourth k step of
// one slab and the first of the next.  The copy after instruction n of them, or -1.
static constexpr int product_copy_at_slot(int n) { return n % 2 == 0 ? n / 2 : -1; }

// 256 threads = 4 waves, 2 (rows of b) x 2 (rows of a), each with a 128 x 128 sub-tile of 4 x 4 accumulator blocks.  One wave per SIMD.
// LDS: two stages of [256 rows][128 bytes] for either operand; the eight 16-byte chunks of a row, one block of 32 elements each, are
// permuted by (row / 2) % 8, so that the reads of 16 consecutive rows spread over the banks.  A slab is four k steps of 64 elements, a
// lane's share of a step one chunk of one row.  The scales of a slab go through LDS too (8 bytes a row).
//
// Where K is an odd number of 128s the last slab of a row is half a slab: its copies fetch its four chunks twice, and its last two k steps
// multiply zeros.
template <int DT, bool HALF>
__global__ __launch_bounds__(kBlock, 1) void mx4_product_kernel(Mx4Product m, Mx4Plan plan)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds_b[2][kMxTile * kMxSlabBytes];  // 32 KB per stage
    __shared__ __attribute__((aligned(16))) uint8_t lds_a[2][kMxTile * kMxSlabBytes];
    __shared__ __attribute__((aligned(16))) uint8_t lds_s[2][2 * kMxTile * 8];          // scales: rows of a, rows of b
    __shared__ __attribute__((aligned(16))) uint8_t lds_out[kWaves][32 * 128];          // 128 bytes of 32 rows of the output
    typedef typename Elem<DT>::type elem;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wv = wave >> 1, wt = wave & 1;
    const int l32 = lane & 31, lh = lane >> 5;

    // Consecutive workgroup ids go to different XCDs; each XCD takes a compact set of token blocks across the ranges of b, so that its
    // L2 sees a tile from several workgroups at about the same time.
    const int G = plan.n_tb * plan.splits;
    int q = blockIdx.x;
    if (G % 8 == 0) q = (q % 8) * (G / 8) + q / 8;
    const int tb = q / plan.splits, sp = q % plan.splits;
    const int vt0 = (int)((int64_t)sp * plan.n_vt / plan.splits), vt1 = (int)((int64_t)(sp + 1) * plan.n_vt / plan.splits);
    const int64_t n0 = (int64_t)tb * kMxTile;
    const uint32_t pitch = (uint32_t)(m.K / 2);  // bytes of a row's codes
    const int nk = (int)((m.K + 255) / 256);
    const int32_t V = (int32_t)m.V;

    // ---- copies: global memory straight into LDS.  Lane i of a copy lands in chunk i % 8 of row i / 8 and fetches the chunk that the
    // permutation puts there; thread -> rows (tid / 8) + 32 p.  Uniform base plus an invariant lane offset.
    const int crow = tid >> 3;
    const int cchunk = (tid & 7) ^ ((crow >> 1) & 7);
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);
    const uint32_t last_a = (uint32_t)((m.N - n0 < kMxTile ? m.N - n0 : kMxTile) - 1);
    uint32_t aoff[8], boff[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) aoff[p] = min((uint32_t)(crow + 32 * p), last_a) * pitch + (uint32_t)cchunk * 16u;
#pragma unroll
    for (int p = 0; p < 8; ++p) boff[p] = (uint32_t)(crow + 32 * p) * pitch + (uint32_t)cchunk * 16u;
    // rows past the end of b (its last tile) re-read the last row
    uint32_t most_b;
    auto set_most = [&](int vt) {
        const int32_t left = (V - vt * kMxTile < kMxTile ? V - vt * kMxTile : kMxTile) - 1;
        most_b = (uint32_t)left * pitch + (uint32_t)cchunk * 16u;
    };
    set_most(vt0);
    // what a lane's offset is less by: in a half slab the upper chunks are those of the lower half again
    const uint32_t back_in_half = HALF && cchunk >= 4 ? 64u : 0u;
    uint32_t back = nk == 1 ? back_in_half : 0u;
    int l_vt = vt0, l_kt = 0;  // the next slab to fetch; past the end it stays on the last tile
    // (no branches: the compiler would carry the matrix instructions before one past it and issue them in one piece)
    auto advance_cursor = [&]() {
        const bool wrap = l_kt + 1 == nk;
        l_kt = wrap ? 0 : l_kt + 1;
        l_vt += wrap && l_vt + 1 < vt1 ? 1 : 0;
        set_most(l_vt);
        if (HALF) back = l_kt + 1 == nk ? back_in_half : 0u;
    };
    const uint8_t *const abase = m.a + n0 * pitch;
    // chunk i (0-7: rows of b, 8-15: rows of a) of the cursor's slab -> LDS stage buf (M0 carries the LDS address of lane 0)
    auto copy_chunk = [&](auto I, int buf) {
        constexpr int i = decltype(I)::value;
        const uint8_t *sbase = i < 8 ? m.b + (int64_t)l_vt * kMxTile * pitch + (int64_t)l_kt * kMxSlabBytes : abase + (int64_t)l_kt * kMxSlabBytes;
        const uint32_t voff = (i < 8 ? min(boff[i & 7], most_b) : aoff[i & 7]) - (HALF ? back : 0u);
        const uint8_t *stage = (i < 8 ? &lds_b[buf][0] : &lds_a[buf][0]) + 8 * wave_u * kMxSlabBytes;
        const uint32_t lds_base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)stage;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0"
                     :
                     : "s"(sbase), "v"(voff), "s"(lds_base), "n"(32 * (i & 7) * kMxSlabBytes)
                     : "memory", "m0", "scc");
#pragma clang diagnostic pop
    };
    auto copies_landed = [&]() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // the cursor's scales: 4 KB, a copy for each wave
    auto copy_scales = [&](int buf) {
        const uint8_t *sbase = wave_u < 2 ? m.ta + ((int64_t)tb * nk + l_kt) * (kMxTile * 8) + wave_u * 1024
                                          : m.tb + ((int64_t)l_vt * nk + l_kt) * (kMxTile * 8) + (wave_u - 2) * 1024;
        const uint32_t voff = (uint32_t)lane * 16u;
        const uint8_t *stage = &lds_s[buf][0] + wave_u * 1024;
        const uint32_t lds_base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)stage;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(sbase), "v"(voff), "s"(lds_base) : "memory", "m0");
#pragma clang diagnostic pop
    };

    // ---- fragments: lane -> row l32 of a 32-row block, chunk 2 step + lh
    const int sw = (l32 >> 1) & 7;
    const int b_row = (wv * 128 + l32) * kMxSlabBytes, a_row = (wt * 128 + l32) * kMxSlabBytes;
    struct Frag {
        i32x4 b[4], a[4];
    };
    auto read_frag = [&](Frag &f, int i, int buf, int step) {
        const int off = ((2 * step + lh) ^ sw) * 16;
        if (i < 4)
            f.b[i] = *reinterpret_cast<const i32x4 *>(&lds_b[buf][b_row + i * 32 * kMxSlabBytes + off]);
        else
            f.a[i - 4] = *reinterpret_cast<const i32x4 *>(&lds_a[buf][a_row + (i - 4) * 32 * kMxSlabBytes + off]);
    };

    struct Scales {
        int b[4], a[4];
    };
    auto read_scales = [&](Scales &f, int buf) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f.a[j] = *reinterpret_cast<const int *>(&lds_s[buf][(wt * 128 + j * 32 + l32) * 8 + 4 * lh]);
            f.b[j] = *reinterpret_cast<const int *>(&lds_s[buf][(kMxTile + wv * 128 + j * 32 + l32) * 8 + 4 * lh]);
        }
    };

    f32x16 acc[4][4];
    Frag F0, F1;
    Scales sc, sc_next;
    auto kstep = [&](auto STEP, const Frag &cur, Frag &nxt, int buf_next, int step_next, auto &&extra) {
        constexpr int step = decltype(STEP)::value;
        static_for<8>([&](auto I) {
            constexpr int i = decltype(I)::value, e0 = 2 * i, e1 = 2 * i + 1;
            acc[e0 >> 2][e0 & 3] = fp4_mfma<step>(cur.b[e0 >> 2], cur.a[e0 & 3], acc[e0 >> 2][e0 & 3], sc.b[e0 >> 2], sc.a[e0 & 3]);
            extra(std::integral_constant<int, e0>());
            acc[e1 >> 2][e1 & 3] = fp4_mfma<step>(cur.b[e1 >> 2], cur.a[e1 & 3], acc[e1 >> 2][e1 & 3], sc.b[e1 >> 2], sc.a[e1 & 3]);
            extra(std::integral_constant<int, e1>());
            read_frag(nxt, i, buf_next, step_next);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    auto drop = [&](Frag &f, int keep) {  // keep: -1, or 0
#pragma unroll
        for (int j = 0; j < 4; ++j) f.a[j] &= keep;
    };
    int par = 0;  // LDS stage of the slab being multiplied
    const std::integral_constant<int, 0> k0;
    const std::integral_constant<int, 1> k1;
    const std::integral_constant<int, 2> k2;
    const std::integral_constant<int, 3> k3;
    auto cp = [&](auto PH, int buf) {
        return [&, buf](auto E) {
            constexpr int c = product_copy_at_slot(16 * decltype(PH)::value + decltype(E)::value);
            if constexpr (c >= 0) copy_chunk(std::integral_constant<int, c>(), buf);
        };
    };
    // One slab.  The stage of slab g is last read in its third k step, so after the barrier that follows it is free, and the copies of
    // slab g + 2 go into it during the fourth step of slab g and the first of slab g + 1; each wave waits for its own copies before
    // the barrier of slab g + 1.  The first fragments of the next slab, of the next tile too, are read in the fourth step.
    auto slab = [&](int keep) {
        copy_scales(par ^ 1);
        kstep(k0, F0, F1, par, 1, cp(k1, par ^ 1));
        kstep(k1, F1, F0, par, 2, [&](auto) {});
        advance_cursor();
        if (HALF) drop(F0, keep);
        kstep(k2, F0, F1, par, 3, [&](auto) {});
        copies_landed();
        barrier();
        read_scales(sc_next, par ^ 1);
        if (HALF) drop(F1, keep);
        kstep(k3, F1, F0, par ^ 1, 0, cp(k0, par));
        sc = sc_next;
        par ^= 1;
    };

    // prologue: slab 0 whole, and of slab 1 what the fourth k step of a slab before it would have issued
    static_for<16>([&](auto I) { copy_chunk(I, 0); });
    copy_scales(0);
    advance_cursor();
    static_for<16>([&](auto E) { cp(k0, 1)(E); });
    copies_landed();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) read_frag(F0, i, 0, 0);
    read_scales(sc, 0);

    for (int vt = vt0; vt < vt1; ++vt) {
        const int64_t v0 = (int64_t)vt * kMxTile;
        const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = zero;
        for (int kt = 0; kt < nk; ++kt) slab(kt + 1 == nk ? 0 : -1);

        // The tile is stored in whole 128-byte lines: a lane's accumulators are 16 bytes of a row at a time, 32 rows of a wave, and the L2
        // takes a piece of a line no faster than a whole one.  So each wave turns 128 bytes of 32 rows in LDS of its own (whose operations
        // keep their order within a wave) and stores eight lines at a time, past the caches, which have better use for the operands.
        // 4096 x 151,936 x 4096, us: 32 bytes of 32 rows at a time 1343, lines 1305, past the caches 1259 (32 bytes past them 1960).
        // (The accumulators are fetched by assembly statements, which the compiler does not keep away from the matrix instructions that
        // write them: the first one read was written fifteen instructions ago, the last four are read hundreds of cycles later.)
        const bool whole = v0 + kMxTile <= m.V && n0 + kMxTile <= m.N;
        uint8_t *const turn = &lds_out[wave][0];
        const int orow = lane >> 3, ochunk = lane & 7;
        constexpr int E = Elem<DT>::kPerVec;
        elem *const out0 = reinterpret_cast<elem *>(m.out) + (n0 + wt * 128 + orow) * m.ld + v0 + wv * 128 + ochunk * E;
        constexpr int kParts = DT == 0 ? 2 : 4;  // of the wave's 128 columns, 128 bytes each
        static_for<4>([&](auto JB) {
            constexpr int jb = decltype(JB)::value;
            static_for<kParts>([&](auto PART) {
                constexpr int part = decltype(PART)::value;
                auto put = [&](int chunk, u32x4 q) { *reinterpret_cast<u32x4 *>(turn + l32 * 128 + (chunk ^ (l32 & 7)) * 16) = q; };
                if constexpr (DT == 0) {
                    static_for<2>([&](auto I) {
                        constexpr int i = decltype(I)::value;
                        u32x4 q[2];
                        pack_block<true>(acc[2 * part + i][jb], q);
                        put(4 * i + lh, q[0]);
                        put(4 * i + 2 + lh, q[1]);
                    });
                } else {
                    float x[16];
                    fetch_block<true>(acc[part][jb], x);
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        put(2 * g + lh, u32x4{__float_as_uint(x[4 * g]), __float_as_uint(x[4 * g + 1]), __float_as_uint(x[4 * g + 2]),
                                              __float_as_uint(x[4 * g + 3])});
                }
                __builtin_amdgcn_wave_barrier();
                u32x4 line[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 8 * i + orow;
                    line[i] = *reinterpret_cast<const u32x4 *>(turn + r * 128 + (ochunk ^ (r & 7)) * 16);
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    elem *p = out0 + (int64_t)(jb * 32 + 8 * i) * m.ld + part * 8 * E;
                    if (whole) {
                        __builtin_nontemporal_store(line[i], reinterpret_cast<u32x4_any *>(p));
                    } else if (n0 + wt * 128 + jb * 32 + 8 * i + orow < m.N) {
                        const int64_t c = v0 + wv * 128 + part * 8 * E + ochunk * E;
                        if (c < m.V) store_vector<DT>(p - c, c / E, m.V, line[i]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);  // (left to itself the compiler fetches many blocks before it stores one)
            });
        });
    }
    copies_landed();  // nothing may still be on its way into LDS that the next workgroup has
}

// Stores a block as it is: p is the lane's row of the output, v the block's first column.
template <int DT>
__device__ __forceinline__ void store_block(const f32x16 acc, typename Elem<DT>::type *p, int32_t v, int lh, int32_t V, bool whole, bool live)
{
    constexpr int E = Elem<DT>::kPerVec, kPieces = DT == 0 ? 2 : 4;
    u32x4 q[kPieces];
    if constexpr (DT == 0) {
        pack_block<false>(acc, q);
    } else {
#pragma unroll
        for (int g = 0; g < 4; ++g)
            q[g] = u32x4{__float_as_uint(acc[4 * g]), __float_as_uint(acc[4 * g + 1]), __float_as_uint(acc[4 * g + 2]), __float_as_uint(acc[4 * g + 3])};
    }
    if (!live) return;
#pragma unroll
    for (int g = 0; g < kPieces; ++g) {
        const int32_t c = v + 2 * E * g + E * lh;
        if (whole || c + E <= V) {
            *reinterpret_cast<u32x4_any *>(p + c) = q[g];
        } else {
            const uint32_t w[4] = {q[g].x, q[g].y, q[g].z, q[g].w};
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (c + j < V) {
                    if constexpr (DT == 0)
                        p[c + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
                    else
                        p[c + j] = __uint_as_float(w[j]);
                }
        }
    }
}

// ---- up to 128 rows of a ----
//
// What bounds these is reading b once: the tile is as wide as the batch (T = 32, 64 or 128 rows of a), and the matrix instructions of a
// slab take a fraction of the time its share of the memory bandwidth does.  A workgroup's four waves own 32 R rows of b each and all rows
// of a.  S LDS stages, so that S - 1 slabs are in flight while one is multiplied, one barrier per slab: wait for the wave's own copies of
// slab s (those of the slabs after it may be in flight), barrier: slab s is in LDS whole, and every wave is done with slab s - 1, whose
// stage takes slab s + S - 1.  Scales are fetched as they are stored, 4 bytes a lane.
//
// The rows of b are dealt out in blocks of 32, so that no workgroup has more than one block beyond another; a workgroup's last tile is
// as short as its blocks say, and re-reads its last row (from the L2) for what is missing.
template <int DT, int T, int R, bool NT>
__global__ __launch_bounds__(kBlock, T <= 64 && R == 1 ? 2 : 1) void mx4_small_kernel(Mx4Product m)
{
    typedef typename Elem<DT>::type elem;
    constexpr int kRows = 128 * R, TB = T / 32, kStages = (T == 128 && R == 1) || (T == 32 && R == 2) ? 4 : 3;
    constexpr int kCopies = 4 * R + TB + R + 1;  // per wave and slab
    __shared__ __attribute__((aligned(16))) uint8_t lds_b[kStages][kRows * kMxSlabBytes];
    __shared__ __attribute__((aligned(16))) uint8_t lds_a[kStages][T * kMxSlabBytes];
    __shared__ __attribute__((aligned(16))) uint8_t lds_sb[kStages][kRows * 8];
    __shared__ __attribute__((aligned(16))) uint8_t lds_sa[kStages][T * 8];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int l32 = lane & 31, lh = lane >> 5;
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);
    const uint32_t pitch = (uint32_t)(m.K / 2), spitch = (uint32_t)(m.K / 32);
    const int nk = (int)((m.K + 255) / 256);
    const bool half = m.K % 256 != 0;
    const int64_t blocks = (m.V + 31) / 32;
    const int32_t row0 = (int32_t)(32 * (blocks * blockIdx.x / gridDim.x)), V = (int32_t)m.V;
    const int64_t row_end = 32 * (blocks * (blockIdx.x + 1) / gridDim.x);
    const int32_t row1 = row_end < m.V ? (int32_t)row_end : V;
    const int tiles = (row1 - row0 + kRows - 1) / kRows, total = tiles * nk;

    const int crow = tid >> 3;
    const int cchunk = (tid & 7) ^ ((crow >> 1) & 7);
    const uint32_t chunk0 = (uint32_t)cchunk * 16u, off0 = (uint32_t)crow * pitch + chunk0, most_a = (uint32_t)(m.N - 1) * pitch + chunk0;
    const uint32_t word = (uint32_t)(lane & 1) * 4u;
    const int srow_b = wave * 32 * R + (lane >> 1), srow_a = (wave & (TB - 1)) * 32 + (lane >> 1);
    const uint32_t soff_a = (uint32_t)(srow_a < m.N ? srow_a : (int)m.N - 1) * spitch + word;
    // in a half slab the upper chunks and the upper four scales are those of the lower half again
    const uint32_t back_in_half = half && cchunk >= 4 ? 64u : 0u, sback_in_half = half ? word : 0u;

    int f_row = row0, f_kt = 0, f_stage = 0;  // the next slab to fetch and the stage it goes to
    auto copy16 = [&](const uint8_t *sbase, uint32_t voff, const uint8_t *stage, auto PAST) {
        const uint32_t to = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)stage;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
        if constexpr (decltype(PAST)::value)
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0 nt" : : "s"(sbase), "v"(voff), "s"(to) : "memory", "m0");
        else
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(sbase), "v"(voff), "s"(to) : "memory", "m0");
#pragma clang diagnostic pop
    };
    auto copy4 = [&](const uint8_t *sbase, uint32_t voff, const uint8_t *stage) {
        const uint32_t to = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)stage;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, %0" : : "s"(sbase), "v"(voff), "s"(to) : "memory", "m0");
#pragma clang diagnostic pop
    };
    auto fetch_slab = [&]() {
        const int32_t last = (row1 - f_row < kRows ? row1 - f_row : kRows) - 1;
        const bool short_slab = half && f_kt + 1 == nk;
        const uint32_t back = short_slab ? back_in_half : 0u, sback = short_slab ? sback_in_half : 0u;
        const uint32_t most_b = (uint32_t)last * pitch + chunk0;
        const uint8_t *cb = m.b + (int64_t)f_row * pitch + (int64_t)f_kt * kMxSlabBytes, *ca = m.a + (int64_t)f_kt * kMxSlabBytes;
        const uint8_t *sb = m.bs + (int64_t)f_row * spitch + (int64_t)f_kt * 8, *sa = m.as + (int64_t)f_kt * 8;
        static_for<4 * R>([&](auto P) {
            constexpr int p = decltype(P)::value;
            copy16(cb, min(off0 + (uint32_t)(32 * p) * pitch, most_b) - back, &lds_b[f_stage][(8 * wave_u + 32 * p) * kMxSlabBytes],
                   std::integral_constant<bool, NT>());
        });
        static_for<TB>([&](auto P) {
            constexpr int p = decltype(P)::value;
            copy16(ca, min(off0 + (uint32_t)(32 * p) * pitch, most_a) - back, &lds_a[f_stage][(8 * wave_u + 32 * p) * kMxSlabBytes], std::false_type());
        });
        static_for<R>([&](auto P) {
            constexpr int p = decltype(P)::value;
            copy4(sb, (uint32_t)min(srow_b + 32 * p, (int)last) * spitch + word - sback, &lds_sb[f_stage][(wave_u * R + p) * 256]);
        });
        copy4(sa, soff_a - sback, &lds_sa[f_stage][(wave_u & (TB - 1)) * 256]);
        f_stage = f_stage + 1 == kStages ? 0 : f_stage + 1;
        if (++f_kt == nk) {
            f_kt = 0;
            f_row += kRows;
        }
    };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    for (int i = 0; i < kStages - 1 && i < total; ++i) fetch_slab();
    const int sw = (l32 >> 1) & 7;
    int stage = 0, done = 0;  // stage of the next slab to multiply, slabs multiplied
    for (int tile = 0; tile < tiles; ++tile) {
        const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        f32x16 acc[R][TB];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = zero;
        for (int kt = 0; kt < nk; ++kt) {
            if (done + kStages - 1 <= total)  // the slabs up to done + kStages - 2 are on their way
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"((kStages - 2) * kCopies) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            barrier();
            if (done + kStages - 1 < total) fetch_slab();
            const int keep = half && kt + 1 == nk ? 0 : -1;
            uint2 sa[TB], sb[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                sb[i] = *reinterpret_cast<const uint2 *>(&lds_sb[stage][((wave * R + i) * 32 + l32) * 8]);
                sb[i].x >>= 8 * lh;
                sb[i].y >>= 8 * lh;
            }
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                sa[j] = *reinterpret_cast<const uint2 *>(&lds_sa[stage][(j * 32 + l32) * 8]);
                sa[j].x >>= 8 * lh;
                sa[j].y >>= 8 * lh;
            }
            static_for<4>([&](auto STEP) {
                constexpr int step = decltype(STEP)::value;
                const int off = ((2 * step + lh) ^ sw) * 16;
                i32x4 fb[R], fa[TB];
#pragma unroll
                for (int i = 0; i < R; ++i) fb[i] = *reinterpret_cast<const i32x4 *>(&lds_b[stage][((wave * R + i) * 32 + l32) * kMxSlabBytes + off]);
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    fa[j] = *reinterpret_cast<const i32x4 *>(&lds_a[stage][(j * 32 + l32) * kMxSlabBytes + off]);
                    if (step >= 2) fa[j] &= keep;
                }
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < TB; ++j)
                        acc[i][j] = fp4_mfma<2 * (step & 1)>(fb[i], fa[j], acc[i][j], (int)(step < 2 ? sb[i].x : sb[i].y), (int)(step < 2 ? sa[j].x : sa[j].y));
            });
            stage = stage + 1 == kStages ? 0 : stage + 1;
            ++done;
        }
        const int32_t v0 = row0 + tile * kRows;
        const bool whole = v0 + kRows <= row1;
        static_for<TB>([&](auto JB) {
            constexpr int jb = decltype(JB)::value;
            const int n = jb * 32 + l32;
            elem *p = reinterpret_cast<elem *>(m.out) + (int64_t)n * m.ld;
            static_for<R>([&](auto IB) {
                constexpr int ib = decltype(IB)::value;
                store_block<DT>(acc[ib][jb], p, v0 + (wave * R + ib) * 32, lh, row1, whole, n < m.N);
            });
        });
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing may still be on its way into LDS that the next workgroup has
}

// Ranges so that the rounds of workgroups (one to a compute unit) times the tiles of the longest range are fewest; the fewest ranges of
// those, because each fills its pipeline anew.
static Mx4Plan mx4_plan(int64_t N, int64_t V)
{
    Mx4Plan p;
    p.n_tb = (int)((N + kMxTile - 1) / kMxTile);
    p.n_vt = (int)((V + kMxTile - 1) / kMxTile);
    int64_t best = INT64_MAX;
    p.splits = 1;
    for (int s = 1; s <= p.n_vt && s <= 512; ++s) {
        const int64_t rounds = ((int64_t)p.n_tb * s + 255) / 256, cost = rounds * ((p.n_vt + s - 1) / s);
        if (cost < best) {
            best = cost;
            p.splits = s;
        }
    }
    return p;
}

constexpr int64_t kMxSmallMost = 128;  // most rows of a of the kernel that reads b once

// Whether the threads that put the scales in tile order (2048 for 256 rows of either matrix) are counted in 32 bits.
bool mx4_product_grid(int64_t N, int64_t V) { return N <= kMxSmallMost || N + V <= ((int64_t)1 << 29) - 1024; }

size_t mx4_product_workspace_bytes(int64_t N, int64_t V, int64_t K)
{
    if (N <= kMxSmallMost) return 0;
    const Mx4Plan p = mx4_plan(N, V);
    return (size_t)(p.n_tb + (int64_t)p.n_vt) * (size_t)((K + 255) / 256) * (kMxTile * 8);
}

template <int DT, int T>
static void run_small(const Mx4Product &m, hipStream_t stream)
{
    // One workgroup to a compute unit with tiles of 256 rows of b where each of them has that many, two with tiles of 128 below.  A
    // matrix larger than the 256 MB Infinity Cache is read past it, as in the fused LM head.
    const int64_t blocks = (m.V + 31) / 32;
    if (blocks >= 256 * 8) {
        const dim3 grid(256);
        if (m.V * m.K / 2 > (int64_t)256 << 20)
            mx4_small_kernel<DT, T, 2, true><<<grid, dim3(kBlock), 0, stream>>>(m);
        else
            mx4_small_kernel<DT, T, 2, false><<<grid, dim3(kBlock), 0, stream>>>(m);
    } else {
        const int64_t most = T <= 64 ? 512 : 256;
        mx4_small_kernel<DT, T, 1, false><<<dim3((unsigned)(blocks < most ? blocks : most)), dim3(kBlock), 0, stream>>>(m);
    }
}

int launch_mx4_product(const uint8_t *a_codes, const uint8_t *a_scales, int64_t N, const uint8_t *b_codes, const uint8_t *b_scales,
                       int64_t V, int64_t K, void *out, int dtype, int64_t ld, void *workspace, hipStream_t stream)
{
    if (N <= kMxSmallMost) {
        const Mx4Product m{a_codes, a_scales, b_codes, b_scales, N, V, K, out, ld, nullptr, nullptr};
#define RUN(DT) N <= 32 ? run_small<DT, 32>(m, stream) : N <= 64 ? run_small<DT, 64>(m, stream) : run_small<DT, 128>(m, stream)
        if (dtype == 0)
            RUN(0);
        else
            RUN(1);
#undef RUN
        return hipGetLastError() == hipSuccess ? 0 : 1;
    }
    const Mx4Plan plan = mx4_plan(N, V);
    const int nk = (int)((K + 255) / 256);
    uint8_t *const tiled = (uint8_t *)workspace;
    const Mx4Product m{a_codes, a_scales, b_codes, b_scales, N, V, K, out, ld, tiled, tiled + (int64_t)plan.n_tb * nk * (kMxTile * 8)};
    mx4_tile_scales_kernel<<<dim3((unsigned)((plan.n_tb + plan.n_vt) * (kMxTile / kScaleRows)), (unsigned)((nk + kScaleSlabs - 1) / kScaleSlabs)), dim3(kBlock), 0, stream>>>(
        a_scales, N, b_scales, V, K, plan.n_tb, tiled);
    const dim3 grid((unsigned)((int64_t)plan.n_tb * plan.splits));
#define RUN(DT, HALF) mx4_product_kernel<DT, HALF><<<grid, dim3(kBlock), 0, stream>>>(m, plan)
    if (dtype == 0)
        K % 256 ? RUN(0, true) : RUN(0, false);
    else
        K % 256 ? RUN(1, true) : RUN(1, false);
#undef RUN
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace difr
