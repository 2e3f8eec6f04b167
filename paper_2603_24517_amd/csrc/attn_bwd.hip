// Attention backward for MI355X (gfx950, CDNA4): dQ, dK and dV from dO, O and LSE, the probabilities recomputed tile by tile.
//
// With P = exp(scale * Q K^T - LSE) and dS = P * (dO V^T - delta), delta = rowsum(dO * O) - dLSE:
//     dV = P^T dO        dK = scale * dS^T Q        dQ = scale * dS K
//
// Three launches: delta and LSE in the units and the layout that the kernel wants (attn_bwd_stats); the products
// (attn_bwd_kernel); and, where items were cut into parts, the sum of the parts (attn_bwd_join).
//
// dK and dV are sums over queries, dQ is one over keys.  One pass for all three would have to add up dQ in memory across
// workgroups (atomics: another order, other bits, every launch, and 16 KiB of FP32 through the caches for 32 rows).
// Here a work item holds one side in registers and streams the other, and the scores are formed in both kinds of items: seven products
// instead of five, but no memory traffic beside inputs and outputs, and the same bits always.
//   * a "keys" item holds K and V of 128 keys and streams Q and dO of every query head that shares them;
//   * a "rows" item holds Q and dO of 128 query rows and streams K and V.
// Both are the same loop with the operands' names exchanged.  X1, X2 stand for what is held, Y1, Y2 for what streams:
//     S = Y1 X1^T     dP = Y2 X2^T - delta     (keys only) acc2 += Y2^T P     acc1 += Y1^T dS
// With v_mfma_f32_32x32x16_bf16 and Y as the A operand, the accumulator layout puts one held row (lane % 32) in each lane
// and 16 of the tile's 32 streamed rows in its registers, so P and dS are, packed to BF16 in registers, directly the B operands of the
// products with Y^T, which the transposing read ds_read_b64_tr_b16 fetches from the same tile in LDS: nothing
// of size rows x keys leaves the registers.  BF16 is what the instruction multiplies, and what the forward pass rounds its P to: with it the 2-norm of the error against
// 64 bits is 0.0024 of the result's in every call timed, of which the rounding of the results alone is 0.0017; P and dS in two BF16 parts each would be twice the
// products.
//
// What bounds it: 14 * 128 FLOP per pair of unmasked row and key on the matrix pipe.  8 x 4096, 16 heads: 3.06 ms, 1.26 PFLOP/s of products (a library
// product of 8192^3 on the same card as much), the pipe 75 % busy at the 1.56 GHz that the board's power leaves; memory reads and writes are
// 0.4 ms of it.  A wavefront holds 32 rows, a workgroup is four of them, and two workgroups share a compute unit: one's vector
// instructions, LDS latencies, first loads and results pass behind the other's products.  The step's order and the place of every vector instruction in it
// are fixed by hand (sched_barrier), because the registers, 256 per wavefront of which sums and held operands take 160, leave no room for the
// order that the compiler picks.  Holding 64 rows per wavefront, one workgroup per unit (512 registers, half the LDS reads), was 4 % faster for the largest calls
// and up to a third slower for small ones, as nothing fills its waits; with two forms of the step, masked or not, the compiler copied up to 300
// registers where they meet.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include <math.h>
#include <atomic>
#include <type_traits>
#include <utility>

#include "../../include/attn.h"
#include "../../include/attn_layer.h"
#include "attn_bwd_plan.h"

namespace {

using namespace attn_bwd_plan;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#define LDS_AS __attribute__((address_space(3)))

constexpr int TILE_BYTES = BT * ROW_BYTES;      // 8 KiB
constexpr int STATS_BYTES = 2 * BT * 4;         // -LSE and -delta of a step's 32 rows
constexpr float LOG2E = 1.4426950408889634f;

// How an item of each kind uses LDS: a ring of stages, each a tile of Y1 and one of Y2 (keys items: and its rows' figures).  While step j runs, step
// j + 1's tiles arrive.  Keys items read nothing of step j - 1's, and hold V there: two stages, and a wavefront waits for its reads in front of the
// barrier that hands a stage on.  Rows items still read Y1 of step j - 1, at the end of the step, so that a read of step j - 2's may be on its way
// when the request that takes its stage leaves: four.  Two workgroups share a compute unit's 160 KiB.
template <bool KEYS>
struct Lds {
    static constexpr bool DRAIN = KEYS;
    static constexpr int STAGES = KEYS ? 2 : 4, X2 = STAGES * 2 * TILE_BYTES, FIGURES = X2 + (KEYS ? 4 * 32 * ROW_BYTES : 0);
    static constexpr int BYTES = FIGURES + (KEYS ? STAGES * STATS_BYTES : 0);
};
constexpr int LDS_BYTES = Lds<true>::BYTES > Lds<false>::BYTES ? Lds<true>::BYTES : Lds<false>::BYTES;
static_assert(LDS_BYTES <= 80 * 1024);

struct Tensors {
    const __bf16 *q, *k, *v, *dout;
    __bf16 *dq, *dk, *dv;
    const float *stats;
    unsigned char *part_q, *part_kv;    // parts: [tile][group][piece][wavefront] PART_BYTES each; of keys items twice that, dk and dv
    float c, scale;                 // c = scale * log2(e)
    float masked;                   // the score whose probability is 0: c * masked = -inf
};
struct Params : Tensors, Sizes {};

// f(0), f(1), ... f(N - 1) with constants (the unroller gives up on a loop of this size)
template <int... I, class F>
__device__ __forceinline__ void static_for(std::integer_sequence<int, I...>, F &&f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void static_for(F &&f) { static_for(std::make_integer_sequence<int, N>{}, f); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    bf16x2 p = __builtin_convertvector((f32x2){a, b}, bf16x2);   // v_cvt_pk_bf16_f32, nearest even
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ const unsigned char *uniform_ptr(const unsigned char *ptr) {
    const uint64_t v = (uint64_t)(uintptr_t)ptr;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const unsigned char *)(uintptr_t)(((uint64_t)hi << 32) | lo);
}
// 16 (4) bytes per lane from global memory straight into LDS, at lds_base + 16 (4) * lane.  Inline assembly, so that the compiler's
// count of outstanding loads does not make every LDS read wait for it; the caller waits with s_waitcnt vmcnt(n).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_dma16(const unsigned char *base, uint32_t voffset, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(lds_base), "v"(voffset), "s"(base)
                 : "memory", "m0");
}
__device__ __forceinline__ void lds_dma4(const unsigned char *base, uint32_t voffset, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 :
                 : "s"(lds_base), "v"(voffset), "s"(base)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
constexpr int wait_vmcnt(int n) { return 0x0F70 | n; }     // s_waitcnt vmcnt(n), n < 16
constexpr int WAIT_LGKMCNT0 = ~0x0F00;                      // (and it also waits for this wavefront's LDS reads)
__device__ __forceinline__ void wg_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

// One physical 16-byte unit of a tile row: unit u of row r stands at u ^ f(r), f(r) = (r & 3) << 2 | (r >> 2) & 3.  f runs through
// all 16 values, so 16 lanes that read one unit of 16 rows touch every bank once; and its upper bits differ within 4 rows in line, so
// the 4 rows x 64 bytes that a half-wave fetches with the transposing read do so too: one copy of a tile serves both.
__device__ __forceinline__ int swz(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

// ------------------------------------------------------------------------------------------------ -LSE and -delta
// stats[(b * Hq + h) * qtiles + tile][64]: -LSE * log2(e) of the tile's 32 rows, then -delta.  Rows past the end, and rows
// without a valid key (LSE = -inf), get -inf and 0, so that their P and dS are 0.
__global__ __launch_bounds__(256) void attn_bwd_stats(const __bf16 *dout, const __bf16 *o, const float *lse, const float *dlse,
                                                      float *stats, int Hq, int Sq, int qtiles, unsigned rows, unsigned blocks)
{
    // 16 lanes per (position, head) row, heads fastest: a wavefront reads 1 KiB in line.  Four rows each, loads first.
    const unsigned b = blockIdx.x / blocks, block = blockIdx.x - b * blocks;
    const int part = threadIdx.x & 15;
    const size_t base = (size_t)b * Sq * Hq;
    unsigned n[4], i[4], h[4];
    bf16x8 x[4], y[4];
    float l[4], dl[4];
    bool real[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        n[k] = block * 64 + k * 16 + (threadIdx.x >> 4);
        i[k] = n[k] / (unsigned)Hq;
        h[k] = n[k] - i[k] * Hq;
        real[k] = i[k] < (unsigned)Sq;
        const size_t at = (base + (real[k] ? n[k] : 0)) * HD + part * 8;
        x[k] = *(const bf16x8 *)(dout + at);
        y[k] = *(const bf16x8 *)(o + at);
        const size_t figure = real[k] ? ((size_t)b * Hq + h[k]) * Sq + i[k] : 0;
        l[k] = lse[figure];
        dl[k] = dlse ? dlse[figure] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf((float)x[k][e], (float)y[k][e], s);
        s += __shfl_xor(s, 1);
        s += __shfl_xor(s, 2);
        s += __shfl_xor(s, 4);
        s += __shfl_xor(s, 8);
        if (part == 0 && n[k] < rows) {
            const bool some = real[k] && l[k] != -INFINITY;
            float *out = stats + (((size_t)b * Hq + h[k]) * qtiles + (i[k] >> 5)) * (2 * BT) + (i[k] & 31);
            out[0] = some ? -l[k] * LOG2E : -INFINITY;
            out[BT] = some ? dl[k] - s : 0.0f;
        }
    }
}

// ------------------------------------------------------------------------------------------------------ the products
// One item: KEYS holds K (X1), V (X2) and streams Q (Y1), dO (Y2); otherwise the reverse.
template <bool KEYS>
__device__ __forceinline__ void item(const Params &p, int group, int tile, int piece)
{
    typedef Lds<KEYS> L;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    LDS_AS unsigned char *lds = (LDS_AS unsigned char *)smem;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // ---- what this wavefront holds, and the steps that it streams
    int b, x_head, x0;
    find_rows(p, KEYS, group, tile, wave, b, x_head, x0);
    const int x_rows = KEYS ? p.Skv : p.Sq, y_rows = KEYS ? p.Sq : p.Skv;
    // KEYS: query tiles t0 .. qtiles - 1 of each head; else: key tiles from 0 on
    const int t0 = KEYS ? keys_skip(p, tile) : 0;
    const int per_head = KEYS ? p.qtiles - t0 : rows_steps(p, tile);
    int steps = KEYS ? per_head * p.G : per_head, step0 = 0;
    const int n_pieces = pieces(steps, KEYS ? p.keys.most : p.rows.most);
    if (piece >= n_pieces) return;
    if (n_pieces > 1) piece_steps(steps, n_pieces, piece, step0, steps);
    // (all of it is wave-uniform: scalar registers)
    auto uniform = [](int &x) __attribute__((always_inline)) { x = __builtin_amdgcn_readfirstlane(x); };
    uniform(b); uniform(x_head); uniform(x0); uniform(steps);
    const int y_head0 = KEYS ? x_head * p.G : fast_div(x_head, p.d_g);
    const int x_heads = KEYS ? p.Hkv : p.Hq, y_heads = KEYS ? p.Hq : p.Hkv;
    const uint32_t y_stride = (uint32_t)y_heads * ROW_BYTES;

    // ---- requests: 4 rows x 256 bytes per instruction, two of each tile per wavefront (and, KEYS, a quarter of 256 bytes of figures)
    const int ld_r = lane >> 4, ld_u = lane & 15;
    // Where steps and requests stand: streamed tile, query head of the group, LDS stages; and, for requests, the tiles' addresses.
    struct At { int tile, head, stage; };
    const int y_tiles = KEYS ? p.qtiles : (y_rows + BT - 1) / BT;
    At cur, req;
    cur.head = KEYS && step0 > 0 ? step0 / per_head : 0;
    cur.tile = KEYS ? min(step0 - cur.head * per_head + t0, y_tiles - 1) : min(step0, y_tiles - 1);
    uniform(cur.head);
    uniform(cur.tile);
    cur.stage = 0;
    req = cur;
    auto tiles_of = [&](int stage) __attribute__((always_inline)) { return lds0 + stage * (2 * TILE_BYTES); };
    auto figures_of = [&](int stage) __attribute__((always_inline)) { return lds0 + L::FIGURES + stage * STATS_BYTES; };
    auto next_stage = [&](int stage) __attribute__((always_inline)) { return (stage + 1) & (L::STAGES - 1); };
    const unsigned char *g1, *g2, *gs = nullptr;
    auto find_tiles = [&]() __attribute__((always_inline)) {
        const size_t at = ((size_t)((size_t)b * y_rows + (size_t)req.tile * BT) * y_heads + y_head0 + req.head) * ROW_BYTES;
        g1 = uniform_ptr((const unsigned char *)(KEYS ? p.q : p.k) + at);
        g2 = uniform_ptr((const unsigned char *)(KEYS ? p.dout : p.v) + at);
        if (KEYS) gs = uniform_ptr((const unsigned char *)(p.stats + ((size_t)((size_t)b * p.Hq + y_head0 + req.head) * p.qtiles + req.tile) * (2 * BT)));
    };
    find_tiles();
    constexpr int PER_STEP = KEYS ? 5 : 4;
    // this lane's place in a tile, and in the last one, where rows past the end read its last row again
    uint32_t row_off[2], row_off_last[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = (wave * 2 + i) * 4 + ld_r;
        row_off[i] = row * y_stride + ((ld_u ^ swz(row)) << 4);
        row_off_last[i] = min(row, y_rows - 1 - (y_tiles - 1) * BT) * y_stride + ((ld_u ^ swz(row)) << 4);
    }
    // part n of the requests for a step
    auto request_part = [&](int n) __attribute__((always_inline)) {
        if (n < 4) {
            const int i = n & 1;
            lds_dma16(n < 2 ? g1 : g2, req.tile == y_tiles - 1 ? row_off_last[i] : row_off[i],
                      __builtin_amdgcn_readfirstlane(tiles_of(req.stage) + (n < 2 ? 0 : TILE_BYTES) + wave * 2048 + i * 1024));
        } else if (lane < 16) {
            lds_dma4(gs, (wave * 16 + lane) * 4, __builtin_amdgcn_readfirstlane(figures_of(req.stage) + wave * 64));
        }
    };
    // past the end the last step's tiles are read again, into a stage that nobody reads (to ask in every step whether there is one more took
    // 1 % longer, 8 x 4096, and gained nothing for 24 x 200)
    int left = steps;
    auto request_done = [&]() __attribute__((always_inline)) {
        req.stage = next_stage(req.stage);
        if (--left <= 0) return;
        if (KEYS && req.tile == y_tiles - 1) {
            req.tile = t0;
            ++req.head;
            find_tiles();
        } else {
            ++req.tile;
            g1 += BT * (size_t)y_stride;
            g2 += BT * (size_t)y_stride;
            if (KEYS) gs += 2 * BT * sizeof(float);
        }
    };

    // ---- held operands
    const uint32_t x2_at = lds0 + L::X2 + wave * (32 * ROW_BYTES);
    bf16x8 x1[8], x2[8];
    f32x16 nd;              // rows items: -delta of the lane's row in every element, the C operand that dP starts from
    float nl = 0.0f;
    const bool dead = x0 >= x_rows;     // this wavefront's rows lie behind the last one
    if (!dead) {
        const __bf16 *from1 = KEYS ? p.k : p.q, *from2 = KEYS ? p.v : p.dout;
        const int row = min(x0 + l32, x_rows - 1);
        const size_t at = ((size_t)((size_t)b * x_rows + row) * x_heads + x_head) * HD + 8 * hh;
#pragma unroll
        for (int s = 0; s < 8; ++s) x1[s] = *(const bf16x8 *)(from1 + at + 16 * s);
        if (KEYS) {         // (V in registers as well: no room beside K, two accumulators of its size and the scores.)  In the order of
                            // its fragments, lane by lane: reads are one address and a constant.
            const unsigned char *g = uniform_ptr((const unsigned char *)(from2 + ((size_t)((size_t)b * x_rows + x0) * x_heads + x_head) * HD));
            const uint32_t o = (uint32_t)(row - x0) * (uint32_t)(x_heads * ROW_BYTES) + 16 * hh;
#pragma unroll
            for (int i = 0; i < 8; ++i) lds_dma16(g, o + 32 * i, __builtin_amdgcn_readfirstlane(x2_at + i * 1024));
        } else {
#pragma unroll
            for (int s = 0; s < 8; ++s) x2[s] = *(const bf16x8 *)(from2 + at + 16 * s);
            const float *st = p.stats + ((size_t)((size_t)b * p.Hq + x_head) * p.qtiles + (row >> 5)) * (2 * BT) + (row & 31);
            nl = st[0];
            const float d = st[BT];
#pragma unroll
            for (int r = 0; r < 16; ++r) nd[r] = d;
        }
    }
    f32x16 acc1[4], acc2[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc1[d][r] = acc2[d][r] = 0.0f;
    auto cleared = [&]() __attribute__((always_inline)) {        // (here, not between the wait for the loads and the first product)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            asm volatile("" : "+v"(acc1[d]));
            if (KEYS) asm volatile("" : "+v"(acc2[d]));
        }
    };

    // ---- LDS reads.  Row l32, unit 2 s + hh: as the swizzle is an exclusive or and tiles are 256-byte aligned, that is the address of
    // unit hh with s << 5 flipped.  Transposed: row 4 hh + i / 4 (+ 8 e, + 16 k) and four d's: likewise with d << 6 and e << 5 flipped.
    const uint32_t r_at = l32 * ROW_BYTES + ((hh ^ swz(l32)) << 4);
    uint32_t t_at;
    {
        const int i16 = lane & 15, g = (lane >> 4) & 1, row = 4 * hh + (i16 >> 2), col = 16 * g + 4 * (i16 & 3);
        t_at = row * ROW_BYTES + (((col >> 3) ^ swz(row)) << 4) + (col & 7) * 2;
    }
    typedef const LDS_AS unsigned char *Ptr;
    auto row_frag = [&](uint32_t at, int s, int tile) __attribute__((always_inline)) -> bf16x8 {         // `at`: tiles_of() + r_at
        return *(const LDS_AS bf16x8 *)((Ptr)(uintptr_t)(at ^ (s << 5)) + tile * TILE_BYTES);
    };
    auto col_frag = [&](uint32_t at, int k, int d, int tile) __attribute__((always_inline)) -> bf16x8 {    // `at`: tiles_of() + t_at
        s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)((Ptr)(uintptr_t)(at ^ (d << 6)) + (tile * TILE_BYTES + 16 * k * ROW_BYTES)));
        s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)((Ptr)(uintptr_t)(at ^ (d << 6) ^ 32) + (tile * TILE_BYTES + (16 * k + 8) * ROW_BYTES)));
        s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, v);
    };

    // ---- a step: phases of 8 products, each with an operand fragment of Y,
    //     KEYS:  S(j)   dP(j)   acc2 += Y2^T P(j)   acc1 += Y1^T dS(j)
    //     rows:  S(j)   dP(j)   acc1 += Y1^T dS(j-1)
    // and between the products the vector work, each piece behind the products that it needs and ahead of those that need it: the exponents of S(j)
    // from dP(j) on, P * dP behind dP(j).  (Rows items have nothing to do between dP(j) and a product with dS(j), so that is a step later.)  Fragments are read
    // LEAD products ahead, across the end of a step too, so the step's barrier stands LEAD products before its end.
    constexpr int LEAD = 2;
    constexpr int NF = KEYS ? 32 : 24;          // products of a step; fragment f lies in frag[f % 4]
    static_assert(LEAD < 4 && NF % 4 == 0);
    constexpr int PH_S = 0, PH_DP = 1, PH_2 = KEYS ? 2 : -1;
    bf16x8 frag[4], frag2[4];
    f32x16 s, dp;
    u32x4 pb[2], ds[2];                         // BF16 pairs, the B operands of acc2 and acc1
    int prev = 0;                               // stage of step j - 1
    uint32_t r_cur, r_next = tiles_of(0) + r_at, t_cur;
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = 0.0f;
    // (held in place once four are complete: the compiler otherwise keeps twice as many FP32 values and rounds them right in front of a product)
    auto pack = [&](u32x4 (&w)[2], int r, float x0, float x1) __attribute__((always_inline)) {       // elements r, r + 1
        w[r >> 3][(r >> 1) & 3] = pack_bf16(x0, x1);
        if ((r & 7) == 6) asm volatile("" : "+v"(w[r >> 3]));
    };
    auto fetch = [&](int f) __attribute__((always_inline)) {
        const int ph = f >> 3, i = f & 7;
        bf16x8 &to = frag[f % 4];
        if (f >= NF) to = row_frag(r_next, i, 0);
        else if (ph == PH_S) to = row_frag(r_cur, i, 0);
        else if (ph == PH_DP) to = row_frag(r_cur, i, 1);
        else to = col_frag(t_cur, i >> 2, i & 3, ph == PH_2 ? 1 : 0);
    };
    auto fetch2 = [&](int i) __attribute__((always_inline)) { frag2[i & 3] = *(const LDS_AS bf16x8 *)((Ptr)(uintptr_t)(x2_at + lane * 16) + i * 1024); };
    auto step = [&]() __attribute__((always_inline)) {
        const int y0 = cur.tile * BT;
        const bool masked = KEYS ? min(x0 + 32, x_rows) - 1 > y0 + p.off : (y0 + BT - 1 > x0 + p.off || y0 + BT > y_rows);
        const Ptr figures = (Ptr)(uintptr_t)figures_of(cur.stage) + 16 * hh;
        r_cur = r_next;
        t_cur = tiles_of(KEYS ? cur.stage : prev) + t_at;
        f32x4 nlv[4];
        // Masked pairs (KEYS: row < key - off; else key > row + off or key >= Skv) give exactly 0, whatever they hold.  A branch around
        // selects alone: two forms of the whole step meet in copies of hundreds of registers.
        auto mask = [&](f32x16 &v, float to) __attribute__((always_inline)) {
            if (masked) {
                int ln = lane;
                asm volatile("" : "+v"(ln));        // formed here, not kept through all steps
                const int x = x0 + (ln & 31), lim = (KEYS ? x - p.off : min(x + p.off, p.Skv - 1)) - y0 - 4 * (ln >> 5);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int y = 8 * (r >> 2) + (r & 3);
                    v[r] = (KEYS ? y >= lim : y <= lim) ? v[r] : to;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        // element e of the vector work
        auto do_exp = [&](int e) __attribute__((always_inline)) {
            s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], p.c, KEYS ? nlv[e >> 2][e & 3] : nl));
            if (KEYS && (e & 1)) pack(pb, e - 1, s[e - 1], s[e]);
        };
        auto do_mul = [&](int e) __attribute__((always_inline)) {
            dp[e] *= s[e];
            if (KEYS && (e & 1)) pack(ds, e - 1, dp[e - 1], dp[e]);
        };
        auto do_round = [&](int e) __attribute__((always_inline)) { pack(ds, 2 * e, dp[2 * e], dp[2 * e + 1]); };
        // the n elements dealt out evenly to `of` slots: those of slot k
        auto spread = [&](int k, int of, int n, auto &&f) __attribute__((always_inline)) {
            if (k < 0 || k >= of) return;
#pragma unroll
            for (int e = 0; e < n; ++e)
                if (e >= k * n / of && e < (k + 1) * n / of) f(e);
        };
        static_for<NF>([&](auto fc) __attribute__((always_inline)) {
            constexpr int f = decltype(fc)::value, ph = f >> 3, i = f & 7;
            if constexpr (KEYS && f == 9) mask(s, p.masked);
            if constexpr (KEYS && f == 17) mask(dp, 0.0f);
            if constexpr (f == NF - LEAD) {
                // the next step's tiles have landed, for every wavefront
                __builtin_amdgcn_s_waitcnt(wait_vmcnt(0) & (L::DRAIN ? WAIT_LGKMCNT0 : ~0));
                wg_barrier();
                r_next = tiles_of(next_stage(cur.stage)) + r_at;
            }
            fetch(f + LEAD);
            if constexpr (KEYS && f >= 6 && f < 14) fetch2(f - 6);
            if (f >= 1 && f <= PER_STEP) request_part(f - 1);
            if (f == PER_STEP + 1) request_done();
            // -LSE, a quarter at a time shortly before its exponents; -delta, where dP starts from
            if constexpr (KEYS && f >= 6 && f < 18 && (f - 6) % 3 == 0) nlv[(f - 6) / 3] = *(const LDS_AS f32x4 *)(figures + 32 * ((f - 6) / 3));
            if constexpr (KEYS && f >= 3 && f < 7) {
                const f32x4 d = *(const LDS_AS f32x4 *)(figures + BT * 4 + 32 * (f - 3));
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[4 * (f - 3) + e] = d[e];
            }
            const bf16x8 a = frag[f % 4];
            if constexpr (ph == PH_S) {
                f32x16 zero;
#pragma unroll
                for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, x1[i], i == 0 ? zero : s, 0, 0, 0);
            } else if constexpr (ph == PH_DP) {
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, KEYS ? frag2[i & 3] : x2[i], !KEYS && i == 0 ? nd : dp, 0, 0, 0);
            } else if constexpr (ph == PH_2) {
                acc2[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, pb[i >> 2]), acc2[i & 3], 0, 0, 0);
            } else {
                acc1[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, ds[i >> 2]), acc1[i & 3], 0, 0, 0);
            }
            if (!KEYS) spread(f, 8, 8, do_round);
            spread(f - 9, KEYS ? 10 : 11, 16, do_exp);
            spread(f - 17, KEYS ? 10 : 7, 16, do_mul);
            __builtin_amdgcn_sched_barrier(0);
        });
        if (!KEYS) mask(dp, 0.0f);
        prev = cur.stage;
        cur.stage = next_stage(cur.stage);
        if (KEYS && cur.tile == y_tiles - 1) cur.tile = t0;
        else ++cur.tile;
    };
    if (steps > 0) {
#pragma unroll
        for (int n = 0; n < PER_STEP; ++n) request_part(n);
        request_done();
        cleared();
        // (all of them, so that the compiler, which counts the loads above but not these, has none left to wait for in the loop)
        __builtin_amdgcn_s_waitcnt(0);
        wg_barrier();
        if (dead) {             // its share of the requests, and the barriers
            for (int j = 0; j < steps; ++j) {
#pragma unroll
                for (int n = 0; n < PER_STEP; ++n) request_part(n);
                request_done();
                __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
                wg_barrier();
            }
            return;
        }
        r_cur = r_next;
#pragma unroll
        for (int f = 0; f < LEAD; ++f) fetch(f);
        for (int j = 0; j < steps; ++j) step();
        if (!KEYS) {            // the last step's dS
#pragma unroll
            for (int r = 0; r < 16; r += 2) pack(ds, r, dp[r], dp[r + 1]);
            t_cur = tiles_of(prev) + t_at;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                acc1[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(col_frag(t_cur, i >> 2, i & 3, 0), __builtin_bit_cast(bf16x8, ds[i >> 2]), acc1[i & 3], 0, 0, 0);
        }
    }

    // ---- results: lane = held row, registers 4 d's; exchanged with lane ^ 32, eight in line, and through LDS into whole rows
    if (dead) return;
    if (n_pieces == 1) {
        if (!KEYS) wg_barrier();        // (keys items: where the wavefront's V was; rows items: stages that every wavefront is done with)
        const uint32_t rows_at = KEYS ? x2_at : lds0 + wave * (32 * ROW_BYTES);
        auto store = [&](f32x16 (&acc)[4], float f, __bf16 *out) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x16 &a = acc[i >> 1];
                const int e = 8 * (i & 1);
                auto u = __builtin_amdgcn_permlane32_swap(pack_bf16(a[e] * f, a[e + 1] * f), pack_bf16(a[e + 4] * f, a[e + 5] * f), false, false);
                auto v = __builtin_amdgcn_permlane32_swap(pack_bf16(a[e + 2] * f, a[e + 3] * f), pack_bf16(a[e + 6] * f, a[e + 7] * f), false, false);
                const u32x4 w = {u[0], v[0], u[1], v[1]};
                *(LDS_AS u32x4 *)(uintptr_t)(rows_at + l32 * ROW_BYTES + (((2 * i + hh) ^ (l32 & 15)) << 4)) = w;
            }
            u32x4 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = 4 * i + ld_r;
                w[i] = *(const LDS_AS u32x4 *)(uintptr_t)(rows_at + row * ROW_BYTES + ((ld_u ^ (row & 15)) << 4));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = x0 + 4 * i + ld_r;
                if (row < x_rows) *(u32x4 *)(out + ((size_t)((size_t)b * x_rows + row) * x_heads + x_head) * HD + 8 * ld_u) = w[i];
            }
        };
        store(acc1, p.scale, KEYS ? p.dk : p.dq);
        if (KEYS) store(acc2, 1.0f, p.dv);
    } else {
        // a part, in the order of the registers: 1 KiB in line at a time
        unsigned char *at = (KEYS ? p.part_kv : p.part_q) + (((size_t)(tile * (KEYS ? p.keys : p.rows).groups + group) * (KEYS ? p.keys : p.rows).splits + piece) * 4 + wave) *
                                                                ((KEYS ? 2 : 1) * PART_BYTES) + lane * 16;
        auto store = [&](f32x16 (&acc)[4], float f) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const f32x16 &a = acc[i >> 2];
                const int e = 4 * (i & 3);
                const f32x4 y = {a[e] * f, a[e + 1] * f, a[e + 2] * f, a[e + 3] * f};
                *(f32x4 *)(at + i * 1024) = y;
            }
            at += PART_BYTES;
        };
        store(acc1, p.scale);
        if (KEYS) store(acc2, 1.0f);
    }
}

__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_bwd_kernel(const Params p)
{
    const Item x = which_item(p, blockIdx.x);
    if (x.keys) item<true>(p, x.group, x.tile, x.piece);
    else item<false>(p, x.group, x.tile, x.piece);
}

// The sum of the parts of each tile that was cut, in the order of its pieces.  A workgroup adds up one wavefront's 32 rows of one result: 8 elements
// per thread and pass.
__global__ __launch_bounds__(256) void attn_bwd_join(const Params p)
{
    const bool keys = (int)blockIdx.x < p.join_keys;
    const Role &r = keys ? p.keys : p.rows;
    int n = keys ? blockIdx.x : blockIdx.x - p.join_keys;
    const int second = keys ? n & 1 : 0;            // dv
    if (keys) n >>= 1;
    const int wave = n & 3;
    n >>= 2;
    const int tile = n / r.groups, group = n - tile * r.groups;
    const int count = pieces(keys ? keys_steps(p, tile) : rows_steps(p, tile), r.most);
    if (count == 1) return;
    int b, head, x0;
    find_rows(p, keys, group, tile, wave, b, head, x0);
    const int rows = keys ? p.Skv : p.Sq, heads = keys ? p.Hkv : p.Hq;
    const int l32 = threadIdx.x & 31;
    if (x0 + l32 >= rows) return;
    const size_t stride = (size_t)4 * (keys ? 2 : 1) * PART_BYTES;
    const unsigned char *from = (keys ? p.part_kv : p.part_q) + (size_t)(tile * r.groups + group) * r.splits * stride + ((size_t)wave * (keys ? 2 : 1) + second) * PART_BYTES;
    __bf16 *out = (keys ? second ? p.dv : p.dk : p.dq) + ((size_t)((size_t)b * rows + x0 + l32) * heads + head) * HD;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int i = pass * 8 + (threadIdx.x >> 5);        // d = 8 i ..: four from lane l32, four from lane l32 + 32
        const unsigned char *at = from + i * 1024 + l32 * 16;
        f32x4 a = {0, 0, 0, 0}, c = {0, 0, 0, 0};
#pragma unroll 4
        for (int s = 0; s < count; ++s, at += stride) {
            a += *(const f32x4 *)at;
            c += *(const f32x4 *)(at + 512);
        }
        const u32x4 w = {pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(c[0], c[1]), pack_bf16(c[2], c[3])};
        *(u32x4 *)(out + 8 * i) = w;
    }
}

// ----------------------------------------------------------------------------------------------------------- host
bool launch(const void *kernel, dim3 grid, int threads, int lds, void **args, hipStream_t st)
{
    if (hipLaunchKernel(kernel, grid, dim3(threads), args, lds, st) == hipSuccess) return true;
    (void)hipGetLastError();
    return false;
}

}  // namespace

extern "C" {

long long attn_bwd_workspace(int B, int Hq, int Hkv, int Sq, int Skv, int D, int causal)
{
    int rc = check_sizes(B, Hq, Hkv, Sq, Skv, D);
    Plan r = {};
    if (rc == ATTN_OK) rc = make_plan(B, Hq, Hkv, Sq, Skv, causal, r);
    return rc == ATTN_OK ? (long long)r.total : rc;
}

int attn_bwd(const void *dout, const float *dlse, const void *q, const void *k, const void *v, const void *o,
             const float *lse, void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes,
             int B, int Hq, int Hkv, int Sq, int Skv, int D, int causal, float scale, void *stream)
{
    if (!dout || !q || !k || !v || !o || !lse || !dq || !dk || !dv || !workspace) return ATTN_E_NULL;
    int rc = check_sizes(B, Hq, Hkv, Sq, Skv, D);
    if (rc != ATTN_OK) return rc;
    if (!isfinite(scale)) return ATTN_E_SCALE;
    if (((uintptr_t)dout | (uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o | (uintptr_t)dq | (uintptr_t)dk | (uintptr_t)dv |
         (uintptr_t)workspace) & 15)
        return ATTN_E_ALIGN;
    if (((uintptr_t)lse | (uintptr_t)dlse) & 3) return ATTN_E_ALIGN;
    Plan r = {};
    rc = make_plan(B, Hq, Hkv, Sq, Skv, causal, r);
    if (rc != ATTN_OK) return rc;
    if (workspace_bytes < r.total) return ATTN_E_WORKSPACE;

    // Once per device: the opt-in that more than 64 KiB of dynamic LDS needs.
    static std::atomic<bool> ready[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return ATTN_E_LAUNCH;
    if (!ready[dev].load(std::memory_order_acquire)) {
        if (hipFuncSetAttribute((const void *)attn_bwd_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES) != hipSuccess)
            return ATTN_E_LAUNCH;
        ready[dev].store(true, std::memory_order_release);
    }
    hipStream_t st = (hipStream_t)stream;

    Params p = {{}, r.p};
    p.q = (const __bf16 *)q; p.k = (const __bf16 *)k; p.v = (const __bf16 *)v; p.dout = (const __bf16 *)dout;
    p.dq = (__bf16 *)dq; p.dk = (__bf16 *)dk; p.dv = (__bf16 *)dv;
    p.stats = (const float *)workspace;
    p.part_kv = (unsigned char *)workspace + r.stats;
    p.part_q = p.part_kv + r.part_kv;
    p.c = scale * LOG2E;
    if (p.c == 0.0f) p.c = 1.2e-38f;        // (no score is large enough to tell it from 0)
    p.masked = p.c > 0 ? -INFINITY : INFINITY;
    p.scale = scale;

    {
        float *stats = (float *)workspace;
        unsigned rows = (unsigned)p.qtiles * BT * (unsigned)Hq, blocks = rows / 64 + (rows % 64 != 0);
        void *args[] = {(void *)&dout, (void *)&o, (void *)&lse, (void *)&dlse, &stats, &Hq, &Sq, &p.qtiles, &rows, &blocks};
        if (!launch((const void *)attn_bwd_stats, dim3(blocks * (unsigned)B), 256, 0, args, st)) return ATTN_E_LAUNCH;
    }
    {
        void *args[] = {&p};
        if (!launch((const void *)attn_bwd_kernel, dim3(p.keys.items + p.rows.items), 256, LDS_BYTES, args, st)) return ATTN_E_LAUNCH;
    }
    if (p.keys.splits > 1 || p.rows.splits > 1) {
        void *args[] = {&p};
        const int rows = p.rows.splits > 1 ? p.rows.groups * p.rows.tiles * 4 : 0;
        if (!launch((const void *)attn_bwd_join, dim3(p.join_keys + rows), 256, 0, args, st)) return ATTN_E_LAUNCH;
    }
    return ATTN_OK;
}

}  // extern "C"
