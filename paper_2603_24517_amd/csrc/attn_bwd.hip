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
// of size rows x keys leaves the registers.
//
// What bounds it: 14 * 128 FLOP per pair of unmasked row and key on the matrix pipe.  8 x 4096, 16 heads: 3.15 ms, 1.22 PFLOP/s of products (a library
// product of 8192^3 on the same card 1.24), the pipe 74 % busy at the 1.56 GHz that the board's power leaves; memory reads and writes are
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

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#define LDS_AS __attribute__((address_space(3)))

constexpr int HD = 128;
constexpr int ROW_BYTES = HD * 2;
constexpr int BT = 32;                          // streamed rows per step
constexpr int TILE_BYTES = BT * ROW_BYTES;      // 8 KiB
constexpr int ITEM_ROWS = 128;                  // held rows of an item, 32 per wavefront
constexpr int STATS_BYTES = 2 * BT * 4;         // -LSE and -delta of a step's 32 rows
constexpr size_t PART_BYTES = 32 * HD * sizeof(float);     // what one wavefront leaves of one sum
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

// n / d for n < 2^31 with constants found on the host
struct Div { uint32_t mul, shift; };
__host__ inline Div make_div(uint32_t d)
{
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    return {(uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1), l};
}
__device__ __forceinline__ int fast_div(int n, Div d) { return (int)((__umulhi((uint32_t)n, d.mul) + (uint32_t)n) >> d.shift); }

// The items of one kind.  A tile's steps (streamed tiles, of all heads of a group) are cut into pieces of at most `most`, so that a call of few or
// uneven tiles fills the chip; a tile of several pieces leaves FP32 parts, which attn_bwd_join adds up.
struct Role {
    int groups, tiles, splits;      // grid: groups x tiles x splits (the largest number of pieces)
    int most;
    int items, per_xcd;             // of all XCDs and of one (of all, where they do not keep to their own groups)
    int window, per_window;         // groups whose tiles are dealt out together, and their items
    Div d_window, d_per_tile, d_per_window;
};
struct Params {
    const __bf16 *q, *k, *v, *dout;
    __bf16 *dq, *dk, *dv;
    const float *stats;
    unsigned char *part_q, *part_kv;    // parts: [tile][group][piece][wavefront] PART_BYTES each; of keys items twice that, dk and dv
    int B, Hq, Hkv, Sq, Skv, G, qtiles;
    int pack_log2, chunks;          // rows items: query heads of a group side by side, and how many such chunks a group has
    int off;                        // key j valid for row i iff j <= i + off (without the mask: always true)
    float c, scale;                 // c = scale * log2(e)
    float masked;                   // the score whose probability is 0: c * masked = -inf
    Role keys, rows;
    int xcd_groups;                 // 0, or the K/V heads (of all batch entries) that each XCD keeps to
    bool together;                  // behind each window's keys items come its rows items; otherwise all rows items come last
    Div d_both;                     // items of a window, of both kinds
    Div d_hkv, d_chunks, d_g;
    int join_keys;                  // workgroups of attn_bwd_join for dk and dv
};

// f(0), f(1), ... f(N - 1) with constants (the unroller gives up on a loop of this size)
template <int... I, class F>
__device__ __forceinline__ void static_for(std::integer_sequence<int, I...>, F &&f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void static_for(F &&f) { static_for(std::make_integer_sequence<int, N>{}, f); }

// Query tiles in front of a tile's first key (keys items); steps of a tile.
__host__ __device__ inline int keys_skip(const Params &p, int tile)
{
    const int first = tile * ITEM_ROWS - p.off;             // first row that sees the tile's first key
    return first > 0 ? (first / BT < p.qtiles ? first / BT : p.qtiles) : 0;
}
__host__ __device__ inline int keys_steps(const Params &p, int tile) { return (p.qtiles - keys_skip(p, tile)) * p.G; }
__host__ __device__ inline int rows_steps(const Params &p, int tile)
{
    const int end = (tile + 1) * (ITEM_ROWS >> p.pack_log2);
    const int last = (end < p.Sq ? end : p.Sq) - 1 + p.off;      // last key that the tile's last row sees
    return last < 0 ? 0 : (last < p.Skv - 1 ? last : p.Skv - 1) / BT + 1;
}
__host__ __device__ inline int pieces(int steps, int most) { return steps <= most ? 1 : (steps + most - 1) / most; }

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
// Batch entry, head and first of the 32 rows that a wavefront of an item holds.
__device__ __forceinline__ void find_rows(const Params &p, bool keys, int group, int tile, int wave, int &b, int &head, int &x0)
{
    const int bh = keys ? group : fast_div(group, p.d_chunks);
    b = fast_div(bh, p.d_hkv);
    head = bh - b * p.Hkv;
    x0 = tile * ITEM_ROWS + wave * 32;
    if (!keys) {
        head = head * p.G + ((group - bh * p.chunks) << p.pack_log2) + (wave & ((1 << p.pack_log2) - 1));
        x0 = tile * (ITEM_ROWS >> p.pack_log2) + (wave >> p.pack_log2) * 32;
    }
}

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
    if (n_pieces > 1) {
        step0 = (int)((unsigned)steps * (unsigned)piece / (unsigned)n_pieces);
        steps = (int)((unsigned)steps * (unsigned)(piece + 1) / (unsigned)n_pieces) - step0;
    }
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

// Which item of a kind has number n in its order (together: in that of window w): window by window, longest tiles first.
__device__ __forceinline__ void find_item(const Role &r, bool together, int n, int w, int first, int &group, int &tile, int &piece)
{
    if (!together) {
        w = fast_div(n, r.d_per_window);
        n -= w * r.per_window;
    }
    tile = fast_div(n, r.d_per_tile);
    n -= tile * r.window * r.splits;
    piece = fast_div(n, r.d_window);
    group = first + w * r.window + n - piece * r.window;
}

// The hardware deals workgroups round-robin to the 8 XCDs, each with an L2 of its own; where the groups (batch entries x K/V heads) divide among them, an
// XCD keeps to its own groups, a window of them at a time, so that the tiles of a group, which stream the same data, meet in one L2.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_bwd_kernel(const Params p)
{
    int n = blockIdx.x, first = 0, w = 0, of_keys = p.keys.per_xcd;
    if (p.xcd_groups) {
        first = (n & 7) * p.xcd_groups;
        n >>= 3;
        if (p.together) {
            w = fast_div(n, p.d_both);
            of_keys = p.keys.per_window;
            n -= w * (of_keys + p.rows.per_window);
        }
    }
    int group, tile, piece;
    if (n < of_keys) {
        find_item(p.keys, p.together, n, w, first, group, tile, piece);
        item<true>(p, group, tile, piece);
    } else {
        find_item(p.rows, p.together, n - of_keys, w, first * p.chunks, group, tile, piece);
        item<false>(p, group, p.rows.tiles - 1 - tile, piece);
    }
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
struct Plan {
    Params p;                                   // sizes and roles
    size_t stats, part_kv, part_q, total;       // bytes: the workspace's three parts
};

int check_sizes(int B, int Hq, int Hkv, int Sq, int Skv, int D)
{
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Skv <= 0 || D <= 0) return ATTN_E_SHAPE;
    if (Hq % Hkv != 0) return ATTN_E_SHAPE;
    if (D != HD) return ATTN_E_UNSUPPORTED;
    if ((long long)Sq + Skv >= (1ll << 31) - 1024 || Hq > 32768 || Hkv > 32768) return ATTN_E_UNSUPPORTED;
    return ATTN_OK;
}

// Workgroups that are resident at a time on the device that this is written for, two per compute unit: how items are cut (and so what the
// workspace needs) does not ask the device.
constexpr int CUS = 256, PLACES = 2 * CUS;
// Microseconds: a step alone on a compute unit, and how much longer it takes beside another; an item beside its steps; how much of the last items
// stands out behind a full chip; the launch and the bytes per microsecond of adding up parts.  Fitted to 100 calls of this range, each cut in
// up to 90 ways: the choice is 2.1 % off the best of those on average, 18 % at most.
constexpr double KEYS_STEP = 0.75, ROWS_STEP = 0.69, SHARED = 1.38, ITEM = 3.8, LAST = 0.7, JOIN = 4.6, JOIN_BYTES = 7.9e6;
constexpr int MOST_PIECES = 32;
constexpr double CACHE_BYTES = 192e6;      // three quarters of the memory-side cache

// The order of the items.  Windows are as many groups as an XCD's 64 places take, or a few more, so that windows are equal.
int fit_window(int groups, int per_group)
{
    int window = (PLACES / 8 + per_group - 1) / per_group;
    if (window > groups) return groups;
    while (groups % window) ++window;
    return window;
}
void deal(Params &p)
{
    const int groups = p.keys.groups, both = p.keys.tiles * p.keys.splits + p.chunks * p.rows.tiles * p.rows.splits;
    p.xcd_groups = groups % 8 == 0 ? groups / 8 : 0;
    // Keys and rows items read the same inputs.  Side by side they find them in L2, which pays where a few tiles to a group leave the rest of the
    // traffic to memory and the cache behind the L2s does not hold the inputs, unless an item is so long that it must not start late: more than a
    // quarter of a place's work.  Together / apart, inputs from memory, us: 96 x 300, 16 heads, masked 347 / 387; 210 x 198, 8 heads, masked 228 / 252;
    // 27 x 642, 24 heads 589 / 626; 34 x 840, 32 on 8 heads 1414 / 1555; longer items 4 x 2401, 32 on 4, masked 877 / 753; smaller inputs 512 x 64, 4 heads,
    // masked 89 / 86.  Of 60 calls drawn 27 are dealt together: 4.4 % faster on average, between 11 % faster and 1.8 % slower.
    p.together = false;
    if (p.xcd_groups && both < PLACES / 8 && 2.0 * ROW_BYTES * ((double)p.G * p.Sq + p.Skv) * groups > CACHE_BYTES) {
        double all = 0;
        int longest = 0;
        for (int t = 0; t < p.keys.tiles; ++t) {
            const int n = keys_steps(p, t);
            all += n;
            longest = n > longest ? n : longest;
        }
        for (int t = 0; t < p.rows.tiles; ++t) {
            const int n = rows_steps(p, t);
            all += (double)n * p.chunks;
            longest = n > longest ? n : longest;
        }
        p.together = 4.0 * longest * PLACES <= all * groups;
    }
    for (Role *r : {&p.keys, &p.rows}) {
        const int heads = r == &p.keys ? 1 : p.chunks, per_group = r->tiles * r->splits;
        r->items = r->groups * per_group;
        r->per_xcd = p.xcd_groups ? r->items / 8 : r->items;
        r->window = r->groups;
        if (p.together)
            r->window = fit_window(p.xcd_groups, both) * heads;
        else if (p.xcd_groups)      // all groups of an XCD at once, longest tiles first, while that is few rounds
            r->window = r->per_xcd <= 4 * PLACES / 8 ? p.xcd_groups * heads : fit_window(p.xcd_groups * heads, per_group);
        r->per_window = r->window * per_group;
        r->d_window = make_div(r->window);
        r->d_per_tile = make_div(r->window * r->splits);
        r->d_per_window = make_div(r->per_window);
    }
    p.d_both = make_div(p.keys.per_window + p.rows.per_window);
}

int make_plan(int B, int Hq, int Hkv, int Sq, int Skv, int causal, Plan &r)
{
    Params &p = r.p;
    const int G = Hq / Hkv;
    p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Sq = Sq; p.Skv = Skv; p.G = G;
    p.pack_log2 = G % 4 == 0 ? 2 : G % 2 == 0 ? 1 : 0;
    p.chunks = G >> p.pack_log2;
    p.qtiles = (Sq + BT - 1) / BT;
    // (i + INT32_MAX - Sq - 256 is above every key for i >= 0 and within 32 bits for the i < Sq + 256 of a tile)
    p.off = causal ? Skv - Sq : INT32_MAX - Sq - 256;
    const int pos = ITEM_ROWS >> p.pack_log2;
    const int tk = (Skv + ITEM_ROWS - 1) / ITEM_ROWS, tr = (Sq + pos - 1) / pos;
    const long long nk = (long long)B * Hkv * tk, nr = (long long)B * Hkv * p.chunks * tr;
    // (a launch has fewer than 2^32 threads; each 64 rows of the figures, with 32 of a head in line, take a workgroup of 256)
    if (nk >= (1ll << 23) || nr >= (1ll << 23) || (long long)p.qtiles * BT * Hq >= (1ll << 30) / B || (long long)p.qtiles * G >= (1ll << 31))
        return ATTN_E_UNSUPPORTED;
    p.d_hkv = make_div(Hkv);
    p.d_chunks = make_div(p.chunks);
    p.d_g = make_div(G);
    p.keys = {B * Hkv, tk, 1, INT32_MAX};
    p.rows = {B * Hkv * p.chunks, tr, 1, INT32_MAX};

    // Calls of few tiles for the chip, or of uneven ones, are cut: the pair of piece lengths whose estimate is the shortest.
    const int long_k = keys_steps(p, 0), long_r = rows_steps(p, tr - 1), short_r = rows_steps(p, 0);
    if (nk + nr < 4 * PLACES && (long long)long_k * MOST_PIECES < (1ll << 31)) {
        double all_k = 0, all_r = 0;
        for (int t = 0; t < tk; ++t) all_k += keys_steps(p, t);
        for (int t = 0; t < tr; ++t) all_r += rows_steps(p, t);
        all_k *= p.keys.groups;
        all_r *= p.rows.groups;
        const double kv_bytes = 2.0 * B * Skv * Hkv * HD * 4, q_bytes = (double)B * Sq * Hq * HD * 4;
        double best = INFINITY;
        int best_k = 1, best_r = 1;
        for (int sk = 1; sk <= MOST_PIECES; sk += sk < 8 ? 1 : sk / 4) {
            const int mk = (long_k + sk - 1) / sk;
            if (sk > 1 && mk < 3) break;
            for (int sr = 1; sr <= MOST_PIECES; sr += sr < 8 ? 1 : sr / 4) {
                const int mr = (long_r + sr - 1) / sr;
                if (sr > 1 && mr < 4) break;
                const double pk = sk > 1 ? all_k / mk : nk, pr = sr > 1 ? all_r / mr : nr, n = pk + pr;       // pieces, about
                const double more = n <= CUS ? 0 : n >= PLACES ? 1 : (n - CUS) / (PLACES - CUS), slow = 1 + (SHARED - 1) * more;
                const double k = slow * KEYS_STEP, q = slow * ROWS_STEP, ik = ITEM + k * mk, ir = ITEM + q * mr;
                double us = (all_k * k + all_r * q + n * ITEM) / PLACES;
                if (n > PLACES) us += LAST * (ITEM + q * (sr > 1 ? mr : short_r));
                if (us < ik) us = ik;
                if (us < ir) us = ir;
                if (sk > 1 || sr > 1) us += JOIN + 2 * ((sk > 1 ? sk * kv_bytes : 0) + (sr > 1 ? sr * q_bytes : 0)) / JOIN_BYTES;
                if (us < best) {
                    best = us;
                    best_k = sk;
                    best_r = sr;
                }
            }
        }
        if (best_k > 1) {
            p.keys.most = (long_k + best_k - 1) / best_k;
            p.keys.splits = pieces(long_k, p.keys.most);
        }
        if (best_r > 1) {
            p.rows.most = (long_r + best_r - 1) / best_r;
            p.rows.splits = pieces(long_r, p.rows.most);
        }
    }
    deal(p);
    auto pad = [](size_t n) { return (n + 255) / 256 * 256; };
    r.stats = pad((size_t)B * Hq * p.qtiles * 2 * BT * sizeof(float));
    p.join_keys = p.keys.splits > 1 ? (int)nk * 8 : 0;
    r.part_kv = p.keys.splits > 1 ? (size_t)p.keys.items * 8 * PART_BYTES : 0;
    r.part_q = p.rows.splits > 1 ? (size_t)p.rows.items * 4 * PART_BYTES : 0;
    r.total = r.stats + r.part_kv + r.part_q;
    return ATTN_OK;
}

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

    Params &p = r.p;
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
