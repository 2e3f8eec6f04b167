// Norm of each head of queries and keys with the position rotation in the same pass, and its gradient, for MI355X (gfx950).
//
// One head of one token is a row of 128 elements, 256 bytes, held by 8 lanes with 16 elements each: two 16-byte loads per lane, and the
// mean over a row is 16 in-lane operations and three exchanges.  Which 16 elements a lane holds is chosen so that both members of a rotated pair
// are in it: of a rotation of halves, 8 elements of the first half and the 8 that they pair with; otherwise 16 in line.
// Everything between load and store is FP32.
//
// A workgroup works on rows of one kind (queries, keys, values), 8 consecutive rows per wavefront at a time, whatever the strides: rows are numbered
// token by token, heads fastest.  Both kernels are bound by memory: they read and write every element once.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include <math.h>

#include "../../include/attn.h"
#include "../../include/attn_layer.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int HD = 128;
constexpr int LANES = 8;                // per row
constexpr int BLOCK_ROWS = 256 / LANES;     // rows of a workgroup at a time.  (Two per lane: 8 x 4096, 48 heads 149 -> 153 us, one token of 64 sequences 2.8 -> 3.5)

// n / d for n < 2^31, found on the host: (umulhi(n, mul) + n) >> shift, or n itself
struct Div { uint32_t mul, shift; };
__host__ Div make_div(uint32_t d)
{
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    return {(uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1), l};
}
__device__ __forceinline__ uint32_t fast_div(uint32_t n, Div d) { return (__umulhi(n, d.mul) + n) >> d.shift; }

struct Tensor {
    unsigned char *at;
    long long batch, token, head;       // bytes
};
struct Kind {
    Tensor x, z, dx;        // the input, the output (or its gradient), the input's gradient
    const void *weight;
    uint32_t rows, heads;
    Div by_heads;
    uint32_t blocks;        // workgroups of this kind
};
struct Params {
    Kind kind[3];           // queries, keys, values
    const float *cos, *sin;
    const void *positions;
    long long places;
    Div by_tokens;          // tokens of a batch entry
    uint32_t S;
    int rotated, wide_positions, wide_weight;
    float eps;
    float *partial;         // backward: [workgroups of queries, then of keys][128]
};

__device__ __forceinline__ const unsigned char *place(const Tensor &t, uint32_t b, uint32_t s, uint32_t h)
{
    return t.at + (long long)b * t.batch + (long long)s * t.token + (long long)h * t.head;
}
__device__ __forceinline__ float sum8(float x)
{
    x += __shfl_xor(x, 1);
    x += __shfl_xor(x, 2);
    return x + __shfl_xor(x, 4);
}

__device__ __forceinline__ float reciprocal_rms(const float (&x)[16], float eps)
{
    float q = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) q = fmaf(x[e], x[e], q);
    return 1.0f / sqrtf(sum8(q) * (1.0f / HD) + eps);
}

// The 16 elements of lane j: [lo, lo + 8) and [hi, hi + 8); its pairs take table elements 8 j .. 8 j + 7.
template <bool ADJACENT>
struct Lane {
    int j, lo, hi;
    bool turns;
    __device__ Lane(int rotated)
    {
        j = threadIdx.x & (LANES - 1);
        turns = 16 * j < rotated;
        lo = 16 * j;
        hi = lo + 8;
        if (!ADJACENT && turns) {
            lo = 8 * j;
            hi = rotated / 2 + 8 * j;
        }
    }
    __device__ void load(const unsigned char *row, float (&x)[16]) const
    {
        const bf16x8 a = *(const bf16x8 *)(row + 2 * lo), c = *(const bf16x8 *)(row + 2 * hi);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = (float)a[e];
            x[8 + e] = (float)c[e];
        }
    }
    __device__ void store(unsigned char *row, const float (&x)[16]) const
    {
        bf16x8 a, c;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a[e] = (__bf16)x[e];
            c[e] = (__bf16)x[8 + e];
        }
        *(bf16x8 *)(row + 2 * lo) = a;
        *(bf16x8 *)(row + 2 * hi) = c;
    }
    __device__ void weights(const void *w, int wide, float (&x)[16]) const
    {
        if (!w) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 1.0f;
        } else if (wide) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = ((const float *)w)[(e < 8 ? lo : hi - 8) + e];
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = (float)((const __bf16 *)w)[(e < 8 ? lo : hi - 8) + e];
        }
    }
    // rotation by +angle, or by -angle: its transpose
    template <bool BACK>
    __device__ void turn(float (&x)[16], const float (&c)[8], const float (&s)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float &a = x[ADJACENT ? 2 * e : e], &b = x[ADJACENT ? 2 * e + 1 : 8 + e];
            const float u = a, v = b, t = BACK ? -s[e] : s[e];
            a = u * c[e] - v * t;
            b = v * c[e] + u * t;
        }
    }
};

struct Spot { uint32_t b, s, h; bool real; };
__device__ __forceinline__ Spot spot(const Params &p, const Kind &k, uint32_t row)
{
    Spot at;
    at.real = row < k.rows;
    const uint32_t n = at.real ? row : 0, token = fast_div(n, k.by_heads);
    at.h = n - token * k.heads;
    at.b = fast_div(token, p.by_tokens);
    at.s = token - at.b * p.S;
    return at;
}
// cos and sin of a token; false: its place is outside the table
__device__ __forceinline__ bool angles(const Params &p, const Spot &at, int j, bool turns, float (&c)[8], float (&s)[8])
{
    long long pos = at.s;
    if (p.positions) {
        const size_t n = (size_t)at.b * p.S + at.s;
        pos = p.wide_positions ? ((const long long *)p.positions)[n] : (long long)((const int *)p.positions)[n];
    }
    const bool inside = pos >= 0 && pos < p.places;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        c[e] = 1.0f;
        s[e] = 0.0f;
    }
    if (turns) {
        const size_t n = (size_t)(inside ? pos : 0) * (p.rotated / 2) + 8 * j;
        const f32x4 c0 = *(const f32x4 *)(p.cos + n), c1 = *(const f32x4 *)(p.cos + n + 4);
        const f32x4 s0 = *(const f32x4 *)(p.sin + n), s1 = *(const f32x4 *)(p.sin + n + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = c0[e];
            c[4 + e] = c1[e];
            s[e] = s0[e];
            s[4 + e] = s1[e];
        }
    }
    return inside;
}

__device__ __forceinline__ void copy_rows(const Params &p, const Kind &k, uint32_t first)
{
    const int j = threadIdx.x & (LANES - 1);
    const Spot at = spot(p, k, first + threadIdx.x / LANES);
    if (!at.real) return;
    const bf16x8 *from = (const bf16x8 *)(place(k.x, at.b, at.s, at.h) + 32 * j);
    bf16x8 *to = (bf16x8 *)(place(k.z, at.b, at.s, at.h) + 32 * j);
    const bf16x8 a = from[0], c = from[1];
    to[0] = a;
    to[1] = c;
}

template <bool ADJACENT>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const Params p)
{
    uint32_t block = blockIdx.x;
    int kind = 0;
    while (block >= p.kind[kind].blocks) block -= p.kind[kind++].blocks;
    const Kind &k = p.kind[kind];
    if (kind == 2) {
        copy_rows(p, k, block * BLOCK_ROWS);
        return;
    }
    const Lane<ADJACENT> lane(p.rotated);
    float x[16], c[8], s[8], w[16];
    const Spot at = spot(p, k, block * BLOCK_ROWS + threadIdx.x / LANES);
    lane.load(place(k.x, at.b, at.s, at.h), x);
    const bool inside = angles(p, at, lane.j, lane.turns, c, s);
    lane.weights(k.weight, p.wide_weight, w);
    const float r = inside ? reciprocal_rms(x, p.eps) : NAN;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = x[e] * r * w[e];
    lane.template turn<false>(x, c, s);
    if (at.real) lane.store((unsigned char *)place(k.z, at.b, at.s, at.h), x);
}

// The gradient.  Each lane adds up dweight of its 16 elements over its rows; the 32 lanes of a workgroup that hold the same
// elements are added in LDS, and the workgroups' sums by the kernel behind, always in the same order.
template <bool ADJACENT>
__global__ __launch_bounds__(256) void qk_norm_rope_bwd_kernel(const Params p)
{
    __shared__ float sums[32][HD];
    uint32_t block = blockIdx.x;
    int kind = 0;
    while (block >= p.kind[kind].blocks) block -= p.kind[kind++].blocks;
    const Kind &k = p.kind[kind];
    const uint32_t stride = k.blocks * BLOCK_ROWS;
    if (kind == 2) {
        for (uint64_t first = (uint64_t)block * BLOCK_ROWS; first < k.rows; first += stride) copy_rows(p, k, (uint32_t)first);
        return;
    }
    const Lane<ADJACENT> lane(p.rotated);
    float w[16], dw[16];
    lane.weights(k.weight, p.wide_weight, w);
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[e] = 0.0f;
    for (uint64_t first = (uint64_t)block * BLOCK_ROWS; first < k.rows; first += stride) {
        float x[16], z[16], c[8], s[8];
        const Spot at = spot(p, k, (uint32_t)first + threadIdx.x / LANES);
        lane.load(place(k.x, at.b, at.s, at.h), x);
        lane.load(place(k.z, at.b, at.s, at.h), z);
        const bool inside = angles(p, at, lane.j, lane.turns, c, s);
        const float r = inside ? reciprocal_rms(x, p.eps) : NAN;
        const bool counts = at.real && inside;      // a token without a place is NaN whatever the weights are: no gradient of theirs
        lane.template turn<true>(z, c, s);
        float m = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] *= r;                                      // xhat
            if (counts) dw[e] = fmaf(z[e], x[e], dw[e]);
            z[e] *= w[e];
            m = fmaf(z[e], x[e], m);
        }
        m = sum8(m) * (1.0f / HD);
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = r * (z[e] - x[e] * m);
        if (at.real) lane.store((unsigned char *)place(k.dx, at.b, at.s, at.h), z);
    }
    if (!p.partial) return;
    float *mine = sums[threadIdx.x / LANES];
#pragma unroll
    for (int e = 0; e < 16; ++e) mine[(e < 8 ? lane.lo : lane.hi - 8) + e] = dw[e];
    __syncthreads();
    if (threadIdx.x < HD) {
        float t = 0.0f;
#pragma unroll
        for (int g = 0; g < 32; ++g) t += sums[g][threadIdx.x];
        p.partial[(size_t)blockIdx.x * HD + threadIdx.x] = t;
    }
}

// dweight: the workgroups' sums, 16 elements of one weight per workgroup, 64 runs of them side by side.
__global__ __launch_bounds__(1024) void qk_norm_rope_weight_kernel(const float *partial, float *dq_weight, float *dk_weight,
                                                                   int q_blocks, int k_blocks)
{
    __shared__ float sums[64][17];
    const bool keys = blockIdx.x >= HD / 16;
    const int col = threadIdx.x & 15, e = (blockIdx.x % (HD / 16)) * 16 + col, run = threadIdx.x >> 4;
    const float *at = partial + (keys ? (size_t)q_blocks * HD : 0) + e;
    const int n = keys ? k_blocks : q_blocks;
    float t = 0.0f;
#pragma unroll 16
    for (int i = run; i < n; i += 64) t += at[(size_t)i * HD];
    sums[run][col] = t;
    __syncthreads();
    if (run < 4) {
        float a = 0.0f;
#pragma unroll
        for (int g = 0; g < 16; ++g) a += sums[run * 16 + g][col];
        sums[run * 16][col] = a;        // (its own run's first, which no other run reads)
    }
    __syncthreads();
    if (run == 0) (keys ? dk_weight : dq_weight)[e] = (sums[0][col] + sums[16][col]) + (sums[32][col] + sums[48][col]);
}

// ----------------------------------------------------------------------------------------------------------- host
constexpr uint32_t MOST_BLOCKS = 1024;      // backward, of one kind: what fills the chip; each leaves 512 bytes of sums

uint32_t bwd_blocks(uint32_t rows)
{
    const uint32_t n = (rows + BLOCK_ROWS - 1) / BLOCK_ROWS, each = (n + MOST_BLOCKS - 1) / MOST_BLOCKS;
    return n == 0 ? 0 : (n + each - 1) / each;
}
int check_rope(const attn_rope *r)
{
    if (!r || !r->cos || !r->sin) return ATTN_E_NULL;
    if (!r->q_weight != !r->k_weight) return ATTN_E_NULL;
    if (r->B <= 0 || r->S <= 0 || r->Hq <= 0 || r->Hkv <= 0 || r->D <= 0 || r->places <= 0) return ATTN_E_SHAPE;
    if (!r->positions && r->S > r->places) return ATTN_E_SHAPE;
    if (r->D != HD || r->rotated < 16 || r->rotated > HD || r->rotated % 16) return ATTN_E_UNSUPPORTED;
    if ((r->pairing != ATTN_ROPE_HALVES && r->pairing != ATTN_ROPE_ADJACENT) || (r->weight_type != ATTN_BF16 && r->weight_type != ATTN_FP32) ||
        (r->position_type != ATTN_INT32 && r->position_type != ATTN_INT64))
        return ATTN_E_UNSUPPORTED;
    // rows of one kind in 31 bits, with room for a last workgroup's
    const long long most = ((1ll << 31) - 2 * BLOCK_ROWS * (long long)MOST_BLOCKS) / ((long long)r->B * r->S);
    if ((long long)r->B * r->S >= (1ll << 31) || r->Hq > most || r->Hkv > most) return ATTN_E_UNSUPPORTED;
    if (!isfinite(r->eps) || r->eps < 0.0f) return ATTN_E_SCALE;
    if (((uintptr_t)r->cos | (uintptr_t)r->sin) & 15) return ATTN_E_ALIGN;
    const uintptr_t weight = r->weight_type == ATTN_FP32 ? 3 : 1, position = r->position_type == ATTN_INT64 ? 7 : 3;
    if ((((uintptr_t)r->q_weight | (uintptr_t)r->k_weight) & weight) || ((uintptr_t)r->positions & position)) return ATTN_E_ALIGN;
    return ATTN_OK;
}
int take_tensor(const attn_heads *t, const attn_rope *r, int heads, Tensor &out)
{
    if (!t || !t->ptr) return ATTN_E_NULL;
    if ((uintptr_t)t->ptr & 15) return ATTN_E_ALIGN;
    if ((r->B > 1 && t->batch % 8) || (r->S > 1 && t->token % 8) || (heads > 1 && t->head % 8)) return ATTN_E_ALIGN;
    const long long most = 1ll << 58;
    if (t->batch > most || t->batch < -most || t->token > most || t->token < -most || t->head > most || t->head < -most) return ATTN_E_UNSUPPORTED;
    out.at = (unsigned char *)t->ptr;
    out.batch = r->B > 1 ? t->batch * 2 : 0;
    out.token = r->S > 1 ? t->token * 2 : 0;
    out.head = heads > 1 ? t->head * 2 : 0;
    return ATTN_OK;
}
void fill(const attn_rope *r, bool values, Params &p)
{
    const int heads[3] = {r->Hq, r->Hkv, r->Hkv};
    for (int i = 0; i < 3; ++i) {
        Kind &k = p.kind[i];
        k.heads = heads[i];
        k.rows = i == 2 && !values ? 0 : (uint32_t)r->B * (uint32_t)r->S * (uint32_t)heads[i];
        k.by_heads = make_div(heads[i]);
        k.weight = i == 0 ? r->q_weight : i == 1 ? r->k_weight : nullptr;
    }
    p.cos = r->cos; p.sin = r->sin;
    p.positions = r->positions;
    p.places = r->places;
    p.by_tokens = make_div(r->S);
    p.S = r->S;
    p.rotated = r->rotated;
    p.wide_positions = r->position_type == ATTN_INT64;
    p.wide_weight = r->weight_type == ATTN_FP32;
    p.eps = r->eps;
}
bool launch(const void *kernel, unsigned grid, void **args, hipStream_t st, int threads = 256)
{
    if (hipLaunchKernel(kernel, dim3(grid), dim3(threads), args, 0, st) == hipSuccess) return true;
    (void)hipGetLastError();
    return false;
}
bool given(const attn_heads *t) { return t && t->ptr; }

}  // namespace

extern "C" {

int attn_qk_norm_rope(const attn_rope *r, const attn_heads *q_in, const attn_heads *k_in, const attn_heads *v_in,
                      const attn_heads *q_out, const attn_heads *k_out, const attn_heads *v_out, void *stream)
{
    int rc = check_rope(r);
    if (rc != ATTN_OK) return rc;
    Params p = {};
    fill(r, given(v_in), p);
    if ((rc = take_tensor(q_in, r, r->Hq, p.kind[0].x)) || (rc = take_tensor(k_in, r, r->Hkv, p.kind[1].x)) ||
        (rc = take_tensor(q_out, r, r->Hq, p.kind[0].z)) || (rc = take_tensor(k_out, r, r->Hkv, p.kind[1].z)))
        return rc;
    if (given(v_in) && ((rc = take_tensor(v_in, r, r->Hkv, p.kind[2].x)) || (rc = take_tensor(v_out, r, r->Hkv, p.kind[2].z)))) return rc;
    unsigned blocks = 0;
    for (Kind &k : p.kind) blocks += k.blocks = (k.rows + BLOCK_ROWS - 1) / BLOCK_ROWS;
    if (blocks >= 1u << 24) return ATTN_E_UNSUPPORTED;      // (a launch has fewer than 2^32 threads)
    void *args[] = {&p};
    const void *kernel = r->pairing == ATTN_ROPE_ADJACENT ? (const void *)qk_norm_rope_kernel<true> : (const void *)qk_norm_rope_kernel<false>;
    return launch(kernel, blocks, args, (hipStream_t)stream) ? ATTN_OK : ATTN_E_LAUNCH;
}

long long attn_qk_norm_rope_bwd_workspace(const attn_rope *r)
{
    const int rc = check_rope(r);
    if (rc != ATTN_OK) return rc;
    const uint32_t tokens = (uint32_t)r->B * (uint32_t)r->S;
    return (long long)(bwd_blocks(tokens * r->Hq) + bwd_blocks(tokens * r->Hkv)) * HD * (long long)sizeof(float);
}

int attn_qk_norm_rope_bwd(const attn_rope *r, const attn_heads *dq_out, const attn_heads *dk_out, const attn_heads *dv_out,
                          const attn_heads *q_in, const attn_heads *k_in, const attn_heads *dq_in, const attn_heads *dk_in,
                          const attn_heads *dv_in, float *dq_weight, float *dk_weight, void *workspace, size_t workspace_bytes,
                          void *stream)
{
    int rc = check_rope(r);
    if (rc != ATTN_OK) return rc;
    if (!dq_weight != !dk_weight || (dq_weight && !workspace)) return ATTN_E_NULL;
    Params p = {};
    fill(r, given(dv_out), p);
    if ((rc = take_tensor(q_in, r, r->Hq, p.kind[0].x)) || (rc = take_tensor(k_in, r, r->Hkv, p.kind[1].x)) ||
        (rc = take_tensor(dq_out, r, r->Hq, p.kind[0].z)) || (rc = take_tensor(dk_out, r, r->Hkv, p.kind[1].z)) ||
        (rc = take_tensor(dq_in, r, r->Hq, p.kind[0].dx)) || (rc = take_tensor(dk_in, r, r->Hkv, p.kind[1].dx)))
        return rc;
    if (given(dv_out) && ((rc = take_tensor(dv_out, r, r->Hkv, p.kind[2].x)) || (rc = take_tensor(dv_in, r, r->Hkv, p.kind[2].z)))) return rc;
    if (((uintptr_t)dq_weight | (uintptr_t)dk_weight) & 3) return ATTN_E_ALIGN;
    unsigned blocks = 0;
    for (Kind &k : p.kind) blocks += k.blocks = bwd_blocks(k.rows);
    if (dq_weight) {
        if ((uintptr_t)workspace & 15) return ATTN_E_ALIGN;
        if ((long long)workspace_bytes < attn_qk_norm_rope_bwd_workspace(r)) return ATTN_E_WORKSPACE;
        p.partial = (float *)workspace;
    }
    hipStream_t st = (hipStream_t)stream;
    void *args[] = {&p};
    const void *kernel = r->pairing == ATTN_ROPE_ADJACENT ? (const void *)qk_norm_rope_bwd_kernel<true> : (const void *)qk_norm_rope_bwd_kernel<false>;
    if (!launch(kernel, blocks, args, st)) return ATTN_E_LAUNCH;
    if (dq_weight) {
        int nq = p.kind[0].blocks, nk = p.kind[1].blocks;
        void *sum[] = {&p.partial, &dq_weight, &dk_weight, &nq, &nk};
        if (!launch((const void *)qk_norm_rope_weight_kernel, 2 * (HD / 16), sum, st, 1024)) return ATTN_E_LAUNCH;
    }
    return ATTN_OK;
}

}  // extern "C"
