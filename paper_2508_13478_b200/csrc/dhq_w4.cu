// Products of few rows with 4-bit weights (include/dhq_groups.h): the codes' preparation and the product.
#include "dhq_group.cuh"
#include "dhq_internal.cuh"
#include "dhq_tmem.cuh"
#include <algorithm>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace dhq {
namespace {

constexpr int kPackThreads = 128;

// One warp per group: lane i holds values i, i + 32, ... of it, so strides 1 to 16 of the butterfly are exchanged and 32, 64
// stay in the lane.  Runs once per matrix.
template <class T, bool ROT>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const T *W, int64_t ldw, int64_t groups, int K, int per_row, int G, uint8_t *codes,
                                                            __nv_bfloat16 *scales)
{
    const int lane = threadIdx.x & 31;
    for (int64_t g = (int64_t)blockIdx.x * (kPackThreads / 32) + threadIdx.x / 32; g < groups; g += (int64_t)gridDim.x * (kPackThreads / 32)) {
        const int64_t n = g / per_row;
        const int first = (int)(g - n * per_row) * G;
        float v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int k = first + 32 * c + lane;
            v[c] = 32 * c < G && k < K ? to_float(W[n * ldw + k]) : 0.0f;
        }
        if (ROT) {
#pragma unroll
            for (int h = 1; h < 32; h <<= 1)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float other = __shfl_xor_sync(0xffffffffu, v[c], h);
                    v[c] = (lane & h) ? __fsub_rn(other, v[c]) : __fadd_rn(v[c], other);
                }
#pragma unroll
            for (int h = 1; h < 4; h <<= 1)
                if (32 * h < G)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (!(c & h)) {
                            const float a = v[c], b = v[c + h];
                            v[c] = __fadd_rn(a, b);
                            v[c + h] = __fsub_rn(a, b);
                        }
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = __fmul_rn(v[c], 1.0f / (float)G); // exact
        }
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) top = max(top, __float_as_uint(v[c]) & 0x7fffffffu);
#pragma unroll
        for (int h = 1; h < 32; h <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, h));
        const bool broken = top >= 0x7f800000u;
        const __nv_bfloat16 rounded = __float2bfloat16_rn(__fdiv_rn(__uint_as_float(top), 7.0f));
        const float inv = __fdiv_rn(1.0f, __bfloat162float(rounded));
        const bool some = !broken && inv <= 3.402823466e+38f; // a scale of 0, or too small to divide by: no code can be formed
        if (lane == 0) scales[g] = broken ? __ushort_as_bfloat16(0x7fffu) : some ? rounded : __ushort_as_bfloat16(0);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (32 * c >= G) break;
            const int q = some ? __float2int_rn(fmaxf(fminf(__fmul_rn(v[c], inv), 7.0f), -7.0f)) : 0;
            // code k of eight goes to nibble k / 2 + 4 (k % 2)
            uint32_t word = (uint32_t)(q + 8) << (4 * (((lane & 7) >> 1) + 4 * (lane & 1)));
#pragma unroll
            for (int h = 1; h < 8; h <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, h);
            if ((lane & 7) == 0) *reinterpret_cast<uint32_t *>(codes + (g * G + 32 * c + lane) / 2) = word;
        }
    }
}

// ---- the product -----------------------------------------------------------------------------------------------------
//
// Bound by reading the codes (half a byte each) once: 6.5 TB/s leaves a scheduler 1.4 cycles for the eight codes of a lane's word, so the
// point is to spend few instructions on each, and to keep enough of them in flight.  A warp owns 16 weight rows and walks over
// blocks of 256 inputs: a block's codes (2 KB) arrive by cp.async in a ring of the warp's own, three blocks deep.  They are the A operand of
// mma.m16n8k16; rows of x (or their terms) are the eight columns of B, so that 1 to 8 columns cost the same.  With so few
// columns the fifth-generation tensor cores have nothing to offer: an operand tile of 128 rows would have to go back to shared
// memory as 16-bit numbers, four times the bytes.
//
// Codes as fp16 numbers.  A stored nibble u = q + 8 in the lowest four bits of a 16-bit number is the fp16 number u 2^-24, one in the next
// four is 16 u 2^-24, both below the normal range and exact on the tensor cores: a mask is the whole conversion, of two codes at a time.  The
// products of the second kind have sums of their own, a sixteenth of which is added, and the 8 is paid back by -8 sum x~ of the
// group, known from the forming of x.  That cancellation costs up to log2(8 |sum x~| / |sum q x~|) of the sums' 24 bits (5 when all of x has one
// sign), which a result of 8 or 11 bits does not notice; for fp32 (EXACT) the nibbles go into the mantissa of 1024 and lose the
// offset by an exact fp16 addition per pair instead.
//
// x as fp16 numbers.  With 2^e the power of two that puts the largest magnitude of a group of x~ into [2^14, 2^15), x~ 2^e = hi + lo with hi
// and lo fp16.  16-bit x is hi itself (values below 2^-28 of their group's largest may lose bits).  Rotated bf16 x is taken as hi, off by
// at most 2^-11 of a value, where its result is rounded by up to 2^-8 (16 rows, 32,768 x 8,192: off by 1.667e-3 of the result's norm in all, a correctly rounded one
// by 1.654e-3; both terms would make twice the columns, 56 -> 89 us).  fp32 and rotated fp16 x take both: lo holds 11 of the rest's bits, so they are off by
// at most 2^-23.  lo makes further columns; the power
// multiplies the finished sum of a group with the weights' scale, in fp32.
//
// Work of a block of 8 warps: 16 WR rows, WK = 8 / WR warps side by side along k.  Where the rows make too few blocks for the GPU
// a cluster of up to 8 splits k, and joins its sums through distributed shared memory in the order of the ranks.
constexpr int kThreads = 256, kWarps = 8, kBlockK = 256, kBlockBytes = 16 * kBlockK / 2, kRing = 3;
constexpr int kFormSmem = 113 * 1024, kMostSmem = 200 * 1024; // the first: two blocks on an SM
// Where blocks do not form x: blocks of 256 inputs of which x is in shared memory at a time, and warps side by side along the
// rows.  (x costs a block of R rows C / 4 R times the bytes of its codes, from L2.)
constexpr __host__ __device__ int part_blocks(int nt) { return nt == 1 ? 4 : nt == 2 ? 2 : 1; }
constexpr __host__ __device__ int row_warps(int nt) { return nt == 1 ? 4 : 8; }
// Where they do: row blocks whose sums are joined together, with one barrier and one turn of writing for all of them.
constexpr __host__ __device__ int join_batch(int columns) { return columns <= 1 ? 8 : columns <= 2 ? 4 : columns <= 4 ? 2 : 1; }

struct LinearArgs {
    const uint8_t *codes;
    const uint16_t *scales; // bf16
    const void *x;          // FORM: x itself; otherwise the terms that form_kernel made of it, [token block][8 NT columns][blocks * 256]
    const float2 *factors;  // and the factor and offset of every group of a column, [token block][block][256 / G][8 NT]
    const void *bias;
    void *out;
    int64_t ldx, ldout, rows;
    int N, K, Kp, G, per_row; // per_row: groups of a weight row
    int tokens, terms;        // of a token block: tokens * terms <= 8 NT columns, term p of token t in column p * tokens + t
    int blocks, per_rank, ranks; // blocks of 256 inputs, and how many of them a rank of the cluster takes
    int stride;               // row blocks in flight
    int wide, wide_scales;    // x can be read 16 bytes at a time; all scales of a block at once
};

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t load_shared(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint4 load_shared16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// A word of eight codes as four pairs of fp16 numbers: exactly the codes, or (the first and third) u 2^-24, (the others) 16 u 2^-24.
template <bool EXACT> __device__ __forceinline__ void numbers(uint32_t w, uint32_t (&p)[4])
{
    // 0x6400 is 1024: a nibble in the lowest four bits of the mantissa adds itself, in the next four sixteen times itself (integers to floating point by
    // masks and one addition: Kim, Henry, Fahim, Awadalla, "Who Says Elephants Can't Run", 2022)
    const __half2 low = __float2half2_rn(-1032.0f), high = __float2half2_rn(-72.0f), sixteenth = __float2half2_rn(0.0625f);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uint32_t v = w >> (4 * i);
        uint32_t a = v & 0x000f000fu, b = v & 0x00f000f0u;
        if (EXACT) {
            a |= 0x64006400u, b |= 0x64006400u;
            const __half2 x = __hadd2(*reinterpret_cast<const __half2 *>(&a), low), y = __hfma2(*reinterpret_cast<const __half2 *>(&b), sixteenth, high);
            a = *reinterpret_cast<const uint32_t *>(&x), b = *reinterpret_cast<const uint32_t *>(&y);
        }
        p[i] = a, p[i + 1] = b;
    }
}
// d += the product of 16 x 16 numbers (two pairs for each of the lane's two rows) and 16 x 8 (not volatile: the compiler may place it)
__device__ __forceinline__ void product(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <class T, bool ROT> constexpr int kTerms = std::is_same<T, float>::value || (ROT && std::is_same<T, __half>::value) ? 2 : 1;

// The span of 128 inputs from column `col` on (a multiple of 128) of a row of x as terms; called by four neighbouring threads, whole
// warps.  term: where the span's first value of the first term goes, `next` elements before the second's; factor: where the factor and the
// offset of the span's first group go, `step` entries before the next group's and `beside` before the second term's.
template <class T, bool ROT>
__device__ __forceinline__ void form_span(const T *row, int col, int K, int G, bool wide, bool any, __half *term, int64_t next, float2 *factor, int step, int beside)
{
    const int j = threadIdx.x & 3;
    float v[4][8];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int k = col + 32 * c + 8 * j, valid = any ? K - k : 0;
        if (wide) load8<T, true>(row + k, valid, v[c]);
        else load8<T, false>(row + k, valid, v[c]);
    }
    if (ROT) rotate_span(v, G);
    uint32_t top[4]; // largest finite magnitude: what is not finite stays so under any scale
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        top[c] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t m = __float_as_uint(v[c][i]) & 0x7fffffffu;
            top[c] = max(top[c], m < 0x7f800000u ? m : 0u);
        }
        top[c] = max(top[c], __shfl_xor_sync(0xffffffffu, top[c], 1));
        top[c] = max(top[c], __shfl_xor_sync(0xffffffffu, top[c], 2));
    }
    if (G > 32) {
        top[0] = top[1] = max(top[0], top[1]);
        top[2] = top[3] = max(top[2], top[3]);
    }
    if (G > 64) top[0] = top[1] = top[2] = top[3] = max(top[0], top[2]);
    float total[kTerms<T, ROT>][4]; // of the terms of a group
    uint32_t field[4];              // of 2^e; tiny groups are not brought up all the way
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        field[c] = min(268u - (top[c] >> 23), 253u);
        const float up = __uint_as_float(field[c] << 23);
        __half hi[8], lo[8];
        float sum_hi = 0.0f, sum_lo = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = __fmul_rn(v[c][i], up);
            hi[i] = __float2half_rn(s);
            const float rest = __fsub_rn(s, __half2float(hi[i]));
            lo[i] = __float2half_rn(fabsf(s) <= 3.0e38f ? rest : 0.0f);
            sum_hi = __fadd_rn(sum_hi, __half2float(hi[i]));
            sum_lo = __fadd_rn(sum_lo, __half2float(lo[i]));
        }
        total[0][c] = sum_hi;
        if (any) *reinterpret_cast<uint4 *>(term + 32 * c + 8 * j) = *reinterpret_cast<const uint4 *>(hi);
        if (kTerms<T, ROT> == 2) {
            total[kTerms<T, ROT> - 1][c] = sum_lo;
            if (any) *reinterpret_cast<uint4 *>(term + next + 32 * c + 8 * j) = *reinterpret_cast<const uint4 *>(lo);
        }
    }
#pragma unroll
    for (int p = 0; p < kTerms<T, ROT>; ++p) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            total[p][c] = __fadd_rn(total[p][c], __shfl_xor_sync(0xffffffffu, total[p][c], 1));
            total[p][c] = __fadd_rn(total[p][c], __shfl_xor_sync(0xffffffffu, total[p][c], 2));
        }
        if (G > 32) {
            total[p][0] = __fadd_rn(total[p][0], total[p][1]);
            total[p][2] = __fadd_rn(total[p][2], total[p][3]);
        }
        if (G > 64) total[p][0] = __fadd_rn(total[p][0], total[p][2]);
        if (any && j == 0)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (((32 * c) & (G - 1)) == 0) {
                    const float down = __uint_as_float((254u - field[c]) << 23);
                    // the offset is -8 2^-24 times the group's sum
                    factor[(32 * c) / G * step + p * beside] = make_float2(down, __fmul_rn(__fmul_rn(total[p][c], -0x1p-21f), down));
                }
    }
}

// Terms, factors and offsets of all rows of x, for products whose blocks would repeat too much of that work.  A span of 128 inputs for
// every four threads.
template <class T, bool ROT>
__global__ void __launch_bounds__(kThreads) form_kernel(const T *x, int64_t ldx, uint32_t rows, int K, int G, int wide, int blocks, int tokens, int columns,
                                                        __half *terms, float2 *factors)
{
    ptx::wait_for_previous_kernels();
    ptx::launch_dependents(); // (not before the wait: the product reads codes before its own)
    const uint32_t spans = (uint32_t)blocks * (kBlockK / kSpan), item = blockIdx.x * (kThreads / 4) + threadIdx.x / 4, t = item / spans;
    const int span = (int)(item - t * spans);
    const bool any = t < rows;
    const uint32_t tb = t / (uint32_t)tokens;
    const int col = (int)(t - tb * (uint32_t)tokens);
    const int64_t width = (int64_t)blocks * kBlockK;
    form_span<T, ROT>(x + (int64_t)t * ldx, span * kSpan, K, G, wide, any, terms + ((int64_t)tb * columns + col) * width + (int64_t)span * kSpan,
                      tokens * width, factors + ((int64_t)tb * spans + span) * (kSpan / G) * columns + col, columns, tokens);
}

// FORM: the block forms the terms of its part of x itself, once; otherwise it copies them part by part, part_blocks(NT) blocks of inputs at a
// time.  SHIFT: a block of 256 inputs has 2^SHIFT groups.  A block (or cluster) takes row blocks blockIdx.x, blockIdx.x + stride, ...;
// the ring runs ahead from one into the next.  Scales come one block ahead, through registers.
template <class T, bool ROT, bool FORM, int SHIFT, int NT>
__global__ void __launch_bounds__(kThreads, NT == 8 ? 1 : 2) linear_kernel(const __grid_constant__ LinearArgs a)
{
    constexpr bool EXACT = std::is_same<T, float>::value;
    constexpr int WR = FORM ? 1 : row_warps(NT), WK = kWarps / WR, R = 16 * WR, C = 8 * NT, CH = part_blocks(NT), GROUPS = 1 << SHIFT;
    extern __shared__ __align__(128) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wr = warp / WK, wk = warp % WK;
    const int g = lane >> 2, t4 = lane & 3;
    const int ranks = a.ranks, rank = ranks > 1 ? (int)cg::this_cluster().block_rank() : 0;
    const int64_t t0 = (int64_t)blockIdx.y * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.rows - t0), columns = a.tokens * a.terms;
    const int first = rank * a.per_rank, count = max(0, min(a.per_rank, a.blocks - first)); // blocks of 256 inputs
    const int chunk = FORM ? a.per_rank : CH, N = a.N, step_n = a.stride * R;

    // shared memory: ring of codes, x and its factors (two parts unless the block forms them), sums (two halves if it does)
    const int parts = FORM ? 1 : 2, pitch = chunk * (kBlockK * 2) + 64; // (columns 64 bytes apart modulo 128: reads of two meet no bank twice)
    uint8_t *xs = smem + kWarps * kRing * kBlockBytes;
    const int x_bytes = (FORM ? columns : C) * pitch;
    float2 *factors = reinterpret_cast<float2 *>(xs + parts * x_bytes);
    const int factor_count = chunk * GROUPS * C;
    float *sums = reinterpret_cast<float *>(factors + parts * factor_count); // [halves][batch][WK][columns][R]
    const int batch = FORM ? join_batch(columns) : 1;

    // ring: a block is 16 rows of 128 bytes; copy i of a lane is piece lane % 8 of row 4 i + lane / 8, which goes to piece (lane % 8) ^ (row % 8), so
    // that the reads below (a word of each of 8 rows) touch every bank once
    const uint32_t row_bytes = (uint32_t)a.Kp / 2;
    const uint32_t ring = smem_at(smem) + warp * (kRing * kBlockBytes);
    const uint32_t ring_to = (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4);
    // Rows behind the last are read as the last one (their results go nowhere), and pieces behind the end of a row, whose x is 0, as
    // the block's first: there is nothing to fill up.
    const int piece = (lane & 7) * 16;
    const int tail = row_bytes % 128 && (uint32_t)piece >= row_bytes % 128 && first + count == a.blocks ? count - 1 : -1;
    int ahead_n = (int)(blockIdx.x / ranks) * R + 16 * wr; // first row and block of inputs that are fetched next
    int ahead = wk;
    const uint8_t *from = nullptr;
    uint32_t row_at[4];
    auto aim = [&] {
        from = a.codes + (uint64_t)(uint32_t)ahead_n * row_bytes + (uint32_t)((first + wk) * 128 + piece);
#pragma unroll
        for (int i = 0; i < 4; ++i) row_at[i] = (uint32_t)min(4 * i + (lane >> 3), N - 1 - ahead_n) * row_bytes; // (at most 15 rows of 2^23 bytes)
    };
    if (ahead_n < N) aim();
    auto fetch = [&](uint32_t slot_at) {
        if (ahead_n >= N) return;
        const uint8_t *at = from - (ahead == tail ? piece : 0);
        const uint32_t to = ring + slot_at + ring_to;
        copy16(to, at + row_at[0]);
        copy16((to ^ 64) + 512, at + row_at[1]);
        copy16(to + 1024, at + row_at[2]);
        copy16((to ^ 64) + 1536, at + row_at[3]);
        ahead += WK;
        from += WK * 128;
        if (ahead >= count) {
            ahead = wk;
            ahead_n += step_n;
            if (ahead_n < N) aim();
        }
    };
    // terms and factors of the part from `block` on
    auto fetch_x = [&](int block, int part) {
        constexpr int per_row = CH * kBlockK / 8; // 16-byte pieces of a column
        const int64_t width = (int64_t)a.blocks * kBlockK;
        const __half *base = (const __half *)a.x + (int64_t)blockIdx.y * C * width + (int64_t)(first + block) * kBlockK;
        const int here = min(CH, count - block);
        for (int i = threadIdx.x; i < columns * per_row; i += kThreads) {
            const int c = i / per_row, k = (i - c * per_row) * 8;
            if (k < here * kBlockK) copy16(smem_at(xs) + part * x_bytes + c * pitch + k * 2, base + c * width + k);
        }
        const float2 *fs = a.factors + ((int64_t)blockIdx.y * a.blocks + first + block) * GROUPS * C;
        for (int i = threadIdx.x; i < here * GROUPS * C / 2; i += kThreads) copy16(smem_at(factors) + (part * factor_count + 2 * i) * 8, fs + 2 * i);
    };
    // scales of a block's groups for the lane's two rows, two to a register; groups behind the row's last (of codes of which x is 0) take that one's
    int scale_block = wk;
    const uint16_t *scales_from[2] = {nullptr, nullptr};
    auto aim_scales = [&](int n) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            scales_from[h] = a.scales + (uint64_t)(uint32_t)min(n + 16 * wr + g + 8 * h, N - 1) * (uint32_t)a.per_row + (uint32_t)((first + wk) << SHIFT);
        scale_block = wk;
    };
    auto next_scales = [&](uint32_t (&s)[2][GROUPS / 2]) {
        if (scale_block >= count) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint16_t *at = scales_from[h];
            if (a.wide_scales) {
                if constexpr (SHIFT == 1) s[h][0] = *reinterpret_cast<const uint32_t *>(at);
                if constexpr (SHIFT == 2) {
                    const uint2 v = *reinterpret_cast<const uint2 *>(at);
                    s[h][0] = v.x, s[h][1] = v.y;
                }
                if constexpr (SHIFT == 3) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(at);
                    s[h][0] = v.x, s[h][1] = v.y, s[h][2] = v.z, s[h][3] = v.w;
                }
            } else {
                const int rest = a.per_row - 1 - ((first + scale_block) << SHIFT);
#pragma unroll
                for (int i = 0; i < GROUPS; i += 2) s[h][i / 2] = (uint32_t)at[min(i, rest)] | (uint32_t)at[min(i + 1, rest)] << 16;
            }
            scales_from[h] += WK << SHIFT;
        }
        scale_block += WK;
    };

    ptx::launch_dependents();
    if (FORM) ptx::wait_for_previous_kernels(); // (otherwise the kernel before this one has waited, and this one waits for it below)
    int n0 = (int)(blockIdx.x / ranks) * R;
    uint32_t scale[2][GROUPS / 2], scale_next[2][GROUPS / 2] = {};
    if (wk < count) {
#pragma unroll
        for (int s = 0; s < kRing - 1; ++s) {
            if (!FORM) copies_commit(); // (the place of a part of x, see below)
            fetch(s * kBlockBytes);
            copies_commit();
        }
        aim_scales(n0);
        next_scales(scale_next);
    }
    if constexpr (FORM) {
        const int spans = a.tokens * chunk * (kBlockK / kSpan);
        for (int base = 0; base < spans; base += kThreads / 4) { // (whole warps: the four of a span exchange values)
            const int i = base + threadIdx.x / 4, t = i / (chunk * (kBlockK / kSpan)), b = i - t * (chunk * (kBlockK / kSpan));
            const bool any = i < spans && t < tokens;
            form_span<T, ROT>((const T *)a.x + (t0 + (any ? t : 0)) * a.ldx, first * kBlockK + b * kSpan, a.K, a.G, a.wide, any,
                              reinterpret_cast<__half *>(xs + t * pitch) + b * kSpan, (int64_t)a.tokens * pitch / 2, factors + b * (GROUPS / 2) * C + t, C, a.tokens);
        }
    } else {
        ptx::wait_for_previous_kernels(); // the terms
        fetch_x(0, 0);
        copies_commit();
        copies_wait<0>();
    }
    __syncthreads();

    const uint32_t word_at = ring + g * 128 + (g << 4) + t4 * 4;
    const uint32_t x_at = smem_at(xs) + (FORM ? min(g, columns - 1) : g) * pitch + t4 * 16 + wk * (kBlockK * 2); // (columns that do not exist: anything)
    const uint32_t factor_at = smem_at(factors) + (wk * GROUPS * C + 2 * t4) * 8;
    uint32_t slot_at = 0;
    int part = 0, half = 0, joint = 0;
    for (; n0 < N; n0 += step_n) {
        float acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
        for (int start = 0; start == 0 || start < count; start += chunk) {
            const bool last = start + chunk >= count; // of this row block
            const bool more = !FORM && (!last || n0 + step_n < N);
            uint32_t xp = x_at + part * x_bytes, fp = factor_at + part * factor_count * 8;
            bool fresh = more;
            const int end = FORM ? count : min(start + CH, count);
            for (int b = start + wk; b < end; b += WK, xp += WK * kBlockK * 2, fp += WK * GROUPS * C * 8) {
                // Groups of copies of a turn: x (if the block does not form it), codes.  All but those of the block after this one are done.
                copies_wait<FORM ? kRing - 2 : 2 * (kRing - 2)>();
                __syncwarp();
                // the slot read a turn ago is free: every lane passed the __syncwarp above
                const uint32_t codes = word_at + slot_at;
                if (!FORM) {
                    if (fresh) fetch_x(last ? 0 : start + CH, part ^ 1);
                    fresh = false;
                    copies_commit();
                }
                fetch(slot_at == 0 ? (kRing - 1) * kBlockBytes : slot_at - kBlockBytes);
                copies_commit();
                slot_at = slot_at == (kRing - 1) * kBlockBytes ? 0 : slot_at + kBlockBytes;
#pragma unroll
                for (int i = 0; i < GROUPS / 2; ++i) scale[0][i] = scale_next[0][i], scale[1][i] = scale_next[1][i];
                if (scale_block >= count && n0 + step_n < N) aim_scales(n0 + step_n);
                next_scales(scale_next);
                float sum[2][NT][4]; // (EXACT: the first only)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t words[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        words[2 * j] = load_shared(codes ^ ((4 * h + j) << 4));
                        words[2 * j + 1] = load_shared((codes ^ ((4 * h + j) << 4)) + 1024);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        constexpr int SPAN = 8 >> SHIFT; // words of a group
                        const int at = 4 * h + j;
                        if (at % SPAN == 0)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int i = 0; i < 4; ++i) sum[0][n][i] = sum[1][n][i] = 0.0f;
                        uint32_t upper[4], lower[4];
                        numbers<EXACT>(words[2 * j], upper);
                        numbers<EXACT>(words[2 * j + 1], lower);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            // pairs (0, 2) and (1, 3) of the word, and the same of x
                            const uint4 x = load_shared16(xp + 8 * n * pitch + 64 * at);
                            product(sum[0][n], upper[0], lower[0], upper[2], lower[2], x.x, x.z);
                            product(sum[EXACT ? 0 : 1][n], upper[1], lower[1], upper[3], lower[3], x.y, x.w);
                        }
                        if ((at + 1) % SPAN == 0) { // the group ends
                            const int gr = at / SPAN;
                            float s[2];
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const uint32_t two = scale[r][gr / 2];
                                s[r] = __uint_as_float(gr % 2 ? two & 0xffff0000u : two << 16);
                                if (!EXACT) s[r] = __fmul_rn(s[r], 0x1p24f);
                            }
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                const uint4 f = load_shared16(fp + (gr * C + 8 * n) * 8);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const float factor = __uint_as_float(i % 2 ? f.z : f.x), offset = __uint_as_float(i % 2 ? f.w : f.y);
                                    const float v = EXACT ? __fmul_rn(sum[0][n][i], factor)
                                                          : __fmaf_rn(__fmaf_rn(sum[1][n][i], 0.0625f, sum[0][n][i]), factor, offset);
                                    acc[n][i] = __fmaf_rn(s[i / 2], v, acc[n][i]);
                                }
                            }
                        }
                    }
                }
            }
            if (more) {
                if (fresh) { // a warp that had no block of this part
                    fetch_x(last ? 0 : start + CH, part ^ 1);
                    copies_commit();
                    copies_wait<0>();
                } else copies_wait<1>(); // all but the codes of the last turn
            }
            if (last) { // this warp's part of the sums
                float *to = sums + ((half * batch + joint) * WK + wk) * columns * R + 16 * wr + g;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int c = 8 * n + 2 * t4 + i;
                        if (c < columns) to[c * R] = acc[n][i], to[c * R + 8] = acc[n][i + 2];
                    }
            }
            if (FORM) break;
            __syncthreads();
            part ^= 1;
        }
        if (++joint < batch && n0 + step_n < N) continue;
        if (FORM) __syncthreads();
        // join, in order: the warps along k, the terms, the ranks
        float *mine = sums + half * batch * WK * columns * R;
        auto joined = [&](int b, int t, int r) {
            const float *s = mine + b * WK * columns * R + t * R + r;
            float v = s[0];
#pragma unroll
            for (int w = 1; w < WK; ++w) v = __fadd_rn(v, s[w * columns * R]);
            if (a.terms == 2) {
                s += a.tokens * R;
#pragma unroll
                for (int w = 0; w < WK; ++w) v = __fadd_rn(v, s[w * columns * R]);
            }
            return v;
        };
        auto put = [&](float v, int n, int t) {
            if (a.bias) v = __fadd_rn(v, to_float(((const T *)a.bias)[n]));
            ((T *)a.out)[(t0 + t) * a.ldout + n] = from_float<T>(v);
        };
        if (ranks == 1) {
            const int n_first = n0 - (joint - 1) * step_n;
            for (int i = threadIdx.x; i < joint * tokens * R; i += kThreads) {
                const int r = i % R, bt = i / R, b = FORM ? bt / tokens : 0, t = bt - b * tokens, n = n_first + b * step_n + r;
                if (n < N) put(joined(b, t, r), n, t);
            }
        } else { // a row block for each cluster: a.stride covers them all
            cg::cluster_group cluster = cg::this_cluster();
            for (int i = threadIdx.x; i < tokens * R; i += kThreads) mine[i] = joined(0, i / R, i % R); // (a thread writes what it alone reads)
            cluster.sync();
            for (int i = threadIdx.x + rank * kThreads; i < tokens * R; i += ranks * kThreads) {
                if (n0 + i % R >= N) continue;
                float v = 0.0f;
                for (int q = 0; q < ranks; ++q) {
                    const float s = cluster.map_shared_rank(mine, q)[i];
                    v = q ? __fadd_rn(v, s) : s;
                }
                put(v, n0 + i % R, i / R);
            }
            cluster.sync(); // nobody leaves, and nobody's sums change, while they are read
        }
        joint = 0;
        if (FORM) half ^= 1;                    // (the next sums are written while slow warps still read these)
        else if (count <= CH) __syncthreads();  // (with more parts there is a barrier before the next sums)
    }
    copies_wait<0>();
}

// What a call's sizes and types make of it.
struct LinearPlan {
    bool form; // blocks form the terms themselves
    int terms, nt, tokens, token_blocks, blocks, ranks, per_rank;
    int64_t smem;
    int64_t term_bytes, factor_bytes; // of the workspace
};
LinearPlan plan_of(int64_t T, int64_t N, int64_t K, int group, bool rot, dhq_dtype_t dtype)
{
    LinearPlan p;
    p.terms = dtype == DHQ_F32 || (rot && dtype == DHQ_F16) ? 2 : 1;
    p.blocks = (int)((K + kBlockK - 1) / kBlockK);
    const int64_t groups = kBlockK / group;
    auto ranks_of = [&](int rows, int warps_k) { // a rank keeps a block of codes for each of its warps
        int r = 1;
        while (r < 8 && (N + rows - 1) / rows * r < 148 && p.blocks / (2 * r) >= warps_k) r *= 2;
        return r;
    };
    auto size = [&](int parts, int64_t chunk, int columns, int sums) {
        return kWarps * kRing * kBlockBytes + parts * (columns * (chunk * kBlockK * 2 + 64) + chunk * groups * 8 * p.nt * 8) + sums * (int64_t)p.tokens * p.terms * 16 * 4;
    };
    // Up to eight columns whose terms fit beside the ring, two blocks to an SM: every block forms them itself (some hundred
    // instructions a thread) and keeps them for all its rows of weights.  One launch, and no reads of x beside those of the codes.
    p.form = T * p.terms <= 8;
    if (p.form) {
        p.nt = 1, p.tokens = (int)std::max<int64_t>(T, 1), p.token_blocks = 1;
        p.ranks = ranks_of(16, kWarps);
        p.per_rank = (p.blocks + p.ranks - 1) / p.ranks;
        p.smem = size(1, p.per_rank, p.tokens * p.terms, 2 * join_batch(p.tokens * p.terms) * kWarps);
        p.form = p.smem <= kFormSmem;
        p.term_bytes = p.factor_bytes = 0;
    }
    if (!p.form) {
        const int columns = (int)std::min<int64_t>(64, std::max<int64_t>(T, 1) * p.terms);
        p.nt = columns <= 8 ? 1 : columns <= 16 ? 2 : columns <= 32 ? 4 : 8;
        p.tokens = (int)std::min<int64_t>(8 * p.nt / p.terms, std::max<int64_t>(T, 1));
        p.token_blocks = (int)((T + p.tokens - 1) / p.tokens);
        p.ranks = p.token_blocks > 1 ? 1 : ranks_of(16 * row_warps(p.nt), kWarps / row_warps(p.nt));
        p.per_rank = (p.blocks + p.ranks - 1) / p.ranks;
        p.smem = size(2, part_blocks(p.nt), 8 * p.nt, kWarps);
        p.term_bytes = (int64_t)p.token_blocks * 8 * p.nt * p.blocks * kBlockK * 2;
        p.factor_bytes = (int64_t)p.token_blocks * p.blocks * groups * 8 * p.nt * 8;
    }
    return p;
}

template <class T, bool ROT, bool FORM, int NT>
dhq_status_t launch_linear(const LinearArgs &a, const LinearPlan &p, bool early, cudaStream_t st)
{
    auto fn = a.G == 128 ? linear_kernel<T, ROT, FORM, 1, NT> : a.G == 64 ? linear_kernel<T, ROT, FORM, 2, NT> : linear_kernel<T, ROT, FORM, 3, NT>;
    constexpr int WR = FORM ? 1 : row_warps(NT);
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || !allow_smem((const void *)fn, dev, kMostSmem)) return DHQ_ERR_CUDA;
    const int row_blocks = (a.N + 16 * WR - 1) / (16 * WR);
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t c = {};
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = (size_t)p.smem;
    c.stream = st;
    c.attrs = attr;
    if (p.ranks > 1) {
        attr[c.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[c.numAttrs].val.clusterDim.x = (unsigned)p.ranks;
        attr[c.numAttrs].val.clusterDim.y = attr[c.numAttrs].val.clusterDim.z = 1;
        ++c.numAttrs;
    }
    if (early) { // set up while the kernels before it end; its codes may be on their way while the terms are formed
        attr[c.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[c.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++c.numAttrs;
    }
    // token blocks in launches of at most 65,535
    LinearArgs part = a;
    part.stride = p.ranks > 1 ? row_blocks : std::min(row_blocks, 148 * (p.smem <= kFormSmem ? 2 : 1));
    part.ranks = p.ranks;
    for (int64_t first = 0; first < p.token_blocks; first += 65535) {
        const int64_t blocks = std::min<int64_t>(65535, p.token_blocks - first);
        c.gridDim = dim3((unsigned)(part.stride * p.ranks), (unsigned)blocks);
        if (cudaLaunchKernelEx(&c, fn, part) != cudaSuccess) {
            cudaGetLastError();
            return DHQ_ERR_CUDA;
        }
        part.rows -= blocks * p.tokens;
        part.out = (T *)part.out + blocks * p.tokens * a.ldout;
        part.x = (const __half *)part.x + blocks * 8 * NT * a.blocks * kBlockK; // (a block that forms x has but one token block)
        part.factors += blocks * a.blocks * (kBlockK / a.G) * 8 * NT;
    }
    return DHQ_OK;
}
template <class T, bool ROT> dhq_status_t launch_linear(const LinearArgs &a, const LinearPlan &p, cudaStream_t st)
{
    if (p.form) return launch_linear<T, ROT, true, 1>(a, p, true, st);
    const bool early = p.token_blocks <= 65535;
    switch (p.nt) { // (formed x is alike with and without the rotation)
    case 1: return launch_linear<T, true, false, 1>(a, p, early, st);
    case 2: return launch_linear<T, true, false, 2>(a, p, early, st);
    case 4: return launch_linear<T, true, false, 4>(a, p, early, st);
    default: return launch_linear<T, true, false, 8>(a, p, early, st);
    }
}

// Forms the terms of all rows in the workspace.
template <class T, bool ROT> dhq_status_t launch_form(const LinearArgs &a, const LinearPlan &p, __half *terms, float2 *factors, cudaStream_t st)
{
    // rows in launches whose spans 32 bits can count, whole token blocks each
    const int64_t spans = (int64_t)p.blocks * (kBlockK / kSpan), most = std::max<int64_t>(1, ((int64_t)1 << 30) / (spans * p.tokens)) * p.tokens;
    for (int64_t first = 0; first < a.rows; first += most) {
        const int64_t rows = std::min(most, a.rows - first), tb = first / p.tokens;
        const dhq_status_t s = launch_behind(form_kernel<T, ROT>, dim3((unsigned)((rows * spans + kThreads / 4 - 1) / (kThreads / 4))), kThreads, 0, st,
                                             (const T *)a.x + first * a.ldx, a.ldx, (uint32_t)rows, a.K, a.G, a.wide, p.blocks, p.tokens, 8 * p.nt,
                                             terms + tb * 8 * p.nt * p.blocks * kBlockK, factors + tb * p.blocks * (kBlockK / a.G) * 8 * p.nt);
        if (s != DHQ_OK) return s;
    }
    return DHQ_OK;
}

} // namespace
} // namespace dhq

using namespace dhq;

extern "C" dhq_status_t dhq_w4_pack(const void *W, dhq_dtype_t dtype, int64_t N, int64_t K, int64_t ldw, int group,
                                    dhq_rot_t rotation, uint8_t *codes, uint16_t *scales, void *stream)
{
    if (!known_dtype(dtype) || N < 1 || N > kMaxColumns || !good_matrix(W, K, ldw, dtype)) return DHQ_ERR_INVALID_ARG;
    if (!codes || !aligned(codes, 16) || !scales || !aligned(scales, 2)) return DHQ_ERR_INVALID_ARG;
    const dhq_status_t s = good_form(group, rotation);
    if (s != DHQ_OK) return s;
    const int per_row = (int)(padded_columns(K, group) / group);
    const int64_t groups = N * per_row;
    const unsigned blocks = (unsigned)std::min<int64_t>((groups + kPackThreads / 32 - 1) / (kPackThreads / 32), 148 * 64);
    with_dtype(dtype, [&](auto tag) {
        using E = typename decltype(tag)::type;
        with_rot(rotation, [&](auto rot) {
            pack_kernel<E, decltype(rot)::value><<<blocks, kPackThreads, 0, (cudaStream_t)stream>>>((const E *)W, ldw, groups, (int)K, per_row, group, codes,
                                                                                                    (__nv_bfloat16 *)scales);
        });
    });
    return launched();
}

extern "C" dhq_status_t dhq_w4_linear_workspace(int64_t T, int64_t N, int64_t K, int group, dhq_rot_t rotation, dhq_dtype_t dtype, int64_t *bytes)
{
    if (!bytes || !known_dtype(dtype) || N < 1 || N > kMaxColumns || K < 1 || K > kMaxColumns || T < 0 || T > kMaxRows) return DHQ_ERR_INVALID_ARG;
    const dhq_status_t s = good_form(group, rotation);
    if (s != DHQ_OK) return s;
    const LinearPlan p = plan_of(T, N, K, group, rotation == DHQ_ROT_INPUT, dtype);
    *bytes = T ? p.term_bytes + p.factor_bytes : 0;
    return DHQ_OK;
}

extern "C" dhq_status_t dhq_w4_linear(const uint8_t *codes, const uint16_t *scales, int64_t N, int64_t K, int group,
                                      dhq_rot_t rotation, const void *x, dhq_dtype_t dtype, int64_t T, int64_t ldx,
                                      const void *bias, void *out, int64_t ldout, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!known_dtype(dtype) || N < 1 || N > kMaxColumns || K < 1 || K > kMaxColumns || T < 0 || T > kMaxRows) return DHQ_ERR_INVALID_ARG;
    dhq_status_t s = good_form(group, rotation);
    if (s != DHQ_OK) return s;
    if (T == 0) return DHQ_OK;
    if (!codes || !aligned(codes, 16) || !scales || !aligned(scales, 2) || (bias && !aligned(bias, elem_bytes(dtype)))) return DHQ_ERR_INVALID_ARG;
    if (!good_matrix(x, K, ldx, dtype) || !good_matrix(out, N, ldout, dtype)) return DHQ_ERR_INVALID_ARG;
    const LinearPlan p = plan_of(T, N, K, group, rotation == DHQ_ROT_INPUT, dtype);
    if (!p.form && (!workspace || !aligned(workspace, 16))) return DHQ_ERR_INVALID_ARG;
    if (!p.form && workspace_bytes < p.term_bytes + p.factor_bytes) return DHQ_ERR_ALLOC;
    LinearArgs a = {};
    a.codes = codes, a.scales = scales, a.x = x, a.bias = bias, a.out = out;
    a.ldx = ldx, a.ldout = ldout, a.rows = T;
    a.N = (int)N, a.K = (int)K, a.Kp = (int)padded_columns(K, group), a.G = group, a.per_row = a.Kp / group;
    a.tokens = p.tokens, a.terms = p.terms, a.blocks = p.blocks, a.per_rank = p.per_rank;
    a.wide = rows_of_16(x, ldx, dtype);
    const int groups = kBlockK / group;
    a.wide_scales = a.per_row % groups == 0 && aligned(scales, 2 * groups);
    with_dtype(dtype, [&](auto tag) {
        using E = typename decltype(tag)::type;
        with_rot(rotation, [&](auto rot) {
            if (!p.form) {
                float2 *factors = (float2 *)((uint8_t *)workspace + p.term_bytes);
                s = launch_form<E, decltype(rot)::value>(a, p, (__half *)workspace, factors, (cudaStream_t)stream);
                if (s != DHQ_OK) return;
                a.x = workspace, a.factors = factors;
            }
            s = launch_linear<E, decltype(rot)::value>(a, p, (cudaStream_t)stream);
        });
    });
    return s;
}
