// Weight gradient of a linear layer from its input's checkpoint (include/dhq_groups.h): dW = dy^T x^.
//
// A plain matrix product but for its second operand, which is stored as 8-bit codes with a power of two per group.  q 2^e is exact
// in 16 bits, so nothing is lost by taking the product in dy's own type on the tensor cores (tcgen05, fp32 sums in tensor memory), and fp32 dy
// is exactly the sum of three bf16 numbers (8 bits each, by truncation), whose products go into the same sums.  The rotation is linear and
// does not touch the rows that the sum runs over: dW = (dy^T q 2^e) H / G, applied once to the finished sums.
//
// fp16 holds 65,504 at most, and q 2^e of a rotated group is up to G times as large as its x (rounded, it is larger without the rotation, too: 64 2^10 for
// 65,504).  A block whose dy is fp16 therefore takes its tile a second time if it has met such numbers: for each group with the least s at which
// 127 2^(e - s) is finite, powers of e - s, and finished sums times 2^s.  Then what lies 2^39 below the group's largest is rounded.
// The warp that makes powers of the exponents sees them anyway.  (8,192 rows, 4,096 x 4,096, groups of 128 / 32: 236 / 240 us without any of this, 237 / 243 with it;
// 253 / 277 where all warps look over the exponents first, 243 / 252 with the second time as a copy of the code, 245 / 265 as a function behind a call.)
//
// What bounds it is the traffic of shared memory (128 bytes per cycle and SM), not only the tensor pipe: with both operands there a
// 128 x 256 tile needs 96 bytes per cycle for the MMAs alone.  So x^ is the operand that lives in tensor memory (lane = input feature,
// column = two rows of the batch): the converting warps read codes as TMA left them in shared memory, transposed on the way as 8 x 8 matrices of
// pairs of bytes (ldmatrix, free of bank conflicts under the 128-byte swizzle: a pair of inputs at two rows ends up in one register), make each
// input's two rows 16-bit numbers in four instructions and store them with tcgen05.st, whose 16x128b form has just that layout.  dy is used as
// it lies in global memory (rows of the batch outside, features inside: MN-major, 128-byte swizzle), by TMA.  8,192 rows, 8,192 x 8,192, bf16:
// 896 to 927 us at full clock, 1,186 to 1,228 TFLOP/s, 0.71 to 0.73 of a plain product by cuBLAS in a short burst (in a loop of seconds, under the power limit, 1,043 to 1,074 us, 0.74 to 0.76 of
// cuBLAS there); a step moves 84 KB through shared memory, 656 of its 730 cycles.
// (Codes read from global memory by the converting warps, 8 rows x 32 bytes a load: 1,109 us; transposed in registers, movmatrix: 930.)
//
// Sums.  The tensor cores cut off what does not fit a sum, so that a sum of n products of 16 is too small by some 2e-8 n / 4 of itself: 3e-7
// after 1,024 rows of bf16, 5e-5 after 65,536 (measured).  A result of 8 or 11 bits does not notice that many, and more are
// split; for fp32 results the sums of every 1,024 rows
// (512 of fp16) are added to a running sum in shared memory (DRAIN) while the MMAs go on with a second set, and the small terms of fp32 dy have
// sums of their own.
//
// Roles: 16 warps convert (and finish the tile; four share a step, each four take every fourth one; 8 warps for fp32 dy, whose steps take three
// times as long), one runs the TMA ring, one brings the exponents, one issues the MMAs; fp32 dy is read by 16 warps and cut into terms.  Tile: 128
// inputs x BN outputs, 64 rows of the batch a step.  Where tiles are few the rows are split over blocks, and a second kernel adds the parts.
#include "dhq_group.cuh"
#include "dhq_tmem.cuh"
#include "dhq_internal.cuh"
#include "dhq_wait.h"
#include <algorithm>
#include <cuda.h>

namespace dhq {
namespace {

constexpr int kTileK = 128, kStep = 64;
constexpr int kLoadWarps = 16, kLoadTurns = 2; // fp32 dy: a half of the warps takes every other step
// Steps between drains: 1,024 rows, 512 for fp16 dy, whose longer products lose more.
template <class T> constexpr int kChunkOf = std::is_same<T, __half>::value ? 8 : 16;
constexpr int kScaleWords = 272; // of a stage: pairs of powers [4 groups][32 pairs of rows], the same for tiny fp16 groups, whether there are any
constexpr int kPitch = kTileK + 4; // floats of a row of the finished tile in shared memory: two rows of a quarter warp meet no bank twice
constexpr unsigned long long kWaitLimit = 2000000000ull; // ns: a wait that long ends the block, with NaN for results

// B operand in shared memory: MN-major, 128-byte swizzle.  64 features (128 bytes) x 64 rows make a box of 8 KB, boxes follow one another.
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(8192 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// kind::f16 with fp32 sums, A K-major (tensor memory), B MN-major; both operands bf16 or both fp16.
__device__ __forceinline__ uint32_t idesc_f16(bool bf16, int M, int N)
{
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (1u << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// Called by a whole warp, issued by one elected thread (see ptx::mma_i8).
__device__ __forceinline__ void mma_f16_tmem(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "elect.sync _|q, 0xffffffff;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
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
// Four 8 x 8 matrices of pairs of bytes, transposed: the address of row (lane % 8) of matrix (lane / 8), 16 bytes; of each the thread gets
// pair lane / 4 of rows 2 (lane % 4) and the next.
__device__ __forceinline__ void load_transposed(uint32_t at, uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(at) : "memory");
}
// 16 lanes x 32 columns: register 2 c + r of thread i is lane 8 r + i / 4, column 4 c + i % 4.
__device__ __forceinline__ void tmem_st_16x128b(uint32_t at, const uint32_t (&v)[16])
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
                   "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}

__device__ __forceinline__ void mbar_inval(uint32_t bar) { asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
template <int WARPS> __device__ __forceinline__ void converters_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory"); }

struct GradArgs {
    const int8_t *codes;
    const uint8_t *exponents;
    const void *dy;
    void *dW;
    float *partial;  // [split][tile][BN][128], or null: a block finishes its tile
    int64_t T, lddy, lddw;
    int N, K, Kp, G;
    int k_tiles, n_tiles, splits, steps; // steps of 64 rows in all
    int rotate, f32_out, wide_in, wide_out; // (wide: rows can be moved 16 bytes at a time)
};

template <class T> constexpr int kTermsOf = std::is_same<T, float>::value ? 3 : 1;
template <class T> constexpr int kConvertWarpsOf = std::is_same<T, float>::value ? 8 : 16;
template <class T> constexpr int kThreadsOf = 32 * (kConvertWarpsOf<T> + (std::is_same<T, float>::value ? kLoadWarps : 0) + 3);
// Tensor memory: sums (two sets where they are drained, one of them in use by the MMAs), for fp32 dy those of the small terms, then stages of x^ of
// 32 columns.
template <class T, int BN, bool DRAIN> constexpr int kFirstA = (std::is_same<T, float>::value ? 3 : DRAIN ? 2 : 1) * BN;
template <class T, int BN, bool DRAIN> constexpr int kStagesA = std::is_same<T, float>::value || (BN == 128 && !DRAIN) ? 4 : 8;
// Shared memory: ring of dy and codes, powers, running sums.  (BN = 128 without running sums is sized for two blocks to an SM, but 19 warps of
// 80 registers a thread leave room for one.  A ring of codes that runs two
// steps ahead of dy's: 936 us for 8,192 rows, 8,192 x 8,192, against 905.)
template <class T, int BN> constexpr int kDyBytes = BN * kStep * 2 * kTermsOf<T>;
template <class T, int BN> constexpr int kStageBytes = kDyBytes<T, BN> + kTileK * kStep;
template <class T, int BN, bool DRAIN> constexpr int kStagesB = std::is_same<T, float>::value ? 2 : BN == 256 ? 5 : DRAIN ? 6 : 4;
template <class T, int BN, bool DRAIN>
constexpr int kRingBytes = DRAIN ? kStagesB<T, BN, DRAIN> * kStageBytes<T, BN> : std::max(kStagesB<T, BN, DRAIN> * kStageBytes<T, BN>, BN *kPitch * 4);
template <class T, int BN, bool DRAIN>
constexpr int kGradSmem = kRingBytes<T, BN, DRAIN> + kStagesB<T, BN, DRAIN> * kScaleWords * 4 + (DRAIN ? BN * kPitch * 4 : 0) + 1024;

struct Waiter {
    volatile int *failed;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const
    {
        return wait_bounded([&] { return ptx::mbar_try_wait_hint(bar, parity, 20000); }, [] { return ptx::globaltimer(); }, kWaitLimit, failed);
    }
};

// Tiles in bands of eight along the outputs, so that blocks that run together share dy and codes in L2.
__device__ __forceinline__ void tile_place(int tile, int k_tiles, int n_tiles, int &kt, int &nt)
{
    const int band = tile / (8 * k_tiles), rest = tile - band * 8 * k_tiles, width = min(8, n_tiles - band * 8);
    kt = rest / width;
    nt = band * 8 + rest - kt * width;
}

// Codes of two rows (bytes 0 and 2 of p; the others are masked off) times the rows' powers.  The seven low bits of a code go into the mantissa of 128, its sign makes 256 of
// the 128 that is taken off again.
__device__ __forceinline__ uint32_t numbers_of(uint32_t p, uint32_t scale, __nv_bfloat16)
{
    const uint32_t a = (p & 0x007f007fu) | 0x43004300u, b = (p & 0x00800080u) | 0x43004300u;
    const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b)),
                                     *reinterpret_cast<const __nv_bfloat162 *>(&scale));
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t numbers_of(uint32_t p, uint32_t scale, __half)
{
    const uint32_t a = ((p & 0x00ff00ffu) ^ 0x64806480u); // 1024 + 128 + q
    const __half2 v = __hmul2(__hsub2(*reinterpret_cast<const __half2 *>(&a), __float2half2_rn(1152.0f)), *reinterpret_cast<const __half2 *>(&scale));
    return *reinterpret_cast<const uint32_t *>(&v);
}
// The powers of two exponent bytes (bits 0 and 16 on) as 16-bit numbers.  fp16 has 2^-14 .. 2^15 and infinity; below, the code is multiplied by
// 2^-14 and then by small16 of the byte.
__device__ __forceinline__ uint32_t powers16(uint32_t bytes, bool &, __nv_bfloat16) { return bytes << 7; }
__device__ __forceinline__ uint32_t powers16(uint32_t bytes, bool &small, __half)
{
    const uint32_t least = __vmaxu2(bytes, 0x00710071u);
    small = small || least != bytes;
    return (__vminu2(least, 0x008f008fu) - 0x00700070u) << 10;
}
constexpr uint32_t kLargestByte = 136; // 127 2^9 is finite in fp16, 64 2^10 is not
// Four exponent bytes less the shifts of their groups; zeros and broken groups stay, and what falls to 0 is nothing beside the largest.
__device__ __forceinline__ uint32_t shifted(uint32_t bytes, uint32_t shifts) { return __vsubus4(bytes, shifts & ~__vcmpeq4(bytes, 0xffffffffu)); }
__device__ __forceinline__ uint32_t small16(uint32_t byte) // 2^(e + 14) for e < -14, else 1; zeros for groups of zeros
{
    return byte == 0 ? 0u : byte >= 113u ? 0x3c00u : __half_as_ushort(__float2half_rn(power_of(byte + 14u)));
}

template <class D> __device__ __forceinline__ void write_span(D *row, int k, int K, bool any, const float (&v)[4][8])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) store8<D, true>(row + k + 32 * c, any ? K - k - 32 * c : 0, v[c]);
}
template <class D> __device__ __forceinline__ void write_values(D *row, int k0, int K, const float *values)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = 32 * i + (threadIdx.x & 31);
        if (k0 + k < K) row[k0 + k] = from_float<D>(values[k]);
    }
}
// Eight neighbouring finished rows of sums, a span of 128 inputs of row n + i with the four threads 4 i .. 4 i + 3 of the warp (v as
// rotate_span wants it).  Rows that cannot be written 16 bytes at a time go through `stage` (rows of kPitch, the warp's own), so that
// neighbouring threads write neighbouring values (1,000 rows, 333 x 777, fp16: 37 -> 22 us).
__device__ __forceinline__ void write_rows(const GradArgs &a, float (&v)[4][8], int n, int k0, bool half_type, float *stage)
{
    if (a.rotate) {
        rotate_span(v, a.G);
        const float inv = 1.0f / (float)a.G; // exact
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = __fmul_rn(v[c][i], inv);
    }
    const int mine = (threadIdx.x & 31) >> 2, at = 8 * (threadIdx.x & 3);
    if (a.wide_out) {
        const int64_t row = (int64_t)(n + mine) * a.lddw;
        const bool any = n + mine < a.N;
        if (a.f32_out) write_span((float *)a.dW + row, k0 + at, a.K, any, v);
        else if (half_type) write_span((__half *)a.dW + row, k0 + at, a.K, any, v);
        else write_span((__nv_bfloat16 *)a.dW + row, k0 + at, a.K, any, v);
        return;
    }
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) store8<float, true>(stage + mine * kPitch + 32 * c + at, 8, v[c]);
    __syncwarp();
    for (int i = 0; i < 8 && n + i < a.N; ++i) {
        const int64_t row = (int64_t)(n + i) * a.lddw;
        const float *values = stage + i * kPitch;
        if (a.f32_out) write_values((float *)a.dW + row, k0, a.K, values);
        else if (half_type) write_values((__half *)a.dW + row, k0, a.K, values);
        else write_values((__nv_bfloat16 *)a.dW + row, k0, a.K, values);
    }
}

// Warps 0 .. CW - 1 convert and finish the tile, then fp32: 16 that load dy; then the one of the TMA ring, that of the powers and that of the MMAs.
template <class T, int BN, bool DRAIN>
__global__ void __launch_bounds__(kThreadsOf<T>)
weight_grad_kernel(const __grid_constant__ GradArgs a, const __grid_constant__ CUtensorMap dy_map, const __grid_constant__ CUtensorMap code_map)
{
    constexpr bool F32 = std::is_same<T, float>::value;
    using M = std::conditional_t<F32, __nv_bfloat16, T>;
    constexpr bool HALF = std::is_same<M, __half>::value;
    constexpr int TERMS = kTermsOf<T>, SB = kStagesB<T, BN, DRAIN>, SA = kStagesA<T, BN, DRAIN>, STAGE = kStageBytes<T, BN>, DY = kDyBytes<T, BN>;
    constexpr int kChunk = kChunkOf<T>, CW = kConvertWarpsOf<T>, TURNS = CW / 4, RING_WARP = kThreadsOf<T> / 32 - 3, POWER_WARP = RING_WARP + 1, MMA_WARP = RING_WARP + 2;
    constexpr int DRAIN_AT = SB < kChunk - TURNS ? SB : kChunk - TURNS; // of a chunk: converters are some SB steps ahead, so the MMAs of the chunk before are done about then
    static_assert(TURNS <= 4 && (!DRAIN || DRAIN_AT > 0), "each turn has a step behind DRAIN_AT");
    // A warp that waits for codes has seen the step of TURNS before full, and steps become full in order (see the powers' warp): so was that of SB
    // before, the stage's last, and its barrier's parity says whether this round's have come.
    static_assert(SB >= TURNS && SA % TURNS == 0, "rounds of the rings");
    constexpr uint32_t COLUMNS = kFirstA<T, BN, DRAIN> + 32 * SA <= 256 ? 256 : 512;
    static_assert(kFirstA<T, BN, DRAIN> + 32 * SA <= 512, "tensor memory");
    extern __shared__ uint8_t raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    uint32_t *powers = (uint32_t *)(smem + kRingBytes<T, BN, DRAIN>);
    float *running = (float *)(DRAIN ? (uint8_t *)(powers + SB * kScaleWords) : smem); // [BN][kPitch]; in the place of the ring where it is only written at the end
    __shared__ uint64_t bars[3 * SB + 2 * SA + 5];
    __shared__ uint32_t tmem_holder;
    __shared__ int failed;
    __shared__ uint32_t large, tops[4]; // HALF: whether a byte above kLargestByte was met; then the largest of each group
    const int warp = (int)ptx::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    auto full_b = [&](int s) { return ptx::smem_u32(bars + s); };               // dy of a stage is there
    auto full_c = [&](int s) { return ptx::smem_u32(bars + SB + s); };          // its codes and powers are
    auto empty_b = [&](int s) { return ptx::smem_u32(bars + 2 * SB + s); };     // all have been used
    auto full_a = [&](int s) { return ptx::smem_u32(bars + 3 * SB + s); };      // x^ of a step is in tensor memory
    auto empty_a = [&](int s) { return ptx::smem_u32(bars + 3 * SB + SA + s); }; // and has been used
    const uint32_t done = ptx::smem_u32(bars + 3 * SB + 2 * SA), chunk_full = done + 8, chunk_empty = done + 24; // (two each)

    const int tiles = a.k_tiles * a.n_tiles, split = blockIdx.x / tiles, tile = blockIdx.x - split * tiles;
    int kt, nt;
    tile_place(tile, a.k_tiles, a.n_tiles, kt, nt);
    const int k0 = kt * kTileK, n0 = nt * BN;
    const int step0 = (int)((int64_t)a.steps * split / a.splits), steps = (int)((int64_t)a.steps * (split + 1) / a.splits) - step0;

    auto init_barriers = [&] {
        for (int s = 0; s < SB; ++s) {
            ptx::mbar_init(full_b(s), F32 ? kLoadWarps / kLoadTurns : 1);
            ptx::mbar_init(full_c(s), 2);
            ptx::mbar_init(empty_b(s), 1); // (the MMAs of a step have waited for those who read its codes)
        }
        for (int s = 0; s < SA; ++s) {
            ptx::mbar_init(full_a(s), 4);
            ptx::mbar_init(empty_a(s), 1);
        }
        ptx::mbar_init(done, 1);
        for (int c = 0; c < 2; ++c) {
            ptx::mbar_init(chunk_full + 8 * c, 1);
            ptx::mbar_init(chunk_empty + 8 * c, CW);
        }
        ptx::fence_mbar_init();
    };
    if (threadIdx.x == 0) {
        failed = 0, large = 0, tops[0] = tops[1] = tops[2] = tops[3] = 0;
        init_barriers();
    }
    // No block takes tensor memory and then waits for a kernel that may not have its own yet, and none of a later kernel starts before this one has.
    ptx::wait_for_previous_kernels();
    if (warp == MMA_WARP) {
        ptx::tmem_alloc(ptx::smem_u32(&tmem_holder), COLUMNS);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    ptx::launch_dependents();
    const uint32_t tmem = ptx::uniform(tmem_holder), first_a = tmem + kFirstA<T, BN, DRAIN>;
    const Waiter wait{&failed};

    uint32_t shifts = 0; // HALF: s of each group, a byte each
    for (;;) {
        if (warp < CW) {
            // x^: inputs 32 * (warp % 4) on of the tile, all rows of a step
            const int quarter = warp & 3, turn = warp >> 2;
            const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
            // sums of the input whose numbers go to this lane of tensor memory, for a part of the outputs
            const int x = 32 * quarter + 16 * (lane >> 4) + 2 * (lane & 7) + ((lane >> 3) & 1);
            constexpr int PART = BN * 4 / CW;
            const int part = (warp >> 2) * PART;
            // (matrix lane / 8: inputs 16 (lane / 8 % 2) on, rows 8 (lane / 16) on of 16)
            const uint32_t code_at = ptx::smem_u32(smem) + DY + (lane >> 4) * 1024 + (lane & 7) * 128 + (((2 * quarter + (lane >> 3 & 1)) ^ (lane & 7)) << 4);
            const uint32_t power_at = ptx::smem_u32(powers) + ((32 * quarter / a.G) * 32 + (lane & 3) * 4) * 4;
            // (stages and their phases are counted, not divided out: 234 instructions a step and warp of 32 rows, with them, were 0.9 of what a
            // scheduler issues in the time of the step's MMAs)
            int sb = turn % SB, round_b = turn / SB & 1;
            auto convert = [&](int i) {
                const int s = i % SA;
                if (!__all_sync(0xffffffffu, wait(full_c(sb), round_b))) return false;
                uint32_t v[2][8];
#pragma unroll
                for (int o = 0; o < 8; o += 2) load_transposed(code_at + sb * STAGE + o * 1024, v[0][o], v[1][o], v[0][o + 1], v[1][o + 1]);
                uint32_t by[8];
                auto powers_of = [&](int which) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 p = load_shared16(power_at + sb * (kScaleWords * 4) + 64 * h + which);
                        by[4 * h] = p.x, by[4 * h + 1] = p.y, by[4 * h + 2] = p.z, by[4 * h + 3] = p.w;
                    }
                };
                powers_of(0);
                uint32_t out[2][16];
#pragma unroll
                for (int o = 0; o < 8; ++o)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        out[m][2 * o] = numbers_of(v[m][o], by[o], M());
                        out[m][2 * o + 1] = numbers_of(v[m][o] >> 8, by[o], M());
                    }
                if (HALF && load_shared(ptx::smem_u32(powers) + sb * (kScaleWords * 4) + 1024)) { // tiny groups
                    powers_of(512);
#pragma unroll
                    for (int o = 0; o < 8; ++o)
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            uint32_t &w = out[y & 1][2 * o + (y >> 1)];
                            const __half2 r = __hmul2(*reinterpret_cast<const __half2 *>(&w), *reinterpret_cast<const __half2 *>(&by[o]));
                            w = *reinterpret_cast<const uint32_t *>(&r);
                        }
                }
                sb += TURNS;
                if (sb >= SB) sb -= SB, round_b ^= 1;
                if (!__all_sync(0xffffffffu, wait(empty_a(s), ((i / SA) & 1) ^ 1))) return false;
                ptx::tc_fence_after();
                const uint32_t to = first_a + lanes + 32 * s;
                tmem_st_16x128b(to, out[0]);
                tmem_st_16x128b(to + (16u << 16), out[1]);
                ptx::tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(full_a(s));
                return true;
            };
            int drained = 0;
            auto drain = [&] { // the sums of chunk `drained` join the running ones (each thread has its own)
                if (!__all_sync(0xffffffffu, wait(chunk_full + 8 * (drained & 1), drained >> 1 & 1))) return false;
                ptx::tc_fence_after();
#pragma unroll 1
                for (int n = part; n < part + PART; n += 32) {
                    uint32_t v[32];
                    ptx::tmem_ld32(tmem + lanes + BN * (drained & 1) + n, v);
                    ptx::tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float *to = running + (n + i) * kPitch + x;
                        *to = drained ? __fadd_rn(*to, __uint_as_float(v[i])) : __uint_as_float(v[i]);
                    }
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(chunk_empty + 8 * (drained & 1));
                ++drained;
                return true;
            };
            const int drains = DRAIN && steps > 0 ? (steps - 1) / kChunk : 0;
            bool on = true;
            for (int i = turn; i < steps && on; i += TURNS) {
                if (DRAIN && drained < i / kChunk && i % kChunk >= DRAIN_AT) on = drain();
                on = on && convert(i);
            }
            while (DRAIN && on && drained < drains) on = drain();
            const bool ok = steps == 0 || wait(done, 0);
            ptx::tc_fence_after();
            converters_sync<CW>(); // everyone is past the ring
            const int64_t out = a.partial ? (int64_t)blockIdx.x * BN * kTileK : 0;
            const float up = HALF ? power_of(127u + (shifts >> (8 * (x / a.G)) & 255u)) : 1.0f;
#pragma unroll 1
            for (int n = part; n < part + PART; n += 32) {
                uint32_t v[32], w[32];
                ptx::tmem_ld32(tmem + lanes + BN * (drains & 1) + n, v);
                if (F32) ptx::tmem_ld32(tmem + lanes + 2 * BN + n, w);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float f = __uint_as_float(v[i]);
                    if (F32) f = __fadd_rn(f, __uint_as_float(w[i]));
                    if (drains > 0) f = __fadd_rn(running[(n + i) * kPitch + x], f);
                    if (HALF) f = __fmul_rn(f, up);
                    f = steps == 0 ? 0.0f : ok && !failed ? f : __uint_as_float(0x7fffffffu);
                    if (a.partial) a.partial[out + (n + i) * kTileK + x] = f;
                    else running[(n + i) * kPitch + x] = f;
                }
            }
            ptx::tc_fence_before();
            if (!a.partial) {
                converters_sync<CW>();
                for (int r = threadIdx.x / 4; r < BN; r += 8 * CW) { // four threads to a row of 128 inputs
                    float v[4][8];
#pragma unroll
                    for (int c = 0; c < 4; ++c) load8<float, true>(running + r * kPitch + 32 * c + 8 * (threadIdx.x & 3), 8, v[c]);
                    write_rows(a, v, n0 + (r & ~7), k0, HALF, running + (r & ~7) * kPitch);
                }
            }
        } else if (warp == MMA_WARP) {
            const uint32_t idesc = idesc_f16(!HALF, kTileK, BN);
            for (int i = 0; i < steps; ++i) {
                const int sa = i % SA, sb = i % SB;
                bool ok = true;
                const int chunk = DRAIN ? i / kChunk : 0;
                if (DRAIN && i > 0 && i % kChunk == 0) {
                    ptx::mma_commit(chunk_full + 8 * ((chunk - 1) & 1));
                    ok = chunk < 2 || wait(chunk_empty + 8 * (chunk & 1), ((chunk >> 1) - 1) & 1);
                }
                ok = ok && wait(full_b(sb), (i / SB) & 1) && wait(full_a(sa), (i / SA) & 1);
                if (!__all_sync(0xffffffffu, ok)) break;
                ptx::tc_fence_after();
#pragma unroll
                for (int p = 0; p < TERMS; ++p)
#pragma unroll
                    for (int kk = 0; kk < kStep / 16; ++kk)
                        mma_f16_tmem(tmem + (p ? 2 * BN : BN * (chunk & 1)), first_a + 32 * sa + 8 * kk, desc_mn(ptx::smem_u32(smem) + sb * STAGE + p * (BN * kStep * 2) + kk * 2048), idesc,
                                     kk | (p ? i | (p - 1) : DRAIN ? i % kChunk : i));
                ptx::mma_commit(empty_a(sa));
                ptx::mma_commit(empty_b(sb));
            }
            if (steps > 0) ptx::mma_commit(done); // (else nobody waits for its arrival)
        } else if (warp == RING_WARP) { // codes and dy by TMA
            for (int i = 0; i < steps; ++i) {
                const int s = i % SB;
                if (!__all_sync(0xffffffffu, wait(empty_b(s), ((i / SB) & 1) ^ 1))) break;
                if (lane == 0) {
                    ptx::mbar_expect_tx(full_c(s), kTileK * kStep);
                    tma_load(ptx::smem_u32(smem) + s * STAGE + DY, &code_map, k0, (step0 + i) * kStep, full_c(s));
                    if (!F32) {
                        ptx::mbar_expect_tx(full_b(s), DY);
#pragma unroll
                        for (int b = 0; b < BN / 64; ++b)
                            tma_load(ptx::smem_u32(smem) + s * STAGE + b * 8192, &dy_map, n0 + 64 * b, (step0 + i) * kStep, full_b(s));
                    }
                }
                __syncwarp();
            }
        } else if (warp == POWER_WARP) {
            // Exponents of rows 2 lane and 2 lane + 1, as pairs of powers.  A row's one, two or four exponents of the tile come in one load where
            // rows are aligned for it (each load of the warp touches 32 lines).  The loads of four steps are issued together, while the four
            // before are handed out, and nothing looks at them until then (waiting for one load of many in flight would wait for all; with a test
            // or a shift behind each load 511 in place of 259 us for 8,192 rows, 4,096 x 4,096).
            const int per_row = a.Kp / a.G, per_tile = kTileK / a.G, last_group = min(per_tile, per_row - k0 / a.G) - 1;
            auto run = [&](auto element, auto many) {
                using E = decltype(element);
                constexpr int LOADS = decltype(many)::value, COUNT = LOADS * (int)sizeof(E), kAhead = 4;
                const uint8_t *const first = a.exponents + (int64_t)step0 * kStep * per_row + k0 / a.G;
                const int rows = (int)min((int64_t)steps * kStep, a.T - (int64_t)step0 * kStep); // of this block
                E e[kAhead][2][LOADS];
                auto load = [&](int i, E (&v)[2][LOADS]) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint8_t *at = first + (int64_t)min(i * kStep + 2 * lane + r, rows - 1) * per_row; // (behind the last row: that one's, see below)
#pragma unroll
                        for (int g = 0; g < LOADS; ++g) v[r][g] = *reinterpret_cast<const E *>(at + (LOADS > 1 ? min(g, last_group) : 0));
                    }
                };
#pragma unroll
                for (int u = 0; u < kAhead; ++u) load(u, e[u]);
                int s = 0, before = 0, round = 0, round_before = 0;
                uint32_t seen = 0;
                // pair p of rows (of 32): half p / 16 of the step, octet (p / 4) % 4, pair p % 4 of it; a reader wants its four octets together
                uint32_t *const mine = powers + (lane >> 4) * 16 + (lane & 3) * 4 + ((lane >> 2) & 3);
                for (int i0 = 0; i0 < steps; i0 += kAhead) {
                    uint32_t byte[kAhead][2]; // up to four exponents of a row
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            byte[u][r] = 0;
#pragma unroll
                            for (int g = 0; g < LOADS; ++g) byte[u][r] |= (uint32_t)e[u][r][g] << (8 * g);
                            if (HALF && shifts) byte[u][r] = shifted(byte[u][r], shifts);
                            if ((i0 + u) * kStep + 2 * lane + r >= rows) byte[u][r] = 0;
                        }
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) load(i0 + kAhead + u, e[u]);
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int i = i0 + u;
                        if (i >= steps) continue;
                        uint32_t pair[COUNT]; // (made before the wait: from there to the arrival others wait for this warp)
                        bool small = false;
#pragma unroll
                        for (int g = 0; g < COUNT; ++g) {
                            const uint32_t bytes = __byte_perm(byte[u][0], byte[u][1], 0x0400 + 0x0101 * g) & 0x00ff00ffu;
                            if (HALF) seen = __vmaxu2(seen, bytes);
                            pair[g] = powers16(bytes, small, M());
                        }
                        if (HALF) small = __any_sync(0xffffffffu, small);
                        if (!__all_sync(0xffffffffu, wait(empty_b(s), round ^ 1))) return;
                        uint32_t *to = mine + s * kScaleWords;
#pragma unroll
                        for (int g = 0; g < COUNT; ++g) to[32 * g] = pair[g];
                        if (HALF) {
                            if (small)
                                for (int g = 0; g < COUNT; ++g)
                                    to[128 + 32 * g] = small16((byte[u][0] >> (8 * g)) & 255u) | small16((byte[u][1] >> (8 * g)) & 255u) << 16;
                            if (lane == 0) powers[s * kScaleWords + 256] = small;
                        }
                        // Steps become full in order, though copies may land in another: a converting warp that has seen step j full knows that all
                        // steps before it were, and with them the round before of the stage that it waits for next.
                        if (i > 0 && !__all_sync(0xffffffffu, wait(full_c(before), round_before))) return;
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(full_c(s));
                        before = s, round_before = round;
                        if (++s == SB) s = 0, round ^= 1;
                    }
                }
                if (HALF && max(seen & 0xffffu, seen >> 16) > kLargestByte) large = 1;
            };
            using std::integral_constant;
            const bool together = per_row % per_tile == 0 && ((uintptr_t)a.exponents & (per_tile - 1)) == 0;
            if (steps == 0) {
            } else if (per_tile == 1) run(uint8_t(), integral_constant<int, 1>());
            else if (!together) run(uint8_t(), integral_constant<int, 4>()); // (with two groups a tile the last two are not used)
            else if (per_tile == 2) run(uint16_t(), integral_constant<int, 1>());
            else run(uint32_t(), integral_constant<int, 1>());
        } else if (F32) {
            // fp32 dy, cut into three bf16 terms: a warp takes every eighth row of a step, four features a thread.  Half of the warps wait for
            // their loads while the other half cuts.
            constexpr int THREADS = 32 * kLoadWarps / kLoadTurns, ROWS = kStep / (THREADS / 32);
            static_assert(!F32 || (BN == 128 && THREADS / 32 == 8), "a row of a tile is four features for each thread of a warp");
            const int turn = (threadIdx.x - 32 * CW) / THREADS, first = (warp - CW) % (THREADS / 32), n = n0 + 4 * lane;
            const bool whole = a.wide_in && n0 + BN <= a.N;
            float4 v[ROWS];
            auto load = [&](int i) {
                if (i >= steps) return;
                const int64_t t = (int64_t)(step0 + i) * kStep + first;
                const float *at = (const float *)a.dy + t * a.lddy + n;
                const int64_t next = 8 * a.lddy;
                if (whole && t - first + kStep <= a.T) {
#pragma unroll
                    for (int u = 0; u < ROWS; ++u, at += next) v[u] = *reinterpret_cast<const float4 *>(at);
                } else {
#pragma unroll
                    for (int u = 0; u < ROWS; ++u, at += next) {
                        const int valid = t + 8 * u < a.T ? a.N - n : 0;
                        v[u] = make_float4(valid > 0 ? at[0] : 0.0f, valid > 1 ? at[1] : 0.0f, valid > 2 ? at[2] : 0.0f, valid > 3 ? at[3] : 0.0f);
                    }
                }
            };
            // 16 bytes of a row of a tile hold eight features: this thread's are a half of piece lane / 2
            uint8_t *const to = smem + (lane >> 4) * 8192 + first * 128 + ((((lane >> 1) & 7) ^ first) << 4) + 8 * (lane & 1);
            auto store = [&](int i) {
                const int s = i % SB;
                float top = 0.0f;
#pragma unroll
                for (int u = 0; u < ROWS; ++u) {
                    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(v[u].x), "f"(v[u].y));
                    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(v[u].z), "f"(v[u].w));
                }
                const bool finite = top <= 3.402823466e+38f;
                if (!__all_sync(0xffffffffu, wait(empty_b(s), ((i / SB) & 1) ^ 1))) return false;
#pragma unroll
                for (int u = 0; u < ROWS; ++u) {
                    const float f[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
                    uint32_t term[3][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        term[0][j] = __float_as_uint(f[j]) & 0xffff0000u;
                        const float rest = __fsub_rn(f[j], __uint_as_float(term[0][j]));
                        term[1][j] = __float_as_uint(rest) & 0xffff0000u;
                        term[2][j] = __float_as_uint(__fsub_rn(rest, __uint_as_float(term[1][j])));
                    }
                    if (!finite) // infinities and NaN are their first term
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t bits = __float_as_uint(f[j]) & 0x7fffffffu;
                            if (bits >= 0x7f800000u) term[1][j] = term[2][j] = 0;
                            if (bits > 0x7f800000u) term[0][j] = 0x7fff0000u;
                        }
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        *reinterpret_cast<uint2 *>(to + s * STAGE + p * (BN * kStep * 2) + u * 1024) =
                            make_uint2(__byte_perm(term[p][0], term[p][1], 0x7632), __byte_perm(term[p][2], term[p][3], 0x7632));
                }
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(full_b(s));
                return true;
            };
            load(turn);
            for (int i = turn; i < steps; i += kLoadTurns) {
                if (!store(i)) break;
                load(i + kLoadTurns);
            }
        }
        if (failed) __nanosleep(1000000); // copies and MMAs in flight end by themselves
        __syncthreads();
        if (!HALF || shifts || !large) break;
        const int per_row = a.Kp / a.G, first = k0 / a.G, groups = min(kTileK / a.G, per_row - first);
        const int64_t end = min((int64_t)(step0 + steps) * kStep, a.T);
        for (int g = 0; g < groups; ++g) {
            uint32_t top = 0;
            for (int64_t r = (int64_t)step0 * kStep + threadIdx.x; r < end; r += kThreadsOf<T>) {
                const uint32_t byte = a.exponents[r * per_row + first + g];
                top = max(top, byte == 255u ? 0u : byte);
            }
            atomicMax(tops + g, top);
        }
        // Barriers and sums as at the beginning.  All copies, MMAs and drains have been waited for; the arrivals that say that stages are empty
        // are, now.
        if (warp == MMA_WARP) {
            for (int s = 0; s < min(SB, steps); ++s) wait(empty_b(s), ((steps - 1 - s) / SB) & 1);
            for (int s = 0; s < min(SA, steps); ++s) wait(empty_a(s), ((steps - 1 - s) / SA) & 1);
        }
        ptx::fence_proxy_async(); // (finished rows were written where copies go)
        ptx::tc_fence_before();
        __syncthreads();
        for (int g = 0; g < groups; ++g) shifts |= (max(tops[g], kLargestByte) - kLargestByte) << (8 * g);
        if (threadIdx.x == 0) {
            for (int i = 0; i < 3 * SB + 2 * SA + 5; ++i) mbar_inval(ptx::smem_u32(bars + i));
            init_barriers();
        }
        const bool again = shifts && !failed; // (without shifts there are broken groups only)
        __syncthreads();
        ptx::tc_fence_after();
        if (!again) break;
    }
    if (warp == MMA_WARP) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, COLUMNS);
    }
}

// 16-bit rows that TMA cannot take (not aligned to 16 bytes), copied to rows that it can.  32 neighbouring threads move neighbouring numbers.
__global__ void __launch_bounds__(256) align_kernel(const uint16_t *from, int64_t ld, int64_t rows, int N, uint16_t *to, int64_t to_ld)
{
    ptx::launch_dependents();
    ptx::wait_for_previous_kernels();
    const int per_row = (N + 255) / 256;
    const int64_t pieces = rows * per_row; // a warp moves 256 numbers of a row
    for (int64_t p = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; p < pieces; p += (int64_t)gridDim.x * 8) {
        const int64_t row = p / per_row;
        const int n = (int)(p - row * per_row) * 256 + (threadIdx.x & 31);
        uint16_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = n + 32 * i < N ? from[row * ld + n + 32 * i] : (uint16_t)0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n + 32 * i < N) to[row * to_ld + n + 32 * i] = v[i];
    }
}

// Adds the parts of every tile, rotates, and writes.  Four threads to a row of 128 inputs, of which Q such groups share the parts: group q
// adds parts q, q + Q, ..., then the groups' sums are added in order (65,536 rows, 256 x 256, 74 parts: with one group a row 70 us).
template <int BN, int Q>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ GradArgs a, int half_type)
{
    __shared__ float4 sums[Q > 1 ? 8 * 256 : 8 * 8 * kPitch / 4]; // [eighth of a thread's values][thread]; then rows to be written
    ptx::launch_dependents();
    ptx::wait_for_previous_kernels();
    const int tiles = a.k_tiles * a.n_tiles;
    const int slot = threadIdx.x / 4, q = slot % Q;
    const int64_t row = (int64_t)blockIdx.x * (64 / Q) + slot / Q;
    const int tile = (int)(row / BN), r = (int)(row - (int64_t)tile * BN);
    int kt, nt;
    tile_place(tile, a.k_tiles, a.n_tiles, kt, nt);
    const bool any = nt * BN + r < a.N; // (tiles * BN is a multiple of 64)
    float v[4][8];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = 0.0f;
    const int64_t next = (int64_t)tiles * BN * kTileK;
    const float *from = a.partial + row * kTileK + 8 * (threadIdx.x & 3) + q * next;
    if (any)
        for (int s = q; s < a.splits; s += Q, from += Q * next)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float p[8];
                load8<float, true>(from + 32 * c, 8, p);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = __fadd_rn(v[c][i], p[i]);
            }
    if (Q > 1) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) sums[(2 * c + i) * 256 + threadIdx.x] = make_float4(v[c][4 * i], v[c][4 * i + 1], v[c][4 * i + 2], v[c][4 * i + 3]);
        __syncthreads();
        if (threadIdx.x >= 256 / Q) return;
        const int mine = threadIdx.x / 4 * Q * 4 + (threadIdx.x & 3);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                for (int g = 0; g < Q; ++g) {
                    const float4 s = sums[(2 * c + i) * 256 + mine + 4 * g];
                    float *to = &v[c][4 * i];
                    to[0] = g ? __fadd_rn(to[0], s.x) : s.x, to[1] = g ? __fadd_rn(to[1], s.y) : s.y;
                    to[2] = g ? __fadd_rn(to[2], s.z) : s.z, to[3] = g ? __fadd_rn(to[3], s.w) : s.w;
                }
        static_assert(256 / (Q > 1 ? Q : 8) == 32, "one warp goes on: the sums are its own now");
        const int64_t out = (int64_t)blockIdx.x * (64 / Q);
        const int out_tile = (int)(out / BN), out_r = (int)(out - (int64_t)out_tile * BN);
        tile_place(out_tile, a.k_tiles, a.n_tiles, kt, nt);
        write_rows(a, v, nt * BN + out_r, kt * kTileK, half_type, (float *)sums);
    } else write_rows(a, v, nt * BN + (r & ~7), kt * kTileK, half_type, (float *)sums + threadIdx.x / 32 * 8 * kPitch);
}

struct GradPlan {
    int bn, k_tiles, n_tiles, splits, steps;
    int64_t blocks, join_blocks; // of the two launches
    int64_t part_bytes, copy_bytes, copy_ld; // of the workspace; elements of a row of the copy
    bool launchable() const { return std::max(blocks, join_blocks) < (int64_t)1 << 31; }
};
// BN = 128 where 256 would leave half of every tile empty, for fp32 dy (three terms, two sets of sums), and for fp32 sums that
// are drained (running sums of 128 x 256 would leave the ring two stages: 527 us for 8,192 rows, 4,096 x 4,096; now 370).  Rows are split where tiles alone do not
// fill the GPU evenly: the rounds of blocks over 148 SMs, in steps of 64 rows (a step of a 128 x 256 tile takes about 0.4 us; a block begins and
// ends within some 4 us), against the traffic of the parts (written and read once, some 4 TB/s, and a launch).
GradPlan plan_of(int64_t T, int64_t N, int64_t K, int group, dhq_dtype_t dtype, dhq_dtype_t dw_dtype, bool aligned_rows)
{
    GradPlan p;
    p.bn = N <= 128 || dtype == DHQ_F32 || (dw_dtype == DHQ_F32 && T > kStep * (dtype == DHQ_F16 ? kChunkOf<__half> : kChunkOf<__nv_bfloat16>)) ? 128 : 256;
    p.k_tiles = (int)((padded_columns(K, group) + kTileK - 1) / kTileK);
    p.n_tiles = (int)((N + p.bn - 1) / p.bn);
    p.steps = (int)((T + kStep - 1) / kStep);
    const int64_t tiles = (int64_t)p.k_tiles * p.n_tiles;
    const double step = dtype == DHQ_F32 ? 0.6 : 0.4 * p.bn / 256;
    double best = 1e300;
    p.splits = 1;
    // 16-bit results: a block sums 16,384 rows of fp16 at most (65,536 of bf16), so that what the tensor cores cut off stays well below half a
    // step of the result (2e-4 of a sum after 65,536 rows of one sign whose products have all their 18 bits).
    const int least = dw_dtype == DHQ_F32 ? 1 : (p.steps - 1) / (dtype == DHQ_F16 ? 256 : 1024) + 1;
    const int most = std::max(least, (int)std::min<int64_t>(std::min<int64_t>(p.steps, 148), std::max<int64_t>(1, ((int64_t)1 << 20) / tiles)));
    for (int s = least; s <= most; ++s) {
        const double rounds = (double)((tiles * s + 147) / 148);
        const double t = rounds * (step * ((p.steps + s - 1) / s) + 4.0) + (s > 1 ? 4.0 + 8.0 * s * tiles * p.bn * kTileK / 4e6 : 0.0);
        if (t < best) best = t, p.splits = s;
    }
    p.blocks = tiles * p.splits;
    p.join_blocks = p.splits > 1 ? tiles * (p.bn / (p.splits >= 8 ? 8 : 64)) : 0;
    p.part_bytes = p.splits > 1 && p.launchable() ? p.splits * tiles * p.bn * kTileK * 4 : 0;
    p.copy_ld = (N + 7) / 8 * 8;
    p.copy_bytes = dtype != DHQ_F32 && !aligned_rows ? T * p.copy_ld * 2 : 0;
    return p;
}

// A map of a matrix for boxes of `width` elements x 64 rows, 128 bytes wide.
dhq_status_t make_map(CUtensorMap *map, CUtensorMapDataType type, int bytes, const void *at, int64_t rows, int64_t columns, int64_t ld)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] { // the driver's function, looked up once
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) fn = nullptr;
        return (Encode)fn;
    }();
    if (!encode) return DHQ_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * bytes};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / bytes), kStep}, unit[2] = {1, 1};
    return encode(map, type, 2, const_cast<void *>(at), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? DHQ_OK
               : DHQ_ERR_CUDA;
}

template <class T, int BN, bool DRAIN> dhq_status_t launch_grad(const GradArgs &a, const CUtensorMap &dy_map, const CUtensorMap &code_map, cudaStream_t st)
{
    auto fn = weight_grad_kernel<T, BN, DRAIN>;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || !allow_smem((const void *)fn, dev, kGradSmem<T, BN, DRAIN>)) return DHQ_ERR_CUDA;
    const int64_t tiles = (int64_t)a.k_tiles * a.n_tiles;
    const dhq_status_t s = launch_behind(fn, dim3((unsigned)(tiles * a.splits)), kThreadsOf<T>, kGradSmem<T, BN, DRAIN>, st, a, dy_map, code_map);
    if (s != DHQ_OK || !a.partial) return s;
    const int half_type = std::is_same<T, __half>::value;
    if (a.splits >= 8) return launch_behind(join_kernel<BN, 8>, dim3((unsigned)(tiles * BN / 8)), 256, 0, st, a, half_type);
    return launch_behind(join_kernel<BN, 1>, dim3((unsigned)(tiles * BN / 64)), 256, 0, st, a, half_type);
}
template <class T> dhq_status_t launch_grad(const GradArgs &a, const GradPlan &p, const CUtensorMap &dy_map, const CUtensorMap &code_map, cudaStream_t st)
{
    if constexpr (std::is_same<T, float>::value) return launch_grad<T, 128, true>(a, dy_map, code_map, st);
    else {
        const bool drain = a.f32_out && (p.steps + p.splits - 1) / p.splits > kChunkOf<T>;
        if (p.bn == 256) return launch_grad<T, 256, false>(a, dy_map, code_map, st); // (for bf16 and fp16 results, or few rows)
        return drain ? launch_grad<T, 128, true>(a, dy_map, code_map, st) : launch_grad<T, 128, false>(a, dy_map, code_map, st);
    }
}

dhq_status_t good_sizes(int64_t T, int64_t N, int64_t K, int group, dhq_rot_t rotation, dhq_dtype_t dtype)
{
    if (!known_dtype(dtype) || T < 0 || T > kMaxRows || K < 1 || K > kMaxColumns || N < 1 || N > kMaxColumns) return DHQ_ERR_INVALID_ARG;
    const dhq_status_t s = good_form(group, rotation);
    // (a block for each tile of 128 x 256)
    return s != DHQ_OK ? s : ((K + 127) / 128) * ((N + 127) / 128) < ((int64_t)1 << 30) ? DHQ_OK : DHQ_ERR_UNSUPPORTED;
}

} // namespace
} // namespace dhq

using namespace dhq;

extern "C" dhq_status_t dhq_checkpoint_weight_grad_workspace(int64_t T, int64_t N, int64_t K, int group, dhq_rot_t rotation, dhq_dtype_t dtype,
                                                             const void *dy, int64_t lddy, dhq_dtype_t dw_dtype, int64_t *bytes)
{
    if (!bytes) return DHQ_ERR_INVALID_ARG;
    const dhq_status_t s = good_sizes(T, N, K, group, rotation, dtype);
    if (s != DHQ_OK) return s;
    if (dw_dtype != DHQ_F32 && dw_dtype != dtype) return DHQ_ERR_INVALID_ARG;
    const GradPlan p = plan_of(T, N, K, group, dtype, dw_dtype, rows_of_16(dy, lddy, dtype));
    if (!p.launchable()) return DHQ_ERR_UNSUPPORTED;
    *bytes = p.part_bytes + p.copy_bytes;
    return DHQ_OK;
}

extern "C" dhq_status_t dhq_checkpoint_weight_grad(const int8_t *codes, const uint8_t *exponents, int64_t T, int64_t K, int group,
                                                   dhq_rot_t rotation, const void *dy, dhq_dtype_t dtype, int64_t N, int64_t lddy,
                                                   void *dW, dhq_dtype_t dw_dtype, int64_t lddw, void *workspace,
                                                   int64_t workspace_bytes, void *stream)
{
    dhq_status_t s = good_sizes(T, N, K, group, rotation, dtype);
    if (s != DHQ_OK) return s;
    if (dw_dtype != DHQ_F32 && dw_dtype != dtype) return DHQ_ERR_INVALID_ARG;
    if (!good_matrix(dW, K, lddw, dw_dtype)) return DHQ_ERR_INVALID_ARG;
    if (T > 0 && (!codes || !aligned(codes, 16) || !exponents || !good_matrix(dy, N, lddy, dtype))) return DHQ_ERR_INVALID_ARG;
    const GradPlan p = plan_of(T, N, K, group, dtype, dw_dtype, rows_of_16(dy, lddy, dtype));
    if (!p.launchable()) return DHQ_ERR_UNSUPPORTED;
    const int64_t need = p.part_bytes + p.copy_bytes;
    if (need && (!workspace || !aligned(workspace, 16))) return DHQ_ERR_INVALID_ARG;
    if (workspace_bytes < need) return DHQ_ERR_ALLOC;
    const cudaStream_t st = (cudaStream_t)stream;
    GradArgs a = {};
    a.codes = codes, a.exponents = exponents, a.dy = dy, a.dW = dW;
    a.partial = p.part_bytes ? (float *)workspace : nullptr;
    a.T = T, a.lddy = lddy, a.lddw = lddw;
    a.N = (int)N, a.K = (int)K, a.Kp = (int)padded_columns(K, group), a.G = group;
    a.k_tiles = p.k_tiles, a.n_tiles = p.n_tiles, a.splits = p.splits, a.steps = p.steps;
    a.rotate = rotation == DHQ_ROT_INPUT, a.f32_out = dw_dtype == DHQ_F32, a.wide_out = rows_of_16(dW, lddw, dw_dtype);
    a.wide_in = rows_of_16(dy, lddy, dtype);
    CUtensorMap dy_map = {}, code_map = {};
    if (T > 0) {
        if (p.copy_bytes) {
            uint16_t *copy = (uint16_t *)((uint8_t *)workspace + p.part_bytes);
            const int64_t pieces = T * ((N + 255) / 256);
            s = launch_behind(align_kernel, dim3((unsigned)std::min<int64_t>((pieces + 7) / 8, 148 * 16)), 256, 0, st, (const uint16_t *)dy, lddy, T, (int)N, copy,
                              p.copy_ld);
            if (s != DHQ_OK) return s;
            a.dy = copy, a.lddy = p.copy_ld;
        }
        if ((s = make_map(&code_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, codes, T, a.Kp, a.Kp)) != DHQ_OK) return s;
        if (dtype != DHQ_F32 &&
            (s = make_map(&dy_map, dtype == DHQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.dy, T, N, a.lddy)) != DHQ_OK)
            return s;
    }
    with_dtype(dtype, [&](auto tag) { s = launch_grad<typename decltype(tag)::type>(a, p, dy_map, code_map, st); });
    return s;
}
