// Activations kept in 8 bits for the backward pass (include/dhq_groups.h): the checkpoint and the activation in one pass
// over x, and the activation's gradient from the checkpoint.
//
// Both are bound by memory, and work on spans of 128 values (dhq_group.cuh).
#include "dhq_group.cuh"
#include "dhq_math.cuh"
#include "dhq_tmem.cuh"
#include "dhq_internal.cuh"
#include <algorithm>
#include <cmath>
#include <type_traits>

namespace dhq {
namespace {

constexpr int kThreads = 256;

struct ActParams {
    float turns_hi, turns_lo; // omega0 / (2 pi) as a sum of two fp32 numbers
    float omega0, s0;
};

// Fraction of a turn of omega0 x, in [-1/2, 1/2] and a rounding: the product is taken with its remainder, so that phases of some
// thousand rad keep the accuracy of small ones (below 2^22 turns; beyond, nothing of the phase is known).
__device__ __forceinline__ Two turn_fraction(Two x, const ActParams &a)
{
    const Two hi = both(a.turns_hi), magic = both(12582912.0f);
    const Two minus = mul2(x, both(-a.turns_hi)), low = fma2(x, both(a.turns_lo), fma2(x, hi, minus));
    return add2(sub2(sub2(add2(minus, magic), magic), minus), low); // (the sum with 1.5 2^23 is rounded to an integer)
}
__device__ __forceinline__ float cos_approx(float x)
{
    float y;
    asm("cos.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^t and 1 / x with results below 2^-126 as 0, which saves the instructions that bring such results out: for what is added to 1, or to
// something of that size.
__device__ __forceinline__ float exp2_flushed(float t)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    return e;
}
__device__ __forceinline__ float reciprocal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <class F> __device__ __forceinline__ Two each(Two v, F f)
{
    float lo, hi;
    apart(v, lo, hi);
    return two(f(lo), f(hi));
}
__device__ __forceinline__ Two sigmoid(Two x)
{
    const Two e = each(mul2(x, both(-1.4426950408889634f)), exp2_flushed);
    return each(add2(e, both(1.0f)), reciprocal);
}
// Phi(x), and exp(-x^2 / 2) beside it.  erfc(z) = (a1 t + ... + a5 t^5) exp(-z^2) + e(z), t = 1 / (1 + p z), z = |x| / sqrt 2, |e| <= 1.5e-7 (Abramowitz
// and Stegun 7.1.26): it shares its exponential with the density; erff and an exponential of its own take more than twice the instructions.
__device__ __forceinline__ Two normal_cdf(Two x, Two &bell)
{
    const Two t = each(x, [](float v) { return reciprocal(__fmaf_rn(fabsf(v), 0.3275911f * 0.70710678f, 1.0f)); });
    bell = each(mul2(mul2(x, both(-0.72134752f)), x), exp2_flushed); // -log2(e) / 2
    // halves of the coefficients: Phi(-|x|) is half of erfc
    Two poly = fma2(both(0.5307027145f), t, both(-0.7265760135f));
    poly = fma2(poly, t, both(0.7107068705f));
    poly = fma2(poly, t, both(-0.142248368f));
    poly = fma2(poly, t, both(0.127414796f));
    const Two tail = mul2(mul2(poly, t), bell);
    float x0, x1, t0, t1;
    apart(x, x0, x1);
    apart(tail, t0, t1);
    return two(x0 < 0.0f ? t0 : __fsub_rn(1.0f, t0), x1 < 0.0f ? t1 : __fsub_rn(1.0f, t1));
}
// exp(-(s0 x)^2), down to the smallest numbers
__device__ __forceinline__ Two envelope(Two g) { return each(mul2(mul2(g, g), both(-1.4426950408889634f)), gabor_envelope); }

constexpr float kTwoPi = 6.2831853071795865f;

template <int ACT> __device__ __forceinline__ Two act_value(Two x, const ActParams &a)
{
    if (ACT == DHQ_ACT_SILU) return mul2(x, sigmoid(x));
    Two bell;
    if (ACT == DHQ_ACT_GELU) return mul2(x, normal_cdf(x, bell));
    const Two s = each(mul2(turn_fraction(x, a), both(kTwoPi)), sin_approx);
    if (ACT == DHQ_ACT_SINE) return s;
    return mul2(s, envelope(mul2(both(a.s0), x)));
}
template <int ACT> __device__ __forceinline__ Two act_slope(Two x, const ActParams &a)
{
    if (ACT == DHQ_ACT_SILU) {
        const Two s = sigmoid(x);
        return mul2(s, fma2(x, sub2(both(1.0f), s), both(1.0f)));
    }
    if (ACT == DHQ_ACT_GELU) { // Phi(x) + x phi(x)
        Two bell;
        const Two cdf = normal_cdf(x, bell);
        return fma2(mul2(x, both(0.39894228f)), bell, cdf);
    }
    const Two t = mul2(turn_fraction(x, a), both(kTwoPi));
    const Two c = mul2(each(t, cos_approx), both(a.omega0));
    if (ACT == DHQ_ACT_SINE) return c;
    const Two g = mul2(both(a.s0), x);
    return mul2(fma2(mul2(g, both(-2.0f * a.s0)), each(t, sin_approx), c), envelope(g));
}

// The span of a group of four threads: row and first column, and whether there is one.
struct Place {
    int64_t row;
    int col;
    bool any;
};
__device__ __forceinline__ Place place_of(uint32_t block, uint32_t rows, uint32_t spans)
{
    const uint32_t item = block * (kThreads / 4) + threadIdx.x / 4, row = item / spans;
    return {(int64_t)row, (int)(item - row * spans) * kSpan, row < rows};
}

__device__ __forceinline__ void copy_some(uint32_t dst, const void *src, int bytes) // of 16, the rest zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void *src, int bytes) // of 8
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// How the rows move.
//   kDirect  fp32 rows aligned to 16 bytes: loads at the beginning of blocks that take one set of 64 spans each.
//   kFed     16-bit rows aligned to 16 bytes: a block works on one set of spans after another, and the pieces of the next ones are on their
//            way to shared memory meanwhile (each thread's own 16 bytes, so there is nothing to wait for but its own copies).  With half the
//            bytes of fp32 rows and the same arithmetic, loads at the beginning leave the memory idle for a third of the time
//            (16,384 x 8,192, bf16, save with silu: 150 -> 122 us).
//   kRagged  other rows: fed too, but a span comes as the 16-byte pieces of memory that it lies in, and leaves the same way, its ragged
//            ends number by number (16,383 x 4,095, bf16, rotated, save with silu, with a load and a store for each number: 188 -> 141 us).
enum Move { kDirect, kFed, kRagged };
constexpr int kFedStages = 3, kGradStages = 2; // of save, of the gradient and of ragged rows
template <class T> constexpr int kRaggedPieces = kSpan * (int)sizeof(T) / 16 + 1;
template <class T> constexpr int kRaggedBytes = 8 * kRaggedPieces<T> * 16; // of a warp and stage
template <class T> constexpr Move move_of(bool wide) { return !wide ? kRagged : sizeof(T) == 2 ? kFed : kDirect; }
template <class T, Move MOVE> constexpr int kSaveSmem = MOVE == kDirect ? 0 : MOVE == kFed ? kFedStages * 4 * kThreads * 16 : kGradStages * (kThreads / 32) * kRaggedBytes<T>;
template <class T, Move MOVE>
constexpr int kGradSmem = MOVE == kDirect ? 0 : kGradStages * (kThreads * 32 + (MOVE == kFed ? 4 * kThreads * 16 : (kThreads / 32) * kRaggedBytes<T>));

// Blocks that the registers have to leave room for on an SM.  kDirect lives off them (16,384 x 4,096, fp32, rotated: save 110 -> 96 us, gradient
// 155 -> 128 us); with more of them the others spill what the rotation holds.
template <Move MOVE> constexpr int kBlocksOf = MOVE == kDirect ? 3 : 2;

// kFed: a thread's four pieces of eight 16-bit numbers to `to`, `to + kThreads`, ...
template <class T> __device__ __forceinline__ void feed(uint4 *to, const T *x, int64_t ld, const Place &at, int K)
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int k = at.col + 32 * c + 8 * (threadIdx.x & 3), valid = at.any ? min(max(K - k, 0), 8) : 0;
        copy_some(smem_at(to + c * kThreads), valid ? x + at.row * ld + k : x, valid * 2);
    }
}
template <class T> __device__ __forceinline__ void fed(const uint4 *from, float (&v)[4][8])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint4 raw[1] = {from[c * kThreads]};
        if constexpr (sizeof(T) == 2) unpack8(raw, v[c], T());
    }
}

// kRagged: the pieces of memory that the warp's eight spans lie in, span s to `to` + s kRaggedPieces 16, its numbers from the offset that the
// span has in its first piece on.
template <class T> __device__ __forceinline__ void feed_ragged(uint8_t *to, const T *x, int64_t ld, const Place &at, int K)
{
    constexpr int P = kRaggedPieces<T>;
    const int lane = threadIdx.x & 31;
    const unsigned long long mine = (unsigned long long)(x + at.row * ld + at.col);
    const int my_bytes = at.any ? min(K - at.col, kSpan) * (int)sizeof(T) : 0; // (a span begins inside the row, or behind it with whole groups: none)
    __syncwarp(); // (everyone has read what was there)
#pragma unroll
    for (int r = 0; r < (8 * P + 31) / 32; ++r) {
        const int i = lane + 32 * r, s = min(i / P, 7), u = i - s * P;
        const unsigned long long start = __shfl_sync(0xffffffffu, mine, 4 * s);
        const int bytes = max(__shfl_sync(0xffffffffu, my_bytes, 4 * s), 0);
        if (u >= P) continue;
        const unsigned long long piece = (start & ~15ull) + 16 * u;
        const int have = (int)min((long long)16, max((long long)0, (long long)(start + bytes - piece)));
        uint8_t *dst = to + (s * P + u) * 16;
        if (bytes && piece < (unsigned long long)x) { // memory before the matrix is not touched: its first numbers one by one
            for (unsigned long long p = start; p < start + min(bytes, (int)(piece + 16 - start)); p += sizeof(T)) *(T *)(dst + (p - piece)) = *(const T *)p;
        } else copy_some(smem_at(dst), have && bytes ? (const void *)piece : (const void *)((uintptr_t)x & ~(uintptr_t)15), bytes ? have : 0);
    }
}
template <class T> __device__ __forceinline__ void fed_ragged(const uint8_t *from, const T *x, int64_t ld, const Place &at, int K, float (&v)[4][8])
{
    const int lane = threadIdx.x & 31, offset = (int)((uintptr_t)(x + at.row * ld + at.col) & 15);
    const uint8_t *span = from + (lane >> 2) * kRaggedPieces<T> * 16 + offset + 8 * (lane & 3) * (int)sizeof(T);
    __syncwarp(); // (the pieces are other threads' copies too)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int valid = at.any ? K - at.col - 32 * c - 8 * (lane & 3) : 0;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = i < valid ? *(const float *)(span + (32 * c + i) * 4) : 0.0f;
        } else {
            const uint8_t *at_word = (const uint8_t *)((uintptr_t)(span + 32 * c * 2) & ~(uintptr_t)3);
            uint32_t w[5];
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = i < 4 || (offset & 2) ? *(const uint32_t *)(at_word + 4 * i) : 0u;
            uint4 raw[1];
            uint32_t *r = reinterpret_cast<uint32_t *>(raw);
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = (offset & 2) ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
            unpack8(raw, v[c], T());
            if (valid < 8) // (numbers behind the row's end)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= valid) v[c][i] = 0.0f;
        }
    }
}
// v to the rows of y through `stage`, the warp's own.
template <class T> __device__ __forceinline__ void store_ragged(uint8_t *stage, T *y, int64_t ld, const Place &at, int K, const float (&v)[4][8])
{
    constexpr int P = kRaggedPieces<T>;
    const int lane = threadIdx.x & 31;
    const unsigned long long mine = (unsigned long long)(y + at.row * ld + at.col);
    const int my_count = at.any ? max(min(K - at.col, kSpan), 0) : 0;
    __syncwarp();
    T *span = (T *)(stage + (lane >> 2) * P * 16 + (int)(mine & 15)) + 8 * (lane & 3);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) span[32 * c + i] = from_float<T>(v[c][i]);
    __syncwarp();
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        const unsigned long long start = __shfl_sync(0xffffffffu, mine, 4 * s), end = start + __shfl_sync(0xffffffffu, my_count, 4 * s) * sizeof(T);
        const unsigned long long base = start & ~15ull, whole = (start + 15) & ~15ull, whole_end = end & ~15ull;
        const uint8_t *from = stage + s * P * 16;
        // whole pieces (at most 16, or 32), then the ends
        const unsigned long long piece = whole + 16 * lane;
        if (piece < whole_end) *(uint4 *)piece = *(const uint4 *)(from + (piece - base));
        const unsigned long long head = start + lane * sizeof(T), tail = max(whole_end, whole) + (lane - 16) * sizeof(T);
        if (lane < 16 && head < min(whole, end)) *(T *)head = *(const T *)(from + (head - base));
        if (lane >= 16 && tail < end) *(T *)tail = *(const T *)(from + (tail - base));
    }
}

// max of magnitudes that keeps a NaN
__device__ __forceinline__ float max_magnitude(float top, float v)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(top), "f"(fabsf(v)));
    return r;
}
__device__ __forceinline__ float max_magnitude(float top, float v, float w)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(top), "f"(v), "f"(w));
    return r;
}

template <class T, bool ROT, int ACT, Move MOVE>
__global__ void __launch_bounds__(kThreads, kBlocksOf<MOVE>) save_kernel(const T *x, int64_t ldx, uint32_t rows, int K, int Kp, int G, uint32_t spans, ActParams act,
                                                        int8_t *codes, uint8_t *exponents, T *y, int64_t ldy)
{
    ptx::launch_dependents();
    ptx::wait_for_previous_kernels();
    const int j = threadIdx.x & 3;
    extern __shared__ uint4 pieces[]; // kFed: [stage][4][thread]; kRagged: [stage][warp][kRaggedBytes]
    constexpr int STAGES = MOVE == kFed ? kFedStages : kGradStages;
    const uint32_t blocks = (uint32_t)(((int64_t)rows * spans + kThreads / 4 - 1) / (kThreads / 4));
    auto own = [&](int s) { return (uint8_t *)pieces + (s * (kThreads / 32) + threadIdx.x / 32) * kRaggedBytes<T>; };
    auto bring = [&](int s, const Place &at) {
        if (MOVE == kFed) feed<T>(pieces + s * 4 * kThreads + threadIdx.x, x, ldx, at, K);
        if (MOVE == kRagged) feed_ragged<T>(own(s), x, ldx, at, K);
        copies_commit();
    };
    if (MOVE != kDirect)
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) bring(s, place_of(blockIdx.x + s * gridDim.x, rows, spans));
    int turn = 0;
    for (uint32_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const Place at = place_of(block, rows, spans);
        const int here = turn;
        float v[4][8];
        if (MOVE == kDirect) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int k = at.col + 32 * c + 8 * j;
                load8<T, true>(x + at.row * ldx + k, at.any ? K - k : 0, v[c]);
            }
        } else {
            bring(turn == 0 ? STAGES - 1 : turn - 1, place_of(block + (STAGES - 1) * gridDim.x, rows, spans));
            copies_wait<STAGES - 1>();
            if (MOVE == kFed) fed<T>(pieces + turn * 4 * kThreads + threadIdx.x, v);
            else fed_ragged<T>(own(turn), x, ldx, at, K, v);
            turn = turn == STAGES - 1 ? 0 : turn + 1;
        }
        if (ACT != DHQ_ACT_NONE) {
            float o[4][8];
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 8; i += 2) apart(act_value<ACT>(two(v[c][i], v[c][i + 1]), act), o[c][i], o[c][i + 1]);
            if (MOVE == kRagged) store_ragged<T>(own(here), y, ldy, at, K, o);
            else
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int k = at.col + 32 * c + 8 * j;
                    store8<T, true>(y + at.row * ldy + k, at.any ? K - k : 0, o[c]);
                }
        }
        if (ACT != DHQ_ACT_NONE && !codes) { // (no checkpoint)
            if (MOVE == kDirect) break;
            continue;
        }
        if (ROT) rotate_span(v, G);
        float top[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            top[c] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i += 2) top[c] = max_magnitude(top[c], v[c][i], v[c][i + 1]);
            top[c] = max_magnitude(top[c], __shfl_xor_sync(0xffffffffu, top[c], 1));
            top[c] = max_magnitude(top[c], __shfl_xor_sync(0xffffffffu, top[c], 2));
        }
        if (G > 32) {
            top[0] = top[1] = max_magnitude(top[0], top[1]);
            top[2] = top[3] = max_magnitude(top[2], top[3]);
        }
        if (G > 64) top[0] = top[1] = top[2] = top[3] = max_magnitude(top[0], top[2]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int k = at.col + 32 * c;
            const uint32_t byte = exponent_byte(top[c]);
            if (byte == 255u) // codes of 0
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = 0.0f;
            const float inv = byte == 255u ? 1.0f : inverse_power(byte);
            // v 2^-e is exact; added to 1.5 2^23 it is rounded half to even, and the sum's lowest byte is the code
            uint32_t word[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t q[4];
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    float lo, hi;
                    apart(fma2(two(v[c][4 * w + i], v[c][4 * w + i + 1]), both(inv), both(12582912.0f)), lo, hi);
                    q[i] = __float_as_uint(lo), q[i + 1] = __float_as_uint(hi);
                }
                word[w] = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            }
            if (at.any && k < Kp) {
                *reinterpret_cast<uint2 *>(codes + at.row * Kp + k + 8 * j) = make_uint2(word[0], word[1]);
                if (j == 0 && (k & (G - 1)) == 0) exponents[at.row * (Kp / G) + k / G] = (uint8_t)byte;
            }
        }
        if (MOVE == kDirect) break; // (a set of spans for each block)
    }
    if (MOVE != kDirect) copies_wait<0>();
}

template <class T, bool ROT, int ACT, Move MOVE>
__global__ void __launch_bounds__(kThreads, kBlocksOf<MOVE>) act_grad_kernel(const int8_t *codes, const uint8_t *exponents, uint32_t rows, int K, int Kp, int G,
                                                            uint32_t spans, ActParams act, const T *dy, int64_t lddy, T *dx, int64_t lddx)
{
    ptx::launch_dependents();
    ptx::wait_for_previous_kernels();
    const int j = threadIdx.x & 3;
    extern __shared__ uint4 pieces[]; // codes [stage][4][thread] of eight bytes, then as in save_kernel
    uint2 *code_pieces = reinterpret_cast<uint2 *>(pieces);
    uint4 *dy_pieces = pieces + kGradStages * kThreads * 2;
    const float inv_g = ROT ? 1.0f / (float)G : 1.0f; // a power of two
    const uint32_t blocks = (uint32_t)(((int64_t)rows * spans + kThreads / 4 - 1) / (kThreads / 4));
    auto own = [&](int s) { return (uint8_t *)dy_pieces + (s * (kThreads / 32) + threadIdx.x / 32) * kRaggedBytes<T>; };
    auto exponents_of = [&](const Place &at, uint32_t (&e)[4]) {
#pragma unroll
        for (int c = 0; c < 4; ++c) e[c] = at.any && at.col + 32 * c < Kp ? exponents[at.row * (Kp / G) + (at.col + 32 * c) / G] : 0u;
    };
    auto bring = [&](int s, const Place &at) {
        if (MOVE == kFed) feed<T>(dy_pieces + s * 4 * kThreads + threadIdx.x, dy, lddy, at, K);
        if (MOVE == kRagged) feed_ragged<T>(own(s), dy, lddy, at, K);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const bool in = at.any && at.col + 32 * c < Kp;
            copy8(smem_at(code_pieces + (s * 4 + c) * kThreads + threadIdx.x), in ? codes + at.row * Kp + at.col + 32 * c + 8 * j : codes, in ? 8 : 0);
        }
        copies_commit();
    };
    uint32_t e[4], e_next[4];
    if (MOVE != kDirect) {
        const Place at = place_of(blockIdx.x, rows, spans);
        bring(0, at);
        exponents_of(at, e_next);
    }
    int turn = 0;
    for (uint32_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const Place at = place_of(block, rows, spans);
        const int here = turn;
        float v[4][8], d[4][8];
        uint2 q[4];
        if (MOVE == kDirect) {
            exponents_of(at, e);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int k = at.col + 32 * c + 8 * j;
                q[c] = at.any && at.col + 32 * c < Kp ? *reinterpret_cast<const uint2 *>(codes + at.row * Kp + k) : make_uint2(0, 0);
                load8<T, true>(dy + at.row * lddy + k, at.any ? K - k : 0, d[c]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) e[c] = e_next[c];
            const Place next = place_of(block + gridDim.x, rows, spans);
            bring(turn ^ 1, next);
            exponents_of(next, e_next);
            copies_wait<1>();
            if (MOVE == kFed) fed<T>(dy_pieces + turn * 4 * kThreads + threadIdx.x, d);
            else fed_ragged<T>(own(turn), dy, lddy, at, K, d);
#pragma unroll
            for (int c = 0; c < 4; ++c) q[c] = code_pieces[(turn * 4 + c) * kThreads + threadIdx.x];
            turn ^= 1;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const uint32_t u = (w ? q[c].y : q[c].x) ^ 0x80808080u; // codes + 128, as the lowest byte of 2^23 + that
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const Two b = two(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 | i)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441 + i)));
                    apart(add2(b, both(-8388736.0f)), v[c][4 * w + i], v[c][4 * w + i + 1]);
                }
            }
        if (ROT) rotate_span(v, G); // on whole numbers: exact
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const Two scale = both(__fmul_rn(power_of(e[c]), inv_g));
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                apart(mul2(two(d[c][i], d[c][i + 1]), act_slope<ACT>(mul2(two(v[c][i], v[c][i + 1]), scale), act)), d[c][i], d[c][i + 1]);
        }
        if (MOVE == kRagged) store_ragged<T>(own(here), dx, lddx, at, K, d);
        else
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int k = at.col + 32 * c + 8 * j;
                store8<T, true>(dx + at.row * lddx + k, at.any ? K - k : 0, d[c]);
            }
        if (MOVE == kDirect) break; // (a set of spans for each block)
    }
    if (MOVE != kDirect) copies_wait<0>();
}

template <class... P, class... A>
dhq_status_t launch_spans(void (*fn)(P...), Move move, int smem, unsigned blocks, cudaStream_t st, A... args)
{
    int dev = -1;
    if (smem && (cudaGetDevice(&dev) != cudaSuccess || !allow_smem((const void *)fn, dev, smem))) return DHQ_ERR_CUDA;
    return launch_behind<P...>(fn, dim3(move == kDirect ? blocks : std::min(blocks, 148u * 4u)), kThreads, (size_t)smem, st, args...);
}
// Rows are handed to the kernels in parts that 32-bit numbers of spans can count; f(first row, rows, blocks).
template <class F> dhq_status_t in_parts(int64_t T, uint32_t spans, F f)
{
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / spans);
    for (int64_t first = 0; first < T; first += most) {
        const int64_t rows = std::min(most, T - first);
        const dhq_status_t s = f(first, (uint32_t)rows, (unsigned)((rows * spans + kThreads / 4 - 1) / (kThreads / 4)));
        if (s != DHQ_OK) return s;
    }
    return DHQ_OK;
}

template <int A> using ActTag = std::integral_constant<int, A>;
template <class F> void with_act(dhq_act_t a, F f)
{
    if (a == DHQ_ACT_NONE) f(ActTag<DHQ_ACT_NONE>());
    else if (a == DHQ_ACT_SINE) f(ActTag<DHQ_ACT_SINE>());
    else if (a == DHQ_ACT_GABOR) f(ActTag<DHQ_ACT_GABOR>());
    else if (a == DHQ_ACT_SILU) f(ActTag<DHQ_ACT_SILU>());
    else f(ActTag<DHQ_ACT_GELU>());
}
ActParams act_params(float omega0, float s0)
{
    const double turns = (double)omega0 / 6.283185307179586476925287;
    ActParams a;
    a.turns_hi = (float)turns;
    a.turns_lo = (float)(turns - (double)a.turns_hi);
    a.omega0 = omega0;
    a.s0 = s0;
    return a;
}
dhq_status_t good_act(dhq_act_t a, float omega0, float s0)
{
    if (a < DHQ_ACT_SINE || a > DHQ_ACT_GELU) return DHQ_ERR_UNSUPPORTED;
    if ((a == DHQ_ACT_SINE || a == DHQ_ACT_GABOR) && !std::isfinite(omega0)) return DHQ_ERR_INVALID_ARG;
    if (a == DHQ_ACT_GABOR && !(s0 > 0.0f && std::isfinite(s0))) return DHQ_ERR_INVALID_ARG;
    return DHQ_OK;
}

} // namespace
} // namespace dhq

using namespace dhq;

extern "C" dhq_status_t dhq_checkpoint_save(const void *x, dhq_dtype_t dtype, int64_t T, int64_t K, int64_t ldx, int group,
                                            dhq_rot_t rotation, dhq_act_t activation, float omega0, float act_s0,
                                            int8_t *codes, uint8_t *exponents, void *y, int64_t ldy, void *stream)
{
    if (!known_dtype(dtype) || T < 0 || T > kMaxRows || K < 1 || K > kMaxColumns) return DHQ_ERR_INVALID_ARG;
    dhq_status_t s = good_form(group, rotation);
    if (s == DHQ_OK) s = good_act(activation, omega0, act_s0);
    if (s != DHQ_OK) return s;
    if (T == 0) return DHQ_OK;
    const bool with_y = activation != DHQ_ACT_NONE;
    const bool keep = codes || exponents; // (else y alone)
    if (!good_matrix(x, K, ldx, dtype) || (keep ? !codes || !aligned(codes, 16) || !exponents : !with_y)) return DHQ_ERR_INVALID_ARG;
    if (with_y ? !good_matrix(y, K, ldy, dtype) : y != nullptr) return DHQ_ERR_INVALID_ARG;
    const int64_t Kp = padded_columns(K, group);
    const uint32_t spans = (uint32_t)((Kp + kSpan - 1) / kSpan);
    const bool wide = rows_of_16(x, ldx, dtype) && (!with_y || rows_of_16(y, ldy, dtype));
    const ActParams act = act_params(omega0, act_s0);
    return in_parts(T, spans, [&](int64_t first, uint32_t rows, unsigned blocks) {
        dhq_status_t done = DHQ_OK;
        with_dtype(dtype, [&](auto tag) {
            using E = typename decltype(tag)::type;
            with_rot(rotation, [&](auto rot) {
                with_act(activation, [&](auto a) {
                    constexpr bool R = decltype(rot)::value;
                    constexpr int A = decltype(a)::value;
                    auto go = [&](auto move) {
                        constexpr Move M = decltype(move)::value;
                        done = launch_spans(save_kernel<E, R, A, M>, M, kSaveSmem<E, M>, blocks, (cudaStream_t)stream, (const E *)x + first * ldx, ldx, rows, (int)K, (int)Kp,
                                            group, spans, act, keep ? codes + first * Kp : nullptr, keep ? exponents + first * (Kp / group) : nullptr, with_y ? (E *)y + first * ldy : (E *)nullptr, ldy);
                    };
                    if (wide) go(std::integral_constant<Move, move_of<E>(true)>());
                    else go(std::integral_constant<Move, kRagged>());
                });
            });
        });
        return done;
    });
}

extern "C" dhq_status_t dhq_checkpoint_act_grad(const int8_t *codes, const uint8_t *exponents, int64_t T, int64_t K, int group,
                                                dhq_rot_t rotation, dhq_act_t activation, float omega0, float act_s0,
                                                const void *dy, dhq_dtype_t dtype, int64_t lddy, void *dx, int64_t lddx, void *stream)
{
    if (!known_dtype(dtype) || T < 0 || T > kMaxRows || K < 1 || K > kMaxColumns) return DHQ_ERR_INVALID_ARG;
    dhq_status_t s = good_form(group, rotation);
    if (s == DHQ_OK) s = activation == DHQ_ACT_NONE ? DHQ_ERR_UNSUPPORTED : good_act(activation, omega0, act_s0);
    if (s != DHQ_OK) return s;
    if (T == 0) return DHQ_OK;
    if (!codes || !aligned(codes, 16) || !exponents || !good_matrix(dy, K, lddy, dtype) || !good_matrix(dx, K, lddx, dtype)) return DHQ_ERR_INVALID_ARG;
    const int64_t Kp = padded_columns(K, group);
    const uint32_t spans = (uint32_t)((Kp + kSpan - 1) / kSpan);
    const bool wide = rows_of_16(dy, lddy, dtype) && rows_of_16(dx, lddx, dtype);
    const ActParams act = act_params(omega0, act_s0);
    return in_parts(T, spans, [&](int64_t first, uint32_t rows, unsigned blocks) {
        dhq_status_t done = DHQ_OK;
        with_dtype(dtype, [&](auto tag) {
            using E = typename decltype(tag)::type;
            with_rot(rotation, [&](auto rot) {
                with_act(activation, [&](auto a) {
                    constexpr int A = decltype(a)::value == DHQ_ACT_NONE ? (int)DHQ_ACT_SINE : decltype(a)::value; // (refused above)
                    constexpr bool R = decltype(rot)::value;
                    auto go = [&](auto move) {
                        constexpr Move M = decltype(move)::value;
                        done = launch_spans(act_grad_kernel<E, R, A, M>, M, kGradSmem<E, M>, blocks, (cudaStream_t)stream, codes + first * Kp,
                                            exponents + first * (Kp / group), rows, (int)K, (int)Kp, group, spans, act, (const E *)dy + first * lddy, lddy,
                                            (E *)dx + first * lddx, lddx);
                    };
                    if (wide) go(std::integral_constant<Move, move_of<E>(true)>());
                    else go(std::integral_constant<Move, kRagged>());
                });
            });
        });
        return done;
    });
}
