// Products of the rollout's weights for GB300 (sm_103a): quantisation to 4-bit
// strips with group scales, matrix-vector products with them, and a
// mixture-of-experts layer for a few tokens (include/rr.h has the definitions).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <type_traits>

#include "rr_internal.h"

namespace {

// ---------------------------------------------------------------------------
// 16-bit element types
// ---------------------------------------------------------------------------

struct BF16 {
    static __device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float(uint32_t(b) << 16); }
    static __device__ __forceinline__ uint16_t round(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
    static constexpr uint16_t kNaN = 0x7FC0;
};
struct F16 {
    static __device__ __forceinline__ float widen(uint16_t b) { return __half2float(__ushort_as_half(b)); }
    static __device__ __forceinline__ uint16_t round(float f) { return __half_as_ushort(__float2half_rn(f)); }
    static constexpr uint16_t kNaN = 0x7E00;
};

template <class T, bool F32>
__device__ __forceinline__ void put(void* out, int64_t i, float f) {
    if (F32) static_cast<float*>(out)[i] = f;
    else static_cast<uint16_t*>(out)[i] = T::round(f);
}

// silu(z) = z / (1 + exp(-z)) as the formula reads.
__device__ __forceinline__ float silu(float z) { return z / (1.0f + expf(-z)); }

// ---------------------------------------------------------------------------
// Packed matrices
// ---------------------------------------------------------------------------

constexpr int kStrip = 16;     // rows of a strip
constexpr int kBlock = 128;    // columns of a block
constexpr int kCodes = kStrip * kBlock / 2;   // bytes of a block's codes
constexpr int kMaxCols = 1 << 18;
constexpr float kLeastScale = 1.17549435e-38f;   // 2^-126

__host__ __device__ constexpr int block_bytes(int group) { return kCodes + 4096 / group; }

// The shape that the kernels take.
struct Packed {
    int64_t rows, cols;
    int64_t strips, blocks;    // of one matrix
    int64_t matrix_bytes;
    int32_t pair;
    // The row in slot r of strip s, or -1 past the edge.
    __device__ __forceinline__ int64_t row(int64_t s, int r) const {
        if (!pair) {
            const int64_t i = s * kStrip + r;
            return i < rows ? i : -1;
        }
        const int64_t i = s * (kStrip / 2) + (r & 7);
        return i < rows / 2 ? (r < 8 ? i : rows / 2 + i) : -1;
    }
};

__device__ __forceinline__ int code(uint32_t word, int i) {
    return int((word >> (4 * (i / 2 + 4 * (i % 2)))) & 15u) - 8;
}

// Eight adjacent 16-bit elements from p on, wherever p lies, of a buffer [begin, end);
// zeros from `left` elements on.  Two aligned 16-byte loads where both are within the
// buffer.
__device__ __forceinline__ uint4 load_any(const uint16_t* p, int left, const uint16_t* begin, const uint16_t* end) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), shift = at & 15;
    const uint4* const from = reinterpret_cast<const uint4*>(at - shift);
    if (left >= 8 && reinterpret_cast<const uint16_t*>(from) >= begin && reinterpret_cast<const uint16_t*>(from + 2) <= end) {
        const uint4 u = from[0], v = from[1];
        uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 6; ++i)
            if (shift & 8) w[i] = w[i + 2];
#pragma unroll
        for (int i = 0; i < 5; ++i)
            if (shift & 4) w[i] = w[i + 1];
        const uint32_t pick = shift & 2 ? 0x5432 : 0x3210;
        return make_uint4(__byte_perm(w[0], w[1], pick), __byte_perm(w[1], w[2], pick), __byte_perm(w[2], w[3], pick),
                          __byte_perm(w[3], w[4], pick));
    }
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = k < left ? p[k] : 0u;
    return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}

// A block of 128 columns by its number within a stack.
struct Item {
    int64_t mat, strip;
    int b;
    __device__ __forceinline__ Item(uint32_t i, const Packed& m) {
        const uint32_t blocks = uint32_t(m.blocks), strips = uint32_t(m.strips);
        b = int(i % blocks);
        i /= blocks;
        strip = i % strips;
        mat = i / strips;
    }
};

// Programmatic dependent launch: the next kernel on the stream may be scheduled
// while this one runs; each waits for the kernels before it to complete before it
// touches memory.
__device__ __forceinline__ void after_previous() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// The code of v in a group of scale s, as the last bits of a float: q + 8 in the low
// four of 0x4B400000 + q + 8.  q is v / s rounded to the nearest integer, ties to
// even, without a division: v (1 / s) is within 2^-21 of the quotient, and a
// quotient of two numbers of at most 11 significant bits that is not m + 1/2 is at
// least 2^-12 from it; rounding the product to multiples of 2^-13 (the sum with
// 1536 does that) thus leaves it on the side where it is, or on m + 1/2 exactly.
template <class T>
__device__ __forceinline__ uint32_t code_bits(float v, float inverse) {
    float q = fmaf(v, inverse, 1536.0f);
    // A float16 scale under its normal range is too coarse to keep q within 7.
    if (std::is_same<T, F16>::value) q = fminf(fmaxf(q, 1536.0f - 7.0f), 1536.0f + 7.0f);
    return __float_as_uint(q + (12582912.0f + 8.0f - 1536.0f));
}

// One warp takes one block: lane 4 g + t holds slots g and g + 8, of each the
// columns 32 j + 8 t + 0..7, so that codes need no exchange between lanes and a
// group's maximum at most two.  VEC: rows can be read 16 bytes at a time.  Bound
// by HBM: 2 bytes read and about half a byte written per element (24576 x 4096: 38.6 us,
// 6.55 TB/s; 30001 x 4097, every vector from two aligned ones: 79 us, 3.9 TB/s).
template <class T, int G, bool VEC>
__global__ void __launch_bounds__(256) rr_quantize_kernel(const __grid_constant__ Packed m, const uint16_t* w,
                                                          const uint16_t* end, int64_t ld, char* packed,
                                                          uint32_t total) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t i = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    after_previous();
    if (i >= total) return;
    const Item it(i, m);
    char* const to = packed + it.mat * m.matrix_bytes + (it.strip * m.blocks + it.b) * block_bytes(G);
    uint32_t v[2][4][4];       // pairs of elements
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int64_t row = m.row(it.strip, 8 * half + g);
        const uint16_t* const src = w + (it.mat * m.rows + max(row, int64_t(0))) * ld;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c = int64_t(it.b) * kBlock + 32 * j + 8 * t;
            uint4 u = make_uint4(0, 0, 0, 0);
            if (VEC && row >= 0 && c + 8 <= m.cols) {
                u = __ldcs(reinterpret_cast<const uint4*>(src + c));
            } else if (row >= 0 && c < m.cols) {
                u = load_any(src + c, int(min(int64_t(8), m.cols - c)), w, end);
            }
            v[half][j][0] = u.x, v[half][j][1] = u.y, v[half][j][2] = u.z, v[half][j][3] = u.w;
        }
    }
    constexpr int kWords = G / 32, kGroups = kBlock / G;
    uint16_t scale[kGroups][2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t words[4];
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            uint32_t top = 0;      // magnitudes are ordered as their bits are
#pragma unroll
            for (int j = k * kWords; j < (k + 1) * kWords; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) top = __vmaxu2(top, v[half][j][q] & 0x7FFF7FFFu);
            top = max(top >> 16, top & 0xFFFFu);
            top = max(top, __shfl_xor_sync(~0u, top, 1));
            top = max(top, __shfl_xor_sync(~0u, top, 2));
            const float a = T::widen(uint16_t(top));
            uint16_t s16 = T::round(a / 7.0f);
            float s = T::widen(s16);
            if (s < kLeastScale) s16 = 0;
            if (!(a < INFINITY)) s16 = T::kNaN;
            const bool dead = s < kLeastScale || !(a < INFINITY);
            const float inverse = 1.0f / s;
            scale[k][half] = s16;
#pragma unroll
            for (int j = k * kWords; j < (k + 1) * kWords; ++j) {
                // The floats' other bits, shifted like the codes, add up to a constant.
                uint32_t word = 0, rest = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    word += code_bits<T>(T::widen(uint16_t(v[half][j][q])), inverse) << (4 * q);
                    word += code_bits<T>(T::widen(uint16_t(v[half][j][q] >> 16)), inverse) << (4 * q + 16);
                    rest += (0x4B400000u << (4 * q)) + (0x4B400000u << (4 * q + 16));
                }
                words[j] = dead ? 0x88888888u : word - rest;
            }
        }
        *reinterpret_cast<uint4*>(to + 512 * half + 16 * lane) =
            make_uint4(words[0], words[1], words[2], words[3]);
    }
    if (t == 0)
#pragma unroll
        for (int k = 0; k < kGroups; ++k)
            reinterpret_cast<uint32_t*>(to + kCodes)[g * kGroups + k] =
                uint32_t(scale[k][0]) | uint32_t(scale[k][1]) << 16;
}

// The inverse, by the same lanes: half a byte read and 2 (or 4) written per element.
// Bound by HBM (24576 x 4096 to bfloat16: 37.8 us, 6.7 TB/s; 30001 x 4097: 86 us, against
// 440 with a store for each element).
template <class T, int G, bool F32, bool VEC>
__global__ void __launch_bounds__(256) rr_dequantize_kernel(const __grid_constant__ Packed m, const char* packed,
                                                            void* w, int64_t ld, uint32_t total) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t i = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    after_previous();
    if (i >= total) return;
    const Item it(i, m);
    const char* const from = packed + it.mat * m.matrix_bytes + (it.strip * m.blocks + it.b) * block_bytes(G);
    uint4 codes_of[2];
    uint32_t scale[kBlock / G];
#pragma unroll
    for (int half = 0; half < 2; ++half)
        codes_of[half] = __ldcs(reinterpret_cast<const uint4*>(from + 512 * half + 16 * lane));
#pragma unroll
    for (int k = 0; k < kBlock / G; ++k)
        scale[k] = reinterpret_cast<const uint32_t*>(from + kCodes)[g * (kBlock / G) + k];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int64_t row = m.row(it.strip, 8 * half + g);
        const uint32_t words[4] = {codes_of[half].x, codes_of[half].y, codes_of[half].z, codes_of[half].w};
        const int64_t c0 = int64_t(it.b) * kBlock + 8 * t, at0 = (it.mat * m.rows + row) * ld + c0;
        uint32_t before[4];        // the 8 elements to the left of this lane's
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float s = T::widen(uint16_t(half ? scale[32 * j / G] >> 16 : scale[32 * j / G]));
            const int64_t c = c0 + 32 * j, at = at0 + 32 * j;
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = s * float(code(words[j], k));
            if (F32) {
                if (row < 0) continue;
                if (VEC && c + 8 <= m.cols) {
                    float4* const p = reinterpret_cast<float4*>(static_cast<float*>(w) + at);
                    p[0] = make_float4(f[0], f[1], f[2], f[3]);
                    p[1] = make_float4(f[4], f[5], f[6], f[7]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (c + k < m.cols) put<T, true>(w, at + k, f[k]);
                }
                continue;
            }
            uint32_t own[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) own[k] = uint32_t(T::round(f[2 * k])) | uint32_t(T::round(f[2 * k + 1])) << 16;
            uint16_t* const p = static_cast<uint16_t*>(w) + at;
            if (VEC) {
                if (row < 0) continue;
                if (c + 8 <= m.cols) {
                    *reinterpret_cast<uint4*>(p) = make_uint4(own[0], own[1], own[2], own[3]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (c + k < m.cols) p[k] = uint16_t(own[k / 2] >> (16 * (k % 2)));
                }
                continue;
            }
            // At any alignment: the 16 aligned bytes that begin with the end of the lane to
            // the left (of lane 0: lane 3's, 32 columns back) and end with this lane's first
            // elements; those that no lane completes, one by one.
            uint32_t left[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t l = __shfl_sync(~0u, own[k], (lane - 1) & 31), far = __shfl_sync(~0u, j ? before[k] : 0, lane | 3);
                left[k] = t ? l : far;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) before[k] = own[k];
            if (row < 0) continue;
            const int over = int(reinterpret_cast<uintptr_t>(p) & 15) / 2;      // elements past an aligned address
            const bool first = j == 0 && t == 0, whole = c + 8 <= m.cols;
            if (whole && over == 0) {
                *reinterpret_cast<uint4*>(p) = make_uint4(own[0], own[1], own[2], own[3]);
            } else if (whole && !first) {
                uint32_t v[8] = {left[0], left[1], left[2], left[3], own[0], own[1], own[2], own[3]};
                const int from = 2 * (8 - over);      // the byte of v that goes to the aligned address
#pragma unroll
                for (int i = 0; i < 6; ++i)
                    if (from & 8) v[i] = v[i + 2];
#pragma unroll
                for (int i = 0; i < 5; ++i)
                    if (from & 4) v[i] = v[i + 1];
                const uint32_t pick = from & 2 ? 0x5432 : 0x3210;
                *reinterpret_cast<uint4*>(p - over) =
                    make_uint4(__byte_perm(v[0], v[1], pick), __byte_perm(v[1], v[2], pick), __byte_perm(v[2], v[3], pick),
                               __byte_perm(v[3], v[4], pick));
            }
            // This lane's own elements from `lo` on: none where the lane to the right
            // completes them, the last `over` where there is none, all of them where this one
            // wrote nothing.
            const bool ended = !(j == 3 && t == 3) && c + 16 <= m.cols;      // the next lane's are whole
            int lo = 8, hi = 8;
            if (over || !whole) {
                if (!whole) lo = 0, hi = int(max(int64_t(0), min(int64_t(8), m.cols - c)));
                else if (first) lo = 0, hi = ended ? 8 - over : 8;
                else if (!ended) lo = 8 - over;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k >= lo && k < hi) p[k] = uint16_t(own[k / 2] >> (16 * (k % 2)));
        }
    }
}

// ---------------------------------------------------------------------------
// Inner products on matrix instructions
// ---------------------------------------------------------------------------

// Weights are the 16-row operand A, tokens the 8-column operand B: a warp's lane
// 4 g + t holds rows g and g + 8 of A, token g of B, and of the sums rows g and
// g + 8 of tokens 2 t and 2 t + 1.  Which columns of a row form an instruction's
// 16 is free as long as A and B agree, so a lane's 8 columns of each 32 are
// adjacent: 16 bytes of tokens, 32 bits of codes, and no exchange between lanes.
template <class T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                    uint32_t b0, uint32_t b1) {
    if (std::is_same<T, BF16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// c = A B.
template <class T>
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
    if (std::is_same<T, BF16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// A word's codes as four pairs of 16-bit numbers q / kUp, exact; pair n is codes
// n and n + 4 (columns 2 n, 2 n + 1).  One shift serves two pairs: codes in bits 0..3
// and 4..7 of a half become numbers where they are.  What bounds the packed products
// is this arithmetic (half the shifts of one per pair: lm_head of Qwen3-8B, one
// token, 59 -> 55 us).
//   bfloat16: the low 8 bits of a pattern without others stand for their value times
//   2^-133 (the subnormals and the binade above them are evenly spaced), so a
//   multiplication by 2^123 or 2^119 brings either code to c 2^-10.  A group's 128
//   products of codes up to 7 2^-10 then stay below the largest element, and no sum
//   overflows that the result does not; results are multiplied by kUp = 2^10 at the end.
//   float16: under the exponent of 1024 they read 1024 + c and 1024 + 16 c (a published
//   conversion: Kim, Henry, Fahim, Awadalla, "Who Says Elephants Can't Run: Bringing Large
//   Scale MoE Models into Cloud Scale Production", 2022).
template <class T>
struct Codes {
    static constexpr float kUp = std::is_same<T, BF16>::value ? 1024.0f : 1.0f;
    static __device__ __forceinline__ uint32_t pair(uint32_t v, bool high) {
        uint32_t d;
        if (std::is_same<T, BF16>::value) {
            // 2^123, 2^119; - 8 * 2^-10.
            asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(v), "r"(high ? 0x7B007B00u : 0x7D007D00u), "r"(0xBC00BC00u));
        } else {
            // 1, 1 / 16; - 1032, - 72.
            asm("fma.rn.f16x2 %0, %1, %2, %3;"
                : "=r"(d) : "r"(v), "r"(high ? 0x2C002C00u : 0x3C003C00u), "r"(high ? 0xD480D480u : 0xE408E408u));
        }
        return d;
    }
    static __device__ __forceinline__ uint32_t mask(uint32_t w, bool high) {
        if (std::is_same<T, BF16>::value) return w & (high ? 0x00F000F0u : 0x000F000Fu);
        uint32_t v;
        if (high) asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0xEA;" : "=r"(v) : "r"(w), "r"(0x64006400u));
        else asm("lop3.b32 %0, %1, 0x000F000F, %2, 0xEA;" : "=r"(v) : "r"(w), "r"(0x64006400u));
        return v;
    }
    static __device__ __forceinline__ void unpack(uint32_t (&to)[4], uint32_t w) {
        const uint32_t u = w >> 8;
        to[0] = pair(mask(w, false), false);
        to[1] = pair(mask(w, true), true);
        to[2] = pair(mask(u, false), false);
        to[3] = pair(mask(u, true), true);
    }
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }

template <int N>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    if (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(N) : "memory");
}
// 16 bytes of shared memory: `bytes` copied, the rest zero.
__device__ __forceinline__ void copy_async_cut(uint32_t to, const void* from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

constexpr int kWarps = 16;         // of a block: one block per SM (24 warps: lm_head 55 -> 61 us)
constexpr int kProdThreads = 32 * kWarps;

// A warp's blocks of codes in flight.  A lane copies the 16-byte runs that it reads
// itself; of the scales, which four lanes share, lanes 0..7 copy a slot pair's each.
template <int G>
struct Block {
    static constexpr int kScale = 512 / G;                      // bytes of a slot pair's scales
    static constexpr int kBytes = kCodes + 8 * kScale;          // = block_bytes(G)
    // from: the block's codes at this lane's run.
    static __device__ __forceinline__ void copy(uint32_t to, const char* from, int lane) {
        copy_async<16>(to + 16 * lane, from);
        copy_async<16>(to + 512 + 16 * lane, from + 512);
        if (lane < 8) copy_async<kScale>(to + kCodes + kScale * lane, from + (kCodes + (kScale - 16) * lane));
    }
};

// How a product's tokens lie in shared memory, 16 bytes per 8 columns and plane:
//   kWhole: 16-bit elements;
//   kHalves, kThirds: the sum of two, of three 16-bit parts, a plane each;
//   kFloats: float32, of each 8 columns the first 4 in one plane, the last 4 in another.
enum Form { kWhole = 1, kHalves = 2, kThirds = 3, kFloats = 4 };
__host__ __device__ constexpr int planes_of(Form f) { return f == kFloats ? 2 : int(f); }

// 8 float32 numbers as three bfloat16 parts each, without an error (but under 2^-110,
// where the last part's bits end): a part is the upper half of what the ones before it
// leave, 8 of the 24 bits.  inf: there are infinities, whose other parts are zeros.
struct Parts {
    uint32_t w[3][4];
    __device__ __forceinline__ Parts(const char* x, int apart, bool inf) {
        const uint4 u = *reinterpret_cast<const uint4*>(x), v = *reinterpret_cast<const uint4*>(x + apart);
        uint32_t f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
        for (int p = 0; p < 3; ++p) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[p][k] = __byte_perm(f[2 * k], f[2 * k + 1], 0x7632);
            if (p == 2) break;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                f[i] = __float_as_uint(__uint_as_float(f[i]) - __uint_as_float(f[i] & 0xFFFF0000u));
            if (p == 0 && inf)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!isfinite(__uint_as_float(f[i]))) f[i] = 0;
        }
    }
};

// sum += W x over one block of 128 columns.  x[n]: this lane's 16 bytes of its
// token's row at the block's first column, in shared memory; planes are `apart` bytes
// apart.  Groups are summed in the matrix unit and scaled in float32; the sums are
// 1 / kUp of the product's.
template <class T, int G, int NT, Form FORM = kWhole>
__device__ __forceinline__ void block_product(float (&sum)[NT][4], const char* stage, const char* const (&x)[NT],
                                              int at, int lane, int apart = 0, bool inf = false) {
    const int g = lane >> 2;
    const uint4 lo = *reinterpret_cast<const uint4*>(stage + 16 * lane);
    const uint4 hi = *reinterpret_cast<const uint4*>(stage + 512 + 16 * lane);
    uint32_t s[128 / G];       // {slot g, slot g + 8}
#pragma unroll
    for (int k = 0; k < 128 / G; ++k)
        s[k] = reinterpret_cast<const uint32_t*>(stage + kCodes)[g * (128 / G) + k];
    const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
    float part[NT][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t al[4], ah[4];
        Codes<T>::unpack(al, wl[j]);
        Codes<T>::unpack(ah, wh[j]);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if constexpr (FORM == kFloats) {
                const Parts v(x[n] + at + 64 * j, apart, inf);
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    if (p == 0 && 32 * j % G == 0) mma_first<T>(part[n], al[0], ah[0], al[1], ah[1], v.w[p][0], v.w[p][1]);
                    else mma<T>(part[n], al[0], ah[0], al[1], ah[1], v.w[p][0], v.w[p][1]);
                    mma<T>(part[n], al[2], ah[2], al[3], ah[3], v.w[p][2], v.w[p][3]);
                }
                continue;
            }
            const uint4 v = *reinterpret_cast<const uint4*>(x[n] + at + 64 * j);
            if (32 * j % G == 0) mma_first<T>(part[n], al[0], ah[0], al[1], ah[1], v.x, v.y);
            else mma<T>(part[n], al[0], ah[0], al[1], ah[1], v.x, v.y);
            mma<T>(part[n], al[2], ah[2], al[3], ah[3], v.z, v.w);
#pragma unroll
            for (int p = 1; p < FORM; ++p) {
                const uint4 r = *reinterpret_cast<const uint4*>(x[n] + p * apart + at + 64 * j);
                mma<T>(part[n], al[0], ah[0], al[1], ah[1], r.x, r.y);
                mma<T>(part[n], al[2], ah[2], al[3], ah[3], r.z, r.w);
            }
        }
        if (32 * (j + 1) % G == 0) {
            const float sl = T::widen(uint16_t(s[32 * j / G])), sh = T::widen(uint16_t(s[32 * j / G] >> 16));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                sum[n][0] = fmaf(sl, part[n][0], sum[n][0]);
                sum[n][1] = fmaf(sl, part[n][1], sum[n][1]);
                sum[n][2] = fmaf(sh, part[n][2], sum[n][2]);
                sum[n][3] = fmaf(sh, part[n][3], sum[n][3]);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Matrix-vector products
// ---------------------------------------------------------------------------

struct MatvecArgs {
    Packed m;
    const char* packed;
    const uint16_t* x;
    void* out;
    int64_t ldx, ldo;
    int32_t tokens, f32;
    int32_t vec;          // x's rows can be read 16 bytes at a time
    int32_t pitch;        // bytes between tokens in shared memory
    int32_t cluster;      // blocks that share the columns
    int32_t batch;        // strips between two joins of a cluster's sums
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive;\nbarrier.cluster.wait;" ::: "memory");
}

// The epilogue of rows g, g + 8 and tokens 2 t, 2 t + 1 (+ 8 n) of a strip.
template <class T>
__device__ __forceinline__ void put_strip(const MatvecArgs& a, int64_t strip, int lane, int n, const float (&v)[4]) {
    const int g = lane >> 2, t = lane & 3;
    const int64_t lo = a.m.row(strip, g), hi = a.m.row(strip, 8 + g);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int tok = 8 * n + 2 * t + i;
        if (tok >= a.tokens || lo < 0) continue;
        const int64_t at = tok * a.ldo;
        if (a.m.pair) {
            const float h = silu(v[i]) * v[2 + i];
            if (a.f32) put<T, true>(a.out, at + lo, h);
            else put<T, false>(a.out, at + lo, h);
        } else {
            if (a.f32) put<T, true>(a.out, at + lo, v[i]);
            else put<T, false>(a.out, at + lo, v[i]);
            if (hi >= 0) {
                if (a.f32) put<T, true>(a.out, at + hi, v[2 + i]);
                else put<T, false>(a.out, at + hi, v[2 + i]);
            }
        }
    }
}

// A run of `total` blocks of weights, shared out evenly over a thread block's warps
// wherever strips begin and end: warp w takes [share_from(w), share_from(w + 1)).
// A strip that lies in one warp's share is finished there; of another, each warp
// leaves its part: the last one (and only it) as its first part, the others as
// their last.  Parts are joined in the order of the warps.
__device__ __forceinline__ int share_from(int w, int total) { return int(uint32_t(w) * uint32_t(total) / kWarps); }
__device__ __forceinline__ int share_of(int p, int total) { return int((kWarps * uint32_t(p + 1) - 1) / uint32_t(total)); }

// A cluster takes a run of strips; each of its blocks takes a share of the
// columns, whose tokens it keeps in shared memory, and a warp an even share of
// the run's blocks of weights, which it streams through stages of U blocks of its own
// without meeting others.  Parts of strips are joined through shared memory at
// the end, and a cluster's sums through its blocks' shared memory after each
// `batch` of strips.  ST: blocks in flight.
// Bound by unpacking codes where there is much to read, by launch, first loads and
// join (4 us) where there is little.  On the GPU: 151936 x 4096, one token 54.5 us (5.9
// TB/s), eight 57.0; 24576 x 4096, four 13.6 us; 5120 x 25600, eight 18.4 us; 6144 x
// 4096, one 5.6 us.  Even shares, rather than whole strips to teams of warps: 24.0 ->
// 18.5 us for 5120 x 25600, whose 320 strips divide badly, 54.5 -> 55.7 for the largest.
template <class T, int G, int NT, int U, int ST>
__global__ void __launch_bounds__(kProdThreads, 1) rr_matvec_kernel(const __grid_constant__ MatvecArgs a) {
    extern __shared__ __align__(128) char smem[];
    using S = Block<G>;
    constexpr int kStages = ST / U, kStageBytes = U * S::kBytes;
    constexpr int kPart = NT * 32;                    // float4 of a strip's sums
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = blockIdx.x % a.cluster, cl = blockIdx.x / a.cluster, n_cl = gridDim.x / a.cluster;
    after_previous();
    // Stages; the tokens; each warp's first part; a cluster's sums by strip.  A warp's
    // last part goes where its stages were.
    char* const fifo = smem + warp * (ST * S::kBytes);
    char* const xs = smem + kWarps * ST * S::kBytes;
    float4* const parts = reinterpret_cast<float4*>(xs + a.tokens * a.pitch);
    float4* const full = parts + kWarps * kPart;
    float4* const last = reinterpret_cast<float4*>(fifo);

    const int64_t s0 = cl * a.m.strips / n_cl, s1 = (cl + 1) * a.m.strips / n_cl;
    const int b0 = int(rank * a.m.blocks / a.cluster), nb = int((rank + 1) * a.m.blocks / a.cluster) - b0;

    // Tokens: this block's columns, zeros past the matrix's.
    const int cols = nb * kBlock;
    const int64_t c0 = int64_t(b0) * kBlock;
    if (a.vec) {
        // 16-byte copies, cut off (and zero-filled) at the row's end.
        for (int n = 0; n < a.tokens; ++n)
            for (int c = 8 * threadIdx.x; c < cols; c += 8 * kProdThreads) {
                const int64_t left = a.m.cols - c0 - c;
                copy_async_cut(smem_at(xs + n * a.pitch + 2 * c), a.x + n * a.ldx + (left > 0 ? c0 + c : 0),
                               left >= 8 ? 16 : left > 0 ? 2 * int(left) : 0);
            }
    } else {
        const uint16_t* const end = a.x + (a.tokens - 1) * a.ldx + a.m.cols;
        const int chunks = cols / 8;
#pragma unroll 4
        for (int k = threadIdx.x; k < a.tokens * chunks; k += kProdThreads) {
            const int n = k / chunks, c = 8 * (k - n * chunks);
            *reinterpret_cast<uint4*>(xs + n * a.pitch + 2 * c) =
                load_any(a.x + n * a.ldx + c0 + c, int(max(int64_t(0), min(int64_t(8), a.m.cols - c0 - c))), a.x, end);
        }
    }
    copy_commit();
    // A lane of an absent token reads the last one's row; its sums go nowhere.
    const char* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
        x[n] = xs + min(8 * n + (lane >> 2), a.tokens - 1) * a.pitch + 16 * (lane & 3);

    const uint32_t fifo_at = smem_at(fifo);
    const int64_t next_strip = (a.m.blocks - nb) * S::kBytes;      // from a strip's last block here to the next's first
    bool staged = false;
    for (int64_t f = s0; f < s1; f += a.batch) {
        const int strips = int(min(int64_t(a.batch), s1 - f)), total = strips * nb;
        const int lo = share_from(warp, total), hi = share_from(warp + 1, total);
        int strip = lo / nb, b = lo - strip * nb;
        // The load cursor, kStages - 1 stages ahead.
        const char* from = a.packed + ((f + strip) * a.m.blocks + b0 + b) * S::kBytes + 16 * lane;
        int lb = b, left = hi - lo, slot = 0;
        auto load = [&](int to) {
            if (a.cluster == 1 && left >= U) {
                // Strip follows strip.
#pragma unroll
                for (int u = 0; u < U; ++u) S::copy(fifo_at + to * kStageBytes + u * S::kBytes, from + u * S::kBytes, lane);
                from += U * S::kBytes;
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (left > u) {
                        S::copy(fifo_at + to * kStageBytes + u * S::kBytes, from, lane);
                        from += S::kBytes;
                        if (++lb == nb) lb = 0, from += next_strip;
                    }
            }
            left -= U;
            copy_commit();
        };
        for (int i = 0; i < kStages - 1; ++i) load(i);
        if (!staged) {
            copy_wait<kStages - 1>();
            __syncthreads();
            staged = true;
        }
        float sum[NT][4] = {};
        bool whole = b == 0;       // this warp has the strip from its first block on
        for (int p = lo; p < hi; p += U) {
            copy_wait<kStages - 2>();
            __syncwarp();          // the scales are there for every lane, and the last stage has been read
            load(slot == 0 ? kStages - 1 : slot - 1);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u > 0 && p + u >= hi) break;
                block_product<T, G, NT>(sum, fifo + slot * kStageBytes + u * S::kBytes, x, b * (2 * kBlock), lane);
                if (++b == nb) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        for (int k = 0; k < 4; ++k) sum[n][k] *= Codes<T>::kUp;
                        if (whole && a.cluster == 1) put_strip<T>(a, f + strip, lane, n, sum[n]);
                        else
                            (whole ? full + strip * kPart : parts + warp * kPart)[n * 32 + lane] =
                                make_float4(sum[n][0], sum[n][1], sum[n][2], sum[n][3]);
                        sum[n][0] = sum[n][1] = sum[n][2] = sum[n][3] = 0.0f;
                    }
                    b = 0;
                    ++strip;
                    whole = true;
                }
            }
            slot = slot + 1 == kStages ? 0 : slot + 1;
        }
        copy_wait<0>();
        __syncwarp();
        if (b != 0)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                for (int k = 0; k < 4; ++k) sum[n][k] *= Codes<T>::kUp;
                last[n * 32 + lane] = make_float4(sum[n][0], sum[n][1], sum[n][2], sum[n][3]);
            }
        __syncthreads();
        for (int i = threadIdx.x; i < strips * kPart; i += kProdThreads) {
            const int k = i / kPart, first = share_of(k * nb, total), end = share_of(k * nb + nb - 1, total);
            if (first == end) continue;
            float v[4] = {};
            for (int w = first; w <= end; ++w) {
                const float4 r = (w < end ? reinterpret_cast<const float4*>(smem + w * (ST * S::kBytes)) : parts + w * kPart)[i % kPart];
                v[0] += r.x, v[1] += r.y, v[2] += r.z, v[3] += r.w;
            }
            if (a.cluster == 1) put_strip<T>(a, f + k, i & 31, i / 32 % NT, v);
            else full[i] = make_float4(v[0], v[1], v[2], v[3]);
        }
        if (a.cluster == 1) continue;      // (one batch)
        cluster_sync();
        for (int i = rank * kProdThreads + threadIdx.x; i < strips * kPart; i += a.cluster * kProdThreads) {
            float v[4] = {};
            for (int r = 0; r < a.cluster; ++r) {
                uint32_t at;
                float4 q;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_at(full + i)), "r"(r));
                asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
                             : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "r"(at) : "memory");
                v[0] += q.x, v[1] += q.y, v[2] += q.z, v[3] += q.w;
            }
            put_strip<T>(a, f + i / kPart, i & 31, i / 32 % NT, v);
        }
        // The sums have been read, here and by the cluster's other blocks, before
        // they are overwritten or this block ends.
        cluster_sync();
    }
}

// ---------------------------------------------------------------------------
// Mixture of experts
// ---------------------------------------------------------------------------

constexpr int kMaxExperts = 512, kMaxTopK = 16, kMaxHidden = 32768, kMaxInter = 16384;
constexpr int kMaxPairs = RR_MOE_MAX_TOKENS * kMaxTopK;
constexpr int kJoinBytes = 2 * kWarps * 2 * 512;   // shared memory of the warps' parts of strips
constexpr int kSmem = 227 * 1024;

// The workspace's control block.
struct MoeControl {
    uint32_t error;        // a wait ran out: calls do nothing until rr_moe_check
    uint32_t barrier[4];   // blocks that have arrived
    uint32_t left;         // blocks that have finished
};

struct MoeArgs {
    const uint16_t* router;
    const char *w13, *w2;
    const uint16_t* x;
    int64_t ldx, ldo;
    uint16_t* out;
    int32_t* ids;
    float* weights;
    MoeControl* control;
    float* logits;     // [tokens, n_experts]
    float* h;          // [pairs, h_ld]: silu(gate) * up, by expert, then token
    float* y;          // [pairs, y_ld]: each pair's product with w2
    uint32_t* h_top;   // [pairs]: the largest finite |h|, as bits (float16)
    int32_t h_ld, y_ld;        // multiples of 4
    int32_t tokens, n_experts, first, n_local, top_k, norm, hidden, inter;
    int32_t x_vec, r_vec;      // rows of x, of the router can be read 16 bytes at a time
    int32_t cap;               // tokens of a pass: at most 16
    int32_t x_pitch, h_pitch;  // bytes between tokens in shared memory
    int32_t x_rows, h_rows;    // tokens' rows of x, of h that fit there
    int32_t all_x;             // shared memory holds every token's row
    int32_t fold;              // rows of h and one of zeros, where shared memory holds all; else 0
    int32_t one;               // the grid is one cluster of as many blocks, or 0
    int64_t m13_bytes, m2_bytes;       // of an expert's matrices
    int32_t* far_chosen;       // [tokens * top_k]: choices made by other blocks
    float* far_c;
};

// A warp's stages of weights.  W: 0 for 16-bit matrices whose rows start at 16
// bytes, 1 for others, or the group of packed ones.
//   0: a block is 64 columns; a lane copies the 16-byte runs that it reads.
//   1: the 9 runs of 16 bytes that hold a row's 64 columns, wherever they start;
//      rows 144 bytes apart.  Lanes read the 20 bytes that theirs are in.
//   Copies end at a row's end, and zeros follow.
template <int W>
struct Weights {
    static constexpr int kCols = 64, kBytes = W ? 16 * 144 : 16 * 128, kStages = 3;
    const char *lo, *hi;      // the block's first column in rows g, g + 8 (null: no such row)
    int32_t left;             // bytes from there to the rows' ends
    __device__ __forceinline__ void seek(const char* base, int64_t mat, const Packed& m, int64_t strip, int b,
                                         int lane) {
        const int64_t l = m.row(strip, lane >> 2), h = m.row(strip, 8 + (lane >> 2));
        const char* const at = base + mat * m.matrix_bytes + b * (2 * kCols);
        lo = l < 0 ? nullptr : at + l * m.cols * 2;
        hi = h < 0 ? nullptr : at + h * m.cols * 2;
        left = int32_t(2 * (m.cols - int64_t(b) * kCols));
    }
    __device__ __forceinline__ void skip(int blocks) {
        if (lo) lo += blocks * (2 * kCols);
        if (hi) hi += blocks * (2 * kCols);
        left -= blocks * (2 * kCols);
    }
    __device__ __forceinline__ void load(uint32_t to, const char* base, int lane) const {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char* const row = half ? hi : lo;
            const int bytes = row ? left : 0;
            if (W == 0) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int at = 64 * j + 16 * t;
                    copy_async_cut(to + 1024 * half + 512 * j + 16 * lane, at < bytes ? row + at : base,
                                   max(0, min(16, bytes - at)));
                }
            } else {
                const int shift = int(reinterpret_cast<uintptr_t>(row) & 15);
#pragma unroll
                for (int j = 0; j < 3; ++j) {
                    const int at = 16 * (4 * j + t) - shift;
                    if (j < 2 || t == 0)
                        copy_async_cut(to + 144 * (8 * half + g) + 64 * j + 16 * t, at < bytes ? row + at : base,
                                       max(0, min(16, bytes - at)));
                }
            }
        }
    }
    // The 4 words of this lane's columns 32 j + 8 t + 0..7 of row g + 8 half.
    static __device__ __forceinline__ uint4 read(const char* stage, int half, int j, int shift, int lane) {
        if (W == 0) return *reinterpret_cast<const uint4*>(stage + 1024 * half + 512 * j + 16 * lane);
        const uint32_t* const p = reinterpret_cast<const uint32_t*>(
            stage + 144 * (8 * half + (lane >> 2)) + 64 * j + 16 * (lane & 3) + (shift & 12));
        const uint32_t w0 = p[0], w1 = p[1], w2 = p[2], w3 = p[3], w4 = shift & 2 ? p[4] : 0;
        const uint32_t pick = shift & 2 ? 0x5432 : 0x3210;
        return make_uint4(__byte_perm(w0, w1, pick), __byte_perm(w1, w2, pick), __byte_perm(w2, w3, pick),
                          __byte_perm(w3, w4, pick));
    }
};

template <int G>
struct PackedWeights {
    using S = Block<G>;
    static constexpr int kCols = kBlock, kBytes = S::kBytes, kStages = 6;
    const char* from;
    __device__ __forceinline__ void seek(const char* base, int64_t mat, const Packed& m, int64_t strip, int b,
                                         int lane) {
        from = base + mat * m.matrix_bytes + (strip * m.blocks + b) * kBytes + 16 * lane;
    }
    __device__ __forceinline__ void skip(int blocks) { from += int64_t(blocks) * kBytes; }
    __device__ __forceinline__ void load(uint32_t to, const char*, int lane) const {
        S::copy(to, from, lane);
    }
};
template <> struct Weights<32> : PackedWeights<32> {};
template <> struct Weights<64> : PackedWeights<64> {};
template <> struct Weights<128> : PackedWeights<128> {};

// sum += W x over one block.  Of 16-bit weights, a block's 64 columns are summed from
// zero and then added: a matrix instruction cuts its sum off, towards zero, and a chain
// of them over a row drifts by 2^-24 a step (2048 x 768, 32 tokens: 0.15% of the outputs
// one step off so, 0.015% as it is, 0.026% with float32 sums elsewhere; 64 tokens 222 ->
// 226 us, one token 30.9 -> 31.9).  low: of the second and third parts of an
// element, whose sums, 2^-8 of the others, then lose nothing beside them.  Where the
// first parts' sum is infinite or NaN it is the result: a part of zero times an infinite
// weight would make NaN of what is infinite (join_low).
template <class T, int W, int NT, Form FORM>
__device__ __forceinline__ void moe_block(float (&sum)[NT][4], float (&low)[NT][4], const char* stage,
                                          const char* const (&x)[NT], int apart, int at, int shift_lo, int shift_hi,
                                          int lane, bool inf) {
    if constexpr (W >= 32) {
        block_product<T, W, NT, FORM>(sum, stage, x, at, lane, apart, inf);
    } else {
        float part[NT][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint4 l = Weights<W>::read(stage, 0, j, shift_lo, lane);
            const uint4 h = Weights<W>::read(stage, 1, j, shift_hi, lane);
            const auto add = [&](int n, int p, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
                if (p == 0 && j == 0) mma_first<T>(part[n], l.x, h.x, l.y, h.y, x0, x1);
                else mma<T>(p ? low[n] : part[n], l.x, h.x, l.y, h.y, x0, x1);
                mma<T>(p ? low[n] : part[n], l.z, h.z, l.w, h.w, x2, x3);
            };
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (FORM == kFloats) {
                    const Parts v(x[n] + at + 64 * j, apart, inf);
#pragma unroll
                    for (int p = 0; p < 3; ++p) add(n, p, v.w[p][0], v.w[p][1], v.w[p][2], v.w[p][3]);
                } else {
#pragma unroll
                    for (int p = 0; p < FORM; ++p) {
                        const uint4 v = *reinterpret_cast<const uint4*>(x[n] + p * apart + at + 64 * j);
                        add(n, p, v.x, v.y, v.z, v.w);
                    }
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[n][k] += part[n][k];
    }
}

__device__ __forceinline__ float join_low(float sum, float low) { return fabsf(sum) < INFINITY ? sum + low : sum; }

// Four elements of h from column c on to the planes of their row.
template <class T, Form H>
__device__ __forceinline__ void put_hidden(char* row, int apart, int c, float (&v)[4]) {
    if (H == kFloats) {
        *reinterpret_cast<float4*>(row + (c & 4 ? apart : 0) + 2 * (c & ~7)) = make_float4(v[0], v[1], v[2], v[3]);
        return;
    }
#pragma unroll
    for (int p = 0; p < planes_of(H); ++p) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            w[q] = H == kThirds ? __float_as_uint(v[q]) >> 16 : T::round(v[q]);
            v[q] -= T::widen(uint16_t(w[q]));
            if (!isfinite(v[q])) v[q] = 0.0f;      // (an infinite element has no rest)
        }
        *reinterpret_cast<uint2*>(row + p * apart + 2 * c) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
}

__device__ __forceinline__ float warp_sum(float v) {
    for (int o = 16; o; o /= 2) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// Descending order of logits as unsigned integers: NaN first, +0 and -0 alike; 0
// is below all of them.
__device__ __forceinline__ uint32_t rank_key(float l) {
    if (isnan(l)) return ~0u;
    const uint32_t b = __float_as_uint(l + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// What every block works out for itself from the logits.
struct MoeTables {
    uint32_t mask[2][kMaxExperts];     // the tokens of a local expert
    float c[kMaxPairs];                // by token and rank
    float pair_c[8 * kMaxTopK];        // by pair (of up to 8 tokens)
    int16_t chosen[kMaxPairs];
    uint16_t first[kMaxExperts];       // a local expert's first pair
    uint16_t pass_expert[kMaxPairs], pass_first[kMaxPairs];
    uint8_t pass_count[kMaxPairs];
    uint8_t token[kMaxPairs];          // of a pair
    float scale[kMaxPairs];            // of h (float16): by pair, or by token
    uint32_t most;                     // tokens of the largest pass
    uint32_t scan[kWarps];
    uint32_t total;                    // pairs << 16 | passes
    uint32_t stop;
    uint32_t inf;                      // an element of h here is not finite
};

// The pair of a local expert and one of its tokens.
__device__ __forceinline__ int pair_of(const MoeTables& tab, int local, int t) {
    const uint32_t m0 = tab.mask[0][local], m1 = tab.mask[1][local];
    return tab.first[local] + (t < 32 ? __popc(m0 & ((1u << t) - 1)) : __popc(m0) + __popc(m1 & ((1u << (t - 32)) - 1)));
}

// Logits of 16 tokens from t0 and 8 experts from e0: a block's warps share the
// columns, tokens are operand A, router rows operand B.  red: 8 KB.
template <class T>
__device__ __forceinline__ void logit_item(const MoeArgs& a, int e0, int t0, float4* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint16_t* const r = a.router + int64_t(min(e0 + g, a.n_experts - 1)) * a.hidden + 8 * t;
    const uint16_t* const lo = a.x + min(t0 + g, a.tokens - 1) * a.ldx + 8 * t;
    const uint16_t* const hi = a.x + min(t0 + 8 + g, a.tokens - 1) * a.ldx + 8 * t;
    float sum[4] = {};
    if (a.x_vec && a.r_vec) {
#pragma unroll 4
        for (int k = 32 * warp; k < a.hidden; k += 32 * kWarps) {
            uint4 w = make_uint4(0, 0, 0, 0), u = w, v = w;
            if (k + 8 * t < a.hidden) {
                w = *reinterpret_cast<const uint4*>(r + k);
                u = *reinterpret_cast<const uint4*>(lo + k);
                if (t0 + 8 < a.tokens) v = *reinterpret_cast<const uint4*>(hi + k);
            }
            mma<T>(sum, u.x, v.x, u.y, v.y, w.x, w.y);
            mma<T>(sum, u.z, v.z, u.w, v.w, w.z, w.w);
        }
    } else {
        const uint16_t* const x_end = a.x + (a.tokens - 1) * a.ldx + a.hidden;
        const uint16_t* const r_end = a.router + int64_t(a.n_experts) * a.hidden;
#pragma unroll 2
        for (int k = 32 * warp; k < a.hidden; k += 32 * kWarps) {
            const int left = a.hidden - k - 8 * t;
            const uint4 w = load_any(r + k, left, a.router, r_end), u = load_any(lo + k, left, a.x, x_end);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (t0 + 8 < a.tokens) v = load_any(hi + k, left, a.x, x_end);
            mma<T>(sum, u.x, v.x, u.y, v.y, w.x, w.y);
            mma<T>(sum, u.z, v.z, u.w, v.w, w.z, w.w);
        }
    }
    red[threadIdx.x] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    if (threadIdx.x < 128) {
        const int i = threadIdx.x;
        float v = 0.0f;
#pragma unroll 4
        for (int q = 0; q < kWarps; ++q) v += reinterpret_cast<const float*>(red)[128 * q + i];
        const int tok = t0 + i / 16 + 8 * (i >> 1 & 1), e = e0 + 2 * (i / 4 % 4) + (i & 1);
        if (tok < a.tokens && e < a.n_experts) __stcg(a.logits + tok * a.n_experts + e, v);
    }
    __syncthreads();
}

// Notes choice i, of token t.
__device__ __forceinline__ void take_choice(const MoeArgs& a, MoeTables& tab, int i, int t, int id, float c) {
    const int local = id - a.first;
    tab.chosen[i] = int16_t(id);
    tab.c[i] = c;
    if (local >= 0 && local < a.n_local) atomicOr(&tab.mask[t >> 5][local], 1u << (t & 31));
    if (blockIdx.x == 0) {
        if (a.ids) a.ids[i] = id;
        if (a.weights) a.weights[i] = c;
    }
}

// One warp: the softmax and the top_k experts of token t.  kEach: experts of a
// lane, every 32nd.  far: for every block to read, else for this one.
template <int kEach>
__device__ __forceinline__ void choose(const MoeArgs& a, MoeTables& tab, int t, int lane, bool far) {
    const float* const row = a.logits + t * a.n_experts;
    float l[kEach];
    uint32_t key[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) l[i] = 32 * i + lane < a.n_experts ? __ldcg(row + 32 * i + lane) : 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) key[i] = 32 * i + lane < a.n_experts ? rank_key(l[i]) : 0;
    float top = 0.0f, mine = 0.0f;
    int my_id = 0;
    for (int j = 0; j < a.top_k; ++j) {
        // The largest key; of equal ones, the lowest index.
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) best = max(best, key[i]);
        best = __reduce_max_sync(~0u, best);
        uint32_t at = ~0u;
        float lv = 0.0f;
#pragma unroll
        for (int i = kEach - 1; i >= 0; --i)
            if (key[i] == best) at = 32 * i + lane, lv = l[i];
        const uint32_t e = __reduce_min_sync(~0u, at);
        lv = __shfl_sync(~0u, lv, e & 31);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (32 * i + lane == int(e)) key[i] = 0;
        if (j == 0) top = lv;       // (NaN where there is one: so are the weights)
        if (lane == j) mine = lv, my_id = int(e);
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (32 * i + lane < a.n_experts) sum += expf(l[i] - top);
    sum = warp_sum(sum);
    float p = lane < a.top_k ? expf(mine - top) / sum : 0.0f;
    if (a.norm) p /= warp_sum(p);
    if (lane < a.top_k) {
        const int i = t * a.top_k + lane;
        if (far) {
            __stcg(a.far_chosen + i, my_id);
            __stcg(a.far_c + i, p);
        } else {
            take_choice(a, tab, i, t, my_id, p);
        }
    }
}

// A barrier of all blocks, in two halves.  What a block wrote before it arrived is
// there for every block that has waited.  Within one cluster it is the hardware's;
// else the wait is bounded: it runs out after about two seconds, which marks the
// workspace.  False then, and where an earlier call's did.
__device__ __forceinline__ void grid_arrive(const MoeArgs& a, int which) {
    if (a.one) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        return;
    }
    __syncthreads();
    if (threadIdx.x == 0)
        asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(&a.control->barrier[which]) : "memory");
}
__device__ __forceinline__ bool grid_wait(const MoeArgs& a, MoeTables& tab, int which) {
    if (a.one) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (tab.stop) copy_wait<0>();
        return tab.stop == 0;
    }
    if (threadIdx.x == 0) {
        uint32_t seen = 0;
        long long since = 0;
        for (;;) {
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(&a.control->barrier[which]) : "memory");
            if (seen >= gridDim.x) {
                // A call whose wait ran out may have left counts behind.
                asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(&a.control->error) : "memory");
                tab.stop = seen;
                break;
            }
            long long now;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
            if (since == 0) since = now;
            if (now - since > 2000000000ll) {
                atomicExch(&a.control->error, 1u);
                tab.stop = 1;
                break;
            }
        }
    }
    __syncthreads();
    if (tab.stop) copy_wait<0>();
    return tab.stop == 0;
}

// One of the two products: a run of (pass, strip) items per block.
struct MoePhase {
    const char* base;
    Packed m;
    int blocks;            // of a strip
    int f0, n;             // this block's items: pass f / strips, strip f % strips
    int tiles;             // groups of 8 tokens of the largest pass
    int strips;
    uint32_t inverse;      // 2^32 / strips, rounded up: exact for f * strips <= 2^32
    __device__ __forceinline__ int pass(int f) const {
        return strips == 1 ? f : int(__umulhi(uint32_t(f), inverse));
    }
    int window;            // passes whose tokens are in shared memory at once
    // The end of the item's window: every `window` passes from the first one's.
    __device__ __forceinline__ int window_end(int i) const {
        const int first = pass(f0), w = (pass(f0 + i) - first) / window + 1;
        return min(n, (first + w * window) * strips - f0);
    }
};

// The order in which a warp takes a phase's blocks of weights: of each window's
// items, whole rounds of 16 one item a warp (adjacent warps then read adjacent
// rows: 120 us for gate and up of 64 tokens, against 131 with a contiguous share for
// each warp), and of the rest an even share of their blocks.
template <int W>
struct Feed {
    Weights<W> w;
    int i, b, left;            // item, block, blocks left in this run
    int rest, end;             // where the window's rounds and the window end
    __device__ __forceinline__ void aim(const MoePhase& p, const MoeTables& tab, int lane) {
        const int f = p.f0 + i, pass = p.pass(f);
        w.seek(p.base, tab.pass_expert[pass], p.m, f - pass * p.strips, b, lane);
    }
    // This warp's first item from i0 on: i0 begins a window, or is the end of its rounds.
    __device__ __forceinline__ void find(const MoePhase& p, const MoeTables& tab, int i0, int warp, int lane) {
        left = 0;
        while (i0 < p.n) {
            end = p.window_end(i0);
            rest = end - (end - i0) % kWarps;
            if (rest > i0) {
                i = i0 + warp;
                b = 0;
                left = p.blocks;
            } else {
                const int total = (end - i0) * p.blocks, lo = share_from(warp, total);
                left = share_from(warp + 1, total) - lo;
                i = i0 + lo / p.blocks;
                b = lo % p.blocks;
                rest = -1;         // the rest itself
            }
            if (left > 0) {
                aim(p, tab, lane);
                return;
            }
            i0 = end;
        }
    }
    // The next block to a stage; an empty group when there is none.
    __device__ __forceinline__ void load(const MoePhase& p, const MoeTables& tab, uint32_t to, int warp, int lane) {
        if (left > 0) {
            w.load(to, p.base, lane);
            if (--left > 0) {
                if (++b < p.blocks) {
                    w.skip(1);
                } else {
                    b = 0;
                    ++i;
                    aim(p, tab, lane);
                }
            } else if (rest < 0) {
                find(p, tab, end, warp, lane);
            } else if (i + kWarps < rest) {
                i += kWarps;
                b = 0;
                left = p.blocks;
                aim(p, tab, lane);
            } else {
                find(p, tab, rest, warp, lane);
            }
        }
        copy_commit();
    }
    // Starts on a phase: all stages but one, from `slot` on.
    __device__ __forceinline__ void start(const MoePhase& p, const MoeTables& tab, uint32_t fifo, int slot, int warp,
                                          int lane) {
        find(p, tab, 0, warp, lane);
        for (int k = 0; k < Weights<W>::kStages - 1; ++k) {
            load(p, tab, fifo + slot * Weights<W>::kBytes, warp, lane);
            slot = slot + 1 == Weights<W>::kStages ? 0 : slot + 1;
        }
    }
};

// Tokens' rows (16-bit) to shared memory, zero-filled to whole blocks: those of
// pairs first, first + 1, ..., or with all_x simply tokens 0, 1, ...  (Copies are in
// flight when this returns: a group of cp.async.)
__device__ __forceinline__ void stage_tokens(const MoeArgs& a, const MoeTables& tab, char* to, int first, int count,
                                             int cols) {
    if (a.x_vec) {
        for (int i = 0; i < count; ++i) {
            const uint16_t* const row = a.x + (a.all_x ? i : tab.token[first + i]) * a.ldx;
            for (int c = 8 * threadIdx.x; c < cols; c += 8 * kProdThreads) {
                const int left = a.hidden - c;
                copy_async_cut(smem_at(to + i * a.x_pitch + 2 * c), row + (left > 0 ? c : 0),
                               left >= 8 ? 16 : left > 0 ? 2 * left : 0);
            }
        }
    } else {
        const uint16_t* const end = a.x + (a.tokens - 1) * a.ldx + a.hidden;
        const int chunks = cols / 8;
#pragma unroll 4
        for (int k = threadIdx.x; k < count * chunks; k += kProdThreads) {
            const int i = k / chunks, c = 8 * (k % chunks);
            const uint16_t* const row = a.x + (a.all_x ? i : tab.token[first + i]) * a.ldx;
            *reinterpret_cast<uint4*>(to + i * a.x_pitch + 2 * c) = load_any(row + c, a.hidden - c, a.x, end);
        }
    }
    copy_commit();
}

// The power of two that brings a float16 token's largest h to 2^14..2^15.
__device__ __forceinline__ int h_exponent(uint32_t top) {
    return top ? max(-100, min(100, 14 - ilogbf(__uint_as_float(top)))) : 0;
}

// A pass's h, which the first product left in float32.
//   bfloat16: three parts, which hold all of its 24 bits, or float32 as it is where three
//   planes leave a pass too few rows (prepare_moe); a lane then splits what it reads.
//   float16: two parts, v = hi + lo to 2^-22 of v, of v times a power of two that brings
//   the token's largest finite element to 2^14..2^15, so that none overflows and what
//   underflows is below 2^-39 of the largest.
template <class T, Form H>
__device__ __forceinline__ void stage_h(const MoeArgs& a, MoeTables& tab, char* to, int first, int count, int cols) {
    const int chunks = cols / 4;
#pragma unroll 4
    for (int k = threadIdx.x; k < count * chunks; k += kProdThreads) {
        const int i = k / chunks, c = 4 * (k % chunks);
        float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (c < a.inter) f = __ldcg(reinterpret_cast<const float4*>(a.h + int64_t(first + i) * a.h_ld + c));
        float up = 1.0f;
        if (H == kHalves) {
            const int e = h_exponent(__ldcg(a.h_top + first + i));
            up = ldexpf(1.0f, e);
            if (c == 0) tab.scale[first + i] = ldexpf(1.0f, -e);
        }
        float v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = c + q < a.inter ? v[q] * up : 0.0f;
            if (H == kFloats && !isfinite(v[q])) tab.inf = 1;
        }
        put_hidden<T, H>(to + i * a.h_pitch, a.h_rows * a.h_pitch, c, v);
    }
}

// Rows g, g + 8 of tokens 2 t, 2 t + 1 (+ 8 n) of a strip and a pass: the first phase
// ends in silu(gate) * up, the second in the pair's part of the output.
template <class T, int PHASE>
__device__ __forceinline__ void moe_put(const MoeArgs& a, const MoePhase& p, const MoeTables& tab, int f, int lane,
                                        int n, const float (&v)[4]) {
    const int pass = p.pass(f), strip = f - pass * p.strips;
    const int first = tab.pass_first[pass], count = tab.pass_count[pass];
    const int64_t lo = p.m.row(strip, lane >> 2), hi = p.m.row(strip, 8 + (lane >> 2));
    uint32_t top[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int tok = 8 * n + 2 * (lane & 3) + k;
        if (tok >= count || lo < 0) continue;
        if (PHASE == 0) {
            const float h = silu(v[k]) * v[2 + k];
            __stcg(a.h + int64_t(first + tok) * a.h_ld + lo, h);
            top[k] = fabsf(h) < INFINITY ? __float_as_uint(fabsf(h)) : 0;
        } else {
            const float s = std::is_same<T, F16>::value ? tab.scale[first + tok] : 1.0f;
            float* const y = a.y + int64_t(first + tok) * a.y_ld;
            __stcg(y + lo, v[k] * s);
            if (hi >= 0) __stcg(y + hi, v[2 + k] * s);
        }
    }
    if (PHASE == 0 && std::is_same<T, F16>::value)
#pragma unroll
        for (int k = 0; k < 2; ++k) {      // of the strip's rows, one lane each
            const int tok = 8 * n + 2 * (lane & 3) + k;
            for (int o = 4; o < 32; o *= 2) top[k] = max(top[k], __shfl_xor_sync(~0u, top[k], o));
            if (lane < 4 && tok < count && top[k]) atomicMax(a.h_top + first + tok, top[k]);
        }
}

// Blocks [b, stop) of item f by one warp: its sums go out where `whole` says that the
// warp has the item from its first block on and this is its last, else to `first`
// (the item ends here) or `last`.  NT: groups of 8 tokens.
template <class T, int W, Form H, int PHASE, int NT>
__device__ __forceinline__ void moe_item(const MoeArgs& a, const MoePhase& p, const MoeTables& tab, Feed<W>& feed,
                                         char* fifo, int& slot, const char* region, float4* firsts, float4* lasts,
                                         int base, int f, int b, int stop, bool whole) {
    constexpr Form kForm = PHASE == 0 ? kWhole : H;
    constexpr int kStages = Weights<W>::kStages, kBytes = Weights<W>::kBytes;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int pitch = PHASE == 0 ? a.x_pitch : a.h_pitch, apart = a.h_rows * a.h_pitch;
    const int pass = p.pass(f), first = tab.pass_first[pass], count = tab.pass_count[pass];
    const uint32_t fifo_at = smem_at(fifo);
    const char* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int pair = first + min(8 * n + g, count - 1);
        x[n] = region + (PHASE == 0 && a.all_x ? tab.token[pair] : pair - base) * pitch + 16 * t;
    }
    int shift_lo = 0, shift_hi = 0;
    if constexpr (W == 1) {
        Weights<1> w;
        w.seek(p.base, tab.pass_expert[pass], p.m, f - pass * p.strips, 0, lane);
        shift_lo = int(reinterpret_cast<uintptr_t>(w.lo) & 15);
        shift_hi = int(reinterpret_cast<uintptr_t>(w.hi) & 15);
    }
    const bool inf = kForm == kFloats && W >= 32 && tab.inf;
    float sum[NT][4] = {}, low[NT][4] = {};
    for (; b < stop; ++b) {
        copy_wait<kStages - 2>();
        __syncwarp();      // what lanes share is there, and the last stage has been read
        feed.load(p, tab, fifo_at + (slot == 0 ? kStages - 1 : slot - 1) * kBytes, warp, lane);
        moe_block<T, W, NT, kForm>(sum, low, fifo + slot * kBytes, x, apart, b * (2 * Weights<W>::kCols), shift_lo,
                                   shift_hi, lane, inf);
        slot = slot + 1 == kStages ? 0 : slot + 1;
    }
    const bool ends = stop == p.blocks;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
    #pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (W >= 32) sum[n][k] *= Codes<T>::kUp;
            else if (kForm != kWhole) sum[n][k] = join_low(sum[n][k], low[n][k]);
        }
        if (ends && whole) moe_put<T, PHASE>(a, p, tab, f, lane, n, sum[n]);
        else (ends ? firsts : lasts)[(warp * 2 + n) * 32 + lane] = make_float4(sum[n][0], sum[n][1], sum[n][2], sum[n][3]);
    }
}

// A window's items [i0, end), whose tokens are in shared memory from pair `base` on, in
// the order of Feed.
template <class T, int W, Form H, int PHASE>
__device__ __forceinline__ void moe_window(const MoeArgs& a, const MoePhase& p, const MoeTables& tab, Feed<W>& feed,
                                           char* fifo, int& slot, const char* region, float4* parts, int base, int i0,
                                           int end) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float4* const firsts = parts;                          // [warp][tile][lane]
    float4* const lasts = parts + kWarps * 2 * 32;
    const auto item = [&](int f, int b, int stop, bool whole) {
        if (tab.pass_count[p.pass(f)] <= 8)
            moe_item<T, W, H, PHASE, 1>(a, p, tab, feed, fifo, slot, region, firsts, lasts, base, f, b, stop, whole);
        else
            moe_item<T, W, H, PHASE, 2>(a, p, tab, feed, fifo, slot, region, firsts, lasts, base, f, b, stop, whole);
    };
    const int rest = end - (end - i0) % kWarps;
    const int total = (end - rest) * p.blocks, lo = share_from(warp, total), hi = share_from(warp + 1, total);
    // First the rounds' items, then the share of the rest, in one loop (one copy of
    // the code).
    int i = i0 + warp, b = 0, at = lo;
    bool whole = true, round = i < rest;
    if (!round) i = rest + lo / p.blocks, b = lo % p.blocks, whole = b == 0;
    while (round || at < hi) {
        const int stop = round ? p.blocks : min(p.blocks, b + hi - at);
        item(p.f0 + i, b, stop, whole);
        if (round) {
            i += kWarps;
            round = i < rest;
            if (!round) i = rest + lo / p.blocks, b = lo % p.blocks, whole = b == 0;
        } else {
            at += stop - b;
            b = 0;
            ++i;
            whole = true;
        }
    }
    if (total == 0) return;
    i0 = rest;
    b = lo % p.blocks;
    if (lo == hi && b != 0) {          // no share, within an item that others have
        lasts[(warp * 2) * 32 + lane] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        lasts[(warp * 2 + 1) * 32 + lane] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    __syncthreads();
    // Items that several warps have: at most one begins in each warp's share.
    for (int k = threadIdx.x; k < kWarps * p.tiles * 32; k += kProdThreads) {
        const int w = k / (p.tiles * 32), n = k / 32 % p.tiles, ln = k & 31;
        const int wlo = share_from(w, total), whi = share_from(w + 1, total);
        if (wlo == whi) continue;
        const int item = (whi - 1) / p.blocks;             // the last one of this warp
        const int from = item * p.blocks, to = from + p.blocks;
        if (from < wlo || to <= whi) continue;             // begun before, or ended here
        if (8 * n >= tab.pass_count[p.pass(p.f0 + i0 + item)]) continue;
        const int last = share_of(to - 1, total);
        float v[4] = {};
        for (int q = w; q <= last; ++q) {
            const float4 r = (q < last ? lasts : firsts)[(q * 2 + n) * 32 + ln];
            v[0] += r.x, v[1] += r.y, v[2] += r.z, v[3] += r.w;
        }
        moe_put<T, PHASE>(a, p, tab, p.f0 + i0 + item, ln, n, v);
    }
}

// Tokens of as many passes as fit are staged at once, so that warps go from one
// pass to the next without meeting.
template <class T, int W, Form H, int PHASE>
__device__ __forceinline__ void moe_phase(const MoeArgs& a, const MoePhase* ph, MoeTables& tab, Feed<W>& feed,
                                          char* fifo, int& slot, char* region, float4* parts) {
    const MoePhase& p = ph[PHASE];
    for (int i0 = 0; i0 < p.n;) {
        const int end = p.window_end(i0), from = p.pass(p.f0 + i0), to = p.pass(p.f0 + end - 1);
        const int base = tab.pass_first[from], pairs = tab.pass_first[to] + tab.pass_count[to] - base;
        if (!(PHASE == 0 && a.all_x)) {
            __syncthreads();
            if (PHASE == 0) stage_tokens(a, tab, region, base, pairs, p.blocks * Weights<W>::kCols);
            else stage_h<T, H>(a, tab, region, base, pairs, p.blocks * Weights<W>::kCols);
            copy_wait<0>();
            __syncthreads();
        }
        moe_window<T, W, H, PHASE>(a, p, tab, feed, fifo, slot, region, parts, base, i0, end);
        i0 = end;
    }
}

// The second phase for few tokens, whose every h fits a block's shared memory: an
// item is a strip of the output over all chosen experts, whose blocks of weights the
// warps share evenly, and the block joins the warps' sums.  No pair's part goes
// through memory, and no barrier follows.
template <int W>
struct FoldFeed {
    Weights<W> w;
    int strip, end, pass, b, left;
    __device__ __forceinline__ void start(const MoePhase& p, const MoeTables& tab, int passes, int warp, int lane) {
        const int total = passes * p.blocks, lo = share_from(warp, total);
        left = share_from(warp + 1, total) - lo;
        if (left == 0) strip = end;
        if (strip >= end) return;
        pass = lo / p.blocks;
        b = lo % p.blocks;
        w.seek(p.base, tab.pass_expert[pass], p.m, strip, b, lane);
    }
    __device__ __forceinline__ void load(const MoePhase& p, const MoeTables& tab, int passes, uint32_t to, int warp,
                                         int lane) {
        if (strip < end) {
            w.load(to, p.base, lane);
            if (--left == 0) {
                ++strip;
                start(p, tab, passes, warp, lane);
            } else if (++b < p.blocks) {
                w.skip(1);
            } else {
                b = 0;
                w.seek(p.base, tab.pass_expert[++pass], p.m, strip, 0, lane);
            }
        }
        copy_commit();
    }
};

template <class T, int W, Form H>
__device__ __forceinline__ void stage_fold(const MoeArgs& a, MoeTables& tab, char* region, int pairs, int cols) {
    const bool half = std::is_same<T, F16>::value;
    if (half) {
        // One power of two for all of a token's parts of the sum.
        if (threadIdx.x < a.tokens) {
            float top = 0.0f;
            for (int j = 0; j < a.top_k; ++j) {
                const int k = threadIdx.x * a.top_k + j, local = tab.chosen[k] - a.first;
                if (local < 0 || local >= a.n_local) continue;
                const float v = tab.c[k] * __uint_as_float(__ldcg(a.h_top + pair_of(tab, local, threadIdx.x)));
                if (v < INFINITY) top = fmaxf(top, v);
            }
            const int e = h_exponent(__float_as_uint(top));
            tab.scale[threadIdx.x] = ldexpf(1.0f, -e);
            tab.scale[8 + threadIdx.x] = ldexpf(1.0f, e);
        }
        __syncthreads();
    }
    const int chunks = cols / 4, apart = a.fold * a.h_pitch;
#pragma unroll 4
    for (int k = threadIdx.x; k < (pairs + 1) * chunks; k += kProdThreads) {
        const int i = k / chunks, c = 4 * (k - i * chunks);
        float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float up = 0.0f;
        if (i < pairs) {
            if (c < a.inter) f = __ldcg(reinterpret_cast<const float4*>(a.h + int64_t(i) * a.h_ld + c));
            up = tab.pair_c[i];
            if (half) up *= tab.scale[8 + tab.token[i]];
        }
        float v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = i < pairs && c + q < a.inter ? v[q] * up : 0.0f;
            if (H == kFloats && !isfinite(v[q])) tab.inf = 1;
        }
        // The row of zeros that absent tokens read is the last.
        put_hidden<T, H>(region + (i < pairs ? i : a.fold - 1) * a.h_pitch, apart, c, v);
    }
}

template <class T, int W, Form H>
__device__ __forceinline__ void moe_fold(const MoeArgs& a, const MoePhase& p, MoeTables& tab, FoldFeed<W>& feed,
                                         char* fifo, int& slot, const char* region, float4* red, int passes) {
    constexpr int kStages = Weights<W>::kStages, kBytes = Weights<W>::kBytes;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int apart = a.fold * a.h_pitch;
    const bool inf = H == kFloats && W >= 32 && tab.inf;
    const uint32_t fifo_at = smem_at(fifo);
    const int total = passes * p.blocks, lo = share_from(warp, total), hi = share_from(warp + 1, total);
    for (int strip = p.f0; strip < p.f0 + p.n; ++strip) {
        float sum[4] = {}, low_sum[4] = {};
        int pass = lo / p.blocks, b = lo % p.blocks;
        for (int at = lo; at < hi; ++pass, b = 0) {
            const int e = tab.pass_expert[pass], stop = min(p.blocks, b + hi - at);
            const uint32_t mask = tab.mask[0][e];
            const int row = mask >> g & 1 ? tab.first[e] + __popc(mask & ((1u << g) - 1)) : a.fold - 1;
            const char* const x[1] = {region + row * a.h_pitch + 16 * t};
            int shift_lo = 0, shift_hi = 0;
            if constexpr (W == 1) {
                Weights<1> w;
                w.seek(p.base, e, p.m, strip, 0, lane);
                shift_lo = int(reinterpret_cast<uintptr_t>(w.lo) & 15);
                shift_hi = int(reinterpret_cast<uintptr_t>(w.hi) & 15);
            }
            float part[1][4] = {}, low[1][4] = {};
            at += stop - b;
            for (; b < stop; ++b) {
                copy_wait<kStages - 2>();
                __syncwarp();
                feed.load(p, tab, passes, fifo_at + (slot == 0 ? kStages - 1 : slot - 1) * kBytes, warp, lane);
                moe_block<T, W, 1, H>(part, low, fifo + slot * kBytes, x, apart, b * (2 * Weights<W>::kCols), shift_lo,
                                      shift_hi, lane, inf);
                slot = slot + 1 == kStages ? 0 : slot + 1;
            }
            // Only of tokens that chose the expert: zeros times its weights are not zero
            // where these are infinite or NaN.
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (mask >> (2 * t + (k & 1)) & 1) {
                    sum[k] += part[0][k];
                    if (W < 32) low_sum[k] += low[0][k];
                }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] = W >= 32 ? sum[k] * Codes<T>::kUp : join_low(sum[k], low_sum[k]);
        red[threadIdx.x] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        __syncthreads();
        if (threadIdx.x < 128) {
            const int i = threadIdx.x, tok = 2 * (i / 4 % 4) + (i & 1);
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < kWarps; ++q) v += reinterpret_cast<const float*>(red)[128 * q + i];
            const int64_t n = p.m.row(strip, i / 16 + 8 * (i >> 1 & 1));
            if (tok < a.tokens && n >= 0) {
                if (std::is_same<T, F16>::value) v *= tab.scale[tok];
                a.out[tok * a.ldo + n] = T::round(v);
            }
        }
        __syncthreads();
    }
}

// Items that a block is about to take, to L2: HBM then has work while the blocks
// wait for one another.  (The rows of a strip, and a packed strip, are one run.)
template <int W>
__device__ __forceinline__ void prefetch_item(const MoePhase& p, int expert, int strip) {
    const char* at;
    int64_t bytes;
    if (W >= 32) {
        at = p.base + expert * p.m.matrix_bytes + strip * p.m.blocks * block_bytes(W >= 32 ? W : 128);
        bytes = p.m.blocks * block_bytes(W >= 32 ? W : 128);
    } else {
        at = p.base + expert * p.m.matrix_bytes + int64_t(strip) * kStrip * p.m.cols * 2;
        bytes = min(int64_t(kStrip), p.m.rows - int64_t(strip) * kStrip) * p.m.cols * 2;
    }
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(at), "r"(uint32_t(bytes)) : "memory");
}

// The last block to finish leaves the counters at zero for the next call.
__device__ __forceinline__ void finish(const MoeArgs& a) {
    if (a.one) return;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&a.control->left, 1u) == gridDim.x - 1) {
            for (int i = 0; i < 4; ++i) a.control->barrier[i] = 0;
            a.control->left = 0;
        }
    }
}

constexpr int kPrefetch = 8;       // strips of the second phase that a block asks for ahead

// The whole layer in one cooperative launch, one block per SM (a small layer: in one
// cluster):
//   logits, a block per 8 experts and 16 tokens            | barrier
//   softmax and choice (over 16 tokens: shared out | barrier), every expert's tokens
//   gate and up of every chosen expert, silu               | barrier
//   down, and for few tokens the weighted sum at once; else | barrier
//   each token's weighted sum
// Bound by HBM where there is much to read (Qwen3-30B-A3B: 64 tokens 1.2 GB in 226 to 234
// us a call, of which gate and up run at 6.3 TB/s and down at 6.2, its last block 12 us
// behind the mean), by the chain of phases where there is little (one token 76 MB in 32
// us, of which 16.5 us are those two phases, 3 us the barrier between them, 7.5 us the
// phases before and 4 us the gap between two launches).
// Each chosen expert's weights are read once per pass of `cap` of its tokens: 16, or as
// many as have room in shared memory (2048 x 768: 16, 4096 x 1536: 8, 7168 x 2048: 5, 4096
// x 14336: 1), the rest from L2 where it still holds them.  Blocks take equal runs of
// (pass, strip of 16 rows) items; warps stream weights through stages that already
// fill with the next phase's while the blocks wait.
template <class T, int W, Form H>
__global__ void __launch_bounds__(kProdThreads, 1) rr_moe_kernel(const __grid_constant__ MoeArgs a) {
    extern __shared__ __align__(128) char smem[];
    constexpr int kFifo = kWarps * Weights<W>::kStages * Weights<W>::kBytes;
    __shared__ MoePhase ph[2];
    MoeTables& tab = *reinterpret_cast<MoeTables*>(smem + kFifo + kJoinBytes);
    char* const region = smem + kFifo + kJoinBytes + (sizeof(MoeTables) + 127) / 128 * 128;
    float4* const red = reinterpret_cast<float4*>(smem + kFifo);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

    after_previous();
    // An earlier call's mark (a grid's blocks look for it when they wait).
    const uint32_t marked = a.one && threadIdx.x == 0 ? __ldcg(&a.control->error) : 0;
    if (threadIdx.x == 0) tab.most = tab.inf = 0;
    for (int i = threadIdx.x; i < a.n_local; i += kProdThreads) tab.mask[0][i] = tab.mask[1][i] = 0;

    // Logits; then, while other blocks are at theirs, tokens to shared memory where all of them fit.
    {
        const int groups = (a.n_experts + 7) / 8;
        for (int i = blockIdx.x; i < groups * ((a.tokens + 15) / 16); i += gridDim.x)
            logit_item<T>(a, i % groups * 8, i / groups * 16, reinterpret_cast<float4*>(smem));
        if (blockIdx.x == gridDim.x - 1)
            for (int i = threadIdx.x; i < a.tokens * min(a.top_k, a.n_local); i += kProdThreads) a.h_top[i] = 0;
        if (threadIdx.x == 0) tab.stop = marked;
        grid_arrive(a, 0);
        if (a.all_x) {
            constexpr int kCols = Weights<W>::kCols;
            stage_tokens(a, tab, region, 0, a.tokens, (a.hidden + kCols - 1) / kCols * kCols);
        }
    }
    if (!grid_wait(a, tab, 0)) return;

    // Up to a token a warp, every block chooses for itself; more tokens are shared out
    // over the blocks (64 of them took every block 9 us, against 2 and a barrier).
    const bool far = a.tokens > kWarps;
    for (int t = far ? warp * gridDim.x + blockIdx.x : warp; t < a.tokens; t += far ? kWarps * gridDim.x : kWarps) {
        if (a.n_experts <= 128) choose<4>(a, tab, t, lane, far);
        else choose<kMaxExperts / 32>(a, tab, t, lane, far);
    }
    if (far) {
        grid_arrive(a, 3);
        if (!grid_wait(a, tab, 3)) return;
        for (int i = threadIdx.x; i < a.tokens * a.top_k; i += kProdThreads)
            take_choice(a, tab, i, i / a.top_k, __ldcg(a.far_chosen + i), __ldcg(a.far_c + i));
    }
    __syncthreads();
    // Pairs by expert, then token; passes of up to `cap` tokens of one expert.
    {
        const int e = threadIdx.x;
        const uint32_t m0 = e < a.n_local ? tab.mask[0][e] : 0, m1 = e < a.n_local ? tab.mask[1][e] : 0;
        const int count = __popc(m0) + __popc(m1), passes = (count + a.cap - 1) / a.cap;
        const uint32_t most = __reduce_max_sync(~0u, uint32_t(min(count, a.cap)));
        if (lane == 0 && most) atomicMax(&tab.most, most);
        uint32_t v = uint32_t(count) << 16 | uint32_t(passes);
        const uint32_t own = v;
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t u = __shfl_up_sync(~0u, v, o);
            if (lane >= o) v += u;
        }
        if (lane == 31) tab.scan[warp] = v;
        __syncthreads();
        uint32_t warps = lane < kWarps ? tab.scan[lane] : 0;      // every warp adds up the warps' sums
#pragma unroll
        for (int o = 1; o < kWarps; o *= 2) {
            const uint32_t u = __shfl_up_sync(~0u, warps, o);
            if (lane >= o) warps += u;
        }
        const uint32_t before = __shfl_sync(~0u, warps, (warp + 31) & 31);
        v += warp ? before : 0;
        if (threadIdx.x == kProdThreads - 1) tab.total = v;
        v -= own;
        const int pair = int(v >> 16);
        int pass = int(v & 0xFFFF);
        if (e < a.n_local) tab.first[e] = uint16_t(pair);
        for (int q = 0; q < passes; ++q, ++pass) {
            tab.pass_expert[pass] = uint16_t(e);
            tab.pass_first[pass] = uint16_t(pair + q * a.cap);
            tab.pass_count[pass] = uint8_t(min(a.cap, count - q * a.cap));
        }
        __syncthreads();
    }
    if (warp < kWarps - 1) {
        for (int i = threadIdx.x; i < a.tokens * a.top_k; i += kProdThreads - 32) {
            const int local = tab.chosen[i] - a.first, t = i / a.top_k;
            if (local < 0 || local >= a.n_local) continue;
            const int pair = pair_of(tab, local, t);
            tab.token[pair] = uint8_t(t);
            if (a.fold) tab.pair_c[pair] = tab.c[i];
        }
    } else {
        // The phases' items: lane k looks at phase k.
        const int k = lane & 1;
        const int passes = int(tab.total & 0xFFFF);
        const int cols = k ? a.inter : a.hidden, strips = k ? (a.hidden + 15) / 16 : (a.inter + 7) / 8;
        const uint32_t all = k && a.fold ? strips : passes * strips;    // at most 1024 passes of 2048 strips
        const uint32_t grid = gridDim.x;
        // (Products under 2^32 for grids of up to 1024 blocks.)
        const int f0 = int(blockIdx.x * all / grid), n = int((blockIdx.x + 1) * all / grid) - f0;
        if (lane < 2) {
            MoePhase p;
            p.base = k ? a.w2 : a.w13;
            p.m.rows = k ? a.hidden : 2 * a.inter;
            p.m.cols = cols;
            p.m.pair = !k;
            p.m.strips = strips;
            p.m.blocks = (cols + kBlock - 1) / kBlock;
            p.m.matrix_bytes = k ? a.m2_bytes : a.m13_bytes;
            p.blocks = (cols + Weights<W>::kCols - 1) / Weights<W>::kCols;
            p.f0 = f0;
            p.n = n;
            p.tiles = tab.most > 8 ? 2 : 1;
            p.strips = strips;
            p.inverse = uint32_t(0xFFFFFFFFu / uint32_t(strips)) + 1;
            p.window = 2 * kMaxPairs;          // no end within the passes
            if (n > 0 && !(k && a.fold) && !(!k && a.all_x)) {
                // All of the block's passes where their tokens fit, else as many as always do.
                const int rows = k ? a.h_rows : a.x_rows, from = p.pass(f0), to = p.pass(f0 + n - 1);
                if (tab.pass_first[to] + tab.pass_count[to] - tab.pass_first[from] > rows)
                    p.window = max(1, rows / int(tab.most));
            }
            ph[k] = p;
        }
    }
    copy_wait<0>();        // the tokens
    __syncthreads();

    char* const fifo = smem + warp * (Weights<W>::kStages * Weights<W>::kBytes);
    int slot = 0;
    Feed<W> feed;
    feed.start(ph[0], tab, smem_at(fifo), slot, warp, lane);
    moe_phase<T, W, H, 0>(a, ph, tab, feed, fifo, slot, region, red);
    grid_arrive(a, 1);
    const int passes = int(tab.total & 0xFFFF);
    if (a.fold) {
        FoldFeed<W> fold;
        fold.strip = ph[1].f0;
        fold.end = ph[1].f0 + ph[1].n;
        fold.start(ph[1], tab, passes, warp, lane);
        for (int i = 0, to = slot; i < Weights<W>::kStages - 1; ++i) {
            fold.load(ph[1], tab, passes, smem_at(fifo) + to * Weights<W>::kBytes, warp, lane);
            to = to + 1 == Weights<W>::kStages ? 0 : to + 1;
        }
        if (W != 1 && warp == kWarps / 2 && ph[1].n > 0)
            for (int i = lane; i < passes; i += 32) prefetch_item<W>(ph[1], tab.pass_expert[i], ph[1].f0);
        if (!grid_wait(a, tab, 1)) return;
        stage_fold<T, W, H>(a, tab, region, int(tab.total >> 16), ph[1].blocks * Weights<W>::kCols);
        __syncthreads();
        moe_fold<T, W, H>(a, ph[1], tab, fold, fifo, slot, region, red, passes);
        copy_wait<0>();
        finish(a);
        return;
    }
    feed.start(ph[1], tab, smem_at(fifo), slot, warp, lane);
    if (W != 1 && warp == kWarps / 2 && lane < min(ph[1].n, kPrefetch)) {
        const int f = ph[1].f0 + lane, pass = ph[1].pass(f);
        prefetch_item<W>(ph[1], tab.pass_expert[pass], f - pass * ph[1].strips);
    }
    if (!grid_wait(a, tab, 1)) return;
    moe_phase<T, W, H, 1>(a, ph, tab, feed, fifo, slot, region, red);
    copy_wait<0>();
    grid_arrive(a, 2);
    if (!grid_wait(a, tab, 2)) return;

    // A warp takes 128 columns of a token.
    const int parts = (a.hidden + 127) / 128;
    for (int i = warp * gridDim.x + blockIdx.x; i < a.tokens * parts; i += kWarps * gridDim.x) {
        const int t = i / parts, n = i % parts * 128 + 4 * lane;
        float sum[4] = {};
        for (int j0 = 0; j0 < a.top_k; j0 += 8) {
            float4 y[8];
            float c[8];
            bool here[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {      // every load before the first sum
                const int k = t * a.top_k + min(j0 + j, a.top_k - 1), e = tab.chosen[k] - a.first;
                here[j] = j0 + j < a.top_k && e >= 0 && e < a.n_local;
                const int le = here[j] ? e : 0;
                const int pair = pair_of(tab, le, t);
                c[j] = tab.c[k];
                y[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (here[j] && n < a.hidden)
                    y[j] = __ldcg(reinterpret_cast<const float4*>(a.y + int64_t(pair) * a.y_ld + n));
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (here[j]) sum[0] += c[j] * y[j].x, sum[1] += c[j] * y[j].y, sum[2] += c[j] * y[j].z, sum[3] += c[j] * y[j].w;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (n + q < a.hidden) a.out[t * a.ldo + n + q] = T::round(sum[q]);
    }
    finish(a);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

rr_status cuda_fail(cudaError_t e, const char* what) {
    return rr_fail(RR_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

#define RR_CUDA(call)                                   \
    do {                                                \
        cudaError_t e_ = (call);                        \
        if (e_ != cudaSuccess) return cuda_fail(e_, #call); \
    } while (0)

#define RR_TRY(call)                     \
    do {                                 \
        rr_status s_ = (call);           \
        if (s_ != RR_OK) return s_;      \
    } while (0)

// Memory of device `dev`, the current one, `align`ed.
rr_status check_device(int dev, const void* p, size_t align, const char* what) {
    if (!p || (uintptr_t)p % align) return rr_fail(RR_EINVAL, "%s is NULL or not %zu-byte aligned", what, align);
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
        cudaGetLastError();
        return rr_fail(RR_EINVAL, "%s is not memory of this GPU", what);
    }
    if (at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev)) return RR_OK;
    return rr_fail(RR_EINVAL, "%s is not memory of this GPU", what);
}

constexpr int kMaxDevices = 16;

rr_status current_device(int* dev) {
    RR_CUDA(cudaGetDevice(dev));
    if (*dev < 0 || *dev >= kMaxDevices) return rr_fail(RR_EINVAL, "device %d: 0..%d", *dev, kMaxDevices - 1);
    return RR_OK;
}

// Lets a kernel have `smem` bytes of dynamic shared memory, once per kernel and device
// (`done`: its own bits, one a device).
template <class K>
cudaError_t allow_smem(K* kernel, int smem, int dev, std::atomic<uint32_t>* done) {
    if (done->load(std::memory_order_relaxed) >> dev & 1) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) done->fetch_or(1u << dev, std::memory_order_relaxed);
    return e;
}

Packed packed_of(int64_t rows, int64_t cols, int group, int pair) {
    Packed m;
    m.rows = rows;
    m.cols = cols;
    m.strips = pair ? (rows / 2 + 7) / 8 : (rows + 15) / 16;
    m.blocks = (cols + kBlock - 1) / kBlock;
    m.matrix_bytes = m.strips * m.blocks * block_bytes(group ? group : 128);
    m.pair = pair;
    return m;
}

rr_status check_quant(const rr_quant* q) {
    if (!q) return rr_fail(RR_EINVAL, "matrix description is NULL");
    if (q->rows < 1 || q->rows > INT32_MAX || q->cols < 1 || q->cols > kMaxCols)
        return rr_fail(RR_ELAYOUT, "matrix of %lld x %lld: 1..2^31-1 rows and 1..2^18 columns",
                       (long long)q->rows, (long long)q->cols);
    if (q->count < 1 || q->count > 65535) return rr_fail(RR_ELAYOUT, "count %d: 1..65535", q->count);
    if (q->group != 32 && q->group != 64 && q->group != 128)
        return rr_fail(RR_ELAYOUT, "group %d: 32, 64 or 128", q->group);
    if (q->dtype != RR_DST_BF16 && q->dtype != RR_DST_F16)
        return rr_fail(RR_EINVAL, "unknown element type %d", q->dtype);
    if (q->pair != 0 && q->pair != 1) return rr_fail(RR_EINVAL, "pair is 0 or 1, not %d", q->pair);
    if (q->pair && q->rows % 2) return rr_fail(RR_ELAYOUT, "paired rows are an even number, not %lld", (long long)q->rows);
    // The kernels number a stack's blocks in 32 bits; its bytes then fit 64.
    const Packed m = packed_of(q->rows, q->cols, q->group, q->pair);
    if (m.strips * m.blocks * q->count > INT32_MAX)
        return rr_fail(RR_ELAYOUT, "%d matrices of %lld x %lld: at most 2^31 - 1 blocks of 16 x 128", q->count,
                       (long long)q->rows, (long long)q->cols);
    return RR_OK;
}

// Calls f with the element type and the group as template arguments.
template <class F>
rr_status with_group(int dtype, int group, F f) {
    using std::integral_constant;
    if (dtype == RR_DST_F16) {
        if (group == 32) return f(F16{}, integral_constant<int, 32>{});
        if (group == 64) return f(F16{}, integral_constant<int, 64>{});
        if (group == 128) return f(F16{}, integral_constant<int, 128>{});
        return f(F16{}, integral_constant<int, 0>{});
    }
    if (group == 32) return f(BF16{}, integral_constant<int, 32>{});
    if (group == 64) return f(BF16{}, integral_constant<int, 64>{});
    if (group == 128) return f(BF16{}, integral_constant<int, 128>{});
    return f(BF16{}, integral_constant<int, 0>{});
}

rr_status check_moe(const rr_moe_layer* L) {
    if (!L) return rr_fail(RR_EINVAL, "layer description is NULL");
    if (L->n_experts < 1 || L->n_experts > kMaxExperts)
        return rr_fail(RR_ELAYOUT, "%d experts: 1..%d", L->n_experts, kMaxExperts);
    if (L->first_expert < 0 || L->n_local < 1 || L->n_local > L->n_experts || L->first_expert > L->n_experts - L->n_local)
        return rr_fail(RR_ELAYOUT, "experts %d + %d are not within 0..%d", L->first_expert, L->n_local, L->n_experts);
    if (L->top_k < 1 || L->top_k > kMaxTopK || L->top_k > L->n_experts)
        return rr_fail(RR_ELAYOUT, "top_k %d: 1..%d, at most the experts", L->top_k, kMaxTopK);
    if (L->hidden < 1 || L->hidden > kMaxHidden || L->inter < 1 || L->inter > kMaxInter)
        return rr_fail(RR_ELAYOUT, "hidden %lld, inter %lld: 1..%d and 1..%d", (long long)L->hidden,
                       (long long)L->inter, kMaxHidden, kMaxInter);
    if (L->dtype != RR_DST_BF16 && L->dtype != RR_DST_F16) return rr_fail(RR_EINVAL, "unknown element type %d", L->dtype);
    if (L->group != 0 && L->group != 32 && L->group != 64 && L->group != 128)
        return rr_fail(RR_ELAYOUT, "group %d: 0, 32, 64 or 128", L->group);
    if (L->norm_topk != 0 && L->norm_topk != 1) return rr_fail(RR_EINVAL, "norm_topk is 0 or 1, not %d", L->norm_topk);
    if (L->reserved != 0) return rr_fail(RR_EINVAL, "reserved is 0, not %d", L->reserved);
    return RR_OK;
}

// Workspace: a control block, then the arrays.  Offsets in bytes.
struct MoeSpace {
    int64_t logits, top, chosen, c, h, y, total;
    int32_t h_ld, y_ld;
};
constexpr int64_t kControlBytes = 256;

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

MoeSpace moe_space(const rr_moe_layer* L, int64_t tokens) {
    MoeSpace s;
    const int64_t pairs = tokens * std::min(L->top_k, L->n_local);
    s.logits = kControlBytes;
    s.h_ld = int32_t((L->inter + 3) / 4 * 4);
    s.y_ld = int32_t((L->hidden + 3) / 4 * 4);
    s.top = s.logits + up16(4 * tokens * L->n_experts);
    s.chosen = s.top + up16(4 * pairs);
    s.c = s.chosen + up16(4 * tokens * L->top_k);
    s.h = s.c + up16(4 * tokens * L->top_k);
    s.y = s.h + 4 * pairs * s.h_ld;
    s.total = s.y + 4 * pairs * s.y_ld;
    return s;
}

// How the rows of a call's tokens share a block's shared memory.
void moe_rows(MoeArgs* a, int room, Form form) {
    const int h_row = planes_of(form) * a->h_pitch, each = std::max(a->x_pitch, h_row);
    a->cap = std::min(16, room / each);
    if (a->cap > 8 && a->cap < 16) a->cap = 8;
    a->cap = std::min(a->cap, a->tokens);
    a->x_rows = room / a->x_pitch;
    a->h_rows = room / h_row;
    a->all_x = a->tokens <= a->x_rows;
    // Every h at once, for up to 8 tokens (one group of columns).
    const int64_t rows = int64_t(a->tokens) * std::min(a->top_k, a->n_local) + 1;
    a->fold = a->tokens <= 8 && a->cap == a->tokens && rows <= a->h_rows ? int32_t(rows) : 0;
}

template <class T, int W, Form H>
rr_status launch_moe(MoeArgs a, int smem, int dev, cudaStream_t stream);

template <class T, int W>
rr_status prepare_moe(MoeArgs a, int dev, cudaStream_t stream) {
    // Tokens that a pass holds in shared memory, by the longer of the two phases' rows.
    constexpr int kFixed = kWarps * Weights<W>::kStages * Weights<W>::kBytes + kJoinBytes +
                           (sizeof(MoeTables) + 127) / 128 * 128 + 1024 /* static */;
    constexpr int kCols = Weights<W>::kCols;
    // Rows 64 bytes past a multiple of 128, as for the matrix-vector products.
    const auto pitch = [](int cols) { return (cols + kCols - 1) / kCols * (2 * kCols) + 64; };
    static_assert(kSmem - kFixed >= 2 * kMaxHidden + 64 && kSmem - kFixed >= 2 * (2 * kMaxInter + 64), "the longest rows fit");
    a.x_pitch = pitch(a.hidden);
    a.h_pitch = pitch(a.inter);
    constexpr int room = kSmem - kFixed, smem = kFixed - 1024 + room;
    if constexpr (std::is_same<T, F16>::value) {
        moe_rows(&a, room, kHalves);
        return launch_moe<T, W, kHalves>(a, smem, dev, stream);
    } else {
        // In three parts (Qwen3-30B-A3B, 64 tokens: 234 us, in float32 260; two parts, which
        // do not hold all of h, 217) where a pass holds as many tokens so, or seven of them
        // (16 experts of 1024 x 1000, 64 tokens, 8 against 16 a pass: 63 and 68 us), or twice
        // an expert's mean.  (16 of 2048 x 4096, 8 tokens, 3 against 4 a pass: 120 and 122 us;
        // 64 tokens 383 and 314; 8 of 4096 x 8192, 64 tokens, 1 against 2: 3527 and 1890.)
        // That float32's two planes leave more calls without a third barrier weighs less:
        // one token of 32 experts of 2880 x 2880 57 us in parts, 64 in float32.
        MoeArgs parts = a;
        moe_rows(&a, room, kFloats);
        moe_rows(&parts, room, kThirds);
        const bool enough = parts.cap >= std::min(a.cap, 7) ||
                            int64_t(parts.cap) * a.n_experts >= 2 * int64_t(a.tokens) * a.top_k;
        if (parts.cap >= 1 && enough) return launch_moe<T, W, kThirds>(parts, smem, dev, stream);
        return launch_moe<T, W, kFloats>(a, smem, dev, stream);
    }
}

// The largest cluster of 16 or 8 blocks that the current device has room for, or 0.
template <class K>
int largest_cluster(K* kernel, int smem) {
    for (int blocks = 16; blocks >= 8; blocks /= 2) {
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = unsigned(blocks);
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(unsigned(blocks));
        cfg.blockDim = dim3(kProdThreads);
        cfg.dynamicSmemBytes = size_t(smem);
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess && n > 0) return blocks;
        cudaGetLastError();
    }
    return 0;
}

template <class T, int W, Form H>
rr_status launch_moe(MoeArgs a, int smem, int dev, cudaStream_t stream) {
    static std::atomic<uint32_t> ready{0};
    static std::atomic<int> clusters[kMaxDevices] = {};        // largest_cluster + 1, once asked
    RR_CUDA(allow_smem(rr_moe_kernel<T, W, H>, kSmem - 1024, dev, &ready));
    int most = clusters[dev].load(std::memory_order_relaxed) - 1;
    if (most < 0) {
        // More than 8 blocks are asked for by name.
        RR_CUDA(cudaFuncSetAttribute(rr_moe_kernel<T, W, H>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        most = largest_cluster(rr_moe_kernel<T, W, H>, smem);
        clusters[dev].store(most + 1, std::memory_order_relaxed);
    }
    a.one = rr_moe_cluster(std::min<int64_t>(int64_t(a.tokens) * a.top_k, a.n_local) * (a.m13_bytes + a.m2_bytes) +
                               int64_t(a.n_experts) * a.hidden * 2 * ((a.tokens + 15) / 16),
                           most);
    if (a.one) {
        const unsigned blocks = unsigned(a.one);
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = blocks;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(blocks);
        cfg.blockDim = dim3(kProdThreads);
        cfg.dynamicSmemBytes = size_t(smem);
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        RR_CUDA(cudaLaunchKernelEx(&cfg, rr_moe_kernel<T, W, H>, a));
        return RR_OK;
    }
    static std::atomic<int> grids[kMaxDevices] = {};
    int grid = grids[dev].load(std::memory_order_relaxed);
    if (!grid) {
        int coop = 0;
        RR_CUDA(cudaDeviceGetAttribute(&grid, cudaDevAttrMultiProcessorCount, dev));
        RR_CUDA(cudaDeviceGetAttribute(&coop, cudaDevAttrCooperativeLaunch, dev));
        if (!coop) return rr_fail(RR_ECUDA, "the device has no cooperative launches");
        grids[dev].store(grid, std::memory_order_relaxed);
    }
    // (Programmatic dependent launch besides left the gap between two launches at
    // the same 4 us.)
    void* args[] = {&a};
    RR_CUDA(cudaLaunchCooperativeKernel((const void*)rr_moe_kernel<T, W, H>, dim3(unsigned(grid)), dim3(kProdThreads), args,
                                        size_t(smem), stream));
    return RR_OK;
}

}  // namespace

extern "C" rr_status rr_quant_bytes(const rr_quant* q, int64_t* matrix_bytes, int64_t* total_bytes) {
    rr_clear_error();
    RR_TRY(check_quant(q));
    const Packed m = packed_of(q->rows, q->cols, q->group, q->pair);
    if (matrix_bytes) *matrix_bytes = m.matrix_bytes;
    if (total_bytes) *total_bytes = m.matrix_bytes * q->count;
    return RR_OK;
}

namespace {

template <class... Params, class... Args>
cudaError_t launch_after(void (*kernel)(Params...), unsigned grid, int threads, cudaStream_t stream, Args... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(unsigned(threads));
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

}  // namespace

extern "C" rr_status rr_quantize(const rr_quant* q, const void* w, int64_t ld, void* packed,
                                 cudaStream_t stream) {
    RR_TRACE("rr_quantize");
    rr_clear_error();
    RR_TRY(check_quant(q));
    if (ld < q->cols) return rr_fail(RR_EINVAL, "row stride %lld of rows of %lld", (long long)ld, (long long)q->cols);
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, w, 2, "w"));
    RR_TRY(check_device(dev, packed, 16, "packed"));
    const Packed m = packed_of(q->rows, q->cols, q->group, q->pair);
    // Eight warps to a block, one item each.
    const uint32_t total = uint32_t(m.strips * m.blocks * q->count);
    const unsigned grid = (total + 7) / 8;
    const bool vec = (uintptr_t)w % 16 == 0 && ld % 8 == 0;
    return with_group(q->dtype, q->group, [&](auto t, auto g) -> rr_status {
        using T = decltype(t);
        constexpr int G = decltype(g)::value ? decltype(g)::value : 128;
        RR_CUDA(launch_after(vec ? rr_quantize_kernel<T, G, true> : rr_quantize_kernel<T, G, false>, grid, 256, stream,
                             m, static_cast<const uint16_t*>(w),
                             static_cast<const uint16_t*>(w) + (q->rows * q->count - 1) * ld + q->cols, ld,
                             static_cast<char*>(packed), total));
        return RR_OK;
    });
}

extern "C" rr_status rr_dequantize(const rr_quant* q, const void* packed, void* w, int64_t ld,
                                   int32_t f32, cudaStream_t stream) {
    RR_TRACE("rr_dequantize");
    rr_clear_error();
    RR_TRY(check_quant(q));
    if (f32 != 0 && f32 != 1) return rr_fail(RR_EINVAL, "f32 is 0 or 1, not %d", f32);
    if (ld < q->cols) return rr_fail(RR_EINVAL, "row stride %lld of rows of %lld", (long long)ld, (long long)q->cols);
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, packed, 16, "packed"));
    RR_TRY(check_device(dev, w, f32 ? 4 : 2, "w"));
    const Packed m = packed_of(q->rows, q->cols, q->group, q->pair);
    // Eight warps to a block, one item each.
    const uint32_t total = uint32_t(m.strips * m.blocks * q->count);
    const unsigned grid = (total + 7) / 8;
    const bool vec = (uintptr_t)w % 16 == 0 && ld % (f32 ? 4 : 8) == 0;
    return with_group(q->dtype, q->group, [&](auto t, auto g) -> rr_status {
        using T = decltype(t);
        constexpr int G = decltype(g)::value ? decltype(g)::value : 128;
        const auto kernel = f32 ? (vec ? rr_dequantize_kernel<T, G, true, true> : rr_dequantize_kernel<T, G, true, false>)
                                : (vec ? rr_dequantize_kernel<T, G, false, true> : rr_dequantize_kernel<T, G, false, false>);
        RR_CUDA(launch_after(kernel, grid, 256, stream, m, static_cast<const char*>(packed), w, ld, total));
        return RR_OK;
    });
}

namespace {

struct MatvecShape {
    unsigned grid;
    int smem;
    bool deep;      // 6 blocks of weights in flight a warp, else 4
};

// Clusters of a size that this GPU runs at once with one block per SM (GB300: 152,
// 76, 36 and 15 of 1, 2, 4 and 8 blocks, since a cluster stays within one GPC).
// Asked once per device.
template <class K>
int clusters_at_once(K* kernel, int dev, int cluster) {
    static std::atomic<int> known[kMaxDevices][9] = {};
    int n = known[dev][cluster].load(std::memory_order_relaxed);
    if (n) return n;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(cluster));
    cfg.blockDim = dim3(kProdThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 1;
    }
    known[dev][cluster].store(n, std::memory_order_relaxed);
    return n;
}

// How a product is shared out, for a.tokens tokens; false if these do not fit.  A
// cluster's blocks share the columns where a block's shared memory would not hold the
// tokens, or where strips are too few to go round.  6 blocks of weights in flight a
// warp, or 4 where that makes room.
bool matvec_shape(MatvecArgs* a, int group, int dev, MatvecShape* shape) {
    const int tiles = a->tokens > 8 ? 2 : 1, part = 512 * tiles;
    int64_t best = INT64_MAX;
    for (int cluster = 1; cluster <= 8 && cluster <= a->m.blocks; cluster *= 2) {
        const int64_t blocks = (a->m.blocks + cluster - 1) / cluster;
        // Rows 64 bytes past a multiple of 128, so that two tokens' rows are on
        // different halves of the banks.
        const int64_t pitch = blocks * 2 * kBlock + 64;
        const int64_t groups = std::min<int64_t>(clusters_at_once(rr_matvec_kernel<BF16, 128, 1, 2, 6>, dev, cluster), a->m.strips);
        const int64_t strips = (a->m.strips + groups - 1) / groups;
        for (int stages = 6; stages >= 4; stages -= 2) {
            const int64_t room = kSmem - kWarps * (stages * block_bytes(group) + part) - pitch * a->tokens;
            const int64_t batch = cluster == 1 ? strips : std::min(strips, room / part);
            if (room < 0 || batch < 1) continue;
            const int64_t joins = cluster == 1 ? 0 : (strips + batch - 1) / batch;
            // In blocks of weights of the busiest warp: those, the copy of the tokens (32 KB
            // of them cost about as much as a block, 12 KB where rows of that length one
            // after another are not aligned), a cluster's joins.  (24576 x 4096, paired, 16
            // tokens: 19.6 us so, in one block's shared memory each, and 21.9 in clusters of 2;
            // 30001 x 4097, 16: 24.1 us so, 25.0 where 32 KB count as a block.)  Where the tokens
            // are does not count, as it would then choose the order of the sums: 2048 x 8192,
            // 8 tokens at an odd address take 10.9 us, and 8.2 with 12 KB.
            const int64_t cost = (strips * blocks + kWarps - 1) / kWarps +
                                 pitch * a->tokens / (a->m.cols % 8 == 0 ? 32768 : 12288) + 4 * joins +
                                 (stages == 4 ? 1 : 0);
            if (cost >= best) continue;
            best = cost;
            a->pitch = int32_t(pitch);
            a->cluster = cluster;
            a->batch = int32_t(batch);
            shape->deep = stages == 6;
            shape->grid = unsigned(groups * cluster);
            shape->smem = int(kSmem - room + (cluster == 1 ? 0 : batch * part));
        }
    }
    return best != INT64_MAX;
}

template <class T, int G, int NT, int U, int ST>
cudaError_t launch_matvec(const MatvecArgs& a, const MatvecShape& shape, int dev, cudaStream_t stream) {
    static std::atomic<uint32_t> ready{0};
    const auto kernel = rr_matvec_kernel<T, G, NT, U, ST>;
    const cudaError_t e = allow_smem(kernel, kSmem, dev, &ready);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(a.cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(shape.grid);
    cfg.blockDim = dim3(kProdThreads);
    cfg.dynamicSmemBytes = size_t(shape.smem);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace

extern "C" rr_status rr_matvec(const rr_quant* q, const void* packed, const void* x, int64_t ldx,
                               int32_t n_tokens, void* out, int64_t ldo, int32_t f32,
                               cudaStream_t stream) {
    RR_TRACE("rr_matvec");
    rr_clear_error();
    RR_TRY(check_quant(q));
    if (q->count != 1) return rr_fail(RR_EINVAL, "rr_matvec takes one matrix, not a stack of %d", q->count);
    if (n_tokens < 0 || n_tokens > RR_MATVEC_MAX_TOKENS)
        return rr_fail(RR_EINVAL, "%d tokens: 0..%d", n_tokens, RR_MATVEC_MAX_TOKENS);
    if (f32 != 0 && f32 != 1) return rr_fail(RR_EINVAL, "f32 is 0 or 1, not %d", f32);
    const int64_t n_out = q->pair ? q->rows / 2 : q->rows;
    if (ldx < q->cols || ldo < n_out)
        return rr_fail(RR_EINVAL, "row strides %lld and %lld of rows of %lld and %lld", (long long)ldx,
                       (long long)ldo, (long long)q->cols, (long long)n_out);
    if (n_tokens == 0) return RR_OK;
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, packed, 16, "packed"));
    RR_TRY(check_device(dev, x, 2, "x"));
    RR_TRY(check_device(dev, out, f32 ? 4 : 2, "out"));
    return with_group(q->dtype, q->group, [&](auto t, auto g) -> rr_status {
        using T = decltype(t);
        constexpr int G = decltype(g)::value ? decltype(g)::value : 128;
        MatvecArgs a;
        a.m = packed_of(q->rows, q->cols, q->group, q->pair);
        a.packed = static_cast<const char*>(packed);
        a.ldx = ldx;
        a.ldo = ldo;
        a.f32 = f32;
        a.vec = (uintptr_t)x % 16 == 0 && (ldx % 8 == 0 || n_tokens == 1);
        // Tokens that one launch takes: all of them but for very long rows, whose
        // tokens would not fit the blocks' shared memory.
        for (int n0 = 0; n0 < n_tokens; n0 += a.tokens) {
            a.tokens = n_tokens - n0;
            a.x = static_cast<const uint16_t*>(x) + n0 * ldx;
            a.out = static_cast<char*>(out) + n0 * ldo * (f32 ? 4 : 2);
            MatvecShape shape;
            while (!matvec_shape(&a, G, dev, &shape)) {
                if (a.tokens == 1) return rr_fail(RR_ELAYOUT, "rows of %lld columns", (long long)q->cols);
                a.tokens = (a.tokens + 1) / 2;
            }
            const cudaError_t e = a.tokens > 8
                                      ? shape.deep ? launch_matvec<T, G, 2, 2, 6>(a, shape, dev, stream)
                                                   : launch_matvec<T, G, 2, 1, 4>(a, shape, dev, stream)
                                      : shape.deep ? launch_matvec<T, G, 1, 2, 6>(a, shape, dev, stream)
                                                   : launch_matvec<T, G, 1, 1, 4>(a, shape, dev, stream);
            if (e != cudaSuccess) return cuda_fail(e, "rr_matvec");
        }
        return RR_OK;
    });
}

extern "C" rr_status rr_moe_workspace(const rr_moe_layer* L, int32_t max_tokens, int64_t* bytes) {
    rr_clear_error();
    RR_TRY(check_moe(L));
    if (max_tokens < 1 || max_tokens > RR_MOE_MAX_TOKENS)
        return rr_fail(RR_EINVAL, "%d tokens: 1..%d", max_tokens, RR_MOE_MAX_TOKENS);
    if (!bytes) return rr_fail(RR_EINVAL, "bytes is NULL");
    *bytes = moe_space(L, max_tokens).total;
    return RR_OK;
}

extern "C" rr_status rr_moe(const rr_moe_layer* L, const void* router, const void* w13, const void* w2,
                            const void* x, int64_t ldx, int32_t n_tokens, void* out, int64_t ldo,
                            int32_t* ids, float* weights, void* workspace, int64_t workspace_bytes,
                            cudaStream_t stream) {
    RR_TRACE("rr_moe");
    rr_clear_error();
    RR_TRY(check_moe(L));
    if (n_tokens < 0 || n_tokens > RR_MOE_MAX_TOKENS)
        return rr_fail(RR_EINVAL, "%d tokens: 0..%d", n_tokens, RR_MOE_MAX_TOKENS);
    if (ldx < L->hidden || ldo < L->hidden)
        return rr_fail(RR_EINVAL, "row strides %lld and %lld of rows of %lld", (long long)ldx, (long long)ldo, (long long)L->hidden);
    if (n_tokens == 0) return RR_OK;
    const MoeSpace S = moe_space(L, n_tokens);
    if (workspace_bytes < S.total)
        return rr_fail(RR_EINVAL, "workspace of %lld bytes, the call needs %lld", (long long)workspace_bytes, (long long)S.total);
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, router, 16, "router"));
    RR_TRY(check_device(dev, w13, 16, "w13"));
    RR_TRY(check_device(dev, w2, 16, "w2"));
    RR_TRY(check_device(dev, x, 2, "x"));
    RR_TRY(check_device(dev, out, 2, "out"));
    if (ids) RR_TRY(check_device(dev, ids, 4, "ids"));
    if (weights) RR_TRY(check_device(dev, weights, 4, "weights"));
    RR_TRY(check_device(dev, workspace, 16, "workspace"));
    char* const ws = static_cast<char*>(workspace);
    MoeArgs a;
    a.router = static_cast<const uint16_t*>(router);
    a.w13 = static_cast<const char*>(w13);
    a.w2 = static_cast<const char*>(w2);
    a.x = static_cast<const uint16_t*>(x);
    a.ldx = ldx;
    a.ldo = ldo;
    a.out = static_cast<uint16_t*>(out);
    a.ids = ids;
    a.weights = weights;
    a.control = reinterpret_cast<MoeControl*>(ws);
    a.logits = reinterpret_cast<float*>(ws + S.logits);
    a.h = reinterpret_cast<float*>(ws + S.h);
    a.y = reinterpret_cast<float*>(ws + S.y);
    a.h_top = reinterpret_cast<uint32_t*>(ws + S.top);
    a.far_chosen = reinterpret_cast<int32_t*>(ws + S.chosen);
    a.far_c = reinterpret_cast<float*>(ws + S.c);
    a.h_ld = S.h_ld;
    a.y_ld = S.y_ld;
    a.tokens = n_tokens;
    a.n_experts = L->n_experts;
    a.first = L->first_expert;
    a.n_local = L->n_local;
    a.top_k = L->top_k;
    a.norm = L->norm_topk;
    a.hidden = int32_t(L->hidden);
    a.inter = int32_t(L->inter);
    a.x_vec = (uintptr_t)x % 16 == 0 && (ldx % 8 == 0 || n_tokens == 1);
    a.r_vec = L->hidden % 8 == 0;
    a.m13_bytes = L->group ? packed_of(2 * L->inter, L->hidden, L->group, 1).matrix_bytes : 4 * L->inter * L->hidden;
    a.m2_bytes = L->group ? packed_of(L->hidden, L->inter, L->group, 0).matrix_bytes : 2 * L->inter * L->hidden;
    return with_group(L->dtype, L->group, [&](auto t, auto g) -> rr_status {
        using T = decltype(t);
        constexpr int G = decltype(g)::value;
        if constexpr (G != 0) return prepare_moe<T, G>(a, dev, stream);
        else if (L->hidden % 8 == 0 && L->inter % 8 == 0) return prepare_moe<T, 0>(a, dev, stream);
        else return prepare_moe<T, 1>(a, dev, stream);
    });
}

extern "C" rr_status rr_moe_check(const rr_moe_layer* L, int32_t max_tokens, void* workspace,
                                  cudaStream_t stream) {
    rr_clear_error();
    RR_TRY(check_moe(L));
    if (max_tokens < 1 || max_tokens > RR_MOE_MAX_TOKENS)
        return rr_fail(RR_EINVAL, "%d tokens: 1..%d", max_tokens, RR_MOE_MAX_TOKENS);
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, workspace, 16, "workspace"));
    uint32_t err = 0;
    RR_CUDA(cudaMemcpyAsync(&err, workspace, 4, cudaMemcpyDeviceToHost, stream));
    RR_CUDA(cudaStreamSynchronize(stream));
    if (!err) return RR_OK;
    RR_CUDA(cudaMemsetAsync(workspace, 0, kControlBytes, stream));
    RR_CUDA(cudaStreamSynchronize(stream));
    return rr_fail(RR_ECUDA, "a wait between the layer's blocks ran out");
}
