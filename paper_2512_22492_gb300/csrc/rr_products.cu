// Products of the rollout's weights for GB300 (sm_103a): quantisation to 4-bit
// strips with group scales, matrix-vector products with them, and a
// mixture-of-experts layer for a few tokens (include/rr.h has the definitions).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <mutex>
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

// One warp takes one block: lane 4 g + t holds slots g and g + 8, of each the
// columns 32 j + 8 t + 0..7, so that a lane's 16 bytes of codes and a group's
// maximum need no memory between lanes.  Bound by HBM: 2 bytes read and about
// half a byte written per element.
template <class T, int G>
__global__ void __launch_bounds__(256) rr_quantize_kernel(Packed m, const uint16_t* w, int64_t ld,
                                                          char* packed, int64_t total) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t item = int64_t(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (item >= total) return;
    const int64_t b = item % m.blocks, strip = item / m.blocks % m.strips;
    const int64_t mat = item / m.blocks / m.strips;
    char* const to = packed + mat * m.matrix_bytes + (strip * m.blocks + b) * block_bytes(G);
    for (int half = 0; half < 2; ++half) {
        const int64_t row = m.row(strip, 8 * half + g);
        float v[4][8];
        const uint16_t* const src = w + (mat * m.rows + row) * ld;
        for (int j = 0; j < 4; ++j) {
            const int64_t c = b * kBlock + 32 * j + 8 * t;
            for (int i = 0; i < 8; ++i)
                v[j][i] = row >= 0 && c + i < m.cols ? T::widen(src[c + i]) : 0.0f;
        }
        uint32_t words[4];
        for (int k = 0; k < kBlock / G; ++k) {
            constexpr int kWords = G / 32;
            float top = 0.0f;
            bool fine = true;
            for (int j = k * kWords; j < (k + 1) * kWords; ++j)
                for (int i = 0; i < 8; ++i) {
                    top = fmaxf(top, fabsf(v[j][i]));
                    fine = fine && isfinite(v[j][i]);
                }
            for (int o = 1; o < 4; o *= 2) {
                top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
                fine = __shfl_xor_sync(~0u, int(fine), o) && fine;
            }
            uint16_t s16 = T::round(top / 7.0f);
            float s = T::widen(s16);
            if (s < kLeastScale) s16 = 0, s = 0.0f;
            if (!fine) s16 = T::kNaN, s = 0.0f;
            if (t == 0)
                reinterpret_cast<uint16_t*>(to + kCodes)[2 * (g * (kBlock / G) + k) + half] = s16;
            for (int j = k * kWords; j < (k + 1) * kWords; ++j) {
                uint32_t word = 0;
                for (int i = 0; i < 8; ++i) {
                    const float q = s > 0.0f ? fminf(fmaxf(rintf(v[j][i] / s), -7.0f), 7.0f) : 0.0f;
                    word |= uint32_t(int(q) + 8) << (4 * (i / 2 + 4 * (i % 2)));
                }
                words[j] = word;
            }
        }
        *reinterpret_cast<uint4*>(to + 512 * half + 16 * lane) =
            make_uint4(words[0], words[1], words[2], words[3]);
    }
}

// The inverse, by the same lanes.
template <class T, int G, bool F32>
__global__ void __launch_bounds__(256) rr_dequantize_kernel(Packed m, const char* packed, void* w,
                                                            int64_t ld, int64_t total) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t item = int64_t(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (item >= total) return;
    const int64_t b = item % m.blocks, strip = item / m.blocks % m.strips;
    const int64_t mat = item / m.blocks / m.strips;
    const char* const from = packed + mat * m.matrix_bytes + (strip * m.blocks + b) * block_bytes(G);
    for (int half = 0; half < 2; ++half) {
        const int64_t row = m.row(strip, 8 * half + g);
        if (row < 0) continue;
        const uint4 q = *reinterpret_cast<const uint4*>(from + 512 * half + 16 * lane);
        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
        for (int j = 0; j < 4; ++j) {
            const float s = T::widen(reinterpret_cast<const uint16_t*>(
                from + kCodes)[2 * (g * (kBlock / G) + 32 * j / G) + half]);
            const int64_t c = b * kBlock + 32 * j + 8 * t;
            for (int i = 0; i < 8; ++i)
                if (c + i < m.cols)
                    put<T, F32>(w, (mat * m.rows + row) * ld + c + i, s * float(code(words[j], i)));
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

// Codes n and n + 4 of a word (columns 2 n, 2 n + 1) as a pair of 16-bit numbers:
// placed in the low mantissa bits of 128 (float16: 1024) they read 128 + q + 8,
// and the subtraction is exact.
template <class T>
__device__ __forceinline__ uint32_t codes(uint32_t word, int n) {
    constexpr bool kB = std::is_same<T, BF16>::value;
    uint32_t v;
    asm("lop3.b32 %0, %1, 0x000F000F, %2, 0xEA;" : "=r"(v) : "r"(word >> (4 * n)), "r"(kB ? 0x43004300u : 0x64006400u));
    if (kB) {
        const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v),
                                         __nv_bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308)));
        return *reinterpret_cast<const uint32_t*>(&d);
    }
    const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&v),
                              __half2(__ushort_as_half(0x6408), __ushort_as_half(0x6408)));
    return *reinterpret_cast<const uint32_t*>(&d);
}

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

constexpr int kWarps = 16;         // of a block: one block per SM
constexpr int kProdThreads = 32 * kWarps;

// A warp's stages of U adjacent blocks of codes each: enough of them that a block
// has 64 to 100 KB in flight, and a wait, a copy's address and a loop's step for
// U blocks at a time.  A lane copies the 16-byte runs that it reads itself; of
// the scales, which four lanes share, lanes 0..7 copy a slot pair's each.
template <int G, int U>
struct Stage {
    static constexpr int kScale = 512 / G;                 // bytes of a slot pair's scales
    static constexpr int kBlockBytes = kCodes + 8 * kScale;     // = block_bytes(G)
    static constexpr int kBytes = U * kBlockBytes;
    static constexpr int kStages = 6 / U;
    // from: the block's codes at this lane's run; scales: at this lane's (< 8) scales.
    static __device__ __forceinline__ void load(uint32_t to, const char* from, const char* scales, int blocks,
                                                int lane) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u > 0 && blocks <= u) break;
            copy_async<16>(to + u * kBlockBytes + 16 * lane, from + u * kBlockBytes);
            copy_async<16>(to + u * kBlockBytes + 512 + 16 * lane, from + u * kBlockBytes + 512);
            if (lane < 8) copy_async<kScale>(to + u * kBlockBytes + kCodes + kScale * lane, scales + u * kBlockBytes);
        }
        copy_commit();
    }
};

// sum += W x over one block of 128 columns.  x[n]: this lane's 16 bytes of its
// token's row at the block's first column, in shared memory.  Groups are summed
// in the matrix unit and scaled in float32.
template <class T, int G, int NT>
__device__ __forceinline__ void block_product(float (&sum)[NT][4], const char* stage, const char* const (&x)[NT],
                                              int at, int lane) {
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
#pragma unroll
        for (int i = 0; i < 4; ++i) al[i] = codes<T>(wl[j], i), ah[i] = codes<T>(wh[j], i);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint4 v = *reinterpret_cast<const uint4*>(x[n] + at + 64 * j);
            if (32 * j % G == 0) mma_first<T>(part[n], al[0], ah[0], al[1], ah[1], v.x, v.y);
            else mma<T>(part[n], al[0], ah[0], al[1], ah[1], v.x, v.y);
            mma<T>(part[n], al[2], ah[2], al[3], ah[3], v.z, v.w);
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
    int32_t team;         // warps that share a strip's columns: 1, 2, 4, 8 or 16
    int32_t cluster;      // blocks that share the columns
    int32_t batch;        // strips between two joins of the teams' sums
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

// A cluster takes a run of strips; each of its blocks takes a share of the
// columns, whose tokens it keeps in shared memory, and of these each warp of a
// team every team-th run of U blocks of 128.  Warps stream their blocks through
// stages of their own without meeting; sums of a batch of strips are joined
// through shared memory in a fixed order.
template <class T, int G, int NT, int U>
__global__ void __launch_bounds__(kProdThreads, 1) rr_matvec_kernel(const __grid_constant__ MatvecArgs a) {
    extern __shared__ __align__(128) char smem[];
    using S = Stage<G, U>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = blockIdx.x % a.cluster, cl = blockIdx.x / a.cluster, n_cl = gridDim.x / a.cluster;
    // Programmatic dependent launch: the next kernel may be scheduled, and waits
    // as this one does for the kernels before it.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    char* const fifo = smem + warp * (S::kStages * S::kBytes);
    char* const xs = smem + kWarps * S::kStages * S::kBytes;
    float4* const red = reinterpret_cast<float4*>(xs + a.tokens * a.pitch);

    const int64_t s0 = cl * a.m.strips / n_cl, s1 = (cl + 1) * a.m.strips / n_cl;
    const int b0 = int(rank * a.m.blocks / a.cluster), b1 = int((rank + 1) * a.m.blocks / a.cluster);
    const int teams = kWarps / a.team, team = warp / a.team, part = warp % a.team;

    // This warp takes runs part, part + team, ... of a strip.  The load cursor
    // goes over them, strip after strip, ahead of the products.
    const int runs = (b1 - b0 + U - 1) / U;
    const int steps = (runs - part + a.team - 1) / a.team;
    int left_strips = steps > 0 ? int((s1 - s0 - team + teams - 1) / teams) : 0;
    int lb = b0 + U * part, slot = 0;
    const char* from = a.packed + ((s0 + team) * a.m.blocks + lb) * S::kBlockBytes + 16 * lane;
    const int64_t scales = kCodes + (S::kScale - 16) * lane;      // from a run's codes to its scales
    const int64_t next_run = int64_t(a.team) * S::kBytes;
    const int64_t next_strip = (teams * a.m.blocks - int64_t(steps - 1) * a.team * U) * S::kBlockBytes;
    const uint32_t fifo_at = smem_at(fifo);
    auto load = [&](int to) {
        if (left_strips > 0) {
            S::load(fifo_at + to * S::kBytes, from, from + scales, b1 - lb, lane);
            lb += a.team * U;
            if (lb >= b1) {
                lb = b0 + U * part;
                --left_strips;
                from += next_strip;
            } else {
                from += next_run;
            }
        } else {
            copy_commit();
        }
    };

    // Tokens: this block's columns, zeros past the matrix's.
    const int cols = (b1 - b0) * kBlock;
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
        for (int n = 0; n < a.tokens; ++n)
#pragma unroll 8
            for (int c = threadIdx.x; c < cols; c += kProdThreads)
                *reinterpret_cast<uint16_t*>(xs + n * a.pitch + 2 * c) =
                    c0 + c < a.m.cols ? a.x[n * a.ldx + c0 + c] : uint16_t(0);
    }
    copy_commit();
    for (int i = 0; i < S::kStages - 1; ++i) load(i);
    copy_wait<S::kStages - 1>();
    __syncthreads();

    // A lane of an absent token reads the last one's row; its sums go nowhere.
    const char* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
        x[n] = xs + min(8 * n + (lane >> 2), a.tokens - 1) * a.pitch + 16 * (lane & 3);
    const bool alone = a.team == 1 && a.cluster == 1;
    for (int64_t from = s0; from < s1; from += a.batch) {
        const int64_t to = min(from + a.batch, s1);
        for (int64_t strip = from + team; strip < to; strip += teams) {
            float sum[NT][4] = {};
            for (int i = 0; i < steps; ++i) {
                copy_wait<S::kStages - 2>();
                __syncwarp();      // the scales are there for every lane, and the last stage has been read
                load(slot == 0 ? S::kStages - 1 : slot - 1);
                const int at = U * (part + i * a.team);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u == 0 || at + u < b1 - b0)
                        block_product<T, G, NT>(sum, fifo + slot * S::kBytes + u * S::kBlockBytes, x,
                                                (at + u) * (2 * kBlock), lane);
                slot = slot + 1 == S::kStages ? 0 : slot + 1;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (alone) put_strip<T>(a, strip, lane, n, sum[n]);
                else
                    red[((part * a.batch + int(strip - from)) * NT + n) * 32 + lane] =
                        make_float4(sum[n][0], sum[n][1], sum[n][2], sum[n][3]);
            }
        }
        if (alone) continue;
        if (a.cluster > 1) cluster_sync();
        else __syncthreads();
        const int count = int(to - from) * NT * 32;
        for (int i = rank * kProdThreads + threadIdx.x; i < count; i += a.cluster * kProdThreads) {
            float v[4] = {};
            for (int r = 0; r < a.cluster; ++r) {
                uint32_t at = smem_at(red + i);
                if (a.cluster > 1) asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(at), "r"(r));
                for (int p = 0; p < a.team; ++p) {
                    float4 f;
                    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
                                 : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w)
                                 : "r"(at + uint32_t(p * a.batch * NT * 32 * sizeof(float4))) : "memory");
                    v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
                }
            }
            put_strip<T>(a, from + i / (NT * 32), i & 31, i / 32 % NT, v);
        }
        // The sums have been read, here and by the cluster's other blocks, before
        // they are overwritten or this block ends.
        if (a.cluster > 1) cluster_sync();
        else __syncthreads();
    }
    copy_wait<0>();
}

// ---------------------------------------------------------------------------
// Mixture of experts
// ---------------------------------------------------------------------------

constexpr int kMaxExperts = 512, kMaxTopK = 16, kMaxInner = 65536;

struct MoeArgs {
    const uint16_t* router;
    const char *w13, *w2;
    const uint16_t* x;
    int64_t ldx, ldo;
    uint16_t* out;
    int32_t* ids;
    float* weights;
    // Workspace.
    float* logits;     // [tokens, n_experts]
    int32_t* chosen;   // [tokens, top_k]
    float* c;          // [tokens, top_k]
    float* h;          // [tokens * top_k, inter]
    int32_t tokens, n_experts, first, n_local, top_k, norm, hidden, inter;
    Packed m13, m2;
};

// A matrix element, whatever the form it is stored in.
template <class T, int G>
__device__ float element(const char* base, const Packed& m, int64_t mat, int64_t row, int64_t col) {
    if (G == 0)
        return T::widen(reinterpret_cast<const uint16_t*>(base)[(mat * m.rows + row) * m.cols + col]);
    const int64_t i = m.pair && row >= m.rows / 2 ? row - m.rows / 2 : row;
    const int64_t strip = m.pair ? i / 8 : i / 16;
    const int half = m.pair ? row >= m.rows / 2 : (i / 8) & 1, g = i & 7;
    const int c = col % kBlock, j = c / 32, t = c % 32 / 8;
    constexpr int kGroup = G ? G : 128;
    const char* const from =
        base + mat * m.matrix_bytes + (strip * m.blocks + col / kBlock) * block_bytes(kGroup);
    const uint32_t word =
        reinterpret_cast<const uint32_t*>(from + 512 * half + 16 * (4 * g + t))[j];
    const uint16_t s =
        reinterpret_cast<const uint16_t*>(from + kCodes)[2 * (g * (kBlock / kGroup) + c / kGroup) + half];
    return T::widen(s) * float(code(word, c % 8));
}

__device__ __forceinline__ float warp_sum(float v) {
    for (int o = 16; o; o /= 2) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

template <class T>
__global__ void __launch_bounds__(128) rr_moe_logits_kernel(const MoeArgs a) {
    const int lane = threadIdx.x & 31;
    const int i = blockIdx.x * 4 + (threadIdx.x >> 5);
    if (i >= a.tokens * a.n_experts) return;
    const int t = i / a.n_experts, e = i % a.n_experts;
    float sum = 0.0f;
    for (int k = lane; k < a.hidden; k += 32)
        sum = fmaf(T::widen(a.x[t * a.ldx + k]), T::widen(a.router[int64_t(e) * a.hidden + k]), sum);
    sum = warp_sum(sum);
    if (lane == 0) a.logits[i] = sum;
}

// Descending order of logits as unsigned integers: NaN first, +0 and -0 alike.
__device__ __forceinline__ uint32_t rank_key(float l) {
    if (isnan(l)) return ~0u;
    const uint32_t b = __float_as_uint(l + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(32) rr_moe_choose_kernel(const MoeArgs a) {
    __shared__ uint32_t key[kMaxExperts];
    const int t = blockIdx.x, lane = threadIdx.x;
    const float* const l = a.logits + t * a.n_experts;
    float top = -INFINITY;
    for (int e = lane; e < a.n_experts; e += 32) {
        key[e] = rank_key(l[e]);
        top = fmaxf(top, l[e]);
    }
    for (int o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    float sum = 0.0f;
    for (int e = lane; e < a.n_experts; e += 32) sum += expf(l[e] - top);
    sum = warp_sum(sum);
    __syncwarp();
    float mine = 0.0f, total = 0.0f;
    int my_id = 0;
    for (int j = 0; j < a.top_k; ++j) {
        unsigned long long best = 0;   // (key, lowest index first)
        for (int e = lane; e < a.n_experts; e += 32)
            if (key[e])
                best = max(best, (unsigned long long)key[e] << 32 | uint32_t(~e));
        for (int o = 16; o; o /= 2) best = max(best, __shfl_xor_sync(~0u, best, o));
        const int e = int(~uint32_t(best));
        const float p = expf(l[e] - top) / sum;
        total += p;
        if (lane == j) mine = p, my_id = e;
        __syncwarp();
        if (lane == e % 32) key[e] = 0;
        __syncwarp();
    }
    if (lane < a.top_k) {
        if (a.norm) mine /= total;
        a.chosen[t * a.top_k + lane] = my_id;
        a.c[t * a.top_k + lane] = mine;
        if (a.ids) a.ids[t * a.top_k + lane] = my_id;
        if (a.weights) a.weights[t * a.top_k + lane] = mine;
    }
}

template <class T, int G>
__global__ void __launch_bounds__(128) rr_moe_up_kernel(const MoeArgs a) {
    const int lane = threadIdx.x & 31;
    const int i = blockIdx.x * 4 + (threadIdx.x >> 5), p = blockIdx.y;
    const int e = a.chosen[p] - a.first;
    if (i >= a.inter || e < 0 || e >= a.n_local) return;
    const uint16_t* const x = a.x + p / a.top_k * a.ldx;
    float gate = 0.0f, up = 0.0f;
    for (int k = lane; k < a.hidden; k += 32) {
        const float v = T::widen(x[k]);
        gate = fmaf(v, element<T, G>(a.w13, a.m13, e, i, k), gate);
        up = fmaf(v, element<T, G>(a.w13, a.m13, e, a.inter + i, k), up);
    }
    gate = warp_sum(gate);
    up = warp_sum(up);
    if (lane == 0) a.h[int64_t(p) * a.inter + i] = silu(gate) * up;
}

template <class T, int G>
__global__ void __launch_bounds__(128) rr_moe_down_kernel(const MoeArgs a) {
    const int lane = threadIdx.x & 31;
    const int n = blockIdx.x * 4 + (threadIdx.x >> 5), t = blockIdx.y;
    if (n >= a.hidden) return;
    float y = 0.0f;
    for (int j = 0; j < a.top_k; ++j) {
        const int p = t * a.top_k + j, e = a.chosen[p] - a.first;
        if (e < 0 || e >= a.n_local) continue;
        float sum = 0.0f;
        for (int k = lane; k < a.inter; k += 32)
            sum = fmaf(a.h[int64_t(p) * a.inter + k], element<T, G>(a.w2, a.m2, e, n, k), sum);
        y += a.c[p] * warp_sum(sum);
    }
    if (lane == 0) a.out[t * a.ldo + n] = T::round(y);
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

// Memory of the current device, `align`ed.
rr_status check_device(const void* p, size_t align, const char* what) {
    if (!p || (uintptr_t)p % align) return rr_fail(RR_EINVAL, "%s is NULL or not %zu-byte aligned", what, align);
    cudaPointerAttributes at;
    int dev = -1;
    RR_CUDA(cudaGetDevice(&dev));
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
        cudaGetLastError();
        return rr_fail(RR_EINVAL, "%s is not memory of this GPU", what);
    }
    if (at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev)) return RR_OK;
    return rr_fail(RR_EINVAL, "%s is not memory of this GPU", what);
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
    return RR_OK;
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
    if (L->hidden < 1 || L->hidden > kMaxInner || L->inter < 1 || L->inter > kMaxInner)
        return rr_fail(RR_ELAYOUT, "hidden %lld, inter %lld: 1..%d", (long long)L->hidden, (long long)L->inter, kMaxInner);
    if (L->dtype != RR_DST_BF16 && L->dtype != RR_DST_F16) return rr_fail(RR_EINVAL, "unknown element type %d", L->dtype);
    if (L->group != 0 && L->group != 32 && L->group != 64 && L->group != 128)
        return rr_fail(RR_ELAYOUT, "group %d: 0, 32, 64 or 128", L->group);
    if (L->norm_topk != 0 && L->norm_topk != 1) return rr_fail(RR_EINVAL, "norm_topk is 0 or 1, not %d", L->norm_topk);
    if (L->reserved != 0) return rr_fail(RR_EINVAL, "reserved is 0, not %d", L->reserved);
    return RR_OK;
}

// Workspace: a control block, then the arrays.  Offsets in bytes.
struct MoeSpace {
    int64_t logits, chosen, c, h, total;
};
constexpr int64_t kControlBytes = 256;   // word 0: the error word

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

MoeSpace moe_space(const rr_moe_layer* L, int64_t tokens) {
    MoeSpace s;
    s.logits = kControlBytes;
    s.chosen = s.logits + up16(4 * tokens * L->n_experts);
    s.c = s.chosen + up16(4 * tokens * L->top_k);
    s.h = s.c + up16(4 * tokens * L->top_k);
    s.total = s.h + up16(4 * tokens * L->top_k * L->inter);
    return s;
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

// Blocks of warps for `items`, or an error where the grid cannot hold them.
rr_status grid_of(int64_t items, int per_block, unsigned* grid) {
    const int64_t n = (items + per_block - 1) / per_block;
    if (n > INT32_MAX) return rr_fail(RR_ELAYOUT, "the stack is too large for one call");
    *grid = unsigned(n);
    return RR_OK;
}

}  // namespace

extern "C" rr_status rr_quantize(const rr_quant* q, const void* w, int64_t ld, void* packed,
                                 cudaStream_t stream) {
    RR_TRACE("rr_quantize");
    rr_clear_error();
    RR_TRY(check_quant(q));
    if (ld < q->cols) return rr_fail(RR_EINVAL, "row stride %lld of rows of %lld", (long long)ld, (long long)q->cols);
    RR_TRY(check_device(w, 2, "w"));
    RR_TRY(check_device(packed, 16, "packed"));
    const Packed m = packed_of(q->rows, q->cols, q->group, q->pair);
    const int64_t total = m.strips * m.blocks * q->count;
    unsigned grid;
    RR_TRY(grid_of(total, 8, &grid));
    return with_group(q->dtype, q->group, [&](auto t, auto g) -> rr_status {
        constexpr int G = decltype(g)::value ? decltype(g)::value : 128;
        rr_quantize_kernel<decltype(t), G><<<grid, 256, 0, stream>>>(
            m, static_cast<const uint16_t*>(w), ld, static_cast<char*>(packed), total);
        RR_CUDA(cudaGetLastError());
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
    RR_TRY(check_device(packed, 16, "packed"));
    RR_TRY(check_device(w, f32 ? 4 : 2, "w"));
    const Packed m = packed_of(q->rows, q->cols, q->group, q->pair);
    const int64_t total = m.strips * m.blocks * q->count;
    unsigned grid;
    RR_TRY(grid_of(total, 8, &grid));
    return with_group(q->dtype, q->group, [&](auto t, auto g) -> rr_status {
        constexpr int G = decltype(g)::value ? decltype(g)::value : 128;
        if (f32)
            rr_dequantize_kernel<decltype(t), G, true><<<grid, 256, 0, stream>>>(
                m, static_cast<const char*>(packed), w, ld, total);
        else
            rr_dequantize_kernel<decltype(t), G, false><<<grid, 256, 0, stream>>>(
                m, static_cast<const char*>(packed), w, ld, total);
        RR_CUDA(cudaGetLastError());
        return RR_OK;
    });
}

namespace {

struct MatvecShape {
    unsigned grid;
    int smem;
    int run;        // blocks of a stage
};
constexpr int kSmem = 227 * 1024;
constexpr int kJoinBytes = 24 * 1024;   // shared memory of the teams' sums

// Clusters of a size that this GPU runs at once with one block per SM (GB300: 152,
// 76, 36 and 15 of 1, 2, 4 and 8 blocks, since a cluster stays within one GPC).
// Asked once per device.
template <class K>
int clusters_at_once(K* kernel, int cluster) {
    static std::mutex mutex;
    static int known[16][4] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev > 15) return 1;
    const int i = cluster == 1 ? 0 : cluster == 2 ? 1 : cluster == 4 ? 2 : 3;
    const std::lock_guard<std::mutex> lock(mutex);
    if (!known[dev][i]) {
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
        int n = 0;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
            cudaGetLastError();
            return 1;
        }
        known[dev][i] = n;
    }
    return known[dev][i];
}

// How a product is shared out, for a.tokens tokens; false if these do not fit.
// The time of a launch goes by the blocks of 128 columns that the busiest warp
// takes; joins cost about one of them.  Measured on GB300: see the table of
// DESIGN.
bool matvec_shape(MatvecArgs* a, int group, MatvecShape* shape) {
    const int tiles = a->tokens > 8 ? 2 : 1;
    const int fifo = kWarps * 6 * block_bytes(group);
    const int room = kSmem - fifo - kJoinBytes;
    int64_t best = INT64_MAX;
    for (int cluster = 1; cluster <= 8; cluster *= 2) {
        if (cluster > a->m.blocks) break;
        const int64_t blocks = (a->m.blocks + cluster - 1) / cluster;
        // Rows 64 bytes past a multiple of 128, so that two tokens' rows are on
        // different halves of the banks.
        const int64_t pitch = blocks * 2 * kBlock + 64;
        if (pitch * a->tokens > room) continue;
        const int64_t groups = std::min<int64_t>(clusters_at_once(rr_matvec_kernel<BF16, 128, 1, 1>, cluster), a->m.strips);
        const int64_t strips = (a->m.strips + groups - 1) / groups;
        for (int team = 1; team <= kWarps; team *= 2) {
            const int teams = kWarps / team;
            // (Warps stream on from batch to batch: whole rounds of the teams.)
            const bool alone = team == 1 && cluster == 1;
            const int64_t fit = kJoinBytes / (512 * tiles * team) / teams * teams;
            const int64_t batch = alone ? strips : std::min(strips, fit);
            const int64_t joins = alone ? 0 : (strips + batch - 1) / batch;
            // Runs of two blocks where they cost nothing.
            const int64_t one = (blocks + team - 1) / team, two = 2 * (((blocks + 1) / 2 + team - 1) / team);
            const int64_t steps = one;
            int64_t cost = 0;
            for (int64_t left = strips; left > 0; left -= batch)
                cost += (std::min(left, batch) + teams - 1) / teams * steps;
            cost += joins * (cluster > 1 ? 2 : 1);
            if (cost >= best) continue;
            best = cost;
            a->pitch = int32_t(pitch);
            a->team = team;
            a->cluster = cluster;
            a->batch = int32_t(batch);
            shape->run = two == one ? 2 : 1;
            shape->grid = unsigned(groups * cluster);
            shape->smem = fifo + int(pitch) * a->tokens
                          + (joins ? int(batch) * 512 * tiles * team : 0);
        }
    }
    return best != INT64_MAX;
}

cudaError_t launch_matvec(void (*kernel)(MatvecArgs), const MatvecArgs& a, const MatvecShape& shape,
                          cudaStream_t stream) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
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
    RR_TRY(check_device(packed, 16, "packed"));
    RR_TRY(check_device(x, 2, "x"));
    RR_TRY(check_device(out, f32 ? 4 : 2, "out"));
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
            while (!matvec_shape(&a, G, &shape)) {
                if (a.tokens == 1) return rr_fail(RR_ELAYOUT, "rows of %lld columns", (long long)q->cols);
                a.tokens = (a.tokens + 1) / 2;
            }
            const cudaError_t e =
                a.tokens > 8
                    ? shape.run == 2 ? launch_matvec(rr_matvec_kernel<T, G, 2, 2>, a, shape, stream)
                                     : launch_matvec(rr_matvec_kernel<T, G, 2, 1>, a, shape, stream)
                    : shape.run == 2 ? launch_matvec(rr_matvec_kernel<T, G, 1, 2>, a, shape, stream)
                                     : launch_matvec(rr_matvec_kernel<T, G, 1, 1>, a, shape, stream);
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
    RR_TRY(check_device(router, 16, "router"));
    RR_TRY(check_device(w13, 16, "w13"));
    RR_TRY(check_device(w2, 16, "w2"));
    RR_TRY(check_device(x, 2, "x"));
    RR_TRY(check_device(out, 2, "out"));
    if (ids) RR_TRY(check_device(ids, 4, "ids"));
    if (weights) RR_TRY(check_device(weights, 4, "weights"));
    RR_TRY(check_device(workspace, 16, "workspace"));
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
    a.logits = reinterpret_cast<float*>(ws + S.logits);
    a.chosen = reinterpret_cast<int32_t*>(ws + S.chosen);
    a.c = reinterpret_cast<float*>(ws + S.c);
    a.h = reinterpret_cast<float*>(ws + S.h);
    a.tokens = n_tokens;
    a.n_experts = L->n_experts;
    a.first = L->first_expert;
    a.n_local = L->n_local;
    a.top_k = L->top_k;
    a.norm = L->norm_topk;
    a.hidden = int32_t(L->hidden);
    a.inter = int32_t(L->inter);
    a.m13 = packed_of(2 * L->inter, L->hidden, L->group, 1);
    a.m2 = packed_of(L->hidden, L->inter, L->group, 0);
    return with_group(L->dtype, L->group, [&](auto t, auto g) -> rr_status {
        using T = decltype(t);
        constexpr int G = decltype(g)::value;
        rr_moe_logits_kernel<T><<<(n_tokens * a.n_experts + 3) / 4, 128, 0, stream>>>(a);
        rr_moe_choose_kernel<<<n_tokens, 32, 0, stream>>>(a);
        rr_moe_up_kernel<T, G><<<dim3((a.inter + 3) / 4, n_tokens * a.top_k), 128, 0, stream>>>(a);
        rr_moe_down_kernel<T, G><<<dim3((a.hidden + 3) / 4, n_tokens), 128, 0, stream>>>(a);
        RR_CUDA(cudaGetLastError());
        return RR_OK;
    });
}

extern "C" rr_status rr_moe_check(const rr_moe_layer* L, int32_t max_tokens, void* workspace,
                                  cudaStream_t stream) {
    rr_clear_error();
    RR_TRY(check_moe(L));
    if (max_tokens < 1 || max_tokens > RR_MOE_MAX_TOKENS)
        return rr_fail(RR_EINVAL, "%d tokens: 1..%d", max_tokens, RR_MOE_MAX_TOKENS);
    RR_TRY(check_device(workspace, 16, "workspace"));
    uint32_t err = 0;
    RR_CUDA(cudaMemcpyAsync(&err, workspace, 4, cudaMemcpyDeviceToHost, stream));
    RR_CUDA(cudaStreamSynchronize(stream));
    if (!err) return RR_OK;
    RR_CUDA(cudaMemsetAsync(workspace, 0, kControlBytes, stream));
    RR_CUDA(cudaStreamSynchronize(stream));
    return rr_fail(RR_ECUDA, "a wait between the layer's blocks ran out");
}
