// Attention of every sequence's newest tokens over the paged cache, for GB300 (sm_103a);
// include/rr.h has the definitions.
//
// Bound by HBM: every key and value of the listed sequences is read once, 4 dim bytes for
// 4 dim x (query heads per key head) x (new tokens) operations.  The work of a call is one
// line of units, 32 keys of one sequence, key head and tile of rows each; every warp of the
// grid takes an even, contiguous run of it, wherever sequences begin and end, so that
// short and long sequences load the SMs alike.  Where a run's edge cuts a tile's keys,
// the pieces (their softmax's maximum and sum, and their normalised output) are joined:
// among a block's warps, then, by the last of a tile's blocks to come, among blocks, in
// the order of the keys each time.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "rr_cache.cuh"

namespace {

constexpr int kUnit = 32;               // keys
constexpr int kMostBlocks = 192;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();
// A row's reference for its exponentials may stay this much (of log2) under its maximum.
constexpr float kSlack = 8.0f;

struct AttendArgs {
    CacheShape c;
    const char* pages;             // of the layer
    const int32_t *table, *lengths;
    int32_t* control;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t ldq, ldo;
    const int32_t *seqs, *starts;
    float* pieces;                 // the warps', then two a block
    uint32_t* arrived;             // per block: arrivals for the tile that starts in it and goes on
    int64_t piece_floats;
    int32_t n, rows, n_q, group;
    float scale;                   // with log2(e)
    int32_t qvec, ovec;
};

template <class T>
__device__ __forceinline__ void mma(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (std::is_same<T, BF16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two floats as one word of 16-bit elements, the first in the low half.
template <class T>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    if (std::is_same<T, BF16>::value) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The transpose of an 8 x 8 matrix of 16-bit elements, a word a lane.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// `bytes` (0..16) from global memory and zeros after them, to shared memory.
__device__ __forceinline__ void copy_async(uint32_t to, const void* from, int bytes) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds2(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void sts(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// What a kernel is compiled for: T, the element type; C, head sizes up to 64 C; NT, tiles
// of up to 8 NT rows.
template <class T_, int C_, int NT_>
struct Kind {
    using T = T_;
    static constexpr int C = C_, NT = NT_;
    static constexpr int kRows = 8 * NT;
    static constexpr int kWarps = C > 2 ? 4 : 8, kThreads = 32 * kWarps;
    static constexpr int kStage = C * 4096;                       // bytes of a unit's keys, or values
    static constexpr int kQ = NT * C * 1024;                      // bytes of a tile's queries
    static constexpr int kRoom = 224 * 1024 / kWarps;    // bytes a warp has
    static constexpr int kMost = (kRoom - kQ) / kStage;
    static constexpr int kStages = kMost > 6 ? 6 : kMost;
    static constexpr int kPieceFloats = kRows * (64 * C + 2);
    static constexpr int kWarpBytes = kQ + kStages * kStage;
    static constexpr int kSmem = kWarps * kWarpBytes;
    static_assert(kStages >= 2, "keys and values in turn");
    static_assert(kPieceFloats * 4 <= kWarpBytes, "a piece takes the place of the stages");
    // Bfloat16 keeps 8 bits of a weight: it enters the second product in two parts, 16
    // bits in all.  Float16's 11 bits are one part: as far off as the result's own
    // rounding is.  Its weights lie between 2^(7 - 2^..) and 2^15, so that those 2^-21 of
    // the largest still have all of their bits (under 2^-32 of it they are 0).
    static constexpr int kParts = std::is_same<T, BF16>::value ? 2 : 1;
    static constexpr float kLift = std::is_same<T, BF16>::value ? 0.0f : 7.0f;
};

// One tile of rows over one sequence's keys.  Row r of a sequence is head r % group of new
// token r / group.
struct Tile {
    int length, first, count;      // tokens of the sequence; its first new one among the call's, and how many
    int slot;                      // the sequence
    int head, tile;                // key head; which 8 NT rows
    int units;                     // of 32 keys
};

// The last key (+ 1) that a row sees.
__device__ __forceinline__ int seen(const Tile& t, int group, int row) { return t.length - t.count + 1 + row / group; }

// Where one warp's tile or one piece goes.
struct Ends {
    int64_t begin, end;            // the tile's units in the call's line; begin < 0: none
    Tile t;
};

// One listed sequence, checked: a sequence that does not fit has no units (and marks
// the cache).
__device__ __forceinline__ void load_seq(const AttendArgs& a, int i, int* slot, int* length, int* first, int* count) {
    *slot = a.seqs[i];
    *first = a.starts ? a.starts[i] : i;
    *count = a.starts ? a.starts[i + 1] - *first : 1;
    *length = a.c.has_seq(*slot) ? __ldg(&a.lengths[*slot]) : -1;
    if (!a.c.has_length(*length) || *first < 0 || *count < 0 || *count > a.rows || *first > a.rows - *count) {
        *length = 0;
        *count = 0;
        atomicOr(&a.control[kLate], kBadRange);
    }
}
__device__ __forceinline__ int units_of(int length) { return max((length + kUnit - 1) / kUnit, 1); }
template <class K>
__device__ __forceinline__ int tiles_of(const AttendArgs& a, int count) {
    return int((int64_t(count) * a.group + K::kRows - 1) / K::kRows);
}
template <class K>
__device__ __forceinline__ int64_t work_of(const AttendArgs& a, int length, int count) {
    return int64_t(a.c.n_kv) * tiles_of<K>(a, count) * units_of(length);
}

// The warps' runs: worker w has units [T w / N, T (w + 1) / N).
struct Line {
    int64_t total;
    int workers;
    __device__ __forceinline__ int64_t begin(int w) const { return total * min(w, workers) / workers; }
    // Whose run holds unit u.
    __device__ __forceinline__ int owner(int64_t u) const { return int(((u + 1) * workers - 1) / total); }
};

// ---------------------------------------------------------------------------
// Results
// ---------------------------------------------------------------------------

// Eight adjacent elements of the result, as T.
template <class T>
__device__ __forceinline__ void put8(uint16_t* to, int d, int dim, bool vec, const float* x) {
    if (vec && d + 8 <= dim) {
        *reinterpret_cast<uint4*>(to + d) =
            make_uint4(pack<T>(x[0], x[1]), pack<T>(x[2], x[3]), pack<T>(x[4], x[5]), pack<T>(x[6], x[7]));
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (d + k < dim) to[d + k] = T::round(x[k]);
}

// Puts a tile's results where they belong: to `piece` if that is given, else to the
// outputs.  o: normalised, as the products leave it: [nt][c][i][.], of the 64 c + 8 g + 2 i-th
// element and the next, of rows 8 nt + 2 t and the next.  top and sum: of those two rows.
template <class K>
__device__ __forceinline__ void emit(const AttendArgs& a, const Tile& t, float* piece, const float (&o)[K::NT][K::C][4][4],
                                     const float (&top)[K::NT][2], const float (&sum)[K::NT][2]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    const int left = t.count * a.group - t.tile * K::kRows;
#pragma unroll
    for (int nt = 0; nt < K::NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * nt + 2 * c4 + e;
            if (r >= left) continue;
            const int row = t.tile * K::kRows + r;
            const int64_t token = t.first + row / a.group;
            const int head = t.head * a.group + row % a.group;
#pragma unroll
            for (int c = 0; c < K::C; ++c) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] = o[nt][c][i][e];
                    x[2 * i + 1] = o[nt][c][i][2 + e];
                }
                if (piece) {
                    float4* to = reinterpret_cast<float4*>(piece + r * (64 * K::C) + 64 * c + 8 * g);
                    to[0] = make_float4(x[0], x[1], x[2], x[3]);
                    to[1] = make_float4(x[4], x[5], x[6], x[7]);
                } else {
                    put8<typename K::T>(a.out + token * a.ldo + int64_t(head) * a.c.dim, 64 * c + 8 * g, a.c.dim, a.ovec, x);
                }
            }
            if (g == 0) {
                if (piece) {
                    piece[64 * K::C * K::kRows + 2 * r] = top[nt][e];
                    piece[64 * K::C * K::kRows + 2 * r + 1] = sum[nt][e];
                } else if (a.lse) {
                    a.lse[token * a.n_q + head] = sum[nt][e] == 0.0f ? -kInf : (top[nt][e] + log2f(sum[nt][e])) * kLn2;
                }
            }
        }
    }
}

// A warp joins row r of n pieces, given by at(i): to `piece`, or, if that is NULL, to
// the outputs.  A piece counts by its sum at the largest of the maxima.
template <class K, bool FAR, class At>
__device__ __forceinline__ void join_row(const AttendArgs& a, const Tile& t, int r, int n, At at, float* piece) {
    constexpr int D = 64 * K::C, kMl = D * K::kRows;
    const int lane = threadIdx.x & 31;
    const auto get = [](const float* x) { return FAR ? __ldcg(x) : *x; };
    const auto get4 = [](const float4* x) { return FAR ? __ldcg(x) : *x; };
    float top = -kInf;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, get(at(i) + kMl + 2 * r));
#pragma unroll
    for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, m));
    const auto share = [&](int i) {
        const float m = get(at(i) + kMl + 2 * r);
        return m == -kInf ? 0.0f : get(at(i) + kMl + 2 * r + 1) * exp2f(m - top);
    };
    float sum = 0;
    for (int i = lane; i < n; i += 32) sum += share(i);
#pragma unroll
    for (int m = 16; m; m >>= 1) sum += __shfl_xor_sync(~0u, sum, m);
    const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
    // 8 adjacent elements a lane; lanes past the head's end help with other pieces.
    constexpr int kLanes = D / 8, kTeams = 32 / kLanes;
    const int d = 8 * (lane % kLanes), team = lane / kLanes;
    float x[8] = {};
    for (int base = 0; base < n; base += 32) {
        const float mine = base + lane < n ? share(base + lane) * inverse : 0.0f;
#pragma unroll 4
        for (int k = 0; k < min(n - base, 32); k += kTeams) {
            const int i = base + k + team;
            const float w = __shfl_sync(~0u, mine, (k + team) & 31);
            if (k + team >= 32 || i >= n || w == 0.0f) continue;
            const float4* from = reinterpret_cast<const float4*>(at(i) + r * D + d);
            const float4 u = get4(from), v = get4(from + 1);
            x[0] = fmaf(w, u.x, x[0]), x[1] = fmaf(w, u.y, x[1]), x[2] = fmaf(w, u.z, x[2]), x[3] = fmaf(w, u.w, x[3]);
            x[4] = fmaf(w, v.x, x[4]), x[5] = fmaf(w, v.y, x[5]), x[6] = fmaf(w, v.z, x[6]), x[7] = fmaf(w, v.w, x[7]);
        }
    }
#pragma unroll
    for (int m = kLanes; m < 32; m <<= 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] += __shfl_xor_sync(~0u, x[k], m);
    }
    if (team) return;
    if (piece) {
        float4* to = reinterpret_cast<float4*>(piece + r * D + d);
        to[0] = make_float4(x[0], x[1], x[2], x[3]);
        to[1] = make_float4(x[4], x[5], x[6], x[7]);
        if (lane == 0) piece[kMl + 2 * r] = top, piece[kMl + 2 * r + 1] = sum;
        return;
    }
    const int row = t.tile * K::kRows + r, head = t.head * a.group + row % a.group;
    const int64_t token = t.first + row / a.group;
    put8<typename K::T>(a.out + token * a.ldo + int64_t(head) * a.c.dim, d, a.c.dim, a.ovec, x);
    if (lane == 0 && a.lse) a.lse[token * a.n_q + head] = sum == 0.0f ? -kInf : (top + log2f(sum)) * kLn2;
}

// FAR: the pieces come from other blocks too.
template <class K, bool FAR, class At>
__device__ __forceinline__ void join(const AttendArgs& a, const Tile& t, int n, At at, float* piece) {
    const int rows = min(t.count * a.group - t.tile * K::kRows, K::kRows);
    for (int r = threadIdx.x >> 5; r < rows; r += K::kWarps) join_row<K, FAR>(a, t, r, n, at, piece);
}

// ---------------------------------------------------------------------------
// One warp's run
// ---------------------------------------------------------------------------

// Lane 4 g + t's part of a tile's query rows: of row 8 nt + g, elements 32 k + 8 t + 0..7.
template <class K>
__device__ __forceinline__ uint4 load_q(const AttendArgs& a, const Tile& t, int nt, int k) {
    const int lane = threadIdx.x & 31, row = t.tile * K::kRows + 8 * nt + (lane >> 2), d = 32 * k + 8 * (lane & 3);
    if (row >= t.count * a.group || d >= a.c.dim) return make_uint4(0, 0, 0, 0);
    const uint16_t* from = a.q + (t.first + row / a.group) * a.ldq + int64_t(t.head * a.group + row % a.group) * a.c.dim + d;
    if (a.qvec) return *reinterpret_cast<const uint4*>(from);
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = d + e < a.c.dim ? from[e] : 0u;
    return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}

// The scores of 32 keys: s[h][nt][.] of keys 8 (h) + g (and 8 more in [2], [3]) of each half h of 16, rows
// 8 nt + 2 t and the next.
template <class K>
__device__ __forceinline__ void mask(const AttendArgs& a, const Tile& t, int key0, float (&s)[2][K::NT][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
#pragma unroll
    for (int nt = 0; nt < K::NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int end = seen(t, a.group, t.tile * K::kRows + 8 * nt + 2 * c4 + e) - key0 - g;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (16 * h >= end) s[h][nt][e] = -kInf;
                if (16 * h + 8 >= end) s[h][nt][2 + e] = -kInf;
            }
        }
    }
}

// The address of 8 adjacent tokens of a page, or NULL past the sequence's end.
__device__ __forceinline__ const char* tokens8(const AttendArgs& a, const Tile& t, int key, int id) {
    if (key >= t.length) return nullptr;
    return a.pages + id * a.c.page_bytes + t.head * a.c.run_bytes + (key & (a.c.page - 1)) * (2 * a.c.pitch);
}

// Units [u0, u1) of a tile once more, one key after another, for values that are not
// finite or nearly too large: a product of weight and value only where the row sees the
// key, weights in float32 and 2^-32 of what they are, so that sums stay finite.
template <class K>
__device__ __noinline__ void carefully(const AttendArgs& a, const Tile& t, int u0, int u1, float* piece) {
    using T = typename K::T;
    const int lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3;
    float o[K::NT][K::C][4][4] = {}, top[K::NT][2], sum[K::NT][2] = {};
#pragma unroll
    for (int nt = 0; nt < K::NT; ++nt) top[nt][0] = top[nt][1] = -kInf;
    for (int pass = 0; pass < 2; ++pass) {
        for (int u = u0; u < u1; ++u) {
            const int key0 = u * kUnit;
            float s[2][K::NT][4] = {};
            const char* at[4];
            for (int h = 0; h < 4; ++h) {
                const int key = key0 + 8 * h;
                int id = key < t.length ? __ldcg(&a.table[int64_t(t.slot) * a.c.max_pages + (key >> a.c.shift)]) : -1;
                at[h] = a.c.has_page(id) ? tokens8(a, t, key, id) : nullptr;
            }
#pragma unroll 1
            for (int k = 0; k < 2 * K::C; ++k) {
                uint4 r[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    r[h] = make_uint4(0, 0, 0, 0);
                    const int d = 32 * k + 8 * c4;
                    if (!at[h] || key0 + 8 * h + g >= t.length || d >= a.c.dim) continue;
                    r[h] = *reinterpret_cast<const uint4*>(at[h] + g * (2 * a.c.pitch) + 2 * d);
                    // (The pad behind the last element is not looked at.)
                    uint32_t* w = &r[h].x;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if (d + 2 * x >= a.c.dim) w[x] = 0;
                        else if (d + 2 * x + 1 >= a.c.dim) w[x] &= 0xFFFFu;
                    }
                }
#pragma unroll
                for (int nt = 0; nt < K::NT; ++nt) {
                    const uint4 b = load_q<K>(a, t, nt, k);
                    mma<T>(s[0][nt], r[0].x, r[1].x, r[0].y, r[1].y, b.x, b.y);
                    mma<T>(s[0][nt], r[0].z, r[1].z, r[0].w, r[1].w, b.z, b.w);
                    mma<T>(s[1][nt], r[2].x, r[3].x, r[2].y, r[3].y, b.x, b.y);
                    mma<T>(s[1][nt], r[2].z, r[3].z, r[2].w, r[3].w, b.z, b.w);
                }
            }
#pragma unroll
            for (int nt = 0; nt < K::NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[h][nt][e] *= a.scale;
            mask<K>(a, t, key0, s);
            if (pass == 0) {
#pragma unroll
                for (int nt = 0; nt < K::NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float m = fmaxf(fmaxf(s[0][nt][e], s[0][nt][2 + e]), fmaxf(s[1][nt][e], s[1][nt][2 + e]));
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, x));
                        top[nt][e] = fmaxf(top[nt][e], m);
                    }
                continue;
            }
#pragma unroll
            for (int nt = 0; nt < K::NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float m = top[nt][e & 1] == -kInf ? 0.0f : top[nt][e & 1];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        s[h][nt][e] = exp2f(s[h][nt][e] - m);
                        sum[nt][e & 1] += s[h][nt][e];
                    }
                }
#pragma unroll 1
            for (int x = 0; x < kUnit; ++x) {
                if (key0 + x >= t.length) break;
                const char* from = at[x >> 3];
#pragma unroll
                for (int nt = 0; nt < K::NT; ++nt) {
                    const int other = (x & 7) * 4 + c4;
                    float p[2];
                    bool sees[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float lo = x & 16 ? s[1][nt][e] : s[0][nt][e], hi = x & 16 ? s[1][nt][2 + e] : s[0][nt][2 + e];
                        p[e] = __shfl_sync(~0u, x & 8 ? hi : lo, other) * 0x1p-32f;
                        sees[e] = key0 + x < seen(t, a.group, t.tile * K::kRows + 8 * nt + 2 * c4 + e);
                    }
#pragma unroll
                    for (int c = 0; c < K::C; ++c) {
                        const int d = 64 * c + 8 * g;
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (from && d < a.c.pitch)
                            v = *reinterpret_cast<const uint4*>(from + int64_t(a.c.n_kv) * a.c.run_bytes + (x & 7) * (2 * a.c.pitch) + 2 * d);
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                if (!sees[e]) continue;
                                o[nt][c][i][e] = fmaf(p[e], T::widen(uint16_t(w[i])), o[nt][c][i][e]);
                                o[nt][c][i][2 + e] = fmaf(p[e], T::widen(uint16_t(w[i] >> 16)), o[nt][c][i][2 + e]);
                            }
                    }
                }
            }
        }
    }
#pragma unroll
    for (int nt = 0; nt < K::NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) sum[nt][e] += __shfl_xor_sync(~0u, sum[nt][e], x);
            const float inverse = sum[nt][e] == 0.0f ? 0.0f : 0x1p32f / sum[nt][e];
#pragma unroll
            for (int c = 0; c < K::C; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    o[nt][c][i][e] *= inverse;
                    o[nt][c][i][2 + e] *= inverse;
                }
        }
    emit<K>(a, t, piece, o, top, sum);
}

// Walks the listed sequences' tiles from a place in the call's line on; 32 sequences'
// numbers at a time, one a lane.
template <class K>
struct Walk {
    const AttendArgs& a;
    int seq, batch;                      // the current sequence, the first one of the loaded ones
    int slot_, length_, first_, count_;  // lane l: of sequence batch + l
    Tile t;
    __device__ __forceinline__ Walk(const AttendArgs& args, int i) : a(args), seq(i), batch(i) { load(); }
    __device__ __forceinline__ void load() {
        const int i = batch + int(threadIdx.x & 31);
        slot_ = length_ = first_ = count_ = 0;
        if (i < a.n) load_seq(a, i, &slot_, &length_, &first_, &count_);
    }
    __device__ __forceinline__ void enter() {
        const int l = seq - batch;
        t.slot = __shfl_sync(~0u, slot_, l);
        t.length = __shfl_sync(~0u, length_, l);
        t.first = __shfl_sync(~0u, first_, l);
        t.count = __shfl_sync(~0u, count_, l);
        t.units = units_of(t.length);
        t.head = t.tile = 0;
    }
    // The next tile; there is one.  The tiles of a key head follow one another.
    __device__ __forceinline__ void next() {
        if (++t.tile < tiles_of<K>(a, t.count)) return;
        t.tile = 0;
        if (++t.head < a.c.n_kv) return;
        do {
            if (++seq >= a.n) return;
            if (seq == batch + 32) {
                batch = seq;
                load();
            }
            enter();
        } while (t.count == 0);
    }
};

// What a unit's copies and its products need to agree on, in shared memory.
template <class K>
struct Shared {
    Ends heads[K::kWarps], tails[K::kWarps];
    int64_t scan[K::kWarps];
    int64_t starts[K::kWarps];       // where a warp's run begins within its first sequence
    int seqs[K::kWarps];
    int last;
    Tile ring[K::kWarps][4];
};

template <class K>
__global__ void __launch_bounds__(K::kThreads, 1) rr_attend_kernel(const __grid_constant__ AttendArgs a) {
    using T = typename K::T;
    constexpr int C = K::C, NT = K::NT, W = K::kWarps;
    extern __shared__ __align__(128) char memory[];
    __shared__ Shared<K> sh;
    after_previous();
    if (__ldcg(&a.control[kState])) return;
    const int lane = threadIdx.x & 31, g = lane >> 2, c4 = lane & 3, w = threadIdx.x >> 5;

    // The line, and where this block's warps begin in it.
    Line line;
    int64_t mine = 0;
    int64_t kept = 0;
    for (int i = threadIdx.x; i < a.n; i += K::kThreads) {
        int slot, length, first, count;
        load_seq(a, i, &slot, &length, &first, &count);
        kept = work_of<K>(a, length, count);
        mine += kept;
    }
    const auto scan = [&](int64_t v, int64_t* total) {
        int64_t s = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t o = __shfl_up_sync(~0u, s, d);
            if (lane >= d) s += o;
        }
        if (lane == 31) sh.scan[w] = s;
        __syncthreads();
        int64_t before = 0, all = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (i < w) before += sh.scan[i];
            all += sh.scan[i];
        }
        __syncthreads();
        *total = all;
        return before + s - v;
    };
    scan(mine, &line.total);
    if (line.total == 0) return;
    // Blocks of a few units a warp where there are few.
    constexpr int kLeast = 2 * W;
    const int blocks = int(min(int64_t(gridDim.x), (line.total + kLeast - 1) / kLeast));
    if (int(blockIdx.x) >= blocks) return;
    line.workers = int(min(int64_t(blocks) * W, line.total));      // (so that none is without units between others)
    const int worker = blockIdx.x * W + w;
    {
        int64_t before = 0;
        const int64_t last = line.begin(blockIdx.x * W + W - 1);
        for (int base = 0; base < a.n && before <= last; base += K::kThreads) {
            const int i = base + int(threadIdx.x);
            int64_t work = kept;
            if (a.n > K::kThreads) {
                int slot, length, first, count;
                work = 0;
                if (i < a.n) {
                    load_seq(a, i, &slot, &length, &first, &count);
                    work = work_of<K>(a, length, count);
                }
            }
            int64_t total;
            const int64_t at = before + scan(work, &total);
#pragma unroll
            for (int x = 0; x < W; ++x) {
                const int64_t u = line.begin(blockIdx.x * W + x);
                if (u >= at && u < at + work) {
                    sh.seqs[x] = i;
                    sh.starts[x] = u - at;
                }
            }
            before += total;
        }
        if (lane == 0) sh.heads[w].begin = sh.tails[w].begin = -1;
        __syncthreads();
    }

    char* const own = memory + w * K::kWarpBytes;
    const uint32_t q_at = uint32_t(__cvta_generic_to_shared(own)), stage_at = q_at + K::kQ;
    const int64_t begin = line.begin(worker), end = line.begin(worker + 1);
    if (begin < end) {
        // The copies' side: iteration `made` is the next whose keys are asked for.
        Walk<K> walk(a, sh.seqs[w]);
        walk.enter();
        int unit;                        // of the walk's tile: the next iteration's
        {
            const int64_t at = sh.starts[w], tile = at / walk.t.units;
            const int tiles = tiles_of<K>(a, walk.t.count);
            unit = int(at - tile * walk.t.units);
            walk.t.head = int(tile / tiles);
            walk.t.tile = int(tile % tiles);
        }
        const int64_t first_tile = begin - unit;      // the first tile's begin in the line
        const int first_unit = unit;
        int64_t made = begin;
        int ids = -1;                    // lane h < 4: the page of the next iteration's tokens 8 h on
        const auto fetch_ids = [&] {
            ids = -1;
            const int key = unit * kUnit + 8 * lane;
            if (made < end && lane < 4 && key < walk.t.length) {
                ids = __ldg(&a.table[int64_t(walk.t.slot) * a.c.max_pages + (key >> a.c.shift)]);
                if (!a.c.has_page(ids)) {
                    ids = -1;
                    atomicOr(&a.control[kLate], kBadTable);
                }
            }
        };
        fetch_ids();
        const char* at[4];               // the tokens whose values are asked for next
        int valid[4];                    // how many of the 8 there are
        uint32_t stage_in = stage_at, stage_out = stage_at;
        const auto step = [&](uint32_t* s) {
            *s += K::kStage;
            if (*s == stage_at + K::kStages * K::kStage) *s = stage_at;
        };
        const int64_t to_values = int64_t(a.c.n_kv) * a.c.run_bytes;
        const int row_bytes = 2 * a.c.pitch, dim_bytes = 2 * a.c.dim;
        const auto ask_keys = [&] {
            if (made < end) {
                if (lane == 0) sh.ring[w][made & 3] = walk.t;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int key = unit * kUnit + 8 * h, id = __shfl_sync(~0u, ids, h);
                    valid[h] = id < 0 ? 0 : min(walk.t.length - key, 8);
                    at[h] = id < 0 ? a.pages
                                   : a.pages + id * a.c.page_bytes + walk.t.head * a.c.run_bytes + (key & (a.c.page - 1)) * row_bytes;
                }
#pragma unroll
                for (int k = 0; k < 2 * C; ++k) {
                    const int d = 64 * k + 16 * c4, bytes = min(max(dim_bytes - d, 0), 16);
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const bool there = g < valid[h] && bytes;
                        copy_async(stage_in + (k * 4 + h) * 512 + lane * 16, there ? at[h] + g * row_bytes + d : a.pages, there ? bytes : 0);
                    }
                }
                // On to the next iteration, but for what the values need.
                ++made;
                if (++unit == walk.t.units) {
                    unit = 0;
                    if (made < end) walk.next();
                }
                fetch_ids();
            } else {
#pragma unroll
                for (int h = 0; h < 4; ++h) valid[h] = -1;
            }
            copies_end();
            step(&stage_in);
        };
        const auto ask_values = [&] {
            if (valid[0] >= 0) {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int d = 128 * c + 16 * g, bytes = min(max(dim_bytes - d, 0), 16);
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const bool there = 2 * c4 + e < valid[h] && bytes;
                            copy_async(stage_in + (c * 8 + h * 2 + e) * 512 + lane * 16,
                                       there ? at[h] + to_values + (2 * c4 + e) * row_bytes + d : a.pages, there ? bytes : 0);
                        }
                    }
                }
            }
            copies_end();
            step(&stage_in);
        };
        bool keys_next = true;
        const auto ask = [&] {
            if (keys_next) ask_keys();
            else ask_values();
            keys_next = !keys_next;
        };
#pragma unroll
        for (int i = 0; i < K::kStages; ++i) ask();

        // The products' side.
        float o[NT][C][4][4], top[NT][2], sum[NT][2];
        uint4 q1[NT == 1 ? 2 * C : 1];
        Tile t;
        int u = 0, u0 = 0;
        int64_t tile_begin = 0;
        bool fresh = true;
        __syncwarp();
        for (int64_t done = begin; done < end; ++done) {
            if (fresh) {
                __syncwarp();
                t = sh.ring[w][done & 3];
                u = u0 = done == begin ? first_unit : 0;
                tile_begin = done == begin ? first_tile : done;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    top[nt][0] = top[nt][1] = -kInf;
                    sum[nt][0] = sum[nt][1] = 0;
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[nt][c][i][e] = 0;
#pragma unroll
                    for (int k = 0; k < 2 * C; ++k) {
                        const uint4 x = load_q<K>(a, t, nt, k);
                        if (NT == 1) q1[k] = x;
                        else sts(q_at + (nt * 2 * C + k) * 512 + lane * 16, x);
                    }
                }
                fresh = false;
            }
            const int key0 = u * kUnit;
            float s[2][NT][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[h][nt][e] = 0;
            copies_wait<K::kStages - 1>();
#pragma unroll
            for (int k = 0; k < 2 * C; ++k) {
                uint4 r[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) r[h] = lds(stage_out + (k * 4 + h) * 512 + lane * 16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 b = NT == 1 ? q1[NT == 1 ? k : 0] : lds(q_at + (nt * 2 * C + k) * 512 + lane * 16);
                    mma<T>(s[0][nt], r[0].x, r[1].x, r[0].y, r[1].y, b.x, b.y);
                    mma<T>(s[1][nt], r[2].x, r[3].x, r[2].y, r[3].y, b.x, b.y);
                    mma<T>(s[0][nt], r[0].z, r[1].z, r[0].w, r[1].w, b.z, b.w);
                    mma<T>(s[1][nt], r[2].z, r[3].z, r[2].w, r[3].w, b.z, b.w);
                }
            }
            step(&stage_out);
            ask();

            // Weights 2^(s - top + lift); `top` moves only where a score is far over it.
            bool far = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[h][nt][e] *= a.scale;
            if (key0 + kUnit > seen(t, a.group, t.tile * K::kRows)) mask<K>(a, t, key0, s);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float m = fmaxf(fmaxf(s[0][nt][e], s[0][nt][2 + e]), fmaxf(s[1][nt][e], s[1][nt][2 + e]));
                    far |= m > top[nt][e] + kSlack;
                }
            if (__any_sync(~0u, far)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float m = fmaxf(fmaxf(s[0][nt][e], s[0][nt][2 + e]), fmaxf(s[1][nt][e], s[1][nt][2 + e]));
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, x));
                        m = fmaxf(m, top[nt][e]);
                        const float f = m == top[nt][e] ? 1.0f : exp2f(top[nt][e] - m);
                        top[nt][e] = m;
                        sum[nt][e] *= f;
#pragma unroll
                        for (int c = 0; c < C; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                o[nt][c][i][e] *= f;
                                o[nt][c][i][2 + e] *= f;
                            }
                    }
            }
            uint32_t p[K::kParts][2][NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m0 = top[nt][0] == -kInf ? 0.0f : top[nt][0] - K::kLift, m1 = top[nt][1] == -kInf ? 0.0f : top[nt][1] - K::kLift;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[h][nt][e] = exp2f(s[h][nt][e] - (e & 1 ? m1 : m0));
                        sum[nt][e & 1] += s[h][nt][e];
                    }
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float lo = s[h][nt][2 * x], hi = s[h][nt][2 * x + 1];
                        const uint32_t big = pack<T>(lo, hi);
                        p[0][h][nt][x] = transposed(big);
                        if (K::kParts == 2)
                            p[K::kParts - 1][h][nt][x] = transposed(pack<T>(lo - T::widen(uint16_t(big)), hi - T::widen(uint16_t(big >> 16))));
                    }
                }
            }

            // Sums over 32 keys from zero by the matrix instructions, which cut off, added in
            // float32, which rounds.
            copies_wait<K::kStages - 1>();
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint2 v[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[x] = lds2(stage_out + (c * 8 + x) * 512 + lane * 16 + half * 8);
#pragma unroll
                    for (int i2 = 0; i2 < 2; ++i2) {
                        uint32_t f[2][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t v0 = i2 ? v[4 * h].y : v[4 * h].x, v1 = i2 ? v[4 * h + 1].y : v[4 * h + 1].x;
                            const uint32_t v2 = i2 ? v[4 * h + 2].y : v[4 * h + 2].x, v3 = i2 ? v[4 * h + 3].y : v[4 * h + 3].x;
                            f[h][0] = __byte_perm(v0, v1, 0x5410);
                            f[h][1] = __byte_perm(v0, v1, 0x7632);
                            f[h][2] = __byte_perm(v2, v3, 0x5410);
                            f[h][3] = __byte_perm(v2, v3, 0x7632);
                        }
                        const int i = 2 * half + i2;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float d[4] = {0, 0, 0, 0};
#pragma unroll
                            for (int part = K::kParts - 1; part >= 0; --part)
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    mma<T>(d, f[h][0], f[h][1], f[h][2], f[h][3], p[part][h][nt][0], p[part][h][nt][1]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[nt][c][i][e] += d[e];
                        }
                    }
                }
            }
            step(&stage_out);
            ask();

            ++u;
            if (u < t.units && done + 1 < end) continue;
            // The run leaves this tile.
            float* piece = nullptr;
            const bool ends = u == t.units, whole = ends && tile_begin >= begin;
            if (!whole && ends) piece = a.pieces + worker * a.piece_floats;
            if (!ends) {
                // The stages are free: nothing is asked for any more.
                copies_wait<0>();
                __syncwarp();
                piece = reinterpret_cast<float*>(own);
            }
            if (lane == 0 && !whole) {
                Ends& e = ends ? sh.heads[w] : sh.tails[w];
                e.begin = tile_begin;
                e.end = tile_begin + t.units;
                e.t = t;
            }
            bool odd = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) sum[nt][e] += __shfl_xor_sync(~0u, sum[nt][e], x);
                    const float inverse = sum[nt][e] == 0.0f ? 0.0f : 1.0f / sum[nt][e];
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            o[nt][c][i][e] *= inverse;
                            o[nt][c][i][2 + e] *= inverse;
                            // (A row whose sum is NaN is all NaN in any case.)
                            odd |= sum[nt][e] == sum[nt][e] && !(fabsf(o[nt][c][i][e]) < kInf && fabsf(o[nt][c][i][2 + e]) < kInf);
                        }
                    if (top[nt][e] != -kInf) top[nt][e] -= K::kLift;
                }
            if (__any_sync(~0u, odd)) carefully<K>(a, t, u0, u, piece);
            else emit<K>(a, t, piece, o, top, sum);
            fresh = true;
        }
        copies_wait<0>();
    }
    __syncthreads();

    // Joins: of the tiles that end here after an earlier warp's run, then of the one that
    // goes on in the next block.
    const int64_t block_begin = line.begin(blockIdx.x * W);
    const auto tail_of = [&](int x) { return reinterpret_cast<const float*>(memory + x * K::kWarpBytes); };
    float* const block_pieces = a.pieces + int64_t(gridDim.x) * W * a.piece_floats;
    for (int x = 0; x <= W; ++x) {
        // (x = W: the tail that goes on.)
        const Ends& e = x < W ? sh.heads[x] : sh.tails[W - 1];
        if (e.begin < 0) continue;
        int from = x < W ? x : W - 1;
        while (from > 0 && sh.tails[from - 1].begin == e.begin) --from;
        const int n = (x < W ? x : W - 1) - from + 1;
        const auto at = [&](int i) { return x < W && i == n - 1 ? a.pieces + (int64_t(blockIdx.x) * W + x) * a.piece_floats : tail_of(from + i); };
        const bool before = e.begin < block_begin, after = x == W;
        if (!before && !after) {
            join<K, false>(a, e.t, n, at, nullptr);
            continue;
        }
        // Of a tile that several blocks share: this block's part, and, for the last of them to
        // come, the whole.
        join<K, false>(a, e.t, n, at, block_pieces + (2 * int64_t(blockIdx.x) + !before) * a.piece_floats);
        const int b0 = line.owner(e.begin) / W, b1 = line.owner(e.end - 1) / W;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            sh.last = atomicAdd(&a.arrived[b0], 1) == unsigned(b1 - b0);
            if (sh.last) a.arrived[b0] = 0;
        }
        __syncthreads();
        if (sh.last) {
            __threadfence();
            join<K, true>(a, e.t, b1 - b0 + 1,
                    [&](int i) { return block_pieces + (2 * int64_t(b0 + i) + (i == 0)) * a.piece_floats; }, nullptr);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int64_t kArrivedBytes = kMostBlocks * 4;

// The largest piece of a cache's head size.
int64_t piece_floats(const rr_cache* C) {
    return C->dim <= 64 ? Kind<BF16, 1, 5>::kPieceFloats : C->dim <= 128 ? Kind<BF16, 2, 5>::kPieceFloats : Kind<BF16, 4, 2>::kPieceFloats;
}
int64_t workspace_of(const rr_cache* C) { return kArrivedBytes + int64_t(kMostBlocks) * (C->dim > 128 ? 4 + 2 : 8 + 2) * piece_floats(C) * 4; }

rr_status check_heads(const rr_cache* C, int32_t n_q) {
    if (n_q < 1 || n_q % C->n_kv || n_q / C->n_kv > 1024)
        return rr_fail(RR_ELAYOUT, "%d query heads of %d key heads: a multiple, up to 1024 times", n_q, C->n_kv);
    return RR_OK;
}

template <class K>
rr_status launch(AttendArgs& a, int dev, cudaStream_t stream) {
    static std::atomic<uint32_t> ready{0};
    static std::atomic<int> sms[kMaxDevices] = {};
    RR_CUDA(allow_smem(rr_attend_kernel<K>, K::kSmem, dev, &ready));
    int grid = sms[dev].load(std::memory_order_relaxed);
    if (!grid) {
        RR_CUDA(cudaDeviceGetAttribute(&grid, cudaDevAttrMultiProcessorCount, dev));
        sms[dev].store(grid, std::memory_order_relaxed);
    }
    grid = std::min(grid, kMostBlocks);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(grid));
    cfg.blockDim = dim3(K::kThreads);
    cfg.dynamicSmemBytes = K::kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    RR_CUDA(cudaLaunchKernelEx(&cfg, rr_attend_kernel<K>, a));
    return RR_OK;
}

// The rows that a tile is to hold: of sequences of the call's mean number of new tokens,
// and up to as many again.
template <class T, int C>
rr_status choose(AttendArgs& a, int dev, cudaStream_t stream) {
    const int mean = (a.rows + a.n - 1) / a.n, most = std::min(2 * mean - 1, a.rows - a.n + 1);
    const int64_t rows = int64_t(a.group) * std::max(most, 1);
    if (rows <= 8) return launch<Kind<T, C, 1>>(a, dev, stream);
    if constexpr (C <= 2) {
        if (rows > 16) return launch<Kind<T, C, 5>>(a, dev, stream);
    }
    return launch<Kind<T, C, 2>>(a, dev, stream);
}

}  // namespace

extern "C" rr_status rr_attend_workspace(const rr_cache* C, int32_t n_q, int64_t* bytes) {
    rr_clear_error();
    RR_TRY(check_cache(C));
    RR_TRY(check_heads(C, n_q));
    if (!bytes) return rr_fail(RR_EINVAL, "bytes is NULL");
    *bytes = workspace_of(C);
    return RR_OK;
}

extern "C" rr_status rr_attend(const rr_cache* C, const void* pages, void* book, int32_t layer, const void* q, int64_t ldq, int32_t n_q,
                               int32_t rows, void* out, int64_t ldo, float* lse, const int32_t* seqs, const int32_t* starts, int32_t n,
                               float scale, void* workspace, int64_t workspace_bytes, cudaStream_t stream) {
    RR_TRACE("rr_attend");
    rr_clear_error();
    RR_TRY(check_cache(C));
    RR_TRY(check_heads(C, n_q));
    if (n < 0 || rows < 0 || (!starts && rows != n)) return rr_fail(RR_EINVAL, "%d rows of %d sequences", rows, n);
    if (layer < 0 || layer >= C->layers) return rr_fail(RR_EINVAL, "layer %d of %d", layer, C->layers);
    const int64_t cols = int64_t(n_q) * C->dim;
    if (ldq < cols || ldo < cols)
        return rr_fail(RR_EINVAL, "row strides %lld and %lld of rows of %lld", (long long)ldq, (long long)ldo, (long long)cols);
    if (workspace_bytes < workspace_of(C))
        return rr_fail(RR_EINVAL, "workspace of %lld bytes, the call needs %lld", (long long)workspace_bytes, (long long)workspace_of(C));
    if (n == 0 || rows == 0) return RR_OK;
    if (int64_t(rows) * (n_q / C->n_kv) > INT_MAX / 2) return rr_fail(RR_ELAYOUT, "%d rows of %d heads", rows, n_q);
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, pages, 16, "pages"));
    RR_TRY(check_device(dev, book, 16, "book"));
    RR_TRY(check_device(dev, q, 2, "q"));
    RR_TRY(check_device(dev, out, 2, "out"));
    if (lse) RR_TRY(check_device(dev, lse, 4, "lse"));
    RR_TRY(check_device(dev, seqs, 4, "seqs"));
    if (starts) RR_TRY(check_device(dev, starts, 4, "starts"));
    RR_TRY(check_device(dev, workspace, 16, "workspace"));
    Book b;
    book_of(C, book, &b);
    AttendArgs a;
    a.c = shape_of(C);
    a.pages = static_cast<const char*>(pages) + layer * a.c.layer_bytes;
    a.table = b.table;
    a.lengths = b.lengths;
    a.control = b.control;
    a.q = static_cast<const uint16_t*>(q);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.ldq = ldq;
    a.ldo = ldo;
    a.seqs = seqs;
    a.starts = starts;
    a.arrived = static_cast<uint32_t*>(workspace);
    a.pieces = reinterpret_cast<float*>(static_cast<char*>(workspace) + kArrivedBytes);
    a.piece_floats = piece_floats(C);
    a.n = n;
    a.rows = rows;
    a.n_q = n_q;
    a.group = n_q / C->n_kv;
    a.scale = scale * kLog2e;
    a.qvec = (uintptr_t)q % 16 == 0 && ldq % 8 == 0 && C->dim % 8 == 0;
    a.ovec = (uintptr_t)out % 16 == 0 && ldo % 8 == 0 && C->dim % 8 == 0;
    const auto with = [&](auto t) -> rr_status {
        using T = decltype(t);
        if (C->dim <= 64) return choose<T, 1>(a, dev, stream);
        if (C->dim <= 128) return choose<T, 2>(a, dev, stream);
        return choose<T, 4>(a, dev, stream);
    };
    return C->dtype == RR_DST_F16 ? with(F16{}) : with(BF16{});
}
