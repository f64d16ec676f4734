// Attention of every sequence's newest tokens over the paged cache, for GB300 (sm_103a);
// include/rr.h has the definitions.
//
// Bound by HBM: every key and value of the listed sequences is read once, 4 dim bytes for
// 4 dim x (query heads per key head) x (new tokens) operations.  The work of a call is one
// line of units, 128 keys of one sequence, key head and tile of rows each; every block (one
// an SM) takes an even, contiguous run of it, wherever sequences begin and end, so that
// short and long sequences load the SMs alike.  Where a run's edge cuts a tile's keys,
// the pieces (their softmax's maximum and sum, and their normalised output) are joined by
// the last of the tile's blocks to come, in the order of the keys each time.
//
// Within a block, per unit: two warps have the pages' keys and values copied to shared
// memory by TMA, which lays them out as the matrix instructions want them and fills what is
// past a head's end with zeros; one thread issues tcgen05 products,
//     S^T [128 keys, rows] = K Q^T,    D^T [dim, rows] = V^T P^T,
// with keys, then head elements, as the 128 rows of the accumulator in TMEM, so that
// a few rows of queries cost few columns and keys and values go from shared memory into the
// product as they lie; eight or twelve warps turn scores into weights; one more warp fetches
// the next tile's queries.  S^T of the next unit is computed while the softmax of this
// one runs.
//
// Measured: 64 sequences of 200 to 16000 tokens, 32 heads over 4 key heads of 128 (1.06 GB):
// 172 to 176 us, 6.1 TB/s (the SMs' mean is done after 155, the last after 166); 96 of 500 to
// 7500, 64 over 8, five tokens each (1.59 GB): 288 us, 5.5 TB/s; one of 40001, 32 over 8
// (164 MB): 36 us, 4.6 TB/s.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include <cuda.h>
#include <cudaTypedefs.h>

#include "rr_cache.cuh"

namespace {

constexpr int kUnit = 128;              // keys
constexpr int kGather = 8;              // units whose sums gather in TMEM
constexpr int kMostBlocks = 192;
constexpr int kListed = 128;            // sequences whose numbers a block keeps (loading them again: 1 us)
constexpr int kMostStages = 12;
constexpr int kSmem = 220 * 1024;       // of a block, beside its static part
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();
// A row's reference for its exponentials may stay this much (of log2) under its maximum.
constexpr float kSlack = 8.0f;
// In place of minus the reference of a row that has seen nothing yet: any score but the least float
// is above it by more than the slack.
constexpr float kNothing = FLT_MAX;
constexpr long long kWaitCycles = 4000000000;

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
    float* pieces;                 // two a block
    uint32_t* arrived;             // per block: arrivals for the tile that starts in it and goes on
    int64_t piece_floats;
    int32_t n, rows, n_q, group;
    int32_t stages, atoms;         // of the ring; 64 elements of a head each
    // Of a unit's keys or values in shared memory, where 8 tokens' 64 elements are 1 KiB together:
    // from 64 elements to the next, from 8 tokens to the next; and how many elements one copy has.
    int32_t atom_bytes, eight_bytes, copy_atoms;
    float scale;                   // with log2(e)
    int32_t qvec, ovec;
};

// What a kernel is compiled for: T, the element type; MT, head sizes up to 128 MT; NG, tiles
// of up to 8 NG rows.
template <class T_, int MT_, int NG_>
struct Kind {
    using T = T_;
    static constexpr int MT = MT_, NG = NG_;
    static constexpr int kRows = 8 * NG;
    static constexpr int D = 128 * MT;
    // Sets of four softmax warps; copies, products and queries have a warp each.  (96 sequences of
    // five tokens of 8 heads each: 2 sets 327 us, 3 314, 4 338)
    static constexpr int kSets = NG == 8 ? 3 : 2;
    static constexpr int kSoft = 128 * kSets, kThreads = kSoft + 128;
    static constexpr int kKeys = kSoft / 32, kValues = kKeys + 1, kProducts = kKeys + 2, kQueries = kKeys + 3;
    // A weight enters the second product in two parts: of bfloat16 16 bits in all, of float16 22.
    // (One part is off by up to half of its last bit: float16's 2^-12 would be as much as a result's
    // own rounding, and more than that where values cancel.)  Float16's weights are 2^7 to 2^15 at
    // a row's maximum, so that those 2^-21 of the largest still have all bits of their first
    // part; the second ends at 2^-32 of it.  (Float16's second part: nothing up to 16 rows, and of 64
    // rows a stage of the ring: 96 sequences of five tokens of 8 heads each 288 us, 263 with one.)
    static constexpr int kParts = 2;
    static constexpr float kLift = std::is_same<T, BF16>::value ? 0.0f : 7.0f;
    static constexpr int kQ = MT * NG * 2048;           // bytes of a tile's queries
    static constexpr int kP = NG * 2048;                // of one part of the weights
    // What a tile costs beside its units, in halves of one (its first reference, its results).
    static constexpr int kOpen = NG == 2 ? 1 : 4;
    // A tile's sums: in registers, or, of many rows, in shared memory.  (With them in registers
    // those of 64 rows spill, to an L1 that shared memory has left next to nothing of:
    // 96 sequences of five tokens of 8 heads each 372 us, so 322.)
    static constexpr bool kKeep = NG == 2;
    static constexpr int kSums = kKeep ? 0 : kRows * D * 4;
    static constexpr int kFixed = 2 * kQ + kParts * kP + kSums;
    // TMEM: S^T twice, then D^T, whose columns are the rows' first parts, then their second ones.
    static constexpr int kD = kParts * kRows, kUsed = 2 * kRows + MT * kD;
    static constexpr int kColumns = kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : 256;
    static_assert(kUsed <= 256, "TMEM");
};

// Two floats as one word of 16-bit elements, the first in the low half.
template <class T>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    if (std::is_same<T, BF16>::value) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// One tile of rows over one sequence's keys.  Row r of a sequence is head r % group of new
// token r / group.
struct Tile {
    int length, first, count;      // tokens of the sequence; its first new one among the call's, and how many
    int slot;                      // the sequence
    int head, tile;                // key head; which 8 NG rows
    int units;                     // of 128 keys
};

// A tile's part in a block's run.
struct Item {
    Tile t;
    int first, n;                  // units; n 0: the block's run has ended
    int64_t begin;                 // of the tile in the call's line
};

// The last key (+ 1) that a row sees.
__device__ __forceinline__ int seen(const Tile& t, int group, int row) { return t.length - t.count + 1 + row / group; }

// One listed sequence, checked: a sequence that does not fit has no units (and marks
// the cache).
__device__ __forceinline__ void load_seq(const AttendArgs& a, int i, int* slot, int* length, int* first, int* count) {
    *slot = a.seqs[i];
    *first = a.starts ? a.starts[i] : i;
    const int end = a.starts ? a.starts[i + 1] : i + 1;
    *length = a.c.has_seq(*slot) ? __ldcg(&a.lengths[*slot]) : -1;
    *count = 0;
    if (a.c.has_length(*length) && *first >= 0 && end >= *first && end <= a.rows) {
        *count = end - *first;
    } else {
        *length = 0;
        atomicOr(&a.control[kLate], kBadRange);
    }
}
__device__ __forceinline__ int units_of(int length) { return max((length + kUnit - 1) / kUnit, 1); }
template <class K>
__device__ __forceinline__ int tiles_of(const AttendArgs& a, int count) {
    return int((int64_t(count) * a.group + K::kRows - 1) / K::kRows);
}
// A tile's length in the call's line: two places a unit, the k-th unit's (from 0) being kOpen + 2 k
// from the tile's begin.
template <class K>
__device__ __forceinline__ int64_t places_of(int units) { return K::kOpen + 2 * int64_t(units); }
template <class K>
__device__ __forceinline__ int64_t place_of(int unit) { return K::kOpen + 2 * int64_t(unit); }
// The first of a tile's units from a place on.
template <class K>
__device__ __forceinline__ int unit_from(int64_t place, int units) {
    return place <= K::kOpen ? 0 : int(min((place - K::kOpen + 1) / 2, int64_t(units)));
}
template <class K>
__device__ __forceinline__ int64_t work_of(const AttendArgs& a, int length, int count) {
    return int64_t(a.c.n_kv) * tiles_of<K>(a, count) * places_of<K>(units_of(length));
}

// The blocks' runs: block b has the units at places T b / N to T (b + 1) / N - 1.
struct Line {
    int64_t total;
    int blocks;
    __device__ __forceinline__ int64_t begin(int b) const { return total * b / blocks; }
    // Whose run holds a place.
    __device__ __forceinline__ int owner(int64_t u) const { return int(((u + 1) * blocks - 1) / total); }
};

// Walks the tiles of a block's run, and the units of each that belong to it; 32
// sequences' numbers at a time, one a lane.
template <class K>
struct Walk {
    const AttendArgs& a;
    const int4* info;                    // NULL, or all sequences' numbers
    int seq, batch;                      // the current sequence, the first one of the loaded ones
    int slot_, length_, first_, count_;  // lane l: of sequence batch + l
    int64_t at, begin, end;              // where the tile begins in the line; the run
    Tile t;
    int first, n;                        // the tile's units in the run
    // From the run's first place on, `inside` places from the begin of sequence i.
    __device__ __forceinline__ Walk(const AttendArgs& args, const int4* info_, int i, int64_t inside, int64_t begin_, int64_t end_)
        : a(args), info(info_), seq(i), batch(i), begin(begin_), end(end_) {
        load();
        enter();
        const int64_t each = places_of<K>(t.units), tile = inside / each;
        const int tiles = tiles_of<K>(a, t.count);
        at = begin - (inside - tile * each);
        t.head = int(tile / tiles);
        t.tile = int(tile % tiles);
        range();
        if (n <= 0) next();
    }
    __device__ __forceinline__ void load() {
        const int i = batch + int(threadIdx.x & 31);
        slot_ = length_ = first_ = count_ = 0;
        if (i >= a.n) return;
        if (info) {
            const int4 x = info[i];
            slot_ = x.x, length_ = x.y, first_ = x.z, count_ = x.w;
        } else {
            load_seq(a, i, &slot_, &length_, &first_, &count_);
        }
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
    __device__ __forceinline__ void range() {
        first = at < begin ? unit_from<K>(begin - at, t.units) : 0;
        n = unit_from<K>(end - at, t.units) - first;
    }
    __device__ __forceinline__ bool ended() const { return n <= 0; }
    // The next tile that has units in the run; n is 0 if there is none.  The tiles of a key head follow
    // one another.
    __device__ __forceinline__ void next() {
        do {
            at += places_of<K>(t.units);
            n = 0;
            if (at >= end) return;
            if (++t.tile < tiles_of<K>(a, t.count)) {
            } else if (++t.head < a.c.n_kv) {
                t.tile = 0;
            } else {
                do {
                    if (++seq >= a.n) return;
                    if (seq == batch + 32) {
                        batch = seq;
                        load();
                    }
                    enter();
                } while (t.count == 0);
            }
            range();
        } while (n <= 0);
    }
};

// ---------------------------------------------------------------------------
// Barriers, copies, products
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_of(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, int parity) {
    uint32_t done;
    asm volatile(
        "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
// Whether the barrier's phase came.  A wait that runs out (two seconds or so) raises *quit, on
// which the block's other waits give up too.
__device__ __forceinline__ bool bar_wait(uint32_t bar, int parity, volatile int* quit, int32_t* control) {
    if (bar_try(bar, parity)) return true;
    const long long t0 = clock64();
#pragma unroll 1
    for (int k = 0; !bar_try(bar, parity); ++k) {
        if (k & 31) continue;
        if (*quit) return false;
        if (clock64() - t0 > kWaitCycles) {
            *quit = 1;
            atomicOr(&control[kLate], kBadWait);
            return false;
        }
    }
    return true;
}

// Of a call that gave up: waits until `landed` is true, for a tenth of a second or so after t0 at most.
template <class Landed>
__device__ __forceinline__ void drain(long long t0, Landed landed) {
#pragma unroll 1
    while (!landed() && clock64() - t0 < kWaitCycles / 20) {}
}

// The softmax warps' own barrier, with the OR of what they bring.
template <int THREADS>
__device__ __forceinline__ bool soft_any(bool x) {
    uint32_t r;
    asm volatile(
        "{ .reg .pred p, q; setp.ne.u32 p, %1, 0; barrier.cta.red.or.pred q, 1, %2, p; selp.u32 %0, 1, 0, q; }"
        : "=r"(r)
        : "r"(uint32_t(x)), "n"(THREADS)
        : "memory");
    return __any_sync(~0u, r);
}
template <int THREADS>
__device__ __forceinline__ void soft_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(THREADS) : "memory"); }

__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, 0, %3, %4, %5}], [%6];" ::"r"(to),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}

// A descriptor of a matrix in shared memory: strides in bytes, layout 2 for rows of 128
// bytes swizzled, 0 for 8 x 16 bytes as they lie.
__device__ __forceinline__ uint64_t descriptor(uint32_t at, uint32_t leading, uint32_t stride, uint64_t layout) {
    return uint64_t((at & 0x3FFFF) >> 4) | uint64_t(leading >> 4) << 16 | uint64_t(stride >> 4) << 32 | uint64_t(1) << 46 | layout << 61;
}
// Of an instruction: float32 sums, 128 x n; which operands have their rows' index adjacent.
template <class T>
__device__ __forceinline__ uint32_t instruction(int n, bool a_rows, bool b_rows) {
    const uint32_t type = std::is_same<T, BF16>::value ? 1 : 0;
    return 1u << 4 | type << 7 | type << 10 | uint32_t(a_rows) << 15 | uint32_t(b_rows) << 16 | uint32_t(n >> 3) << 17 | (128u >> 4) << 24;
}
// (All lanes come here; the one that `mine` names issues.)
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool add, uint32_t mine) {
    asm volatile(
        "{ .reg .pred p, q; setp.ne.u32 p, %4, 0; setp.ne.u32 q, %5, 0; @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(instr), "r"(uint32_t(add)), "r"(mine)
        : "memory");
}
// The barrier's arrival when all products issued so far are done.
__device__ __forceinline__ void products_arrive(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Eight columns of this lane's row, in pairs.
__device__ __forceinline__ void tmem_load(uint32_t at, unsigned long long* x) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(at)
                 : "memory");
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (unsigned long long)(r[2 * e + 1]) << 32 | r[2 * e];
}
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Generic writes to shared memory, before the copies' and products' side reads them.
__device__ __forceinline__ void to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Two floats, for which one instruction does.
using F2 = unsigned long long;
__device__ __forceinline__ F2 both(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float low(F2 x) { return __uint_as_float(uint32_t(x)); }
__device__ __forceinline__ float high(F2 x) { return __uint_as_float(uint32_t(x >> 32)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(r));
    return r;
}
// The same in all lanes, and known to be.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(~0u, x, 0); }

__device__ __forceinline__ float exp2_fast(float x) {
    // (Weights under 2^-126 are 0.)
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

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

// Element d of row r's result, or its maximum and sum, where they belong: in `piece` if
// that is given, else in the outputs.
template <class K>
struct Place {
    float* piece;
    uint16_t* out;
    float* lse;
    __device__ __forceinline__ Place(const AttendArgs& a, const Tile& t, int r, float* to) {
        const int row = t.tile * K::kRows + r, head = t.head * a.group + row % a.group;
        const int64_t token = t.first + row / a.group;
        piece = to ? to + r * K::D : nullptr;
        out = a.out + token * a.ldo + int64_t(head) * a.c.dim;
        lse = to ? to + K::kRows * K::D + 2 * r : a.lse ? a.lse + token * a.n_q + head : nullptr;
    }
    __device__ __forceinline__ void element(const AttendArgs& a, int d, float x) const {
        if (piece) piece[d] = x;
        else if (d < a.c.dim) out[d] = K::T::round(x);
    }
    __device__ __forceinline__ void sums(float top, float sum) const {
        if (piece) lse[0] = top, lse[1] = sum;
        else if (lse) *lse = sum == 0.0f ? -kInf : (top + log2f(sum)) * kLn2;
    }
};

// A warp joins row r of n pieces, given by at(i), in the outputs.  A piece counts by its sum
// at the largest of the maxima.  What bounds it is the time of a load: those of 8 pieces are on
// their way at once, the first of them with the maxima and sums.
template <class K, class At>
__device__ __forceinline__ void join_row(const AttendArgs& a, const Tile& t, int r, int n, At at) {
    constexpr int kMl = K::D * K::kRows;
    // 8 adjacent elements a lane; with 16 lanes' worth of them, half the lanes take every
    // other piece.
    constexpr int kLanes = K::D / 8, kTeams = 32 / kLanes, kBatch = 8 / kTeams;
    const int lane = threadIdx.x & 31, d = 8 * (lane % kLanes), team = lane / kLanes;
    float4 u[kBatch], v[kBatch];
    const auto load = [&](int k) {
#pragma unroll
        for (int e = 0; e < kBatch; ++e) {
            const float4* from = reinterpret_cast<const float4*>(at(min(k + e * kTeams + team, n - 1)) + r * K::D + d);
            u[e] = __ldcg(from), v[e] = __ldcg(from + 1);
        }
    };
    // (Maximum, sum) of a piece.
    const auto sums_of = [&](int i) { return i < n ? __ldcg(reinterpret_cast<const float2*>(at(i) + kMl + 2 * r)) : make_float2(-kInf, 0); };
    // (Maxima may be infinite; one without a score but NaN has the sum NaN, one without any 0.)
    const auto share_of = [](float2 y, float top) { return y.x == top ? y.y : y.y * exp2f(y.x - top); };
    load(0);
    float2 mine = sums_of(lane);
    float top = mine.x;
    for (int i = 32 + lane; i < n; i += 32) top = fmaxf(top, sums_of(i).x);
#pragma unroll
    for (int y = 16; y; y >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, y));
    float sum = share_of(mine, top);
    for (int i = 32 + lane; i < n; i += 32) sum += share_of(sums_of(i), top);
#pragma unroll
    for (int y = 16; y; y >>= 1) sum += __shfl_xor_sync(~0u, sum, y);
    const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
    float share = share_of(mine, top) * inverse, x[8] = {};
#pragma unroll 1
    for (int k = 0; k < n; k += 8) {
        if (k) {
            load(k);
            if (k % 32 == 0) share = share_of(sums_of(k + lane), top) * inverse;
        }
#pragma unroll
        for (int e = 0; e < kBatch; ++e) {
            const float w = __shfl_sync(~0u, share, (k + e * kTeams + team) & 31);
            if (k + e * kTeams + team >= n) continue;
            x[0] = fmaf(w, u[e].x, x[0]), x[1] = fmaf(w, u[e].y, x[1]), x[2] = fmaf(w, u[e].z, x[2]), x[3] = fmaf(w, u[e].w, x[3]);
            x[4] = fmaf(w, v[e].x, x[4]), x[5] = fmaf(w, v[e].y, x[5]), x[6] = fmaf(w, v[e].z, x[6]), x[7] = fmaf(w, v[e].w, x[7]);
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
#pragma unroll
        for (int m = kLanes; m < 32; m <<= 1) x[k] += __shfl_xor_sync(~0u, x[k], m);
    }
    if (team) return;
    const Place<K> place(a, t, r, nullptr);
    put8<typename K::T>(place.out, d, a.c.dim, a.ovec, x);
    if (lane == 0) place.sums(top, sum);
}

// Keys [k0, k1) of one row once more, by one warp, one key after another, for values
// that are not finite or nearly too large, and scores of infinity: a product of weight and value
// only where the row sees the key, weights in float32 and 2^-32 of what they are, so that sums stay
// finite.  A score of infinity has the weight NaN (infinity less infinity) in the result; in the
// sum it counts 1, so that lse is infinity unless a score is NaN.
template <class K>
__device__ __noinline__ void carefully(const AttendArgs& a, const Tile& t, int r, int k0, int k1, float* piece) {
    using T = typename K::T;
    constexpr int kEach = K::D / 32;
    const int lane = threadIdx.x & 31, row = t.tile * K::kRows + r;
    const int end = min(k1, seen(t, a.group, row));
    const uint16_t* q = a.q + (t.first + row / a.group) * a.ldq + int64_t(t.head * a.group + row % a.group) * a.c.dim;
    float top = -kInf, sum = 0, o[kEach] = {};
    for (int pass = 0; pass < 2; ++pass) {
        for (int key0 = k0; key0 < end; key0 += 32) {
            const int key = key0 + lane;
            const int id = key < end ? __ldcg(&a.table[int64_t(t.slot) * a.c.max_pages + (key >> a.c.shift)]) : -1;
            const char* at = nullptr;
            float s = -kInf;
            if (a.c.has_page(id)) {
                at = a.pages + id * a.c.page_bytes + t.head * a.c.run_bytes + (key & (a.c.page - 1)) * (2 * a.c.pitch);
                s = 0;
                for (int d = 0; d < a.c.dim; d += 8) {
                    const uint4 k = *reinterpret_cast<const uint4*>(at + 2 * d);
                    const uint32_t w[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (d + e < a.c.dim) s = fmaf(T::widen(q[d + e]), T::widen(uint16_t(w[e / 2] >> (16 * (e & 1)))), s);
                }
                s *= a.scale;
            }
            if (pass == 0) {
                top = fmaxf(top, s);
                continue;
            }
            const float p = exp2f(s - (top == -kInf ? 0.0f : top));
            sum += s == kInf ? 1.0f : p;
            float part[kEach] = {};
            for (int x = 0; x < min(end - key0, 32); ++x) {
                const float w = __shfl_sync(~0u, p, x) * 0x1p-32f;
                const char* from = reinterpret_cast<const char*>(__shfl_sync(~0u, reinterpret_cast<unsigned long long>(at), x));
                if (!from) continue;
                const uint16_t* v = reinterpret_cast<const uint16_t*>(from + int64_t(a.c.n_kv) * a.c.run_bytes);
#pragma unroll
                for (int e = 0; e < kEach; ++e)
                    if (lane + 32 * e < a.c.dim) part[e] = fmaf(w, T::widen(v[lane + 32 * e]), part[e]);
            }
#pragma unroll
            for (int e = 0; e < kEach; ++e) o[e] += part[e];
        }
        if (pass == 0) {
#pragma unroll
            for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
        }
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(~0u, sum, x);
    const float inverse = sum == 0.0f ? 0.0f : 0x1p32f / sum;
    const Place<K> place(a, t, r, piece);
#pragma unroll
    for (int e = 0; e < kEach; ++e) place.element(a, lane + 32 * e, o[e] * inverse);
    if (lane == 0) place.sums(top, sum);
}

// ---------------------------------------------------------------------------
// The kernel
// ---------------------------------------------------------------------------

template <class K>
struct Shared {
    uint64_t full[kMostStages], empty[kMostStages];   // of the ring's stages
    uint64_t scores[2], weights, sums;                // S^T is there (two of them, in turn); P^T; D^T
    uint64_t drained;                                 // (of a call that gave up) no product is under way
    uint64_t q_full[2], q_free[2];                    // a tile's queries and all that is said of it below
    Item items[2];
    alignas(16) int seen[2][K::kRows];
    int64_t out[2][K::kRows];                         // where a row's result begins
    // Of a row: what a score has added before its exponential; what sums are multiplied by
    // when that moves; 1 / the sum of weights.
    alignas(16) float zero[8], bias[K::kRows], factor[K::kRows], inverse[K::kRows];
    float parts[4][K::kRows];
    int4 info[kListed];                               // the listed sequences, where there are no more
    int64_t scan[K::kThreads / 32];
    int64_t start;                                    // where the block's run begins within its first sequence
    int seq;                                          // that sequence
    int quit, last;
    int fresh[2];                                     // whether a unit's sums begin anew (of two, in turn)
    uint32_t tmem;
};

// Eight rows' values, one a lane each, over the warp's lanes: lane l ends with row
// 4 (l / 16) + 2 (l / 8 % 2) + l / 4 % 2 of them.
template <class F>
__device__ __forceinline__ float over_lanes(const F2* pairs, F f) {
    const int lane = threadIdx.x & 31;
    const float x[8] = {low(pairs[0]), high(pairs[0]), low(pairs[1]), high(pairs[1]), low(pairs[2]), high(pairs[2]), low(pairs[3]), high(pairs[3])};
    float a[4], b[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float keep = lane & 16 ? x[i + 4] : x[i], give = lane & 16 ? x[i] : x[i + 4];
        a[i] = f(keep, __shfl_xor_sync(~0u, give, 16));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float keep = lane & 8 ? a[i + 2] : a[i], give = lane & 8 ? a[i] : a[i + 2];
        b[i] = f(keep, __shfl_xor_sync(~0u, give, 8));
    }
    const float keep = lane & 4 ? b[1] : b[0], give = lane & 4 ? b[0] : b[1];
    float c = f(keep, __shfl_xor_sync(~0u, give, 4));
    c = f(c, __shfl_xor_sync(~0u, c, 2));
    return f(c, __shfl_xor_sync(~0u, c, 1));
}
__device__ __forceinline__ int row_of_lane() { return (threadIdx.x >> 4 & 1) * 4 + (threadIdx.x >> 3 & 1) * 2 + (threadIdx.x >> 2 & 1); }

// A unit's place in the ring's order, K0 K1 V0 K2 V1 ...  (The place of the keys behind the
// last ones stays empty.)
__device__ __forceinline__ int keys_at(int i) { return i ? 2 * i - 1 : 0; }
__device__ __forceinline__ int values_at(int i) { return 2 * i + 2; }

// A place in the ring, and the parity of its turn.
struct Stage {
    int at = 0, turn = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++at == stages) at = 0, turn ^= 1;
    }
};

template <class K>
__global__ void __launch_bounds__(K::kThreads, 1) rr_attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map) {
    using T = typename K::T;
    constexpr int NG = K::NG, MT = K::MT, N = K::kRows;
    extern __shared__ char memory[];
    __shared__ Shared<K> sh;
    const int lane = threadIdx.x & 31, w = uniform(threadIdx.x >> 5);

    // What needs no memory of the call's, while the launch before may still run.
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) {
            bar_init(smem_of(&sh.full[i]), 1);
            bar_init(smem_of(&sh.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_of(&sh.scores[i]), 1);
            bar_init(smem_of(&sh.q_full[i]), 1);
            bar_init(smem_of(&sh.q_free[i]), K::kSoft / 32);
        }
        bar_init(smem_of(&sh.weights), K::kSoft / 32);
        bar_init(smem_of(&sh.sums), 1);
        bar_init(smem_of(&sh.drained), 1);
        sh.quit = 0;
        for (int i = 0; i < 8; ++i) sh.zero[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == K::kProducts) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_of(&sh.tmem)), "n"(K::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    const uint32_t tmem = sh.tmem;
    // (All of the block's threads come here.)
    const auto leave = [&] {
        tmem_before();
        __syncthreads();
        // (Of a call that gave up: the products under way end before their memory is given back.)
        if (w == K::kProducts && sh.quit) {
            if (elected()) {
                products_arrive(smem_of(&sh.drained));
                drain(clock64(), [&] { return bar_try(smem_of(&sh.drained), 0); });
            }
            __syncwarp();
        }
        if (w == K::kProducts) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(K::kColumns) : "memory");
    };
    after_previous();
    if (__ldcg(&a.control[kState])) return leave();

    // The line, and where this block's run begins in it.
    Line line;
    int64_t begin, end;
    {
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
            for (int i = 0; i < K::kThreads / 32; ++i) {
                if (i < w) before += sh.scan[i];
                all += sh.scan[i];
            }
            __syncthreads();
            *total = all;
            return before + s - v;
        };
        const auto work = [&](int i) -> int64_t {
            if (i >= a.n) return 0;
            int slot, length, first, count;
            load_seq(a, i, &slot, &length, &first, &count);
            if (a.n <= kListed) sh.info[i] = make_int4(slot, length, first, count);
            return work_of<K>(a, length, count);
        };
        int64_t mine = 0, kept = 0;
        for (int i = threadIdx.x; i < a.n; i += K::kThreads) mine += kept = work(i);
        int64_t at = scan(mine, &line.total);
        if (line.total == 0) return leave();
        // (So many places that each run has a unit.)
        line.blocks = int(max(min(int64_t(gridDim.x), line.total / (2 + K::kOpen)), int64_t(1)));
        if (int(blockIdx.x) >= line.blocks) return leave();
        begin = line.begin(blockIdx.x), end = line.begin(blockIdx.x + 1);
        int64_t before = 0;
        for (int base = 0; base < a.n && before <= begin; base += K::kThreads) {
            int64_t total = line.total;
            if (a.n > K::kThreads) {
                kept = work(base + int(threadIdx.x));
                at = before + scan(kept, &total);
            }
            if (begin >= at && begin < at + kept) {
                sh.seq = base + int(threadIdx.x);
                sh.start = begin - at;
            }
            before += total;
        }
    }

    const uint32_t ring = (smem_of(memory) + 1023) / 1024 * 1024, stage_bytes = a.atoms * 16384;
    const uint32_t q_at = ring + a.stages * stage_bytes, p_at = q_at + 2 * K::kQ;
    float* const sums_at = reinterpret_cast<float*>(memory + (p_at + K::kParts * K::kP - smem_of(memory)));
    __syncthreads();
    const int4* const info = a.n <= kListed ? sh.info : nullptr;
    const auto wait = [&](uint64_t& bar, int parity) { return bar_wait(smem_of(&bar), parity, &sh.quit, a.control); };

    if (w == K::kKeys || w == K::kValues) {
        // Copies: one warp the keys', one the values'.  A lane asks for one page's.
        const bool values = w == K::kValues;
        Walk<K> walk(a, info, sh.seq, sh.start, begin, end);
        int unit = walk.first, left = walk.n;
        const int tokens = a.c.page, pages = kUnit >> a.c.shift, eights = tokens / 8;
        const auto fetch = [&] {
            const int key = unit * kUnit + lane * tokens;
            if (lane >= pages || key >= walk.t.length) return -1;
            const int id = __ldcg(&a.table[int64_t(walk.t.slot) * a.c.max_pages + (key >> a.c.shift)]);
            if (a.c.has_page(id)) return id;
            atomicOr(&a.control[kLate], kBadTable);
            return -1;
        };
        int id = fetch(), i = 0;
        bool ok = true;
        for (; !walk.ended(); ++i) {
            const int here = id, head = (values ? a.c.n_kv : 0) + walk.t.head;
            // (The next unit's pages, ahead of the wait.)
            ++unit;
            if (--left == 0) {
                walk.next();
                unit = walk.first, left = walk.n;
            }
            if (!walk.ended()) id = fetch();
            const int k = values ? values_at(i) : keys_at(i), at = k % a.stages, turn = k / a.stages & 1;
            if (!(ok = __all_sync(~0u, wait(sh.empty[at], turn ^ 1)))) break;
            const uint32_t bar = smem_of(&sh.full[at]);
            const int there = __popc(__ballot_sync(~0u, here >= 0));
            if (elected()) bar_expect(bar, uint32_t(there * a.atoms * tokens * 128));
            __syncwarp();
            if (here >= 0) {
                const uint32_t to = ring + at * stage_bytes + lane * eights * a.eight_bytes;
                for (int y = 0; y < a.atoms; y += a.copy_atoms)
                    tma_load(to + y * a.atom_bytes, &map, a.copy_atoms > 1 ? 0 : 64 * y, 0, head * eights, here, bar);
            }
        }
        if (!ok) {
            // What is on its way has to land before the block ends.  (A stage that has been used since may
            // have been filled once more, by the other warp: its first copy is seen by its use then.)
            const long long t0 = clock64();
            for (int back = max(i - a.stages, 0); back < i; ++back) {
                const int k = values ? values_at(back) : keys_at(back), at = k % a.stages, turn = k / a.stages & 1;
                drain(t0, [&] { return bar_try(smem_of(&sh.full[at]), turn) || bar_try(smem_of(&sh.empty[at]), turn); });
            }
        }
    } else if (w == K::kProducts) {
        // Products.  (All lanes go along; one of them issues.)
        const int k16 = (a.c.dim + 15) / 16;
        // The ring's order: K0 K1 V0 K2 V1 ...
        Stage st;
        int q_item = 0, v_item = 0, q_left = 0, v_left = 0, v_unit = 0, v_length = 0;
        uint32_t q_instr = 0, v_instr = 0;
        const auto rows_of = [&](const Tile& t) { return min(t.count * a.group - t.tile * K::kRows, N); };
        const auto columns = [&](const Tile& t) { return uniform((rows_of(t) + 15) / 16 * 16); };
        const uint32_t first_tmem = uniform(tmem);
        bool more = true;
        for (int i = 0, done = 0;;) {
            const int slot = q_item & 1;
            if (more && q_left == 0) {
                if (!__all_sync(~0u, wait(sh.q_full[slot], q_item >> 1 & 1))) break;
                q_left = uniform(sh.items[slot].n);
                q_instr = instruction<T>(columns(sh.items[slot].t), false, false);
                if (!(more = q_left > 0)) st.next(a.stages);
            }
            if (more) {
                if (!__all_sync(~0u, wait(sh.full[st.at], st.turn))) break;
                tmem_after();
                {
                    // (A descriptor's address counts 16 bytes.)
                    const uint32_t mine = elected();
                    const uint64_t dk = descriptor(ring + st.at * stage_bytes, 16, a.eight_bytes, 2);
                    const uint64_t dq = descriptor(q_at + slot * K::kQ, N * 16, 128, 0);
#pragma unroll
                    for (int j = 0; j < 8 * MT; ++j)
                        if (j < k16)
                            product(first_tmem + uint32_t(i & 1) * N, dk + (j >> 2) * (a.atom_bytes / 16) + (j & 3) * 2, dq + j * (2 * N), q_instr,
                                    j > 0, mine);
                    if (mine) {
                        products_arrive(smem_of(&sh.empty[st.at]));
                        products_arrive(smem_of(&sh.scores[i & 1]));
                    }
                    __syncwarp();
                }
                st.next(a.stages);
                if (--q_left == 0) ++q_item;
                ++i;
            }
            // (Of the unit before; of the last one, if there is none left.)
            if (done == i) break;
            if (done + 1 < i || !more) {
                if (v_left == 0) {
                    const Item& item = sh.items[v_item & 1];
                    v_left = uniform(item.n);
                    v_unit = uniform(item.first);
                    v_length = uniform(item.t.length);
                    // (One product for both parts of the weights, side by side: a product takes about 75
                    // cycles and one more for each column or so.)
                    v_instr = instruction<T>(2 * uniform((rows_of(item.t) + 7) / 8 * 8), true, true);
                    ++v_item;
                }
                if (!__all_sync(~0u, wait(sh.full[st.at], st.turn))) break;
                if (!__all_sync(~0u, wait(sh.weights, done & 1))) break;
                tmem_after();
                const int steps = max((min(v_length - v_unit * kUnit, kUnit) + 15) / 16, 1);
                const bool add = !uniform(sh.fresh[done & 1]);
                {
                    const uint64_t dv = descriptor(ring + st.at * stage_bytes, a.atom_bytes, a.eight_bytes, 2), dp = descriptor(p_at, 128, 2048, 0);
                    const uint32_t mine = elected();
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (j < steps)
                                product(first_tmem + 2 * N + m * K::kD, dv + m * (a.atom_bytes / 8) + j * (a.eight_bytes / 8), dp + j * 16, v_instr,
                                        add || j > 0, mine);
                    if (mine) {
                        products_arrive(smem_of(&sh.empty[st.at]));
                        products_arrive(smem_of(&sh.sums));
                    }
                    __syncwarp();
                }
                st.next(a.stages);
                ++v_unit;
                --v_left;
                ++done;
            }
        }
    } else if (w == K::kQueries) {
        // Queries, and what the others need to know of a tile.
        Walk<K> walk(a, info, sh.seq, sh.start, begin, end);
        const int chunks = (a.c.dim + 15) / 16 * 2;
        for (int item = 0;; ++item) {
            const int slot = item & 1;
            if (!__all_sync(~0u, wait(sh.q_free[slot], (item >> 1 & 1) ^ 1))) break;
            const Tile& t = walk.t;
            const int left = walk.ended() ? 0 : min(t.count * a.group - t.tile * K::kRows, K::kRows), rows = (left + 15) / 16 * 16;
            const uint32_t to = q_at + slot * K::kQ;
            for (int base = 0; base < rows * chunks; base += 8 * 32) {
                uint4 x[8];
                uint32_t where[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = base + 32 * e + lane, r = i / chunks, c = i - r * chunks, d = 8 * c, row = t.tile * K::kRows + r;
                    where[e] = i < rows * chunks ? to + c * (N * 16) + r * 16 : 0;
                    x[e] = make_uint4(0, 0, 0, 0);
                    if (r >= left || d >= a.c.dim || i >= rows * chunks) continue;
                    const uint16_t* from = a.q + (t.first + row / a.group) * a.ldq + int64_t(t.head * a.group + row % a.group) * a.c.dim + d;
                    if (a.qvec) {
                        x[e] = *reinterpret_cast<const uint4*>(from);
                    } else {
                        uint32_t v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = d + k < a.c.dim ? from[k] : 0u;
                        x[e] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (where[e])
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(where[e]), "r"(x[e].x), "r"(x[e].y), "r"(x[e].z), "r"(x[e].w)
                                     : "memory");
            }
            for (int r = lane; r < N; r += 32) {
                const int row = t.tile * K::kRows + r, token = row / a.group;
                sh.seen[slot][r] = r < left ? t.length - t.count + 1 + token : 0;
                sh.out[slot][r] = (t.first + token) * a.ldo + int64_t(t.head * a.group + row - token * a.group) * a.c.dim;
            }
            if (lane == 0) {
                Item& it = sh.items[slot];
                it.t = t;
                it.first = walk.first;
                it.n = max(walk.n, 0);
                it.begin = walk.at;
            }
            to_async();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_of(&sh.q_full[slot]));
            if (walk.ended()) break;
            walk.next();
        }
    } else {
        // Softmax and sums.  Lane l of warp w has key, or element, 32 (w % 4) + l; the sets of four
        // warps share the groups of 8 rows in turn (MT 2: of the sums, half of the sets each 128
        // elements).
        constexpr int kSets = K::kSets, GS = (NG + kSets - 1) / kSets, kSumSets = kSets / MT, GO = (NG + kSumSets - 1) / kSumSets;
        const int set = w >> 2, key = threadIdx.x & 127, half = MT == 2 ? set & 1 : 0, d = key + 128 * half;
        const uint32_t lanes = uint32_t(w & 3) << 21;
        const auto group_of = [&](int j) { return set + kSets * j; };
        const F2 scale2 = both(a.scale, a.scale);
        const auto sum_group = [&](int j) { return set / MT + kSumSets * j; };
        int i = 0;
        bool over = false;
        for (int item = 0; !over; ++item) {
            const int slot = item & 1;
            bool ok = __all_sync(~0u, wait(sh.q_full[slot], (item >> 1 & 1)));
            // (The first scores are over any reference: it is set then.)
            if (int(threadIdx.x) < N) sh.bias[threadIdx.x] = kNothing;
            if (soft_any<K::kSoft>(!ok)) break;
            const Item it = sh.items[slot];
            const int units = uniform(it.n);
            if (units == 0) break;
            const int left = uniform(min(it.t.count * a.group - it.t.tile * K::kRows, K::kRows)), groups = (left + 7) / 8;
            const int first_seen = uniform(seen(it.t, a.group, it.t.tile * K::kRows));
            const int first_key = uniform(it.first * kUnit);
            F2 o[K::kKeep ? GO : 1][4], sum[GS][4];
            bool begun = false;            // whether o has anything
            bool odd = false;              // whether a result is not finite
            // Adds TMEM's sums to o, and multiplies by factor[row] where that is given.
            const auto add_sums = [&](const float* factor, bool last) {
#pragma unroll
                for (int j = 0; j < GO; ++j) {
                    if (sum_group(j) >= groups) continue;
                    F2 x[4], y[4];
                    const uint32_t columns = tmem + lanes + 2 * N + half * K::kD + 8 * sum_group(j);
                    tmem_load(columns, x);
                    tmem_load(columns + 8 * groups, y);
                    tmem_loaded();
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = add2(x[e], y[e]);
                    float* const at = sums_at + 8 * sum_group(j) * K::D + d;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (begun) x[e] = add2(x[e], K::kKeep ? o[K::kKeep ? j : 0][e] : both(at[2 * e * K::D], at[(2 * e + 1) * K::D]));
                        if (factor) {
                            const F2 f = reinterpret_cast<const F2*>(factor + 8 * sum_group(j))[e];
                            x[e] = mul2(x[e], f);
                            // (Rows whose sum is NaN are all NaN in any case.)
                            const int r = 8 * sum_group(j) + 2 * e;
                            if (last) {
                                odd |= r < left && low(f) == low(f) && !(fabsf(low(x[e])) < kInf);
                                odd |= r + 1 < left && high(f) == high(f) && !(fabsf(high(x[e])) < kInf);
                            }
                        }
                        if (K::kKeep) o[K::kKeep ? j : 0][e] = x[e];
                        else at[2 * e * K::D] = low(x[e]), at[(2 * e + 1) * K::D] = high(x[e]);
                    }
                }
                begun = true;
            };
#pragma unroll
            for (int j = 0; j < GS; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[j][e] = 0;
            for (int u = 0; u < units; ++u, ++i) {
                const int key0 = first_key + u * kUnit;
                ok &= __all_sync(~0u, wait(sh.scores[i & 1], i >> 1 & 1));
                tmem_after();
                F2 s[GS][4];
#pragma unroll
                for (int j = 0; j < GS; ++j)
                    if (group_of(j) < groups) tmem_load(tmem + lanes + uint32_t(i & 1) * N + 8 * group_of(j), s[j]);
                tmem_loaded();
                // Which keys the rows see, where that is not all.
                const bool edge = key0 + kUnit > first_seen;
                uint32_t sees[GS];
                if (edge) {
#pragma unroll
                    for (int j = 0; j < GS; ++j) {
                        if (group_of(j) >= groups) continue;
                        sees[j] = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) sees[j] |= uint32_t(key0 + key < sh.seen[slot][8 * group_of(j) + e]) << e;
                    }
                }
                // Weights are 2^x, x = scale s - reference, with scale s rounded first: what a fused
                // product keeps of it, half a bit of a score of 2^32, would be a weight of 2^128.
#pragma unroll
                for (int j = 0; j < GS; ++j) {
                    if (group_of(j) >= groups) continue;
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][e] = mul2(s[j][e], scale2);
                }
                const auto refer = [&](int j, F2* x, const float* from) {
                    const float4* const bias = reinterpret_cast<const float4*>(from);
                    const float4 b0 = bias[0], b1 = bias[1];
                    x[0] = add2(s[j][0], both(b0.x, b0.y));
                    x[1] = add2(s[j][1], both(b0.z, b0.w));
                    x[2] = add2(s[j][2], both(b1.x, b1.y));
                    x[3] = add2(s[j][3], both(b1.z, b1.w));
                    if (edge) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[e] = both(sees[j] >> (2 * e) & 1 ? low(x[e]) : -kInf, sees[j] >> (2 * e + 1) & 1 ? high(x[e]) : -kInf);
                    }
                };
                float most = -kInf;
#pragma unroll
                for (int j = 0; j < GS; ++j) {
                    if (group_of(j) >= groups) continue;
                    F2 x[4];
                    refer(j, x, &sh.bias[8 * group_of(j)]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(low(x[e]), high(x[e])));
                }
                const bool moved = soft_any<K::kSoft>(!ok || most > kSlack + K::kLift);
                if (moved) {
                    if (soft_any<K::kSoft>(!ok || *(volatile int*)&sh.quit)) {
                        over = true;
                        break;
                    }
#pragma unroll
                    for (int j = 0; j < GS; ++j) {
                        if (group_of(j) >= groups) continue;
                        F2 y[4];
                        refer(j, y, sh.zero);
                        const float m = over_lanes(y, [](float p, float q) { return fmaxf(p, q); });
                        if ((lane & 3) == 0) sh.parts[w & 3][8 * group_of(j) + row_of_lane()] = m;
                    }
                    soft_sync<K::kSoft>();
                    if (int(threadIdx.x) < 8 * groups) {
                        const int r = threadIdx.x;
                        const float m = fmaxf(fmaxf(sh.parts[0][r], sh.parts[1][r]), fmaxf(sh.parts[2][r], sh.parts[3][r]));
                        const float before = sh.bias[r], after = m == -kInf ? kNothing : K::kLift - m;
                        const bool moves = after < before;
                        sh.factor[r] = moves ? exp2f(after - before) : 1.0f;
                        if (moves) sh.bias[r] = after;
                    }
                    soft_sync<K::kSoft>();
#pragma unroll
                    for (int j = 0; j < GS; ++j) {
                        if (group_of(j) >= groups) continue;
                        const F2* const f = reinterpret_cast<const F2*>(&sh.factor[8 * group_of(j)]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[j][e] = mul2(sum[j][e], f[e]);
                    }
                }
                uint32_t p[GS][K::kParts][4];
#pragma unroll
                for (int j = 0; j < GS; ++j) {
                    if (group_of(j) >= groups) continue;
                    F2 x[4];
                    refer(j, x, &sh.bias[8 * group_of(j)]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float lo = exp2_fast(low(x[e])), hi = exp2_fast(high(x[e]));
                        const F2 y = both(lo, hi);
                        sum[j][e] = add2(sum[j][e], y);
                        const uint32_t big = pack<T>(lo, hi);
                        p[j][0][e] = big;
                        const F2 rest = fma2(both(T::widen(uint16_t(big)), T::widen(uint16_t(big >> 16))), both(-1.0f, -1.0f), y);
                        p[j][1][e] = pack<T>(low(rest), high(rest));
                    }
                }
                // The weights may be overwritten once the products of the unit before are done.
                if (u > 0) {
                    wait(sh.sums, (i - 1) & 1);
                    tmem_after();
                }
                // Sums gather in TMEM over 8 units, by the matrix instructions, which cut off; then,
                // and where the reference moves, they are added up in float32, which rounds.
                const bool fresh = moved || u % kGather == 0;
                if (fresh && u > 0) {
                    __syncwarp();
                    add_sums(moved ? sh.factor : nullptr, false);
                }
                if (threadIdx.x == 0) sh.fresh[i & 1] = fresh;
#pragma unroll
                for (int j = 0; j < GS; ++j) {
                    if (group_of(j) >= groups) continue;
#pragma unroll
                    for (int x = 0; x < K::kParts; ++x)
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(p_at + (x * groups + group_of(j)) * 2048 + key * 16),
                                     "r"(p[j][x][0]), "r"(p[j][x][1]), "r"(p[j][x][2]), "r"(p[j][x][3])
                                     : "memory");
                }
                const int valid = min(it.t.length - key0, kUnit);
                if (valid < kUnit) {
                    // Behind the sequence's end the page holds anything: values there become 0.
                    const int k = values_at(i);
                    const int stage = k % a.stages;
                    wait(sh.full[stage], k / a.stages & 1);
                    const int rows = max((valid + 15) / 16 * 16, 16) - valid;
                    for (int x = threadIdx.x; x < rows * a.atoms * 8; x += K::kSoft) {
                        const int atom = x / (rows * 8), y = x - atom * (rows * 8), token = valid + (y >> 3);
                        const uint32_t at = ring + stage * stage_bytes + atom * a.atom_bytes + (token >> 3) * a.eight_bytes +
                                            (token & 7) * 128 + (y & 7) * 16;
                        asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at), "r"(0) : "memory");
                    }
                }
                to_async();
                tmem_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_of(&sh.weights));
            }
            if (over) break;

            // The run leaves the tile.
            __syncwarp();
            wait(sh.sums, (i - 1) & 1);
            tmem_after();
            __syncwarp();
#pragma unroll
            for (int j = 0; j < GS; ++j) {
                if (group_of(j) >= groups) continue;
                const float m = over_lanes(sum[j], [](float x, float y) { return x + y; });
                if ((lane & 3) == 0) sh.parts[w & 3][8 * group_of(j) + row_of_lane()] = m;
            }
            soft_sync<K::kSoft>();
            const bool starts = it.first == 0, ends = it.first + it.n == it.t.units;
            float* const piece = starts && ends ? nullptr : a.pieces + (2 * int64_t(blockIdx.x) + starts) * a.piece_floats;
            bool far = false;              // whether a score is infinity
            if (int(threadIdx.x) < left) {
                const int r = threadIdx.x;
                const float total = sh.parts[0][r] + sh.parts[1][r] + sh.parts[2][r] + sh.parts[3][r], bias = sh.bias[r];
                far = bias == -kInf;
                sh.inverse[r] = total == 0.0f ? 0.0f : 1.0f / total;
                Place<K>(a, it.t, r, piece).sums(-bias, total);
            }
            soft_sync<K::kSoft>();
            // (Each sum times 1 / the row's.)
            add_sums(sh.inverse, true);
            if (soft_any<K::kSoft>(far || (odd && d < a.c.dim))) {
                for (int r = w; r < left; r += K::kSoft / 32) carefully<K>(a, it.t, r, it.first * kUnit, (it.first + it.n) * kUnit, piece);
            } else if (K::kKeep) {
#pragma unroll
                for (int j = 0; j < GO; ++j) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int r = 8 * sum_group(j) + e;
                        const float x = e & 1 ? high(o[K::kKeep ? j : 0][e / 2]) : low(o[K::kKeep ? j : 0][e / 2]);
                        if (r >= left) continue;
                        if (piece) piece[r * K::D + d] = x;
                        else if (d < a.c.dim) a.out[sh.out[slot][r] + d] = T::round(x);
                    }
                }
            } else {
                // A warp takes a row, a lane four elements.
                for (int r = w; r < left; r += K::kSoft / 32) {
#pragma unroll
                    for (int e = 4 * lane; e < K::D; e += 128) {
                        const float4 x = *reinterpret_cast<const float4*>(sums_at + r * K::D + e);
                        if (piece) {
                            *reinterpret_cast<float4*>(piece + r * K::D + e) = x;
                        } else if (a.ovec) {
                            if (e < a.c.dim)
                                *reinterpret_cast<uint2*>(a.out + sh.out[slot][r] + e) = make_uint2(pack<T>(x.x, x.y), pack<T>(x.z, x.w));
                        } else {
                            const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (e + k < a.c.dim) a.out[sh.out[slot][r] + e + k] = T::round(y[k]);
                        }
                    }
                }
            }
            if (piece) {
                // Of a tile that several blocks share: the last of them to come joins its pieces.
                const int b0 = line.owner(it.begin + place_of<K>(0)), b1 = line.owner(it.begin + place_of<K>(it.t.units - 1));
                __threadfence();
                soft_sync<K::kSoft>();
                if (threadIdx.x == 0) {
                    sh.last = atomicAdd(&a.arrived[b0], 1) == unsigned(b1 - b0);
                    if (sh.last) a.arrived[b0] = 0;
                }
                soft_sync<K::kSoft>();
                if (sh.last) {
                    __threadfence();
                    for (int r = w; r < left; r += K::kSoft / 32)
                        join_row<K>(a, it.t, r, b1 - b0 + 1, [&](int x) { return a.pieces + (2 * int64_t(b0 + x) + (x == 0)) * a.piece_floats; });
                }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(smem_of(&sh.q_free[slot]));
        }
    }
    leave();
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int64_t kArrivedBytes = kMostBlocks * 4;

// The largest piece of a cache's head size: rows of D elements, a maximum and a sum.
int64_t piece_floats(const rr_cache* C) { return C->dim <= 128 ? 64 * (128 + 2) : 32 * (256 + 2); }
int64_t workspace_of(const rr_cache* C) { return kArrivedBytes + int64_t(kMostBlocks) * 2 * piece_floats(C) * 4; }

rr_status check_heads(const rr_cache* C, int32_t n_q) {
    if (n_q < 1 || n_q % C->n_kv || n_q / C->n_kv > 1024)
        return rr_fail(RR_ELAYOUT, "%d query heads of %d key heads: a multiple, up to 1024 times", n_q, C->n_kv);
    return RR_OK;
}

// The pages as TMA sees them: 64 elements, 8 tokens, 64 elements after 64, 8 tokens after
// 8 (through a page's heads, keys and values), pages.  A copy is one page's tokens of a
// head, swizzled as the products read them: heads of whole 64s at once; others 64 elements
// at a time, zeros past the end.
rr_status map_pages(const AttendArgs& a, int dtype, CUtensorMap* map) {
    const CacheShape& c = a.c;
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> known{nullptr};
    PFN_cuTensorMapEncodeTiled_v12000 encode = known.load(std::memory_order_relaxed);
    if (!encode) {
        cudaDriverEntryPointQueryResult found;
        void* f = nullptr;
        RR_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found));
        if (!f || found != cudaDriverEntryPointSuccess) return rr_fail(RR_ECUDA, "the driver has no cuTensorMapEncodeTiled");
        encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
        known.store(encode, std::memory_order_relaxed);
    }
    const bool joined = a.copy_atoms > 1;
    const cuuint64_t size[5] = {cuuint64_t(joined ? 64 : c.dim), 8, cuuint64_t(joined ? a.atoms : 1), cuuint64_t(2 * c.n_kv * (c.page / 8)),
                                cuuint64_t(c.n_pages)};
    const cuuint64_t stride[4] = {cuuint64_t(2 * c.pitch), 128, cuuint64_t(16 * c.pitch), cuuint64_t(c.page_bytes)};
    const cuuint32_t box[5] = {64, 8, cuuint32_t(a.copy_atoms), cuuint32_t(c.page / 8), 1}, step[5] = {1, 1, 1, 1, 1};
    const CUresult e = encode(map, dtype == RR_DST_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5,
                              const_cast<char*>(a.pages), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (e != CUDA_SUCCESS) return rr_fail(RR_ECUDA, "cuTensorMapEncodeTiled: error %d", int(e));
    return RR_OK;
}

template <class K>
rr_status launch(AttendArgs& a, const CUtensorMap& map, int dev, cudaStream_t stream) {
    static std::atomic<uint32_t> ready{0};
    static std::atomic<int> sms[kMaxDevices] = {};
    RR_CUDA(allow_smem(rr_attend_kernel<K>, kSmem, dev, &ready));
    int grid = sms[dev].load(std::memory_order_relaxed);
    if (!grid) {
        RR_CUDA(cudaDeviceGetAttribute(&grid, cudaDevAttrMultiProcessorCount, dev));
        sms[dev].store(grid, std::memory_order_relaxed);
    }
    // No more blocks than there can be units.
    const int64_t tiles = a.c.n_kv * (int64_t(a.rows) * a.group / K::kRows + a.n);
    const int64_t each = (int64_t(a.c.max_pages) * a.c.page + kUnit - 1) / kUnit;
    grid = int(std::min<int64_t>(std::min(grid, kMostBlocks), tiles * each));
    // The ring has what the queries and weights leave.  (The products of a head of an odd number
    // of 64s read, and leave out, 16 KiB behind its values: within the block's memory.)
    const int room = kSmem - 1024 - K::kFixed, stage = a.atoms * 16384;
    a.stages = std::min(room / stage, kMostStages);
    if (a.atoms % 2 && a.stages * stage + 16384 > kSmem - 1024) --a.stages;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(grid));
    cfg.blockDim = dim3(K::kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    RR_CUDA(cudaLaunchKernelEx(&cfg, rr_attend_kernel<K>, a, map));
    return RR_OK;
}

// The rows that a tile is to hold: of sequences of the call's mean number of new tokens,
// and up to as many again.  Tiles of 16 rows are a little faster than larger ones that are as empty; where
// they do not hold a sequence's rows, its keys are read once a tile.  (Of 16 / 64 rows, 96 sequences
// of 500 to 7500 tokens, 8 key heads of 128: 8 rows 254 / 257 us, 16 257 / 260, 24 487 / 265, 40 726 / 281; of 16 / 32,
// 32 sequences, heads of 256: 8 rows 164 / 166, 16 170 / 171, 24 316 / 176, 40 465 / 328.)
template <class T>
rr_status choose(AttendArgs& a, const CUtensorMap& map, int dev, cudaStream_t stream) {
    const int mean = (a.rows + a.n - 1) / a.n, most = std::min(2 * mean - 1, a.rows - a.n + 1);
    const int64_t rows = int64_t(a.group) * std::max(most, 1);
    if (a.c.dim > 128) return rows <= 16 ? launch<Kind<T, 2, 2>>(a, map, dev, stream) : launch<Kind<T, 2, 4>>(a, map, dev, stream);
    if (rows <= 16) return launch<Kind<T, 1, 2>>(a, map, dev, stream);
    return launch<Kind<T, 1, 8>>(a, map, dev, stream);
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
    CUtensorMap map;
    a.atoms = (a.c.dim + 63) / 64;
    a.copy_atoms = a.c.dim % 64 == 0 ? a.atoms : 1;
    a.atom_bytes = a.copy_atoms > 1 ? 1024 : 16384;
    a.eight_bytes = a.copy_atoms > 1 ? 1024 * a.atoms : 1024;
    RR_TRY(map_pages(a, C->dtype, &map));
    const auto with = [&](auto t) -> rr_status {
        using T = decltype(t);
        return choose<T>(a, map, dev, stream);
    };
    return C->dtype == RR_DST_F16 ? with(F16{}) : with(BF16{});
}
