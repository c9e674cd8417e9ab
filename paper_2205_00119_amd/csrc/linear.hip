// Products of matrices with their epilogue: the linear layer and the gradients of its input and weight.
#include "rows.h"

#include <algorithm>
#include <utility>

#include "activation.h"
#include "columns.h"
#include "linear_internal.h"

namespace mics {
namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A tile of an operand in the LDS holds 128 bytes of k for every row of the tile, in chunks of 16 bytes:
//   k contiguous   [row][8 chunks], chunk c of row r in place c ^ (r mod 8), so that the 16 rows that a matrix instruction takes
//                  come out of all banks;
//   turned         [k][chunks of the tile's rows], chunk c of k in place c ^ f(k): 16-bit elements are turned while they are
//                  read (ds_read_b64_tr_b16: lane i of 16 gives the address of four elements of k = i / 4 and gets element i of four
//                  k), 32-bit ones one by one.
// The k that a lane's chunk holds is the same in both, which is all that a sum needs.
constexpr int kRowBytes = 128;
template <int KIND> constexpr int kDepth = kRowBytes / (int)kWidth<KIND>;          // k of a tile
template <int KIND> constexpr int kChunk = 16 / (int)kWidth<KIND>;                 // elements of a chunk

template <int KIND> __device__ __forceinline__ int twist(int k)
{
    return KIND == kF32 ? 4 * (k >> 2 & 3) : 2 * ((k & 3) | (k >> 3 & 1) << 2);
}

// One chunk of an operand, elements from `valid` on are 0.
template <int KIND> __device__ __forceinline__ u32x4 load_chunk(const char* p, ptrdiff_t valid)
{
    if constexpr (KIND != kF32) return load_vec<KIND>(p, (int)min(valid, (ptrdiff_t)kVec)).q[0];
    else {
        u32x4 q{};
        if (valid >= 4) q = *(const u32x4_a4*)p;
        else if (valid > 0) {
            q.x = *(const uint32_t*)p;
            if (valid > 1) q.y = ((const uint32_t*)p)[1];
            if (valid > 2) q.z = ((const uint32_t*)p)[2];
        }
        return q;
    }
}

// The chunk's elements from `by` on, less than a chunk has, come to its front; zeros follow.
template <int KIND> __device__ __forceinline__ void move_up(u32x4& q, int by)
{
    #pragma unroll
    for (int step = 2; step; step /= 2) {
        const bool go = by & (KIND == kF32 ? step : 2 * step);
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t from = i + step < 4 ? q[i + step < 4 ? i + step : 3] : 0u, own = q[i];
            q[i] = go ? from : own;
        }
    }
    if constexpr (KIND != kF32) {
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t next = i < 3 ? q[i < 3 ? i + 1 : 3] : 0u, own = q[i];
            q[i] = by & 1 ? own >> 16 | next << 16 : own;
        }
    }
}

// How the lanes of a workgroup bring a tile of ROWS rows into the LDS: chunk i * LANES + t in the order of the places there, t: the lane.
template <int KIND, bool TURNED, int ROWS, int LANES> struct Stage {
    static constexpr int kCount = ROWS * 8 / LANES, kAcross = ROWS * (int)kWidth<KIND> / 16;
    static_assert(ROWS * 8 % LANES == 0 && (!TURNED || kAcross >= 16), "whole rounds of lanes, and places that stay in their row");
    // row (turned: first of the rows) and k (first of them; turned: the k) of the tile that chunk i holds
    static __device__ __forceinline__ int row(int t, int i)
    {
        const int s = i * LANES + t;
        return TURNED ? ((s % kAcross) ^ twist<KIND>(s / kAcross)) * kChunk<KIND> : s / 8;
    }
    static __device__ __forceinline__ int depth(int t, int i)
    {
        const int s = i * LANES + t;
        return TURNED ? s / kAcross : ((s % 8) ^ (s / 8 % 8)) * kChunk<KIND>;
    }
    // Chunk i, whatever lies behind the last of `rows` rows or of `k` from this tile on read as 0.
    static __device__ __forceinline__ u32x4 load(const ConstRows& m, size_t row0, size_t k0, size_t rows, size_t k, int t, int i)
    {
        const int r = row(t, i), d = depth(t, i);
        const ptrdiff_t right = (ptrdiff_t)(rows - row0) - r, deep = (ptrdiff_t)(k - k0) - d;
        const size_t at = TURNED ? (k0 + d) * m.stride + row0 + r : (row0 + r) * m.stride + k0 + d;
        return load_chunk<KIND>((const char*)m.data + at * kWidth<KIND>, right <= 0 || deep <= 0 ? 0 : TURNED ? right : deep);
    }
    // The fast ways: every chunk is loaded whole, from 32-bit offsets to one address.  `rows` are there from the tile's first on; rows
    // behind them repeat the last: what they give is not stored.  Turned, the last chunk of the rows begins early, so that it ends
    // with them, and is moved up in registers; where that is in front of the tile, the address is that much lower.
    static __device__ __forceinline__ int lower(size_t rows) { return TURNED ? max(kChunk<KIND> - (int)min(rows, (size_t)ROWS), 0) : 0; }
    // What chunk i is moved up by.
    static __device__ __forceinline__ int early(size_t rows, int t, int i)
    {
        return max(row(t, i) - ((int)min(rows, (size_t)ROWS) - kChunk<KIND>), 0);
    }
    static __device__ __forceinline__ uint32_t offset(size_t stride, size_t rows, int t, int i)
    {
        const int r = TURNED ? row(t, i) - early(rows, t, i) + lower(rows) : (int)min((size_t)row(t, i), rows - 1);
        const uint32_t step = (uint32_t)stride, d = depth(t, i);
        return (TURNED ? d * step + r : r * step + d) * (uint32_t)kWidth<KIND>;
    }
    // Chunk i of the last part of a tile of k, which begins at k0 and ends at `last`, loaded without a branch: from a place inside, and
    // moved up and cleared by settle().
    static __device__ __forceinline__ u32x4 rest(const ConstRows& m, size_t row0, size_t k0, size_t rows, size_t last, int t, int i)
    {
        const size_t k = min(k0 + depth(t, i), last - (TURNED ? 1 : kChunk<KIND>));
        const size_t at = TURNED ? k * m.stride + row0 + row(t, i) - early(rows, t, i) : (row0 + min((size_t)row(t, i), rows - 1)) * m.stride + k;
        return *(const u32x4_a2*)((const char*)m.data + at * kWidth<KIND>);
    }
    static __device__ __forceinline__ void settle(u32x4& q, size_t k0, size_t rows, size_t last, int t, int i)
    {
        const ptrdiff_t behind = (ptrdiff_t)(k0 + depth(t, i)) - (ptrdiff_t)last;      // of its first k; 0 and more: nothing is there
        move_up<KIND>(q, TURNED ? early(rows, t, i) & (kChunk<KIND> - 1) : (int)max(behind + kChunk<KIND>, (ptrdiff_t)0) & (kChunk<KIND> - 1));
        if (behind >= 0) q = u32x4{};
    }
    static __device__ __forceinline__ const char* first(const ConstRows& m, size_t row0, size_t k0, size_t rows)
    {
        return (const char*)m.data + (TURNED ? k0 * m.stride + row0 - lower(rows) : row0 * m.stride + k0) * kWidth<KIND>;
    }
    static __device__ __forceinline__ size_t step(const ConstRows& m) { return TURNED ? m.stride * kRowBytes : kRowBytes; }
};

// 16 bytes for each lane from `base` + `offset` into the LDS from byte `to` + TO on, lane after lane.  It counts as a load in flight that
// the compiler does not know of: landed() waits.  m0, which the LDS address goes through, has to settle first.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"        // that no value is kept in m0, which is reserved, is what is meant
template <int TO> __device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t to)
{
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(base), "v"(offset), "s"(to), "i"(TO)
                 : "memory", "scc", "m0");
}
#pragma clang diagnostic pop
// f(std::integral_constant<int, i>) for every i below N.
template <int... I, typename F> __device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void each(F&& f) { each_of(std::make_integer_sequence<int, N>{}, f); }
// All loads and LDS accesses of this wavefront are over, then all wavefronts are here.
__device__ __forceinline__ void landed()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// What a lane hands to the matrix instructions of 16 rows and half the k of a tile: chunk lane / 16 of row lane % 16.
template <int KIND> struct Piece {
    u32x4 q;
};
template <int KIND, bool TURNED, int ROWS> struct Reader {
    const lds_char* tile;
    uint32_t at;                               // of the tile; turned: without the rows' place
    int row0;
    __device__ __forceinline__ Reader(const lds_char* from, int first_row) : tile(from)
    {
        const int lane = threadIdx.x & 63, g = lane / 16, i = lane % 16;
        row0 = first_row;
        constexpr int pitch = ROWS * (int)kWidth<KIND>;
        if constexpr (!TURNED) at = (first_row + i) * kRowBytes;
        else if constexpr (KIND == kF32) at = g * 4 * pitch + (g << 6) + i * 4;
        else at = (g * 8 + i / 4) * pitch + (twist<KIND>(g * 8 + i / 4) * 16) + (i % 4) * 8;
    }
    __device__ __forceinline__ Piece<KIND> read(int block, int half) const
    {
        const int lane = threadIdx.x & 63, g = lane / 16;
        constexpr int pitch = ROWS * (int)kWidth<KIND>;
        Piece<KIND> p;
        if constexpr (!TURNED) {
            p.q = *(const __attribute__((address_space(3))) u32x4*)(tile + at + block * 16 * kRowBytes + ((half * 4 + g) ^ (lane & 7)) * 16);
        } else {
            // the rows' place is below the bits that k sets
            const uint32_t place = (uint32_t)(row0 / 16 + block) * 16 * (uint32_t)kWidth<KIND>;
            const lds_char* const from = tile + (at ^ place);
            if constexpr (KIND == kF32) {
                #pragma unroll
                for (int j = 0; j < 4; ++j) p.q[j] = *(const __attribute__((address_space(3))) uint32_t*)(from + (half * 16 + j) * pitch);
            } else {
                typedef __attribute__((address_space(3))) s16x4 turned_t;
                const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned_t*)(from + half * 32 * pitch));
                const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned_t*)(from + (half * 32 + 4) * pitch));
                const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
                p.q = u32x4{x.x, x.y, y.x, y.y};
            }
        }
        return p;
    }
};

// acc[n][m] += the product of 16 rows of b and 16 of a: a lane gets row lane % 16 of a, rows lane / 16 * 4 on of b.
template <int KIND> __device__ __forceinline__ void multiply(f32x4& acc, const Piece<KIND>& a, const Piece<KIND>& b)
{
    if constexpr (KIND == kBf16) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b.q), __builtin_bit_cast(bf16x8, a.q), acc, 0, 0, 0);
    } else if constexpr (KIND == kF16) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b.q), __builtin_bit_cast(f16x8, a.q), acc, 0, 0, 0);
    } else {
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t y = b.q[j], x = a.q[j];
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, y), __builtin_bit_cast(float, x), acc, 0, 0, 0);
        }
    }
}

struct ProductArgs {
    Product p;
    unsigned bm, bn, tiles_m, tiles_n;
    unsigned units, whole, shared, splits;     // units: whole tiles and parts of the shared ones
    size_t depth;                              // k of a part
    size_t a_rows, b_rows;                     // m and n, or so many elements as rows of a turned copy have
};

// The unit that a workgroup takes: neighbours on one of the 8 L2 caches (workgroups go round them) share rows of the operands.
__device__ __forceinline__ unsigned unit_of(unsigned i, unsigned units)
{
    const unsigned each = units / 8, rest = units % 8, cache = i % 8;
    return cache * each + min(cache, rest) + i / 8;
}

// Tiles of rows that are taken together, column by column: what runs at one time under one of the 8 L2 caches is then 8 x 4 tiles.
// us, 4 / 8 / 16 rows of tiles / all: 4096 x 8192 x 32768 bf16 1673 / 1678 / 1904 / 1909, 8192 x 8192 x 8192 846 / 842 / 859 / 1167.
constexpr unsigned kBand = 8;
// The first row and column of tile t.
struct Origin {
    size_t m, n;
};
__device__ __forceinline__ Origin origin_of(const ProductArgs& g, unsigned t)
{
    const unsigned of_band = kBand * g.tiles_n, band = t / of_band, in_band = t % of_band, high = min(kBand, g.tiles_m - band * kBand);
    return {(size_t)(band * kBand + in_band % high) * g.bm, (size_t)(in_band / high) * g.bn};
}
// What workgroup i computes: the tile, its part of k, and where a part goes.
struct Unit {
    unsigned tile;
    size_t first, last;                        // of k
    float* parts;                              // NULL: the whole tile
};
__device__ __forceinline__ Unit unit_at(const ProductArgs& g, unsigned i)
{
    if (i < g.whole) return {unit_of(i, g.whole), 0, g.p.k, nullptr};
    const unsigned j = unit_of(i - g.whole, g.units - g.whole), split = j / g.shared, at = j % g.shared;
    const size_t first = split * g.depth;
    return {g.whole + at, first, min(g.p.k, first + g.depth), g.p.parts + ((size_t)at * g.splits + split) * (g.bm * g.bn)};
}

// One workgroup for a tile of BM x BN results, WM x WN wavefronts with 64 columns each.
// WAY kDirect: whole chunks begin on 16 bytes, so tiles of k go straight into the LDS, the next one and the one behind it on their
// way; while a wavefront multiplies one half of a tile it reads the next half.  Reads and loads are spread among the matrix
// instructions (us, in front of them / spread: 4096 x 8192 x 4096 bf16 210 / 194, input gradient 4096 x 20480 x 5120 725 / 678, weight
// gradient 8192 x 4096 x 16384 930 / 851).  Neither the LDS (its ports are busy a quarter of the time, 1 % of that with conflicts) nor
// memory bounds it: the matrix units are busy 63 to 70 % of the time, the rest goes to the barrier of each tile.  Slower were tiles of 64
// bytes of k in a ring of four, which wait less for loads and more for barriers (830 / 915 at 8192 x 8192 x 8192), instructions of
// 32 x 32 (830 / 919), and four wavefronts of 128 x 128 (823 / 887).
// kThrough: chunks begin on any element; a tile waits in registers while the one before is multiplied.
// kGuarded: rows shorter than a chunk, tiles of more than 2^31 bytes; every chunk is looked at.
enum { kDirect, kThrough, kGuarded };
template <int KIND, bool AT, bool BT, int BM, int BN, int WM, int WN, int WAY>
__global__ __launch_bounds__(64 * WM * WN, WAY == kThrough && WM * WN == 4 ? 2 : 1) void product_kernel(ProductArgs g)
{
    constexpr int kLanes = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, kOut = TM < 4 ? TM : 4;
    static_assert(TN % 4 == 0, "a wavefront's columns are whole blocks of a checkpoint");
    constexpr int kTileBytes = (BM + BN) * kRowBytes;
    // a wavefront's results on their way out: floats from row to row in the LDS, and lanes for a row
    constexpr int kStagePitch = TN * 16 + 4, kOutBytes = WM * WN * kOut * 16 * kStagePitch * 4, kAcross = TN * 16 / kVec;
    __shared__ __attribute__((aligned(1024))) char lds[std::max(2 * kTileBytes, kOutBytes)];
    typedef Stage<KIND, AT, BM, kLanes> StageA;
    typedef Stage<KIND, BT, BN, kLanes> StageB;
    const Product& p = g.p;
    const int wave = wave_index(), lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    lds_char* const tile = (lds_char*)lds;

    for (unsigned i = blockIdx.x; i < g.units; i += gridDim.x) {
        // Not known to be the same in every turn, so that what a lane derives from it is not kept, in memory, over the loop: us, kept /
        // formed anew, input gradient 4096 x 20480 x 5120 664 / 637, weight gradient 8192 x 4096 x 16384 838 / 825.
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
        const Unit unit = unit_at(g, i);
        const Origin origin = origin_of(g, unit.tile);
        const size_t m0 = origin.m, n0 = origin.n, first = unit.first, last = unit.last;
        f32x4 acc[TM][TN] = {};
        typedef Piece<KIND> PieceA[TM];
        typedef Piece<KIND> PieceB[TN];
        auto read = [&](PieceA& pa, PieceB& pb, int at, int half) {
            const Reader<KIND, AT, BM> a(tile + at * kTileBytes, wm * TM * 16);
            const Reader<KIND, BT, BN> b(tile + at * kTileBytes + BM * kRowBytes, wn * TN * 16);
            #pragma unroll
            for (int n = 0; n < TN; ++n) pb[n] = b.read(n, half);
            #pragma unroll
            for (int m = 0; m < TM; ++m) pa[m] = a.read(m, half);
        };
        auto add = [&](const PieceA& pa, const PieceB& pb) {
            #pragma unroll
            for (int m = 0; m < TM; ++m) {
                #pragma unroll
                for (int n = 0; n < TN; ++n) multiply<KIND>(acc[m][n], pa[m], pb[n]);
            }
        };
        auto fetch = [&](u32x4 (&ra)[StageA::kCount], u32x4 (&rb)[StageB::kCount], size_t k0) {
            #pragma unroll
            for (int c = 0; c < StageA::kCount; ++c) ra[c] = StageA::load(p.a, m0, k0, p.m, last, t, c);
            #pragma unroll
            for (int c = 0; c < StageB::kCount; ++c) rb[c] = StageB::load(p.b, n0, k0, p.n, last, t, c);
        };
        auto put = [&](const u32x4 (&ra)[StageA::kCount], const u32x4 (&rb)[StageB::kCount], int at) {
            lds_char* const to = tile + at * kTileBytes + t * 16;
            #pragma unroll
            for (int c = 0; c < StageA::kCount; ++c) *(__attribute__((address_space(3))) u32x4*)(to + c * kLanes * 16) = ra[c];
            #pragma unroll
            for (int c = 0; c < StageB::kCount; ++c)
                *(__attribute__((address_space(3))) u32x4*)(to + BM * kRowBytes + c * kLanes * 16) = rb[c];
        };
        if constexpr (WAY != kGuarded) {
            if (const size_t rest = last > first ? (last - first) % kDepth<KIND> : 0) {      // in front: a sum has no order
                u32x4 ra[StageA::kCount], rb[StageB::kCount];
                #pragma unroll
                for (int c = 0; c < StageA::kCount; ++c) ra[c] = StageA::rest(p.a, m0, last - rest, g.a_rows - m0, last, t, c);
                #pragma unroll
                for (int c = 0; c < StageB::kCount; ++c) rb[c] = StageB::rest(p.b, n0, last - rest, g.b_rows - n0, last, t, c);
                #pragma unroll
                for (int c = 0; c < StageA::kCount; ++c) StageA::settle(ra[c], last - rest, g.a_rows - m0, last, t, c);
                #pragma unroll
                for (int c = 0; c < StageB::kCount; ++c) StageB::settle(rb[c], last - rest, g.b_rows - n0, last, t, c);
                put(ra, rb, 0);
                __syncthreads();
                #pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (AT && rest <= (size_t)half * (kDepth<KIND> / 2)) break;      // the gradient of a weight may have few rows
                    PieceA pa;
                    PieceB pb;
                    read(pa, pb, 0, half);
                    add(pa, pb);
                }
                __syncthreads();
            }
            const size_t whole = last > first ? (last - first) / kDepth<KIND> : 0;
            if (whole) {
                uint32_t oa[StageA::kCount], ob[StageB::kCount];
                #pragma unroll
                for (int c = 0; c < StageA::kCount; ++c) oa[c] = StageA::offset(p.a.stride, g.a_rows - m0, t, c);
                #pragma unroll
                for (int c = 0; c < StageB::kCount; ++c) ob[c] = StageB::offset(p.b.stride, g.b_rows - n0, t, c);
                const char *from_a = StageA::first(p.a, m0, first, g.a_rows - m0), *from_b = StageB::first(p.b, n0, first, g.b_rows - n0);
                const size_t step_a = StageA::step(p.a), step_b = StageB::step(p.b);
                if constexpr (WAY == kThrough) {
                    u32x4 ra[StageA::kCount], rb[StageB::kCount];
                    auto load = [&] {
                        #pragma unroll
                        for (int c = 0; c < StageA::kCount; ++c) ra[c] = *(const u32x4_a2*)(from_a + oa[c]);
                        #pragma unroll
                        for (int c = 0; c < StageB::kCount; ++c) rb[c] = *(const u32x4_a2*)(from_b + ob[c]);
                        from_a += step_a;
                        from_b += step_b;
                    };
                    auto place = [&](int at) {
                        if (AT && p.m - m0 < BM) {              // the tile at the rows' end
                            #pragma unroll
                            for (int c = 0; c < StageA::kCount; ++c) move_up<KIND>(ra[c], StageA::early(p.m - m0, t, c));
                        }
                        if (BT && p.n - n0 < BN) {
                            #pragma unroll
                            for (int c = 0; c < StageB::kCount; ++c) move_up<KIND>(rb[c], StageB::early(p.n - n0, t, c));
                        }
                        put(ra, rb, at);
                    };
                    load();
                    place(0);
                    if (whole > 1) load();
                    int at = 0;
                    for (size_t left = whole; left; --left, at ^= 1) {
                        barrier_lds();
                        PieceA pa;
                        PieceB pb;
                        read(pa, pb, at, 0);
                        if (left > 1) place(at ^ 1);
                        if (left > 2) load();
                        add(pa, pb);
                        read(pa, pb, at, 1);
                        add(pa, pb);
                    }
                    __syncthreads();
                } else {
                const uint32_t place = (uint32_t)(uintptr_t)tile + wave * 1024;
                constexpr int kLoads = StageA::kCount + StageB::kCount;
                // loads I to I + N - 1 of a tile
                auto some = [&](uint32_t to, auto first_of, auto count) {
                    each<decltype(count)::value>([&](auto c) {
                        constexpr int I = decltype(first_of)::value + decltype(c)::value;
                        if constexpr (I < StageA::kCount) load_to_lds<I * kLanes * 16>(from_a, oa[I], to);
                        else if constexpr (I < kLoads)
                            load_to_lds<BM * kRowBytes + (I - StageA::kCount) * kLanes * 16>(from_b, ob[I - StageA::kCount], to);
                    });
                };
                auto load = [&](int at) {
                    some(place + at * kTileBytes, std::integral_constant<int, 0>{}, std::integral_constant<int, kLoads>{});
                    from_a += step_a;
                    from_b += step_b;
                };
                // Half a tile: row by row of results the products of what has been read, what is multiplied next, and with LOADS a part of
                // the loads of another tile, so that none of them comes in one piece.
                auto half_of = [&](const PieceA& pa, const PieceB& pb, PieceA& na, PieceB& nb, int at, auto half, auto loads) {
                    const Reader<KIND, AT, BM> a(tile + at * kTileBytes, wm * TM * 16);
                    const Reader<KIND, BT, BN> b(tile + at * kTileBytes + BM * kRowBytes, wn * TN * 16);
                    const uint32_t to = place + (at ^ 1) * kTileBytes;
                    each<TM>([&](auto r) {
                        constexpr int M = decltype(r)::value, share = (kLoads + TM - 1) / TM;
                        constexpr int columns = (TN + TM - 1) / TM;
                        each<columns>([&](auto c) {
                            constexpr int N = M * columns + decltype(c)::value;
                            if constexpr (N < TN) nb[N] = b.read(N, decltype(half)::value);
                        });
                        na[M] = a.read(M, decltype(half)::value);
                        if constexpr (decltype(loads)::value) some(to, std::integral_constant<int, M * share>{}, std::integral_constant<int, share>{});
                        #pragma unroll
                        for (int n = 0; n < TN; ++n) multiply<KIND>(acc[M][n], pa[M], pb[n]);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                    if constexpr (decltype(loads)::value) {
                        from_a += step_a;
                        from_b += step_b;
                    }
                };
                PieceA a0, a1;
                PieceB b0, b1;
                load(0);
                if (whole > 1) load(1);
                landed();
                read(a0, b0, 0, 0);
                int at = 0;
                size_t k = whole;
                for (; k > 2; --k, at ^= 1) {                   // the tile behind the next one takes this one's place
                    half_of(a0, b0, a1, b1, at, std::integral_constant<int, 1>{}, std::false_type{});
                    landed();
                    half_of(a1, b1, a0, b0, at ^ 1, std::integral_constant<int, 0>{}, std::true_type{});
                }
                for (; k; --k, at ^= 1) {                       // behind the last tile is read what nothing uses
                    half_of(a0, b0, a1, b1, at, std::integral_constant<int, 1>{}, std::false_type{});
                    landed();
                    half_of(a1, b1, a0, b0, at ^ 1, std::integral_constant<int, 0>{}, std::false_type{});
                }
                }
            }
        } else {
            u32x4 ra[StageA::kCount], rb[StageB::kCount];
            int at = 0;
            if (first < last) {
                fetch(ra, rb, first);
                put(ra, rb, 0);
            }
            for (size_t k0 = first; k0 < last; k0 += kDepth<KIND>, at ^= 1) {
                __syncthreads();
                const bool more = k0 + kDepth<KIND> < last;
                if (more) fetch(ra, rb, k0 + kDepth<KIND>);
                #pragma unroll
                for (int half = 0; half < 2; ++half) {
                    PieceA pa;
                    PieceB pb;
                    read(pa, pb, at, half);
                    add(pa, pb);
                }
                if (more) put(ra, rb, at ^ 1);
            }
        }
        // A wavefront's results pass through the LDS into rows of its columns, eight to a lane, whose bias is loaded once.
        typedef __attribute__((address_space(3))) f32x4 lds_f4;
        constexpr int kStep = 64 / kAcross;                     // rows at a time
        lds_char* const mine = tile + wave * kOut * 16 * kStagePitch * 4;
        const size_t col = n0 + wn * TN * 16 + lane % kAcross * kVec;
        const int valid = col < p.n ? (int)min(p.n - col, (size_t)kVec) : 0;
        Epilogue e = p.e;
        float bias[kVec] = {};
        if (e.bias && !unit.parts) load_any((const char*)e.bias, e.param, (unsigned)(col / kVec), valid, bias);
        const bool bare = !unit.parts && !e.bias && !e.pre.data && !e.codes.data && !e.residual.data && !e.act && e.out_kind == KIND;
        e.bias = nullptr;
        __syncthreads();
        #pragma unroll
        for (int part = 0; part < TM / kOut; ++part) {
            #pragma unroll
            for (int m = 0; m < kOut; ++m) {
                #pragma unroll
                for (int n = 0; n < TN; ++n)
                    *(lds_f4*)(mine + ((m * 16 + lane % 16) * kStagePitch + n * 16 + lane / 16 * 4) * 4) = acc[part * kOut + m][n];
            }
            wave_lds_order();                                   // other lanes' sums are read
            const size_t row0 = m0 + wm * TM * 16 + part * kOut * 16 + lane / kAcross;
            const int rows = row0 < p.m ? (int)min((p.m - row0 + kStep - 1) / kStep, (size_t)(kOut * 16 / kStep)) : 0;
            const lds_char* from = mine + (lane / kAcross * kStagePitch + lane % kAcross * kVec) * 4;
            auto take = [&](float (&v)[kVec]) {
                const f32x4 low = *(const lds_f4*)from, high = *(const lds_f4*)(from + 16);
                from += kStep * kStagePitch * 4;
                #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = low[i];
                    v[i + 4] = high[i];
                }
            };
            float v[kVec];
            if (unit.parts) {
                float* to = unit.parts + (row0 - m0) * BN + (col - n0);
                for (int r = 0; r < rows; ++r, to += kStep * BN) {
                    take(v);
                    store_vec<kF32>((char*)to, pack<kF32>(v), kVec);
                }
            } else if (bare) {
                char* to = (char*)e.out.data + (row0 * e.out.stride + col) * kWidth<KIND>;
                for (int r = 0; r < rows; ++r, to += e.out.stride * (kStep * kWidth<KIND>)) {
                    take(v);
                    store_vec<KIND>(to, pack<KIND>(v), valid);
                }
            } else {
                for (int r = 0; r < rows; ++r) {
                    take(v);
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) v[i] += bias[i];
                    finish<KIND>(e, row0 + r * kStep, (unsigned)(col / kVec), (unsigned)p.n, valid, v);
                }
            }
            wave_lds_order();                                   // before the next part takes their place
        }
        __syncthreads();
    }
}

// Products of few rows: all that counts is that the weights are read once, as fast as memory gives them.  A workgroup takes BN
// columns; its wavefronts take turns at the tiles of k, 128 bytes of each row of b at a time, straight into the operands of the
// matrix instructions, and their sums are added in the LDS.
//   b not turned   16 columns to an instruction, lane i of 16 has chunk lane / 16 of row i;
//   b turned       a lane has a chunk of columns of kChunk k, which it turns around in registers: instruction j takes column j of
//                  every chunk.
// us, in tiles of 32 to 128 rows, with parts of k / so, two sets of weights in turn: 1 x 2560 x 10240 bf16 17.4 / 12.0 (12 in the kernel's
// own trace; the weights alone take 7.7), 1 x 4096 x 4096 12.9 / 7.9, 16 x 4096 x 4096 13.6 / 10.1, 32 x 4096 x 4096 14.2 / 13.5, the
// input's gradient of 16 x 2560 x 10240 f32 25.6 / 22.5.  Every wavefront loads a for itself, once for every 16 columns, so tiles are
// faster where rows and columns are many, and the rule, which takes this kernel for all it can serve, loses there: 16 x 5120 x 20480
// bf16 47.7 / 61.0, 32 x 5120 x 20480 49.2 / 75.3, 8 x 2560 x 10240 f32 23.9 / 25.3, 32 x 20480 x 5120 f32 88.0 / 186, input's gradient
// 32 x 2560 x 10240 f32 26.4 / 32.8.
// Rows of b off 16 bytes are left to the tiles unless b is turned: 16 rows at a time from 64 bytes each, 56 / 150.  Two tiles of k at a
// time and 32 or 64 columns were slower (39 / 51).
constexpr int kFewWaves = 8;
template <int KIND, bool BT, int TM, int BN>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows_kernel(ProductArgs g)
{
    constexpr int C = kChunk<KIND>, NF = BN / 16, BM = TM * 16, kPitch = BN + 4;
    static_assert(!BT || NF == C, "");
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][BM * kPitch];
    const Product& p = g.p;
    const int wave = wave_index(), lane = threadIdx.x & 63, i16 = lane % 16, g4 = lane / 16;
    for (unsigned i = blockIdx.x; i < g.units; i += gridDim.x) {
        const Unit unit = unit_at(g, i);
        const size_t n0 = (size_t)unit.tile * BN;
        const char* a_row[TM];
        #pragma unroll
        for (int m = 0; m < TM; ++m) a_row[m] = (const char*)p.a.data + min((size_t)(m * 16 + i16), p.m - 1) * p.a.stride * kWidth<KIND>;
        // turned: the last chunk of a row of b begins early and is moved up
        const size_t column = n0 + (size_t)i16 * C, start = BT ? min(column, p.n - C) : 0;
        const int early = (int)min(column - start, (size_t)C);
        const char* b_row[BT ? 1 : NF];
        if constexpr (BT) b_row[0] = (const char*)p.b.data + start * kWidth<KIND>;
        else {
            #pragma unroll
            for (int n = 0; n < NF; ++n) b_row[n] = (const char*)p.b.data + min(n0 + n * 16 + i16, p.n - 1) * p.b.stride * kWidth<KIND>;
        }
        f32x4 acc[TM][NF] = {};
        // one half of a tile of k from k0 on, of which the first `there` are there
        auto half = [&](size_t k0, auto all, size_t there) {
            constexpr bool ALL = decltype(all)::value;
            Piece<KIND> a[TM], b[NF];
            const ptrdiff_t rest = (ptrdiff_t)there - g4 * C;
            if constexpr (BT) {
                u32x4 rows[C];
                const char* const from = b_row[0] + (k0 + g4 * C) * p.b.stride * kWidth<KIND>;
                const uint32_t step = (uint32_t)p.b.stride * (uint32_t)kWidth<KIND>;
                #pragma unroll
                for (int r = 0; r < C; ++r) {
                    rows[r] = u32x4{};
                    if (ALL || r < rest) rows[r] = *(const u32x4_a2*)(from + r * step);
                }
                if (early) {
                    #pragma unroll
                    for (int r = 0; r < C; ++r) move_up<KIND>(rows[r], early);
                }
                #pragma unroll
                for (int n = 0; n < NF; ++n) {
                    if constexpr (KIND == kF32) {
                        #pragma unroll
                        for (int r = 0; r < 4; ++r) b[n].q[r] = rows[r % C][n % 4];
                    } else {
                        #pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint32_t low = rows[(2 * r) % C][n / 2 % 4], high = rows[(2 * r + 1) % C][n / 2 % 4];
                            b[n].q[r] = n % 2 ? low >> 16 | (high & 0xFFFF0000u) : (low & 0xFFFFu) | high << 16;
                        }
                    }
                }
            } else {
                #pragma unroll
                for (int n = 0; n < NF; ++n) {
                    const char* const from = b_row[n] + (k0 + g4 * C) * kWidth<KIND>;
                    if constexpr (ALL) b[n].q = *(const u32x4_a2*)from;
                    else b[n].q = load_chunk<KIND>(from, rest);
                }
            }
            #pragma unroll
            for (int m = 0; m < TM; ++m) {
                const char* const from = a_row[m] + (k0 + g4 * C) * kWidth<KIND>;
                if constexpr (ALL) a[m].q = *(const u32x4_a2*)from;
                else a[m].q = load_chunk<KIND>(from, rest);
            }
            #pragma unroll
            for (int m = 0; m < TM; ++m) {
                #pragma unroll
                for (int n = 0; n < NF; ++n) multiply<KIND>(acc[m][n], a[m], b[n]);
            }
        };
        size_t k0 = unit.first + (size_t)wave * kDepth<KIND>;
        constexpr size_t turn = kFewWaves * kDepth<KIND>;
        for (; k0 + kDepth<KIND> <= unit.last; k0 += turn) {
            half(k0, std::true_type{}, 0);
            half(k0 + kDepth<KIND> / 2, std::true_type{}, 0);
        }
        for (; k0 < unit.last; k0 += turn) {                    // the last tile of k, for one wavefront
            half(k0, std::false_type{}, unit.last - k0);
            if (k0 + kDepth<KIND> / 2 < unit.last) half(k0 + kDepth<KIND> / 2, std::false_type{}, unit.last - k0 - kDepth<KIND> / 2);
        }
        // a lane has row lane % 16 and the columns that belong to rows lane / 16 * 4 + r of the instructions' first operand
        __syncthreads();
        #pragma unroll
        for (int m = 0; m < TM; ++m) {
            float* const to = sums[wave] + (m * 16 + i16) * kPitch;
            #pragma unroll
            for (int n = 0; n < NF; ++n) {
                #pragma unroll
                for (int r = 0; r < 4; ++r) to[BT ? (g4 * 4 + r) * C + n : n * 16 + g4 * 4 + r] = acc[m][n][r];
            }
        }
        __syncthreads();
        for (int at = threadIdx.x; at < BM * BN / kVec; at += 64 * kFewWaves) {
            const int row = at / (BN / kVec), c = at % (BN / kVec);
            float v[kVec] = {};
            for (int w = 0; w < kFewWaves; ++w) {
                const float* const from = sums[w] + row * kPitch + c * kVec;
                #pragma unroll
                for (int e = 0; e < kVec; ++e) v[e] += from[e];
            }
            const size_t col = n0 + (size_t)c * kVec;
            const int valid = col < p.n ? (int)min(p.n - col, (size_t)kVec) : 0;
            if (unit.parts) store_vec<kF32>((char*)(unit.parts + row * BN + c * kVec), pack<kF32>(v), kVec);
            else if ((size_t)row < p.m) finish<KIND>(p.e, row, (unsigned)(col / kVec), (unsigned)p.n, valid, v);
        }
        __syncthreads();
    }
}

// The sums of the shared tiles' parts, in ascending order, and what happens to them: 3.9 us for few parts, which is the launch.
constexpr int kJoinLanes = 64;
template <int KIND> __global__ __launch_bounds__(kJoinLanes) void join_kernel(ProductArgs g)
{
    const Product& p = g.p;
    const unsigned across = g.bn / kVec, size = g.bm * g.bn;
    const size_t lanes = (size_t)g.shared * (size / kVec);
    for (size_t i = (size_t)blockIdx.x * kJoinLanes + threadIdx.x; i < lanes; i += (size_t)gridDim.x * kJoinLanes) {
        const unsigned at = (unsigned)(i / (size / kVec)), in = (unsigned)(i % (size / kVec)), r = in / across, c = in % across;
        const Origin origin = origin_of(g, g.whole + at);
        const size_t row = origin.m + r, col = origin.n + (size_t)c * kVec;
        if (row >= p.m) continue;                               // whole blocks of lanes
        const float* const from = p.parts + (size_t)at * g.splits * size + (size_t)in * kVec;
        float v[kVec] = {};
        #pragma unroll 4
        for (unsigned s = 0; s < g.splits; ++s) {
            const f32x4 low = *(const f32x4_a4*)(from + (size_t)s * size), high = *(const f32x4_a4*)(from + (size_t)s * size + 4);
            #pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] += low[e];
                v[e + 4] += high[e];
            }
        }
        finish<KIND>(p.e, row, (unsigned)(col / kVec), (unsigned)p.n, col < p.n ? (int)min(p.n - col, (size_t)kVec) : 0, v);
    }
}

template <int KIND, bool BT> int launch_few(const ProductArgs& g, void* stream)
{
    constexpr int wide = BT ? 16 * kChunk<KIND> : 64;
    const dim3 grid(grid_of(g.units)), block(64 * kFewWaves);
    auto go = [&](auto TM) {
        if constexpr (!BT)
            if (g.bn == 16) return launch_args(few_rows_kernel<KIND, BT, decltype(TM)::value, 16>, grid, block, 0, stream, g);
        return launch_args(few_rows_kernel<KIND, BT, decltype(TM)::value, wide>, grid, block, 0, stream, g);
    };
    return g.bm == 16 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 2>{});
}

// Operands copied into rows on 16 bytes, chunk by chunk; blockIdx.y: which.  Behind the rows and their ends are zeros, so that no tile
// of k is in part (2047 x 5121 x 2561 binary16 103 / 78 us).  47 MB take 16 us, 5.9 TB/s read and written.
struct Copy {
    const char* from;
    char* to;
    size_t there, rows, stride, chunks;        // rows of the operand, of the copy; bytes from one to the next; chunks of the copy's
    size_t bytes;                              // of the operand's
};
struct CopyArgs {
    Copy c[2];
};
constexpr int kCopyLanes = 256;
template <int KIND> __global__ __launch_bounds__(kCopyLanes) void copy_kernel(CopyArgs g)
{
    const Copy& c = g.c[blockIdx.y];
    const size_t all = c.rows * c.chunks;
    for (size_t base = (size_t)blockIdx.x * kCopyLanes; base < all; base += (size_t)gridDim.x * kCopyLanes) {
        const size_t row0 = base / c.chunks;                                    // the same in all lanes
        const unsigned at = (unsigned)(base - row0 * c.chunks) + threadIdx.x, chunks = (unsigned)c.chunks, up = at / chunks;
        const size_t row = row0 + up, i = base + threadIdx.x;
        if (i >= all) break;
        const ptrdiff_t place = (ptrdiff_t)(at - up * chunks) * 16, valid = row < c.there ? ((ptrdiff_t)c.bytes - place) / (ptrdiff_t)kWidth<KIND> : 0;
        const u32x4 q = load_chunk<KIND>(c.from + row * c.stride + place, valid);
        *(u32x4*)(c.to + i * 16) = q;
    }
}

template <int KIND, bool AT, bool BT, int BM, int BN, int WM, int WN, int WAY> int launch_tiles(const ProductArgs& g, void* stream)
{
    return launch_args(product_kernel<KIND, AT, BT, BM, BN, WM, WN, WAY>, dim3(grid_of(g.units)), dim3(64 * WM * WN), 0, stream, g);
}

}  // namespace

int launch_product(const Product& p, const ProductPlan& plan, int kind, void* stream)
{
    const size_t width = kind == kF32 ? 4 : 2;
    ProductArgs g{p, (unsigned)plan.bm, (unsigned)plan.bn, (unsigned)ceil_div(p.m, plan.bm), (unsigned)ceil_div(p.n, plan.bn),
                  (unsigned)(plan.whole + plan.shared * plan.splits), (unsigned)plan.whole, (unsigned)plan.shared, (unsigned)plan.splits,
                  plan.depth * (kRowBytes / width), p.m, p.n};
    if (plan.a_copy + plan.b_copy) {
        char* to = (char*)(((uintptr_t)p.parts + parts_bytes(plan) + 15) / 16 * 16);
        CopyArgs c{};
        size_t most = 0;
        int n = 0;
        if (plan.a_copy && plan.b_copy) g.p.k = copy_k(p.k, width);
        auto take = [&](ConstRows& m, bool turned, size_t& rows, size_t bytes) {
            if (!bytes) return;
            const size_t there = turned ? p.k : rows, high = turned ? g.p.k : rows, wide = turned ? rows : p.k;
            const size_t stride = copy_stride(turned ? rows : g.p.k, width);
            c.c[n++] = {(const char*)m.data, to, there, high, m.stride * width, stride * width / 16, wide * width};
            most = std::max(most, bytes / 16);
            m = {to, stride};
            if (turned) rows = stride;
            to += bytes;
        };
        take(g.p.a, p.a_turned, g.a_rows, plan.a_copy);
        take(g.p.b, p.b_turned, g.b_rows, plan.b_copy);
        const int err = dispatch_kind(kind, [&](auto K) {
            return launch_args(copy_kernel<decltype(K)::value>, dim3(grid_of((most + kCopyLanes - 1) / kCopyLanes), (unsigned)n), dim3(kCopyLanes), 0,
                               stream, c);
        });
        if (err) return err;
    }
    const int err = dispatch_kind(kind, [&](auto K) { return dispatch_flag(p.a_turned, [&](auto A) { return dispatch_flag(p.b_turned, [&](auto B) {
        constexpr int KIND = decltype(K)::value;
        constexpr bool AT = decltype(A)::value, BT = decltype(B)::value;
        constexpr size_t W = kWidth<KIND>;
        if constexpr (AT && !BT) return 0;
        else {
            if constexpr (!AT)
                if (plan.few) return launch_few<KIND, BT>(g, stream);
            if (!in_chunks(p.a, AT, p.m, p.k, W) || !in_chunks(p.b, BT, p.n, p.k, W))
                return launch_tiles<KIND, AT, BT, 128, 128, 2, 2, kGuarded>(g, stream);
            return dispatch_flag(on_16(g.p.a, AT, g.a_rows, W) && on_16(g.p.b, BT, g.b_rows, W), [&](auto D) {
                constexpr int WAY = decltype(D)::value ? kDirect : kThrough;
                if constexpr (KIND == kF32 && !AT)
                    if (plan.bm == 32) return launch_tiles<KIND, AT, BT, 32, 128, 2, 2, WAY>(g, stream);
                if constexpr (KIND == kF32)
                    if (plan.bm == 64) return launch_tiles<KIND, AT, BT, 64, 64, 4, 1, WAY>(g, stream);
                if constexpr (KIND != kF32 && !(AT && WAY == kThrough))
                    if (plan.bm == 256) return launch_tiles<KIND, AT, BT, 256, 256, 2, 4, WAY>(g, stream);
                return launch_tiles<KIND, AT, BT, 128, 128, 2, 2, WAY>(g, stream);
            });
        }
    }); }); });
    if (err || plan.splits == 1) return err;
    return dispatch_kind(kind, [&](auto K) {
        const size_t lanes = plan.shared * plan.bm * (plan.bn / kVec);
        return launch_args(join_kernel<decltype(K)::value>, dim3(grid_of((lanes + kJoinLanes - 1) / kJoinLanes)), dim3(kJoinLanes), 0, stream, g);
    });
}

}  // namespace mics
