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
    u32x4 q{};
    if (valid >= kChunk<KIND>) {
        if constexpr (KIND == kF32) q = *(const u32x4_a4*)p;
        else q = *(const u32x4_a2*)p;
    } else {
        #pragma unroll
        for (int i = 0; i < kChunk<KIND>; ++i)
            if (i < valid) {
                if constexpr (KIND == kF32) q[i] = ((const uint32_t*)p)[i];
                else q[i / 2] |= (uint32_t)((const uint16_t*)p)[i] << (i % 2 * 16);
            }
    }
    return q;
}

// How the lanes of a workgroup bring a tile of ROWS rows into the LDS: chunk i * LANES + lane in the order of the places there.
template <int KIND, bool TURNED, int ROWS, int LANES> struct Stage {
    static constexpr int kCount = ROWS * 8 / LANES, kAcross = ROWS * (int)kWidth<KIND> / 16;
    static_assert(ROWS * 8 % LANES == 0, "");
    // row (turned: first of the rows) and k (first of them; turned: the k) of the tile that chunk i holds
    static __device__ __forceinline__ int row(int i)
    {
        const int s = i * LANES + (int)threadIdx.x;
        return TURNED ? ((s % kAcross) ^ twist<KIND>(s / kAcross)) * kChunk<KIND> : s / 8;
    }
    static __device__ __forceinline__ int depth(int i)
    {
        const int s = i * LANES + (int)threadIdx.x;
        return TURNED ? s / kAcross : ((s % 8) ^ (s / 8 % 8)) * kChunk<KIND>;
    }
    // Chunk i, whatever lies behind the last of `rows` rows or of `k` from this tile on read as 0.
    static __device__ __forceinline__ u32x4 load(const ConstRows& m, size_t row0, size_t k0, size_t rows, size_t k, int i)
    {
        const int r = row(i), d = depth(i);
        const ptrdiff_t right = (ptrdiff_t)(rows - row0) - r, deep = (ptrdiff_t)(k - k0) - d;
        const size_t at = TURNED ? (k0 + d) * m.stride + row0 + r : (row0 + r) * m.stride + k0 + d;
        return load_chunk<KIND>((const char*)m.data + at * kWidth<KIND>, right <= 0 || deep <= 0 ? 0 : TURNED ? right : deep);
    }
    // The fast ways: every chunk is loaded whole, from 32-bit offsets to one address.  `rows` are there from the tile's first on; rows
    // behind them repeat the last: what they give is not stored.  Turned, the last chunk of the rows begins early, so that it ends
    // with them, and is moved up in registers; where that is in front of the tile, the address is that much lower.
    static __device__ __forceinline__ int lower(size_t rows) { return TURNED ? max(kChunk<KIND> - (int)min(rows, (size_t)ROWS), 0) : 0; }
    // What chunk i is moved up by.
    static __device__ __forceinline__ int early(size_t rows, int i)
    {
        return max(row(i) - ((int)min(rows, (size_t)ROWS) - kChunk<KIND>), 0);
    }
    static __device__ __forceinline__ uint32_t offset(size_t stride, size_t rows, int i)
    {
        const int r = TURNED ? row(i) - early(rows, i) + lower(rows) : (int)min((size_t)row(i), rows - 1);
        const uint32_t step = (uint32_t)stride, d = depth(i);
        return (TURNED ? d * step + r : r * step + d) * (uint32_t)kWidth<KIND>;
    }
    static __device__ __forceinline__ const char* first(const ConstRows& m, size_t row0, size_t k0, size_t rows)
    {
        return (const char*)m.data + (TURNED ? k0 * m.stride + row0 - lower(rows) : row0 * m.stride + k0) * kWidth<KIND>;
    }
    static __device__ __forceinline__ size_t step(const ConstRows& m) { return TURNED ? m.stride * kRowBytes : kRowBytes; }
};

// 16 bytes for each lane from `base` + `offset` into the LDS from byte `to` + TO on, lane after lane.  It counts as a load in flight that
// the compiler does not know of: landed() waits.  m0, which nothing else here uses, has to settle first.
template <int TO> __device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t to)
{
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(base), "v"(offset), "s"(to), "i"(TO) : "memory", "scc");
}
// The chunk's elements from `by` on come to its front.
template <int KIND> __device__ __forceinline__ void move_up(u32x4& q, int by)
{
    #pragma unroll
    for (int step = 2; step; step /= 2) {
        const bool go = by & (KIND == kF32 ? step : 2 * step);
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t from = q[i + step < 4 ? i + step : 3];
            q[i] = go ? from : q[i];
        }
    }
    if constexpr (KIND != kF32) {
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t next = q[i < 3 ? i + 1 : 3], own = q[i];
            q[i] = by & 1 ? own >> 16 | next << 16 : own;
        }
    }
}
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
    size_t tiles_m, tiles_n, units;            // units: tiles times splits
    size_t depth;                              // tiles of k in a split
    int splits;
};

// The unit that a workgroup takes: neighbours on one of the 8 L2 caches (workgroups go round them) share rows of the operands.
__device__ __forceinline__ size_t unit_of(size_t i, size_t units)
{
    const size_t each = units / 8, rest = units % 8, cache = i % 8;
    return cache * each + min(cache, rest) + i / 8;
}

// Tiles of rows that are taken together, column by column: what runs at one time under one of the 8 L2 caches is then 8 x 4 tiles.
// us, 4 / 8 / 16 rows of tiles / all: 4096 x 8192 x 32768 bf16 1673 / 1678 / 1904 / 1909, 8192 x 8192 x 8192 846 / 842 / 859 / 1167.
constexpr size_t kBand = 8;
constexpr int kStagePitch = 64 + 4;            // floats of a row of a wavefront's results in the LDS

// One workgroup for a tile of BM x BN results, WM x WN wavefronts with 64 columns each.
// WAY kDirect: whole chunks begin on 16 bytes, so tiles of k go straight into the LDS, two of them in flight; while a wavefront
// multiplies one half of a tile it reads the next half.
// kThrough: chunks begin on any element; a tile waits in registers while the one before is multiplied.
// kGuarded: rows shorter than a chunk, tiles of more than 2^31 bytes; every chunk is looked at.  So is the last part of a tile of k
// in the other two.
enum { kDirect, kThrough, kGuarded };
template <int KIND, bool AT, bool BT, int BM, int BN, int WM, int WN, int WAY>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(ProductArgs g)
{
    constexpr int kLanes = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, kOut = TM < 4 ? TM : 4;
    static_assert(TN == 4, "a wavefront's columns are one block of a checkpoint");
    constexpr int kTileBytes = (BM + BN) * kRowBytes, kOutBytes = WM * WN * kOut * 16 * kStagePitch * 4;
    __shared__ __attribute__((aligned(1024))) char lds[std::max(2 * kTileBytes, kOutBytes)];
    typedef Stage<KIND, AT, BM, kLanes> StageA;
    typedef Stage<KIND, BT, BN, kLanes> StageB;
    const Product& p = g.p;
    const int wave = wave_index(), lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    lds_char* const tile = (lds_char*)lds;

    for (size_t i = blockIdx.x; i < g.units; i += gridDim.x) {
        const size_t unit = unit_of(i, g.units), tiles = g.tiles_m * g.tiles_n;
        const size_t split = unit / tiles, t = unit % tiles;
        const size_t band = t / (kBand * g.tiles_n), in_band = t % (kBand * g.tiles_n), high = min(kBand, g.tiles_m - band * kBand);
        const size_t m0 = (band * kBand + in_band % high) * BM, n0 = in_band / high * BN;
        size_t first = split * g.depth * kDepth<KIND>;
        const size_t last = min(p.k, first + g.depth * kDepth<KIND>);
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
            for (int c = 0; c < StageA::kCount; ++c) ra[c] = StageA::load(p.a, m0, k0, p.m, last, c);
            #pragma unroll
            for (int c = 0; c < StageB::kCount; ++c) rb[c] = StageB::load(p.b, n0, k0, p.n, last, c);
        };
        auto put = [&](const u32x4 (&ra)[StageA::kCount], const u32x4 (&rb)[StageB::kCount], int at) {
            lds_char* const to = tile + at * kTileBytes + threadIdx.x * 16;
            #pragma unroll
            for (int c = 0; c < StageA::kCount; ++c) *(__attribute__((address_space(3))) u32x4*)(to + c * kLanes * 16) = ra[c];
            #pragma unroll
            for (int c = 0; c < StageB::kCount; ++c)
                *(__attribute__((address_space(3))) u32x4*)(to + BM * kRowBytes + c * kLanes * 16) = rb[c];
        };
        if constexpr (WAY != kGuarded) {
            if (const size_t rest = last > first ? (last - first) % kDepth<KIND> : 0) {      // in front: a sum has no order
                u32x4 ra[StageA::kCount], rb[StageB::kCount];
                fetch(ra, rb, last - rest);
                put(ra, rb, 0);
                __syncthreads();
                #pragma unroll
                for (int half = 0; half < 2; ++half) {
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
                for (int c = 0; c < StageA::kCount; ++c) oa[c] = StageA::offset(p.a.stride, p.m - m0, c);
                #pragma unroll
                for (int c = 0; c < StageB::kCount; ++c) ob[c] = StageB::offset(p.b.stride, p.n - n0, c);
                const char *from_a = StageA::first(p.a, m0, first, p.m - m0), *from_b = StageB::first(p.b, n0, first, p.n - n0);
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
                    auto settled = [&] {                        // the tile at the rows' end
                        if (AT && p.m - m0 < BM) {
                            #pragma unroll
                            for (int c = 0; c < StageA::kCount; ++c) move_up<KIND>(ra[c], StageA::early(p.m - m0, c));
                        }
                        if (BT && p.n - n0 < BN) {
                            #pragma unroll
                            for (int c = 0; c < StageB::kCount; ++c) move_up<KIND>(rb[c], StageB::early(p.n - n0, c));
                        }
                    };
                    load();
                    settled();
                    put(ra, rb, 0);
                    if (whole > 1) load();
                    int at = 0;
                    for (size_t k = whole; k; --k, at ^= 1) {
                        barrier_lds();
                        PieceA pa;
                        PieceB pb;
                        read(pa, pb, at, 0);
                        if (k > 1) {
                            settled();
                            put(ra, rb, at ^ 1);
                        }
                        if (k > 2) load();
                        add(pa, pb);
                        read(pa, pb, at, 1);
                        add(pa, pb);
                    }
                    __syncthreads();
                } else {
                const uint32_t place = (uint32_t)(uintptr_t)tile + wave * 1024;
                auto load = [&](int at) {
                    const uint32_t to = place + at * kTileBytes;
                    each<StageA::kCount>([&](auto c) {
                        load_to_lds<decltype(c)::value * kLanes * 16>(from_a, oa[decltype(c)::value], to);
                    });
                    each<StageB::kCount>([&](auto c) {
                        load_to_lds<BM * kRowBytes + decltype(c)::value * kLanes * 16>(from_b, ob[decltype(c)::value], to);
                    });
                    from_a += step_a;
                    from_b += step_b;
                };
                PieceA a0, a1;
                PieceB b0, b1;
                load(0);
                if (whole > 1) load(1);
                landed();
                read(a0, b0, 0, 0);
                int at = 0;
                for (size_t k = whole; k; --k, at ^= 1) {
                    read(a1, b1, at, 1);
                    __builtin_amdgcn_sched_barrier(0);          // reads are issued before the products that they pass by
                    add(a0, b0);
                    __builtin_amdgcn_sched_barrier(0);
                    landed();
                    if (k > 2) load(at);
                    read(a0, b0, at ^ 1, 0);                    // behind the last tile: what nothing uses
                    __builtin_amdgcn_sched_barrier(0);
                    add(a1, b1);
                    __builtin_amdgcn_sched_barrier(0);
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
        // A wavefront's results pass through the LDS into rows of 64 columns, eight to a lane.
        typedef __attribute__((address_space(3))) f32x4 lds_f4;
        lds_char* const mine = tile + wave * kOut * 16 * kStagePitch * 4;
        #pragma unroll
        for (int part = 0; part < TM / kOut; ++part) {
            __syncthreads();
            #pragma unroll
            for (int m = 0; m < kOut; ++m) {
                #pragma unroll
                for (int n = 0; n < TN; ++n)
                    *(lds_f4*)(mine + ((m * 16 + lane % 16) * kStagePitch + n * 16 + lane / 16 * 4) * 4) = acc[part * kOut + m][n];
            }
            __syncthreads();
            for (int r = lane / 8; r < kOut * 16; r += 8) {
                const size_t row = m0 + wm * TM * 16 + part * kOut * 16 + r, col = n0 + wn * TN * 16 + lane % 8 * kVec;
                if (row >= p.m) break;
                const lds_char* const from = mine + (r * kStagePitch + lane % 8 * kVec) * 4;
                const f32x4 low = *(const lds_f4*)from, high = *(const lds_f4*)(from + 16);
                float v[kVec] = {low.x, low.y, low.z, low.w, high.x, high.y, high.z, high.w};
                const int valid = col < p.n ? (int)min(p.n - col, (size_t)kVec) : 0;
                if (g.splits > 1) store_vec<kF32>((char*)(p.parts + (split * p.m + row) * p.n + col), pack<kF32>(v), valid);
                else finish<KIND>(p.e, row, (unsigned)(col / kVec), (unsigned)p.n, valid, v);
            }
        }
        __syncthreads();
    }
}

// Whether an operand's rows hold whole chunks and a tile's chunks lie within 31 bits of its first; and whether on 16 bytes.
bool in_chunks(const ConstRows& m, bool turned, size_t rows, size_t width)
{
    return (!turned || rows * width >= 16) && m.stride < (size_t{1} << 31) / width / 256;
}
bool direct(const ConstRows& m, bool turned, size_t rows, size_t width)
{
    return (uintptr_t)m.data % 16 == 0 && m.stride * width % 16 == 0 && (!turned || rows * width % 16 == 0);
}

template <int KIND, bool AT, bool BT, int BM, int BN, int WM, int WN, int WAY> int launch_tiles(ProductArgs g, void* stream)
{
    g.tiles_m = ceil_div(g.p.m, BM);
    g.tiles_n = ceil_div(g.p.n, BN);
    g.units = g.tiles_m * g.tiles_n * g.splits;
    return launch_args(product_kernel<KIND, AT, BT, BM, BN, WM, WN, WAY>, dim3(grid_of(g.units)), dim3(64 * WM * WN), 0, stream, g);
}

}  // namespace

int launch_product(const Product& p, int kind, void* stream)
{
    ProductArgs g{p, 0, 0, 0, 0, linear_splits(p.m, p.n, p.k)};
    const int err = dispatch_kind(kind, [&](auto K) { return dispatch_flag(p.a_turned, [&](auto A) { return dispatch_flag(p.b_turned, [&](auto B) {
        constexpr int KIND = decltype(K)::value;
        constexpr bool AT = decltype(A)::value, BT = decltype(B)::value;
        if constexpr (AT && !BT) return 0;
        else {
            constexpr size_t W = kWidth<KIND>;
            g.depth = ceil_div(ceil_div(p.k, kDepth<KIND>), g.splits);
            if (!in_chunks(p.a, AT, p.m, W) || !in_chunks(p.b, BT, p.n, W)) return launch_tiles<KIND, AT, BT, 128, 128, 2, 2, kGuarded>(g, stream);
            return dispatch_flag(direct(p.a, AT, p.m, W) && direct(p.b, BT, p.n, W), [&](auto D) {
                constexpr int WAY = decltype(D)::value ? kDirect : kThrough;
                if constexpr (KIND != kF32)
                    if (ceil_div(p.m, 256) * ceil_div(p.n, 256) >= 200) return launch_tiles<KIND, AT, BT, 256, 256, 2, 4, WAY>(g, stream);
                return launch_tiles<KIND, AT, BT, 128, 128, 2, 2, WAY>(g, stream);
            });
        }
    }); }); });
    if (err || g.splits == 1) return err;
    return launch_activation({p.e, {nullptr, 0}, p.parts, g.splits, p.m, (unsigned)p.n}, kind, stream);
}

}  // namespace mics
