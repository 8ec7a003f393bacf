// Tiled products of 16-bit operands with 32-bit sums: the core of the softmax head and of the
// Newton-Schulz products.  Internal linkage: every translation unit gets its own copy.
//
//   acc[m, n] = sum over segments s, k of A_s[m, k] B_s[k, n]
//
// A stands with k contiguous; B with k contiguous (KMajor: rows n) or with n contiguous (NMajor: rows
// k, read through the LDS transpose).  A segment is one pair of parts: fp32 operands come as the sum of
// 16-bit parts, and a product of two such sums is a list of part products over one accumulator.
//
// A workgroup owns a BM x BN tile.  Tiles of 64 k of both operands go from global memory straight into
// LDS (16 bytes a lane, no registers), two buffers in turn.  16-byte chunks are permuted inside a row,
// by permuting what each lane fetches, so that the operand reads of a wavefront spread over all banks:
//   KMajor  row of 64 k = 8 chunks:    chunk c of row r at c ^ ((r >> 1) & 7)
//   NMajor  row of BN n, 32-byte pairs: pair p of row k at p ^ ((k & 3) | (k >> 3 & 1) << 2), as far as there are pairs
#pragma once
#include "lc_internal.h"

namespace lc {
namespace {

typedef _Float16 f16_t;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int kTileK = 64;
constexpr int kMaxSegments = 6;

__device__ __forceinline__ f32x4 mma32(bf16_t, s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma32(f16_t, s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// One operand as the kernels read it.  Strides in elements.  What lies outside `rows` x `len` is never
// read: addresses are held inside, and what a lane fetches twice is either not stored (rows of the
// result) or multiplied with the zeros that stand behind A's k (`len` of B ends before A's).
struct TileOperand {
    const uint16_t* p;
    int64_t row, batch;
    int64_t part[kMaxSegments];   // offset of the part that a segment takes
    int rows, len;                // KMajor: rows of k, `len` of them; NMajor: `rows` k of `len` n.  len % 8 == 0,
                                  // the k padded to 64 are those of the product
};
constexpr int64_t kMaxRowStride = 1 << 22;   // offsets inside a tile of 256 rows stay below 2^31 bytes

struct TileArgs {
    TileOperand a, b;
    int M, N, K;                  // K: padded to 64, A is zero behind its own length
    int segments;
    int rescale_after;            // the sums are multiplied by `rescale` before this segment (0: never)
    float rescale;
    int batches, mt, nt, splits;  // tiles in M and N, shares of the K axis
    int upper;                    // symmetric result: only tiles with tm <= tn, (mt (mt + 1) / 2 of them)
    const int* m_count;           // [batches] rows of A that count, or null; tiles behind them run no product
    const int* k_count;           // [batches] k that count (a multiple of 64 is taken), or null
    int count_base;               // first row of the chunk: what is left of a count is max(0, count - base)
};

enum BLayout { KMajor, NMajor };

template <int BM_, int BN_, int WM_, int WN_>
struct TileShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;   // WM x WN wavefronts
    static constexpr int kThreads = 64 * WM * WN;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;     // 16 x 16 tiles of a wavefront
    static constexpr int kStage = (BM + BN) * kTileK;              // elements of one LDS buffer
};

typedef __attribute__((address_space(3))) void* LdsPtr;
typedef const __attribute__((address_space(1))) void* GlobalPtr;

// 16 bytes a lane from base + off (bytes) to consecutive places in LDS from `to` on.
__device__ __forceinline__ void fetch16(const char* base, uint32_t off, uint16_t* to) {
    __builtin_amdgcn_global_load_lds((GlobalPtr)(base + off), (LdsPtr)to, 16, 0, 0);
}

// What a lane fetches of R rows of a KMajor operand: offsets (bytes) from the tile's first row and column; `base` of
// fetch() is the tile's first row.
template <int R, int THREADS>
struct KMajorFetch {
    static constexpr int kPer = THREADS / 8, kLoads = R / kPer;   // rows per load instruction of the workgroup
    uint32_t off[kLoads];
    int c8;   // the lane's first k inside a tile
    __device__ __forceinline__ void init(const TileOperand& o, int row0) {
        const int t = threadIdx.x;
        static_assert(kPer % 16 == 0, "the permutation of a lane's chunk is the same in all its rows");
        c8 = ((t & 7) ^ ((t >> 4) & 7)) * 8;
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            off[q] = ((uint32_t)(min(row0 + q * kPer + (t >> 3), o.rows - 1) - row0) * (uint32_t)o.row + c8) * 2u;
    }
    __device__ __forceinline__ void fetch(const TileOperand& o, const char* base, int k0, uint16_t* to) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        to += wave * 8 * kTileK;
        const char* at = base + 2 * (int64_t)k0;
        if (k0 + kTileK <= o.len) {
#pragma unroll
            for (int q = 0; q < kLoads; ++q) fetch16(at, off[q], to + q * kPer * kTileK);
        } else {
            const int back = max(0, k0 + c8 + 8 - o.len);   // k0 < len, both multiples of 8: it stays inside the tile
#pragma unroll
            for (int q = 0; q < kLoads; ++q) fetch16(at, off[q] - 2u * (uint32_t)back, to + q * kPer * kTileK);
        }
    }
};
// ... of BN columns of an NMajor operand: offsets from the k tile's first row.
template <int BN, int THREADS>
struct NMajorFetch {
    static constexpr int kChunks = BN / 8, kPer = THREADS / kChunks, kLoads = kTileK / kPer;
    uint32_t col;   // bytes
    int k;
    uint32_t row2;  // bytes of a row
    __device__ __forceinline__ static int swizzle(int k) { return (((k & 3) | ((k >> 3 & 1) << 2)) & (BN / 16 - 1)) << 1; }
    uint32_t off[kLoads];
    __device__ __forceinline__ void init(const TileOperand& o, int n0) {
        const int t = threadIdx.x;
        k = t / kChunks;
        row2 = (uint32_t)o.row * 2u;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int kk = q * kPer + k, c = (t % kChunks) ^ swizzle(kk);
            off[q] = (uint32_t)kk * row2 + (uint32_t)min(n0 + c * 8, o.len - 8) * 2u;
        }
    }
    __device__ __forceinline__ void fetch(const TileOperand& o, const char* base, int k0, uint16_t* to) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        to += wave * 512;
        const char* at = base + (int64_t)k0 * row2;
        if (k0 + kTileK <= o.rows) {
#pragma unroll
            for (int q = 0; q < kLoads; ++q) fetch16(at, off[q], to + q * THREADS * 8);
        } else {
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const int back = max(0, q * kPer + k + k0 + 1 - o.rows);   // k0 < rows: at most q * kPer + k
                fetch16(at, off[q] - (uint32_t)back * row2, to + q * THREADS * 8);
            }
        }
    }
};

__device__ __forceinline__ s16x8 read_kmajor(const uint16_t* tile, int row, int ks, int lane) {
    const int c = (ks * 4 + (lane >> 4)) ^ ((lane >> 1) & 7);
    return *reinterpret_cast<const s16x8*>(tile + (row + (lane & 15)) * kTileK + c * 8);
}
// A 16-lane group reads 4 rows of k, 16 columns; lane i gets column i of all four.
template <int BN>
__device__ __forceinline__ s16x8 read_nmajor(const uint16_t* tile, int col, int ks, int lane) {
    const int g = lane >> 4, i = lane & 15;
    const int k = ks * 32 + g * 8 + (i >> 2);
    const int pair = (col >> 4) ^ (((i >> 2) | ((g & 1) << 2)) & (BN / 16 - 1));
    const uint16_t* at = tile + k * BN + pair * 16 + (i & 3) * 4;
    typedef __attribute__((address_space(3))) s16x4* P;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 4 * BN));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <BLayout L, int BN, int THREADS>
struct FetchB {
    typedef KMajorFetch<BN, THREADS> type;
};
template <int BN, int THREADS>
struct FetchB<NMajor, BN, THREADS> {
    typedef NMajorFetch<BN, THREADS> type;
};

struct TilePlace {
    int batch, tm, tn, split;   // batch < 0: nothing to do
};

// Workgroup id -> tile.  Each XCD takes a contiguous range; inside it, blocks of 8 tiles of M by all of N, M fastest,
// so that what runs together shares rows of A and columns of B in the L2.
__device__ __forceinline__ TilePlace tile_place(const TileArgs& a) {
    const int per = a.upper ? a.mt * (a.mt + 1) / 2 : a.mt * a.nt;
    const int64_t total = (int64_t)per * a.batches * a.splits;
    const int64_t chunk = (total + kXcds - 1) / kXcds;
    const int64_t id = (int64_t)(blockIdx.x % kXcds) * chunk + blockIdx.x / kXcds;
    TilePlace pl{-1, 0, 0, 0};
    if (blockIdx.x / kXcds >= chunk || id >= total) return pl;
    const int64_t one = id % ((int64_t)per * a.splits);
    pl.batch = (int)(id / ((int64_t)per * a.splits));
    pl.split = (int)(one / per);
    const int t = (int)(one % per);
    if (a.upper) {
        // column tn holds tn + 1 tiles
        int tn = __builtin_amdgcn_readfirstlane((int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f));
        while ((tn + 1) * (tn + 2) / 2 <= t) ++tn;
        while (tn * (tn + 1) / 2 > t) --tn;
        pl.tn = tn;
        pl.tm = t - tn * (tn + 1) / 2;
    } else {
        constexpr int kG = 8;
        const int g = t / (kG * a.nt), first = g * kG, size = min(kG, a.mt - first);
        pl.tm = first + (t - g * kG * a.nt) % size;
        pl.tn = (t - g * kG * a.nt) / size;
    }
    return pl;
}

inline unsigned tile_grid(const TileArgs& a) {
    const int64_t per = a.upper ? (int64_t)a.mt * (a.mt + 1) / 2 : (int64_t)a.mt * a.nt;
    const int64_t total = per * a.batches * a.splits;
    return (unsigned)((total + kXcds - 1) / kXcds * kXcds);
}

// The sums of one tile.  On return acc[i][j][e] of lane l of wavefront (wm, wn) is row
// wm * TM * 16 + 16 i + (l & 15), column wn * TN * 16 + 16 j + 4 (l >> 4) + e of the tile.
template <typename T, typename S, BLayout L>
__device__ __forceinline__ void tile_sums(const TileArgs& a, const TilePlace pl, int kt0, int kt1, uint16_t* lds,
                                          f32x4 (&acc)[S::TM][S::TN]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / S::WN, wn = wave % S::WN;
    const int m0 = pl.tm * S::BM, n0 = pl.tn * S::BN;
    const int per_seg = kt1 - kt0, total = per_seg * a.segments;
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (total <= 0) return;
    const char* ab = reinterpret_cast<const char*>(a.a.p + (int64_t)pl.batch * a.a.batch + (int64_t)m0 * a.a.row);
    const char* bb = reinterpret_cast<const char*>(a.b.p + (int64_t)pl.batch * a.b.batch + (L == KMajor ? (int64_t)n0 * a.b.row : 0));
    KMajorFetch<S::BM, S::kThreads> fa_;
    typename FetchB<L, S::BN, S::kThreads>::type fb_;
    fa_.init(a.a, m0);
    fb_.init(a.b, n0);
    int seg = 0, next_k = kt0;   // of the tile that is fetched next
    auto fetch = [&](uint16_t* to) {
        fa_.fetch(a.a, ab + 2 * a.a.part[seg], next_k * kTileK, to);
        fb_.fetch(a.b, bb + 2 * a.b.part[seg], next_k * kTileK, to + S::BM * kTileK);
        if (++next_k == kt1) next_k = kt0, ++seg;
    };
    const int rescale_at = a.rescale_after ? a.rescale_after * per_seg : -1;
    fetch(lds);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int t = 0; t < total; ++t) {
        uint16_t* cur = lds + (t & 1) * S::kStage;
        if (t + 1 < total) fetch(lds + ((t + 1) & 1) * S::kStage);
        if (t == rescale_at) {
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int j = 0; j < S::TN; ++j) acc[i][j] *= a.rescale;
        }
        const uint16_t* ta = cur + wm * S::TM * 16 * kTileK;
        const uint16_t* tb = cur + S::BM * kTileK;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            s16x8 fa[S::TM], fb[S::TN];
#pragma unroll
            for (int j = 0; j < S::TN; ++j) {
                if constexpr (L == KMajor)
                    fb[j] = read_kmajor(tb, (wn * S::TN + j) * 16, ks, lane);
                else
                    fb[j] = read_nmajor<S::BN>(tb, (wn * S::TN + j) * 16, ks, lane);
            }
#pragma unroll
            for (int i = 0; i < S::TM; ++i) fa[i] = read_kmajor(ta, i * 16, ks, lane);
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int j = 0; j < S::TN; ++j) acc[i][j] = mma32(T(), fb[j], fa[i], acc[i][j]);
        }
        __builtin_amdgcn_s_waitcnt(0);   // the next tile is in LDS, this one's reads are done
        __syncthreads();
    }
}

// The k tiles [kt0, kt1) of a workgroup's share.
__device__ __forceinline__ void tile_k_range(const TileArgs& a, const TilePlace pl, int bm, int& kt0, int& kt1) {
    int kt = a.K / kTileK;
    if (a.k_count)
        kt = min(kt, (max(0, __builtin_amdgcn_readfirstlane(a.k_count[pl.batch]) - a.count_base) + kTileK - 1) / kTileK);
    if (a.m_count && pl.tm * bm >= __builtin_amdgcn_readfirstlane(a.m_count[pl.batch]) - a.count_base) kt = 0;
    kt0 = (int)((int64_t)kt * pl.split / a.splits);
    kt1 = (int)((int64_t)kt * (pl.split + 1) / a.splits);
}

}  // namespace
}  // namespace lc
