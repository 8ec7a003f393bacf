// The direction that Newton-Schulz products make of a matrix, and the momentum step that takes it.
//
//   X_0 = M / |M|_F,   A = X X^T,   B = b A + c A A,   X <- a X + B X,   (a, b, c) = (3.4445, -4.7750, 2.0315)
//
// Every step maps each singular value s of X to a s + b s^3 + c s^5 and leaves the singular vectors alone; values in
// (0, 1] go to about 0.7 .. 1.2 in five steps (the slope at zero is a: a value below 1 / 485 arrives below that).
// X is taken with its smaller side as rows (a higher matrix is transposed on the way in and out).
//
// Bound by the products, 2 S S L + (S S S + S S L) multiply-adds a step for S x L: A and A A are symmetric, only tiles
// on and above the diagonal are formed and stored twice.  The products run on the 16-bit matrix cores.  All factors
// are bounded: from |X_0|_F = 1 on, no singular value passes 1.2024, none of A 1.446, and b x + c x x stays in [-2.81, 0]
// there.  That is what fp16 wants: they are stored times 2^14 (at most 46000), with 11 significant bits down to 4e-9.
//   bf16 matrices with more than 384 rows and columns: factors rounded to fp16; X itself stays in 32 bits, and a X is added in 32 bits.  That matters:
//     directions with singular values near zero are blown up by a per step, and so would be what rounding X puts
//     there (a rounded X: 2e-2 of the result at 64 directions of 512; so: 7e-4, less than bf16 itself).  The result is
//     1.02 to 1.5 times as far from 64 bits as its rounding to bf16 alone (the most with all singular values alike).
//   fp32 matrices, and smaller bf16 ones (whose result one part leaves up to 2.8 times as far off, and whose products
//   cost little): each factor as the sum of two fp16 parts, h = fp16(x), l = fp16(x - h), 22 bits and a sign down to
//     4e-6, an error of 2e-12 below;  h l + l h + h h.  What is left out, l l, is below 2^-24 of the product of the elements: results
//     are as far from 64 bits as those of fp32 products (1.5e-6 at 512 x 512, both).
#include "lc_operators.h"
#include "lc_tile_product.h"

namespace lc {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kUp = 16384.f, kDown2 = 1.f / (16384.f * 16384.f);   // scale of stored factors, and of a product of two undone
constexpr int kOnePartSide = 384;   // see above
constexpr int kBlock = 256;
constexpr int kNormParts = 1024;   // partial sums of squares of a replica at most

enum OrthStep { kGram, kPoly, kNext, kLast };

// The matrix that comes in, and the momentum step's arrays.
struct OrthIn {
    const void* src;            // G (update) or M
    int64_t row, rep;
    float* v;                   // update: momentum, read and written first
    int64_t v_row, v_rep;
    float beta;
    int rows, cols;
    double* parts;              // [m][kNormParts]
};

template <typename T>
__global__ void __launch_bounds__(kBlock) orth_square_kernel(OrthIn in) {
    __shared__ double lds[4];
    const int i = blockIdx.y;
    const T* src = static_cast<const T*>(in.src) + i * in.rep;
    double s = 0.0;
    for (int r = blockIdx.x; r < in.rows; r += gridDim.x)
        for (int c = threadIdx.x; c < in.cols; c += kBlock) {
            float x = static_cast<float>(src[r * in.row + c]);
            if (in.v) {
                float* v = in.v + i * in.v_rep + r * in.v_row + c;
                x = in.beta != 0.f ? fmaf(in.beta, *v, x) : x;   // a momentum that counts as zero is not read
                *v = x;
            }
            s += static_cast<double>(x) * x;
        }
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) in.parts[i * kNormParts + blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

struct Factors {
    uint16_t *h, *l;   // parts; l null: one part
};

__device__ __forceinline__ void split(float x, uint16_t& h, uint16_t& l) {
    const f16_t a = static_cast<f16_t>(x);
    h = __builtin_bit_cast(uint16_t, a);
    l = __builtin_bit_cast(uint16_t, static_cast<f16_t>(x - static_cast<float>(a)));
}

// M / |M| into X (32 bits and parts), 64 x 64 a workgroup, transposed where M is higher than wide.
template <typename T>
__global__ void __launch_bounds__(kBlock) orth_start_kernel(OrthIn in, int n_parts, int tall, float* x, Factors f, int S, int L, int Lp) {
    __shared__ float tile[64][65];
    __shared__ float inv_s;
    const int i = blockIdx.z, r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;   // of X
    const T* src = static_cast<const T*>(in.src) + i * in.rep;
    const float* v = in.v ? in.v + i * in.v_rep : nullptr;
    if (threadIdx.x < 64) {
        double part = 0.0;
        for (int k = threadIdx.x; k < n_parts; k += 64) part += in.parts[i * kNormParts + k];
        const double s = wave_sum(part);
        // a zero matrix stays zero; a norm below what 1 / norm can be in 32 bits: as far as that goes
        if (threadIdx.x == 0) inv_s = s > 0.0 ? static_cast<float>(fmin(1.0 / sqrt(s), 3e38)) : s == 0.0 ? 0.f : static_cast<float>(s);
    }
    __syncthreads();
    const float inv = inv_s;
    const int tc = threadIdx.x & 63, tr = threadIdx.x >> 6;
#pragma unroll 4
    for (int q = 0; q < 16; ++q) {
        const int a = q * 4 + tr;   // row of the tile of M as it stands
        const int r = (tall ? c0 : r0) + a, c = (tall ? r0 : c0) + tc;
        float val = 0.f;
        if (r < in.rows && c < in.cols) val = v ? v[r * in.v_row + c] : static_cast<float>(src[r * in.row + c]);
        tile[a][tc] = val * inv;
    }
    __syncthreads();
#pragma unroll 4
    for (int q = 0; q < 16; ++q) {
        const int r = r0 + q * 4 + tr, c = c0 + tc;
        if (r >= S) continue;
        const float val = tall ? tile[tc][q * 4 + tr] : tile[q * 4 + tr][tc];
        const int64_t at = ((int64_t)i * S + r) * Lp + c;
        uint16_t h, l;
        split(val * kUp, h, l);
        x[at] = val;
        f.h[at] = h;
        if (f.l) f.l[at] = l;
    }
    (void)L;
}

struct OrthOut {
    int S, Sp, L, Lp;
    float* a;                   // [m][S][Sp] A in 32 bits, tiles on and above the diagonal
    float* x;                   // [m][S][Lp] X in 32 bits
    Factors to;                 // A, B or the next X
    // last step
    int tall, update, out_bf16;
    void* out;                  // M's place of the result, or X of the update
    int64_t out_row, out_rep;
    float lr, scale, wd;
};

__device__ __forceinline__ void store_factors(const Factors& f, int64_t at, const float (&v)[4]) {
    s16x4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint16_t a, b;
        split(v[e] * kUp, a, b);
        h[e] = (short)a;
        l[e] = (short)b;
    }
    *reinterpret_cast<s16x4*>(f.h + at) = h;
    if (f.l) *reinterpret_cast<s16x4*>(f.l + at) = l;
}

template <typename S, BLayout LB, OrthStep STEP>
__global__ void __launch_bounds__(S::kThreads) orth_product_kernel(TileArgs a, OrthOut o) {
    __shared__ __align__(1024) uint16_t lds[S::kLds];
    const TilePlace pl = tile_place(a);
    if (pl.batch < 0) return;
    f32x4 acc[S::TM][S::TN];
    tile_sums<f16_t, S, LB>(a, pl, 0, a.K / S::BK, lds, acc);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int mw = pl.tm * S::BM + (w / S::WN) * S::TM * 16 + (lane & 15), nw = pl.tn * S::BN + (w % S::WN) * S::TN * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
        const int m = mw + i * 16;
        if (m >= o.S) continue;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            const int n = nw + j * 16;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e] * kDown2;
            if constexpr (STEP == kGram || STEP == kPoly) {
                if (n >= o.Sp) continue;
                const int64_t at = ((int64_t)pl.batch * o.S + m) * o.Sp + n;
                if constexpr (STEP == kPoly) {
                    const f32x4 g = *reinterpret_cast<const f32x4*>(o.a + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = kNsB * g[e] + kNsC * v[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e >= o.S) v[e] = 0.f;   // behind the matrix: zeros, which a product takes as its last k
                if constexpr (STEP == kGram) *reinterpret_cast<f32x4*>(o.a + at) = f32x4{v[0], v[1], v[2], v[3]};
                store_factors(o.to, at, v);
                if (pl.tm != pl.tn) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (n + e >= o.S) continue;
                        const int64_t mirror = ((int64_t)pl.batch * o.S + n + e) * o.Sp + m;
                        uint16_t h, l;
                        split(v[e] * kUp, h, l);
                        o.to.h[mirror] = h;
                        if (o.to.l) o.to.l[mirror] = l;
                    }
                }
            } else {
                if (n >= o.Lp) continue;
                const int64_t at = ((int64_t)pl.batch * o.S + m) * o.Lp + n;
                const f32x4 x = *reinterpret_cast<const f32x4*>(o.x + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fmaf(kNsA, x[e], v[e]);
                if constexpr (STEP == kNext) {
                    *reinterpret_cast<f32x4*>(o.x + at) = f32x4{v[0], v[1], v[2], v[3]};
                    store_factors(o.to, at, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (n + e >= o.L) continue;
                        const int64_t to = pl.batch * o.out_rep + (o.tall ? (int64_t)(n + e) * o.out_row + m : (int64_t)m * o.out_row + n + e);
                        if (o.update) {
                            float* p = static_cast<float*>(o.out) + to;
                            *p = *p - o.lr * (o.scale * v[e] + o.wd * *p);
                        } else if (o.out_bf16) {
                            static_cast<bf16_t*>(o.out)[to] = static_cast<bf16_t>(v[e]);
                        } else {
                            static_cast<float*>(o.out)[to] = v[e];
                        }
                    }
                }
            }
        }
    }
}

template <int NP>
struct Tiles {
    typedef TileShape<256, 256, 2, 4, 64, 1, 2> Large;
    typedef TileShape<128, 128, 2, 2, 64, 1, 2> Medium;
    typedef TileShape<64, 64, 2, 2, 64, 1, 4> Small;
};
template <>
struct Tiles<2> {
    typedef TileShape<256, 256, 2, 4, 32, 2, 2> Large;
    typedef TileShape<128, 128, 2, 2, 32, 2, 2> Medium;
    typedef TileShape<64, 64, 2, 2, 64, 2, 4> Small;
};

template <typename S>
void launch_product(TileArgs a, const OrthOut& o, OrthStep step, hipStream_t st) {
    a.mt = (a.M + S::BM - 1) / S::BM;
    a.nt = (a.N + S::BN - 1) / S::BN;
    const unsigned g = tile_grid(a);
    switch (step) {
        case kGram: orth_product_kernel<S, KMajor, kGram><<<g, S::kThreads, 0, st>>>(a, o); break;
        case kPoly: orth_product_kernel<S, KMajor, kPoly><<<g, S::kThreads, 0, st>>>(a, o); break;
        case kNext: orth_product_kernel<S, NMajor, kNext><<<g, S::kThreads, 0, st>>>(a, o); break;
        case kLast: orth_product_kernel<S, NMajor, kLast><<<g, S::kThreads, 0, st>>>(a, o); break;
    }
}

// Tile size: the largest that still gives most compute units a workgroup.
template <int NP>
void launch_step_parts(const TileArgs& a, const OrthOut& o, OrthStep step, hipStream_t st) {
    auto tiles = [&](int b) {
        const int64_t mt = (a.M + b - 1) / b, nt = (a.N + b - 1) / b;
        return (a.upper ? mt * (mt + 1) / 2 : mt * nt) * a.batches;
    };
    if (tiles(256) >= 128) launch_product<typename Tiles<NP>::Large>(a, o, step, st);
    else if (tiles(128) >= 128) launch_product<typename Tiles<NP>::Medium>(a, o, step, st);
    else launch_product<typename Tiles<NP>::Small>(a, o, step, st);
}
void launch_step(const TileArgs& a, const OrthOut& o, OrthStep step, int parts, hipStream_t st) {
    if (parts == 2) launch_step_parts<2>(a, o, step, st);
    else launch_step_parts<1>(a, o, step, st);
}

struct OrthPlan {
    int S, L, Sp, Lp, parts;
    double* norm;
    float *x, *a;
    uint16_t *xp[2], *ap, *bp;   // [parts][m][..]
    size_t bytes;
};
OrthPlan orth_plan(int m, int rows, int cols, int dtype, void* ws) {
    OrthPlan p;
    p.S = std::min(rows, cols);
    p.L = std::max(rows, cols);
    p.Sp = static_cast<int>(round_up(p.S, kPadK));
    p.Lp = static_cast<int>(round_up(p.L, kPadK));
    p.parts = dtype == LC_GEMM_BF16 && p.S > kOnePartSide ? 1 : 2;
    const int64_t nx = (int64_t)m * p.S * p.Lp, na = (int64_t)m * p.S * p.Sp;
    Carver c{static_cast<char*>(ws)};
    p.norm = c.take<double>((int64_t)m * kNormParts);
    p.x = c.take<float>(nx);
    p.a = c.take<float>(na);
    p.xp[0] = c.take<uint16_t>(nx * p.parts);
    p.xp[1] = c.take<uint16_t>(nx * p.parts);
    p.ap = c.take<uint16_t>(na * p.parts);
    p.bp = c.take<uint16_t>(na * p.parts);
    p.bytes = c.used;
    return p;
}

// M (or the momentum that the step has just formed) through `steps` steps into o's place.
int orthogonalise(int m, const OrthIn& in, int dtype, int steps, OrthOut o, const OrthPlan& p, hipStream_t st) {
    const bool bf16 = dtype == LC_GEMM_BF16;
    const int tall = in.rows > in.cols, blocks = std::min(in.rows, std::max(16, kNormParts / m));
    const int64_t nx = (int64_t)m * p.S * p.Lp, na = (int64_t)m * p.S * p.Sp;
    const dim3 gs(blocks, m), g0(p.Lp / 64, (p.S + 63) / 64, m);
    auto factors = [&](uint16_t* q, int64_t n) { return Factors{q, p.parts == 2 ? q + n : nullptr}; };
    if (bf16) {
        orth_square_kernel<bf16_t><<<gs, kBlock, 0, st>>>(in);
        orth_start_kernel<bf16_t><<<g0, kBlock, 0, st>>>(in, blocks, tall, p.x, factors(p.xp[0], nx), p.S, p.L, p.Lp);
    } else {
        orth_square_kernel<float><<<gs, kBlock, 0, st>>>(in);
        orth_start_kernel<float><<<g0, kBlock, 0, st>>>(in, blocks, tall, p.x, factors(p.xp[0], nx), p.S, p.L, p.Lp);
    }
    o.S = p.S; o.Sp = p.Sp; o.L = p.L; o.Lp = p.Lp;
    o.a = p.a; o.x = p.x;
    o.tall = tall;
    TileArgs t{};
    t.batches = m;
    t.splits = 1;
    auto operand = [&](const uint16_t* q, int64_t n, int row, int64_t batch, int rows, int len) {
        return TileOperand{q, row, batch, {0, n, 0}, rows, len};
    };
    for (int k = 0; k < steps; ++k) {
        const uint16_t* x = p.xp[k & 1];
        const int64_t bx = (int64_t)p.S * p.Lp, ba = (int64_t)p.S * p.Sp;
        t.M = t.N = p.S;
        t.K = p.Lp;
        t.upper = 1;
        t.a = operand(x, nx, p.Lp, bx, p.S, p.Lp);
        t.b = operand(x, nx, p.Lp, bx, p.S, p.Lp);
        o.to = factors(p.ap, na);
        launch_step(t, o, kGram, p.parts, st);
        t.K = p.Sp;
        t.a = operand(p.ap, na, p.Sp, ba, p.S, p.Sp);
        t.b = operand(p.ap, na, p.Sp, ba, p.S, p.Sp);
        o.to = factors(p.bp, na);
        launch_step(t, o, kPoly, p.parts, st);
        t.upper = 0;
        t.N = p.Lp;
        t.a = operand(p.bp, na, p.Sp, ba, p.S, p.Sp);
        t.b = operand(x, nx, p.Lp, bx, p.S, p.Lp);   // S rows of k
        o.to = factors(p.xp[(k + 1) & 1], nx);
        launch_step(t, o, k + 1 < steps ? kNext : kLast, p.parts, st);
    }
    return hipGetLastError() == hipSuccess ? LC_OK : LC_ERR_HIP;
}

// Biases of a run: g = G + wd x, v <- beta v + g, x <- x - lr v.
struct Biases {
    int64_t off[LC_MAX_LAYERS];
    int n[LC_MAX_LAYERS];
};
__global__ void __launch_bounds__(kBlock) update_biases_kernel(float* X, float* V, const float* G, int64_t Ps, Biases b, float lr, float beta,
                                                               float wd) {
    const int c = blockIdx.x * kBlock + threadIdx.x;
    if (c >= b.n[blockIdx.y]) return;
    const int64_t at = blockIdx.z * Ps + b.off[blockIdx.y] + c;
    const float x = X[at], g = fmaf(wd, x, G[at]);
    const float v = beta != 0.f ? fmaf(beta, V[at], g) : g;
    V[at] = v;
    X[at] = fmaf(-lr, v, x);
}

// Sizes that the kernels' 32-bit offsets inside a matrix hold.
bool orth_sizes_ok(int m, int32_t rows, int32_t cols) {
    return m >= 1 && m <= kMaxReplicas && rows >= 1 && cols >= 1 && rows <= LC_ORTHOGONAL_MAX_SIDE && cols <= LC_ORTHOGONAL_MAX_SIDE;
}
bool steps_ok(int steps) { return steps >= 1 && steps <= 16; }

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" {

size_t lc_orthogonal_workspace_bytes(int m, int32_t rows, int32_t cols, int dtype) {
    if (!orth_sizes_ok(m, rows, cols) || (dtype != LC_GEMM_FP32 && dtype != LC_GEMM_BF16)) return 0;
    return orth_plan(m, rows, cols, dtype, nullptr).bytes;
}

int lc_orthogonalize(int m, int32_t rows, int32_t cols, int dtype, lc_rows src, lc_rows dst, int steps, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (!orth_sizes_ok(m, rows, cols) || !steps_ok(steps) || (dtype != LC_GEMM_FP32 && dtype != LC_GEMM_BF16)) return LC_ERR_ARG;
    int rc = check_input(src, m, rows, cols, dtype);
    if (rc == LC_OK) rc = check_output(dst, m, rows, cols, dtype);
    if (rc != LC_OK) return rc;
    if (!workspace || workspace_bytes < lc_orthogonal_workspace_bytes(m, rows, cols, dtype)) return LC_ERR_WORKSPACE;
    if (!aligned_to(workspace, 256)) return LC_ERR_ALIGN;
    const OrthPlan p = orth_plan(m, rows, cols, dtype, workspace);
    const OrthIn in{src.p, src.row, src.replica, nullptr, 0, 0, 0.f, rows, cols, p.norm};
    OrthOut o{};
    o.out_bf16 = dtype == LC_GEMM_BF16;
    o.out = dst.p;
    o.out_row = dst.row;
    o.out_rep = dst.replica;
    return orthogonalise(m, in, dtype, steps, o, p, static_cast<hipStream_t>(stream));
}

int lc_update_orthogonal(int m, int32_t rows, int32_t cols, lc_rows X, lc_rows V, lc_rows G, float lr, float beta, float wd,
                         int steps, void* workspace, size_t workspace_bytes, void* stream) {
    if (!orth_sizes_ok(m, rows, cols) || !steps_ok(steps)) return LC_ERR_ARG;
    if (!(lr > 0.f) || !(beta >= 0.f && beta < 1.f) || !(wd >= 0.f)) return LC_ERR_ARG;
    int rc = check_output(X, m, rows, cols, LC_GEMM_FP32);
    if (rc == LC_OK) rc = check_output(V, m, rows, cols, LC_GEMM_FP32);
    if (rc == LC_OK) rc = check_input(G, m, rows, cols, LC_GEMM_FP32);
    if (rc != LC_OK) return rc;
    if (X.p == V.p || X.p == G.p || V.p == G.p) return LC_ERR_ARG;
    if (!workspace || workspace_bytes < lc_orthogonal_workspace_bytes(m, rows, cols, LC_GEMM_FP32)) return LC_ERR_WORKSPACE;
    if (!aligned_to(workspace, 256)) return LC_ERR_ALIGN;
    const OrthPlan p = orth_plan(m, rows, cols, LC_GEMM_FP32, workspace);
    const OrthIn in{G.p, G.row, G.replica, static_cast<float*>(V.p), V.row, V.replica, beta, rows, cols, p.norm};
    OrthOut o{};
    o.update = 1;
    o.out = X.p;
    o.out_row = X.row;
    o.out_rep = X.replica;
    o.lr = lr;
    o.wd = wd;
    o.scale = sqrtf(std::max(1.f, static_cast<float>(cols) / static_cast<float>(rows)));
    return orthogonalise(m, in, LC_GEMM_FP32, steps, o, p, static_cast<hipStream_t>(stream));
}

size_t lc_update_orthogonal_bytes(const lc_handle* h) {
    size_t most = 0;
    if (h && h->md.kind == LC_KIND_MLP)
        for (int l = 1; l <= h->L; ++l)
            most = std::max(most, lc_orthogonal_workspace_bytes(h->m, h->layer[l].d_in, h->layer[l].d_out, LC_GEMM_FP32));
    return most;
}

int lc_update_from_grad_orthogonal(lc_handle* h, int steps, void* workspace, size_t workspace_bytes) {
    if (!h || steps < 1 || steps > 16) return LC_ERR_ARG;
    if (!h->attached || !h->G) return LC_ERR_STATE;
    if (h->md.kind != LC_KIND_MLP) return LC_ERR_UNSUPPORTED;
    if (!(h->md.lr > 0.f) || !(effective_beta(h) >= 0.f && effective_beta(h) < 1.f) || !(h->md.wd >= 0.f)) return LC_ERR_ARG;
    for (int l = 1; l <= h->L; ++l)
        if (std::max(h->layer[l].d_in, h->layer[l].d_out) > LC_ORTHOGONAL_MAX_SIDE) return LC_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < lc_update_orthogonal_bytes(h)) return LC_ERR_WORKSPACE;
    if (!aligned_to(workspace, 256)) return LC_ERR_ALIGN;
    const int mrc = lc_materialize(h);   // a pending broadcast is written to the rows first
    if (mrc != LC_OK) return mrc;
    Biases b{};
    int widest = 0;
    for (int l = 1; l <= h->L; ++l) {
        const LayerGeom& g = h->layer[l];
        auto rows = [&](const float* p) { return lc_rows{const_cast<float*>(p) + g.w_off, g.d_out, h->Ps}; };
        const int rc = lc_update_orthogonal(h->m, g.d_in, g.d_out, rows(h->X), rows(h->V), rows(h->G), h->md.lr, effective_beta(h),
                                            h->md.wd, steps, workspace, workspace_bytes, h->stream);
        if (rc != LC_OK) return rc;
        b.off[l - 1] = g.b_off;
        b.n[l - 1] = g.d_out;
        widest = std::max(widest, g.d_out);
    }
    update_biases_kernel<<<dim3((widest + kBlock - 1) / kBlock, h->L, h->m), kBlock, 0, h->stream>>>(h->X, h->V, h->G, h->Ps, b, h->md.lr,
                                                                                                   effective_beta(h), h->md.wd);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        h->last_hip = static_cast<int>(e);
        return LC_ERR_HIP;
    }
    h->v_cleared = false;
    return LC_OK;
}

}  // extern "C"
