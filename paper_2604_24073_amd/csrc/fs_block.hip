// The norms around a block with its gate and residual scale, forward and backward, and rows in 8 bits.
//
//   y = x + scale * w_post * rms(a) * silu(g),  h = w_pre * rms(y)
//
// With r = 1 / sqrt(mean(t^2) + eps) and that = t r, the gradient of rms(t) applied to u is  r (u - that mean(u that)).  So
//   dY = dy + rms'(w_pre dh; y)           u = dY scale w_post
//   dg = u ahat silu'(g)                  da = rms'(u silu(g); a)
//   dw_post = scale T, dscale = w_post T  with T = sum over rows of dY ahat silu(g);   dw_pre = sum over rows of dh yhat
// Every row needs itself twice (once for its mean), and rows are at most 4 KB: a row stays in the registers of the lanes that
// loaded it, eight columns each, so that everything is read once and written once, and the norms of the backward pass are
// computed anew from the rows instead of being kept.  Bound by memory; no product is shared between rows, hence no MFMA.
// 297 k rows of 128 columns, residual rows fp32 and the block's bf16: forward 532 MB in 102 us, backward 836 MB in 160, both
// 5.2 TB/s, where a large copy has 6.2; with a and g kept in 8 bits besides (200 k x 256) 822 MB in 148 and 1027 MB in 203.
// Few rows are launches: 256 x 512 4.6 us forward.
#include <type_traits>

#include "fs_rowvec.h"

using namespace fs;

namespace {

constexpr int kBlockThreads = 256;
constexpr int kBlockWaves = kBlockThreads / kWave;
constexpr int64_t kMaxGrid = 1 << 22;    // workgroups of a launch: a launch has fewer than 2^32 threads
constexpr int kMaxPartials = 768;        // workgroups of a backward pass, each with column sums of its own: three a CU, which is what
                                         // its registers leave room for (297 k rows of 128 columns: 190 us with 1024, 165 with 768)

// LPR lanes share a row, NC times eight columns each: lane l of them holds columns 8 l + 8 LPR c.
template <typename TR, typename TA, int LPR, int NC, bool JOIN>
__global__ __launch_bounds__(kBlockThreads) void block_norm_kernel(fs_block_args p) {
    constexpr int kRows = kWave / LPR;
    const int lane = threadIdx.x & (kWave - 1), sub = lane & (LPR - 1);
    const TR *x = static_cast<const TR *>(p.x);
    const TA *a = static_cast<const TA *>(p.a), *g = static_cast<const TA *>(p.g);
    TR *y = static_cast<TR *>(p.y);
    TA *h = static_cast<TA *>(p.h);
    const float inv_dim = 1.f / (float)p.dim;
    const int64_t groups = (p.n + kRows * kBlockWaves - 1) / (kRows * kBlockWaves);
    for (int64_t b = blockIdx.x; b < groups; b += gridDim.x) {
        const int64_t row = (b * kBlockWaves + threadIdx.x / kWave) * kRows + lane / LPR;
        // lanes behind the last row go along with nothing to load: sums and maxima are taken across lanes
        const bool live = row < p.n;
        float xv[NC][8];
        int left[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = 8 * (sub + LPR * c);
            left[c] = live ? p.dim - col : 0;
            load8(x + row * p.dim + col, left[c], xv[c]);
        }
        if constexpr (JOIN) {
            float av[NC][8], gv[NC][8];
            float ss = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = 8 * (sub + LPR * c);
                load8(a + row * p.a_stride + col, left[c], av[c]);
                load8(g + row * p.g_stride + col, left[c], gv[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += av[c][i] * av[c][i];
            }
            const float r = 1.f / sqrtf(row_sum<LPR>(ss) * inv_dim + p.eps);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = 8 * (sub + LPR * c);
                const int64_t byte = row * p.dim + col;
                const int cols = p.dim - col;
                if (p.a_codes) {
                    uint32_t e;
                    const u32x2 codes = rows8_encode(av[c], e);
                    if (left[c] > 0) {
                        *reinterpret_cast<u32x2 *>(p.a_codes + byte) = codes;
                        if ((sub & 3) == 0) p.a_exps[byte / FS_ROWS8_GROUP] = (uint8_t)e;
                    }
                }
                if (p.g_codes) {
                    uint32_t e;
                    const u32x2 codes = rows8_encode(gv[c], e);
                    if (left[c] > 0) {
                        *reinterpret_cast<u32x2 *>(p.g_codes + byte) = codes;
                        if ((sub & 3) == 0) p.g_exps[byte / FS_ROWS8_GROUP] = (uint8_t)e;
                    }
                }
                float sc[8], wp[8];
                load8(p.scale + col, cols, sc);
                load8(p.w_post + col, cols, wp);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    xv[c][i] += sc[i] * wp[i] * (av[c][i] * r) * (gv[c][i] / (1.f + __expf(-gv[c][i])));
                store8(y + byte, left[c], xv[c]);
            }
        }
        if (p.y_codes) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int64_t byte = row * p.dim + 8 * (sub + LPR * c);
                float kept[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) kept[i] = as_stored(xv[c][i], y);
                uint32_t e;
                const u32x2 codes = rows8_encode(kept, e);
                if (left[c] > 0) {
                    *reinterpret_cast<u32x2 *>(p.y_codes + byte) = codes;
                    if ((sub & 3) == 0) p.y_exps[byte / FS_ROWS8_GROUP] = (uint8_t)e;
                }
            }
        }
        if (!h) continue;
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) ss += xv[c][i] * xv[c][i];
        const float r = 1.f / sqrtf(row_sum<LPR>(ss) * inv_dim + p.eps);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = 8 * (sub + LPR * c);
            float wv[8], hv[8];
            load8(p.w_pre + col, p.dim - col, wv);
#pragma unroll
            for (int i = 0; i < 8; ++i) hv[i] = xv[c][i] * r * wv[i];
            store8(h + row * p.dim + col, left[c], hv);
        }
    }
}

// eight columns of a kept row, plain or in 8 bits
template <typename T>
__device__ __forceinline__ void load_kept(const void *rows, int64_t stride, const int8_t *codes, const uint8_t *exps, int dim,
                                          int64_t row, int col, int left, float (&v)[8]) {
    if (rows) {
        load8(static_cast<const T *>(rows) + row * stride + col, left, v);
    } else {
        u32x2 c = {0u, 0u};
        uint32_t e = 1;
        if (left > 0) {
            c = *reinterpret_cast<const u32x2 *>(codes + row * dim + col);
            e = exps[(row * dim + col) / FS_ROWS8_GROUP];
        }
        rows8_decode(c, e, v);
    }
}

// A workgroup takes the row groups blockIdx.x, blockIdx.x + gridDim.x, ... and keeps the column sums of its rows in
// registers; they are added up across its lanes and written down, part[2 * workgroup + {0: T, 1: dw_pre}][dim].
template <typename TR, typename TA, int LPR, int NC, bool JOIN, bool NORM>
__global__ __launch_bounds__(kBlockThreads) void block_norm_backward_kernel(fs_block_args p, float *__restrict__ part) {
    constexpr int kRows = kWave / LPR;
    __shared__ float sums[kBlockWaves][2 * NC * LPR * 8];
    const int lane = threadIdx.x & (kWave - 1), sub = lane & (LPR - 1), w = threadIdx.x / kWave;
    const TR *dy = static_cast<const TR *>(p.dy);
    const TA *dh = static_cast<const TA *>(p.dh);
    TR *dx = static_cast<TR *>(p.dx);
    TA *da = static_cast<TA *>(p.da), *dg = static_cast<TA *>(p.dg);
    const float inv_dim = 1.f / (float)p.dim;
    float sum_t[NC][8] = {}, sum_pre[NC][8] = {};
    float wpre[NC][8], wsc[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = 8 * (sub + LPR * c), cols = p.dim - col;
        if constexpr (NORM) load8(p.w_pre + col, cols, wpre[c]);
        if constexpr (JOIN) {
            float s[8], v[8];
            load8(p.scale + col, cols, s);
            load8(p.w_post + col, cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) wsc[c][i] = s[i] * v[i];
        }
    }
    const int64_t groups = (p.n + kRows * kBlockWaves - 1) / (kRows * kBlockWaves);
    for (int64_t b = blockIdx.x; b < groups; b += gridDim.x) {
        const int64_t row = (b * kBlockWaves + w) * kRows + lane / LPR;
        const bool live = row < p.n;
        float dv[NC][8], yv[NC][8], hv[NC][8], av[NC][8], gv[NC][8];
        int left[NC];
        float ssy = 0.f, dot = 0.f, ssa = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = 8 * (sub + LPR * c);
            left[c] = live ? p.dim - col : 0;
            load8(dy + row * p.dim + col, dy ? left[c] : 0, dv[c]);
            if constexpr (NORM) {
                load8(dh + row * p.dim + col, left[c], hv[c]);
                load_kept<TR>(p.y, p.dim, p.y_codes, p.y_exps, p.dim, row, col, left[c], yv[c]);
            }
            if constexpr (JOIN) {
                load_kept<TA>(p.a, p.a_stride, p.a_codes, p.a_exps, p.dim, row, col, left[c], av[c]);
                load_kept<TA>(p.g, p.g_stride, p.g_codes, p.g_exps, p.dim, row, col, left[c], gv[c]);
            }
        }
        if constexpr (NORM) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    ssy += yv[c][i] * yv[c][i];
                    dot += hv[c][i] * wpre[c][i] * yv[c][i];
                }
            const float r = 1.f / sqrtf(row_sum<LPR>(ssy) * inv_dim + p.eps);
            const float m = row_sum<LPR>(dot) * r * inv_dim;               // mean of (w_pre dh) yhat
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float yhat = yv[c][i] * r;
                    dv[c][i] += r * (hv[c][i] * wpre[c][i] - yhat * m);
                    sum_pre[c][i] += left[c] > 0 ? hv[c][i] * yhat : 0.f;
                }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) store8(dx + row * p.dim + 8 * (sub + LPR * c), left[c], dv[c]);
        if constexpr (JOIN) {
            // gv becomes silu(g), dgv what dg is made of
            float dgv[NC][8];
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) ssa += av[c][i] * av[c][i];
            const float r = 1.f / sqrtf(row_sum<LPR>(ssa) * inv_dim + p.eps);
            float dota = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float ahat = av[c][i] * r, gate = 1.f / (1.f + __expf(-gv[c][i]));
                    const float silu = gv[c][i] * gate;
                    const float u = dv[c][i] * wsc[c][i];
                    dgv[c][i] = u * ahat * (gate * (1.f + gv[c][i] * (1.f - gate)));
                    sum_t[c][i] += left[c] > 0 ? dv[c][i] * ahat * silu : 0.f;
                    gv[c][i] = u * silu;
                    av[c][i] = ahat;
                    dota += u * silu * ahat;
                }
            const float m = row_sum<LPR>(dota) * inv_dim;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = 8 * (sub + LPR * c);
#pragma unroll
                for (int i = 0; i < 8; ++i) gv[c][i] = r * (gv[c][i] - av[c][i] * m);
                store8(da + row * p.da_stride + col, left[c], gv[c]);
                store8(dg + row * p.dg_stride + col, left[c], dgv[c]);
            }
        }
    }
    // across the row groups of the wavefront, then across the wavefronts
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int m = LPR; m < kWave; m <<= 1) {
                sum_t[c][i] += __shfl_xor(sum_t[c][i], m, kWave);
                sum_pre[c][i] += __shfl_xor(sum_pre[c][i], m, kWave);
            }
            if (lane < LPR) {
                const int col = 8 * (sub + LPR * c) + i;
                sums[w][col] = sum_t[c][i];
                sums[w][NC * LPR * 8 + col] = sum_pre[c][i];
            }
        }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * NC * LPR * 8; k += kBlockThreads) {
        const int which = k / (NC * LPR * 8), col = k % (NC * LPR * 8);
        if (col < p.dim) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < kBlockWaves; ++v) s += sums[v][k];
            part[((int64_t)blockIdx.x * 2 + which) * p.dim + col] = s;
        }
    }
}

// The column sums of the workgroups added up in 64 bits: sixteen columns a workgroup, 64 threads a column, for it is one chain of
// loads (768 x 128 columns twice: 5 us, with 16 threads a column 21).
constexpr int kSumSlices = 64;
__global__ __launch_bounds__(16 * kSumSlices) void block_norm_weights_kernel(fs_block_args p, const float *__restrict__ part, int parts,
                                                                            bool join, bool norm) {
    __shared__ double sh[kSumSlices][17];
    const int c = threadIdx.x & 15, s = threadIdx.x >> 4;
    const int k = blockIdx.x * 16 + c;                   // column of the T sums, then of the dw_pre sums
    const bool in = k < 2 * p.dim && (k < p.dim ? join : norm);
    double sum = 0.0;
    if (in) {
#pragma unroll 4
        for (int b = s; b < parts; b += kSumSlices) sum += (double)part[(int64_t)b * 2 * p.dim + k];
    }
    sh[s][c] = sum;
    __syncthreads();
    for (int half = kSumSlices / 2; half >= 1; half >>= 1) {
        if (s < half) sh[s][c] += sh[s + half][c];
        __syncthreads();
    }
    if (s != 0 || !in) return;
    sum = sh[0][c];
    if (k < p.dim) {
        p.dw_post[k] = parts > 0 ? (float)(sum * (double)p.scale[k]) : 0.f;
        p.dscale[k] = parts > 0 ? (float)(sum * (double)p.w_post[k]) : 0.f;
    } else {
        p.dw_pre[k - p.dim] = (float)sum;
    }
}

// ---- rows in 8 bits, on their own: a thread has eight columns ---------------------------------------------------------------
// Bound by memory: 297 k rows of 128 fp32 columns, 191 MB each way, 39 us there (4.9 TB/s) and 29 back (6.6).
template <typename T>
__global__ __launch_bounds__(kBlockThreads) void rows_pack8_kernel(const T *__restrict__ rows, int64_t stride, int64_t pieces,
                                                                   int per_row, int8_t *__restrict__ codes,
                                                                   uint8_t *__restrict__ exps) {
    // pieces is a multiple of four: the lanes of a group are all in or all out
    for (int64_t k = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x; k < pieces; k += (int64_t)gridDim.x * kBlockThreads) {
        const int64_t row = k / per_row;
        float v[8];
        load8(rows + row * stride + 8 * (k - row * per_row), 8, v);
        uint32_t e;
        const u32x2 c = rows8_encode(v, e);
        *reinterpret_cast<u32x2 *>(codes + 8 * k) = c;
        if ((k & 3) == 0) exps[k >> 2] = (uint8_t)e;
    }
}

template <typename T>
__global__ __launch_bounds__(kBlockThreads) void rows_unpack8_kernel(const int8_t *__restrict__ codes,
                                                                     const uint8_t *__restrict__ exps, int64_t pieces,
                                                                     int per_row, T *__restrict__ rows, int64_t stride) {
    for (int64_t k = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x; k < pieces; k += (int64_t)gridDim.x * kBlockThreads) {
        const int64_t row = k / per_row;
        float v[8];
        rows8_decode(*reinterpret_cast<const u32x2 *>(codes + 8 * k), exps[k >> 2], v);
        store8(rows + row * stride + 8 * (k - row * per_row), 8, v);
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------------
// lanes that share a row: eight columns each; four at least, for the groups of 32 columns
int block_lanes(int32_t dim) {
    const int l = lanes_per_row((dim + 7) / 8);
    return l < 4 ? 4 : l > kWave ? kWave : l;
}
unsigned capped_grid(int64_t groups) { return (unsigned)(groups < kMaxGrid ? groups : kMaxGrid); }
int64_t block_row_groups(int64_t n, int32_t dim) { return ceil_div(n, (int64_t)kBlockWaves * (kWave / block_lanes(dim))); }
int block_partials(int64_t n, int32_t dim) {
    const int64_t g = block_row_groups(n, dim);
    return (int)(g < kMaxPartials ? g : kMaxPartials);
}

bool stride_ok(int64_t stride, int32_t dim, int dt) { return stride >= dim && (stride * elem_size(dt)) % 16 == 0; }

#define FS_NEED(cond, msg)                                   \
    do {                                                     \
        if (!(cond)) return set_err(ctx, FS_EINVAL, msg);    \
    } while (0)

int check_block(fs_ctx *ctx, const fs_block_args &p, bool packed) {
    FS_NEED(p.rows_dt == FS_F32 || p.rows_dt == FS_BF16, "block norm: unknown dtype of the rows");
    FS_NEED(p.dt == FS_F32 || p.dt == FS_BF16, "block norm: unknown dtype");
    FS_NEED(p.n >= 0, "block norm: negative size");
    FS_NEED(p.n < (1ll << 31), "block norm: more than 2^31-1 rows");
    const int unit = packed ? FS_ROWS8_GROUP : p.rows_dt == FS_F32 && p.dt == FS_F32 ? 4 : 8;
    FS_NEED(p.dim > 0 && p.dim <= FS_MAX_BLOCK_DIM && p.dim % unit == 0,
            "block norm: dim must be a multiple of 4 (both fp32) / 8 / 32 (rows in 8 bits), at most FS_MAX_BLOCK_DIM");
    FS_NEED(p.eps >= 0.f && p.eps < 1e30f, "block norm: eps must be a number, not negative");
    return FS_OK;
}

template <typename F>
int by_width(int32_t dim, F &&f) {
    switch (block_lanes(dim)) {
        case 4: return f(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
        case 8: return f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
        case 16: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
        case 32: return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
        default:
            if (dim <= 8 * kWave) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
            return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    }
}
template <typename F>
int by_types(int rows_dt, int dt, F &&f) {
    if (rows_dt == FS_F32) return dt == FS_F32 ? f((float *)nullptr, (float *)nullptr) : f((float *)nullptr, (bf16_t *)nullptr);
    return dt == FS_F32 ? f((bf16_t *)nullptr, (float *)nullptr) : f((bf16_t *)nullptr, (bf16_t *)nullptr);
}

}  // namespace

extern "C" {

int fs_block_norm(fs_ctx *ctx, const fs_block_args *args, fs_stream stream) {
    if (!ctx) return FS_EINVAL;
    FS_NEED(args, "block norm: null pointer");
    fs_block_args p = *args;
    const bool join = p.a != nullptr;
    const int rc = check_block(ctx, p, (join && (p.a_codes || p.g_codes)) || p.y_codes);
    if (rc != FS_OK) return rc;
    if (!join) p.a_codes = p.g_codes = nullptr;
    if (p.n == 0) return FS_OK;
    FS_NEED(p.x && aligned16(p.x), "block norm: x is null or not 16-byte aligned");
    if (join) {
        FS_NEED(p.g && p.w_post && p.scale && p.y, "block norm: null pointer");
        FS_NEED(aligned16(p.a) && aligned16(p.g) && aligned16(p.y) && aligned16(p.w_post) && aligned16(p.scale),
                "block norm: pointer not 16-byte aligned");
        FS_NEED(stride_ok(p.a_stride, p.dim, p.dt) && stride_ok(p.g_stride, p.dim, p.dt),
                "block norm: a stride is less than dim or not a multiple of 16 bytes");
    }
    FS_NEED(join || p.h || p.y_codes, "block norm: nothing to compute");
    if (p.h) FS_NEED(p.w_pre && aligned16(p.h) && aligned16(p.w_pre), "block norm: h or w_pre is null or not 16-byte aligned");
    FS_NEED((!p.a_codes || p.a_exps) && (!p.g_codes || p.g_exps) && (!p.y_codes || p.y_exps),
            "block norm: codes without exponents");
    FS_NEED(aligned16(p.a_codes) && aligned16(p.g_codes) && aligned16(p.y_codes), "block norm: codes not 16-byte aligned");
    device_scope on(ctx->device);
    if (!on.ok) return set_err(ctx, FS_EHIP, "block norm: the context's GPU cannot be made current");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid(capped_grid(block_row_groups(p.n, p.dim)));
    by_types(p.rows_dt, p.dt, [&](auto *r, auto *t) {
        using TR = std::remove_pointer_t<decltype(r)>;
        using TA = std::remove_pointer_t<decltype(t)>;
        return by_width(p.dim, [&](auto lpr, auto nc) {
            if (join) block_norm_kernel<TR, TA, lpr(), nc(), true><<<grid, kBlockThreads, 0, s>>>(p);
            else block_norm_kernel<TR, TA, lpr(), nc(), false><<<grid, kBlockThreads, 0, s>>>(p);
            return 0;
        });
    });
    FS_LAUNCH_CHECK(ctx, "block_norm");
    return FS_OK;
}

size_t fs_block_norm_work_bytes(int64_t n, int32_t dim) {
    if (n <= 0 || dim <= 0 || dim > FS_MAX_BLOCK_DIM) return 0;
    return (size_t)block_partials(n, dim) * 2 * (size_t)dim * sizeof(float);
}

int fs_block_norm_backward(fs_ctx *ctx, const fs_block_args *args, fs_stream stream) {
    if (!ctx) return FS_EINVAL;
    FS_NEED(args, "block norm backward: null pointer");
    fs_block_args p = *args;
    // without rows there may be no addresses to tell what is wanted but those of the sums
    const bool join = p.n > 0 ? p.a || p.a_codes : p.dw_post || p.dscale;
    const bool norm = p.n > 0 ? p.dh != nullptr : p.dw_pre != nullptr;
    const bool packed = p.n > 0 && ((join && (!p.a || !p.g)) || (norm && !p.y));
    const int rc = check_block(ctx, p, packed);
    if (rc != FS_OK) return rc;
    FS_NEED(join || norm, "block norm backward: nothing to compute");
    FS_NEED(!join || (p.dw_post && p.dscale), "block norm backward: null pointer");
    if (p.n > 0) {
        if (join) {
            FS_NEED(p.a || p.a_exps, "block norm backward: codes without exponents");
            FS_NEED(p.g || (p.g_codes && p.g_exps), "block norm backward: g is null, or codes without exponents");
            FS_NEED(p.w_post && p.scale && p.da && p.dg, "block norm backward: null pointer");
            FS_NEED(aligned16(p.w_post) && aligned16(p.scale) && aligned16(p.a ? p.a : p.a_codes) && aligned16(p.g ? p.g : p.g_codes) &&
                        aligned16(p.da) && aligned16(p.dg),
                    "block norm backward: pointer not 16-byte aligned");
            FS_NEED((!p.a || stride_ok(p.a_stride, p.dim, p.dt)) && (!p.g || stride_ok(p.g_stride, p.dim, p.dt)) &&
                        stride_ok(p.da_stride, p.dim, p.dt) && stride_ok(p.dg_stride, p.dim, p.dt),
                    "block norm backward: a stride is less than dim or not a multiple of 16 bytes");
        }
        if (norm) {
            FS_NEED(p.y || (p.y_codes && p.y_exps), "block norm backward: y is null, or codes without exponents");
            FS_NEED(p.w_pre && p.dw_pre, "block norm backward: null pointer");
            FS_NEED(aligned16(p.y ? p.y : p.y_codes) && aligned16(p.dh) && aligned16(p.w_pre),
                    "block norm backward: pointer not 16-byte aligned");
        }
        FS_NEED(p.dx && aligned16(p.dx) && aligned16(p.dy), "block norm backward: dx is null, or dx or dy not 16-byte aligned");
        FS_NEED(p.work && p.work_bytes >= fs_block_norm_work_bytes(p.n, p.dim), "block norm backward: work is too small");
    }
    device_scope on(ctx->device);
    if (!on.ok) return set_err(ctx, FS_EHIP, "block norm backward: the context's GPU cannot be made current");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    float *part = static_cast<float *>(p.work);
    const int parts = p.n > 0 ? block_partials(p.n, p.dim) : 0;
    if (parts > 0) {
        by_types(p.rows_dt, p.dt, [&](auto *r, auto *t) {
            using TR = std::remove_pointer_t<decltype(r)>;
            using TA = std::remove_pointer_t<decltype(t)>;
            return by_width(p.dim, [&](auto lpr, auto nc) {
                if (join && norm)
                    block_norm_backward_kernel<TR, TA, lpr(), nc(), true, true><<<parts, kBlockThreads, 0, s>>>(p, part);
                else if (join)
                    block_norm_backward_kernel<TR, TA, lpr(), nc(), true, false><<<parts, kBlockThreads, 0, s>>>(p, part);
                else
                    block_norm_backward_kernel<TR, TA, lpr(), nc(), false, true><<<parts, kBlockThreads, 0, s>>>(p, part);
                return 0;
            });
        });
        FS_LAUNCH_CHECK(ctx, "block_norm_backward");
    }
    block_norm_weights_kernel<<<(unsigned)ceil_div(2 * p.dim, 16), 16 * kSumSlices, 0, s>>>(p, part, parts, join, norm);
    FS_LAUNCH_CHECK(ctx, "block_norm_weights");
    return FS_OK;
}

int fs_rows_pack8(fs_ctx *ctx, const void *rows, int64_t stride, fs_dtype dt, int64_t n, int32_t dim, int8_t *codes,
                  uint8_t *exps, fs_stream stream) {
    if (!ctx) return FS_EINVAL;
    FS_NEED(dt == FS_F32 || dt == FS_BF16, "rows pack8: unknown dtype");
    FS_NEED(n >= 0 && n < (1ll << 31), "rows pack8: n is negative or beyond 2^31-1");
    FS_NEED(dim > 0 && dim <= FS_MAX_BLOCK_DIM && dim % FS_ROWS8_GROUP == 0,
            "rows pack8: dim must be a multiple of FS_ROWS8_GROUP, at most FS_MAX_BLOCK_DIM");
    FS_NEED(stride_ok(stride, dim, dt), "rows pack8: the stride is less than dim or not a multiple of 16 bytes");
    if (n == 0) return FS_OK;
    FS_NEED(rows && codes && exps, "rows pack8: null pointer");
    FS_NEED(aligned16(rows) && aligned16(codes), "rows pack8: pointer not 16-byte aligned");
    device_scope on(ctx->device);
    if (!on.ok) return set_err(ctx, FS_EHIP, "rows pack8: the context's GPU cannot be made current");
    const int64_t pieces = n * (dim / 8);
    const unsigned grid = capped_grid(ceil_div(pieces, kBlockThreads));
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dt == FS_F32)
        rows_pack8_kernel<float><<<grid, kBlockThreads, 0, s>>>(static_cast<const float *>(rows), stride, pieces, dim / 8, codes, exps);
    else
        rows_pack8_kernel<bf16_t><<<grid, kBlockThreads, 0, s>>>(static_cast<const bf16_t *>(rows), stride, pieces, dim / 8, codes, exps);
    FS_LAUNCH_CHECK(ctx, "rows_pack8");
    return FS_OK;
}

int fs_rows_unpack8(fs_ctx *ctx, const int8_t *codes, const uint8_t *exps, int64_t n, int32_t dim, void *rows, int64_t stride,
                    fs_dtype dt, fs_stream stream) {
    if (!ctx) return FS_EINVAL;
    FS_NEED(dt == FS_F32 || dt == FS_BF16, "rows unpack8: unknown dtype");
    FS_NEED(n >= 0 && n < (1ll << 31), "rows unpack8: n is negative or beyond 2^31-1");
    FS_NEED(dim > 0 && dim <= FS_MAX_BLOCK_DIM && dim % FS_ROWS8_GROUP == 0,
            "rows unpack8: dim must be a multiple of FS_ROWS8_GROUP, at most FS_MAX_BLOCK_DIM");
    FS_NEED(stride_ok(stride, dim, dt), "rows unpack8: the stride is less than dim or not a multiple of 16 bytes");
    if (n == 0) return FS_OK;
    FS_NEED(rows && codes && exps, "rows unpack8: null pointer");
    FS_NEED(aligned16(rows) && aligned16(codes), "rows unpack8: pointer not 16-byte aligned");
    device_scope on(ctx->device);
    if (!on.ok) return set_err(ctx, FS_EHIP, "rows unpack8: the context's GPU cannot be made current");
    const int64_t pieces = n * (dim / 8);
    const unsigned grid = capped_grid(ceil_div(pieces, kBlockThreads));
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dt == FS_F32)
        rows_unpack8_kernel<float><<<grid, kBlockThreads, 0, s>>>(codes, exps, pieces, dim / 8, static_cast<float *>(rows), stride);
    else
        rows_unpack8_kernel<bf16_t><<<grid, kBlockThreads, 0, s>>>(codes, exps, pieces, dim / 8, static_cast<bf16_t *>(rows), stride);
    FS_LAUNCH_CHECK(ctx, "rows_unpack8");
    return FS_OK;
}

}  // extern "C"
