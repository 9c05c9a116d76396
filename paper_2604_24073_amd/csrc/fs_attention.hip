// Attention over a jagged batch with a learned relative position bias, forward.
//
//   s_ij = scale q_i . k_j + bias[bucket(pos_i - pos_j), head],  o_i = sum_j softmax(s_i)_j v_j
//
// One pass over the keys with the running maximum m and sum l of a row's softmax: a workgroup has 64 query rows of one user
// and head, a wavefront 16 of them, and the keys come by in tiles of 64 through LDS, the next tile on its way while
// this one is worked on.  The products are turned over: S^T = K Q^T and O^T = V^T P^T, so that a lane has one query
// row, its m and l are a register each, and the scores stay in registers from one product to the other.
//
// Bound by the vector units, which have 12 to 14 instructions for a score where out is wanted unrounded (five or six of them
// split P into three terms), and by how little of that the matrix units' time hides under: 73 % and 38 % of the time with 64
// columns (four wavefronts a SIMD), 84 % and 20 % with 32 (five).  160 histories with 150 k rows, 8 of them of 16384, 4 heads of
// 64 columns over 2 key heads, out unrounded for the bias's gradient: 2.7 to 2.9 ms, 400 TFLOP/s of the formula's products and
// 800 of those that are made.  1024 histories with 262 k rows, 4 heads of 32: 0.51 ms.  Tried without gain: the next tile's
// scores made beside this tile's powers (registers: a wavefront a SIMD less, 0.51 ms to 0.62), priorities for wavefronts in their
// products.
#include "fs_attention.h"

using namespace fs;

namespace {

// Sixteens of query rows of a wavefront.  Two halve what a score reads from LDS, but leave registers for fewer wavefronts and more
// rows that are none.  us with one / two, bf16: 506 / 545 (1024 histories of 256 on average, 32 columns), 718 / 838 (64 columns),
// 209 / 232 (300 of 400 up, 64), 1562 / 1600 (64 of 4000 up, 64), 2877 / 2809 (8 of 16384, 64), 1040 / 1750 (64 of 2000 up, 128).
constexpr int QT = 1;

// EXACT, of bf16 rows whose unrounded out is wanted: P goes into its product as three terms of bf16, which hold its 24 bits.  The
// bias's gradient adds up differences of dO V^T and D = dO . out that cancel over a row, and an out made of rounded P leaves its
// errors in them.  dbias is off by 6e-4 of itself with one term, 1e-6 with two, 4e-7 with three (1024 histories with 262 k rows,
// 64 buckets, and histories of 16384 rows alike); the pass over the former, 4 heads of 32 columns, took 0.41, 0.47 and 0.54 ms.
// Without out_f32 P is one term: a bf16 out is rounded to half a step of bf16 anyway, and half a step of every P, independent of each
// other, adds no more than that to it (2.4e-3 off in all against 1.7e-3 for the rounding of out alone).
template <typename T, int DH, bool EXACT>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_forward_kernel(attn_params p) {
    constexpr int kRows = 16 * kAttnWaves * QT, kShift = 6, kPad = row_pad(QT);
    constexpr int KC = DH / 32, MT = DH / 16;
    extern __shared__ __align__(16) char lds[];
    tile<T, DH> &K = *reinterpret_cast<tile<T, DH> *>(lds), &V = (&K)[1];
    uint32_t *odd = reinterpret_cast<uint32_t *>(&V + 1);            // [wavefronts]: the tile had values that are no numbers
    float *bias_lds = reinterpret_cast<float *>(odd + kAttnWaves);

    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15, w = wave_id();
    const int head = blockIdx.x % p.heads;
    const int slot = (int)(blockIdx.x / p.heads);
    if (head == 0) check_layout(p, slot, (int)(gridDim.x / p.heads));
    user u;
    int index;
    if (!find_user(p, p.q_offsets, slot, kShift, u, index) || (int64_t)index * kRows >= u.nq) return;
    index = (u.nq - 1) / kRows - index;                              // the last rows, which see most, begin first
    const int row0 = index * kRows;                                  // first query row of the workgroup
    const int rows = u.nq - row0 < kRows ? u.nq - row0 : kRows;
    const int pos0 = u.first + row0, pos_last = pos0 + rows - 1;
    const int end = p.causal ? (pos_last + 1 < u.nk ? pos_last + 1 : u.nk) : u.nk;
    const int tiles = end <= 0 ? 0 : (end + kTile - 1) / kTile;
    const T *kbase = static_cast<const T *>(p.k) + u.k0 * p.k_stride + (head / p.group) * p.width;
    const T *vbase = static_cast<const T *>(p.v) + u.k0 * p.v_stride + (head / p.group) * p.width;

    tile_regs<T, DH> kr, vr;
    kr.place(p.k_stride, p.width);
    vr.place(p.v_stride, p.width);
    kr.load(kbase, p.k_stride, tiles ? u.nk : 0);
    vr.load(vbase, p.v_stride, tiles ? u.nk : 0);

    // the wavefront's query rows, and where they stand among the keys
    const int wrow = row0 + 16 * QT * w, wpos = u.first + wrow;
    piece<T> qf[QT][KC];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int row = wrow + 16 * t + j;
        const T *qbase = static_cast<const T *>(p.q) + u.q0 * p.q_stride + head * p.width;
#pragma unroll
        for (int c = 0; c < KC; ++c) global_rows(qf[t][c], qbase, p.q_stride, row, row < u.nq, 32 * c, p.width);
    }
    strip<kPad> bias;
    const bool hides = bias.fill(p, head, bias_lds, pos0 - (end > 0 ? end - 1 : 0), pos_last);
    const float scale2 = p.scale * kLog2e;

    // the products with P's further terms have a sum of their own: an infinity among the values meets zeros and negative terms there
    f32x4 acc[QT][MT] = {}, acc_rest[EXACT ? QT : 1][MT] = {};
    // m: what the row's scores are less by (less: the same in the product's own terms); it follows the row's
    // maximum once that is 2^8 ahead, which is enough to keep the powers in range, and at once from the first key seen on
    float m[QT], l[QT], less[QT], ahead[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = l[t] = less[t] = 0.f;
        ahead[t] = neg_inf();
    }
    // From this tile on some rows do not see all keys: what they do not see must not reach them, not even as 0 * NaN.  Below zero
    // where the bias hides: one register tells both.
    const int first_edge = hides ? -1 : p.causal ? max((pos0 + 1) >> 6, 0) : 0x7fffffff;
    const auto edge = [&](int n) { return n >= first_edge; };
    const auto stage = [&](int n) {
        kr.store(K);
        if (edge(n)) {
            const bool any = __any(vr.clean());
            if (lane == 0) odd[w] = any;
        }
        vr.store(V);
    };
    if (tiles) stage(0);
    for (int n = 0; n < tiles; ++n) {
        __syncthreads();
        const int key0 = n * kTile;
        if (n + 1 < tiles) {
            kr.load(kbase + (int64_t)(key0 + kTile) * p.k_stride, p.k_stride, u.nk - key0 - kTile);
            vr.load(vbase + (int64_t)(key0 + kTile) * p.v_stride, p.v_stride, u.nk - key0 - kTile);
        }
        if (wrow < u.nq && !(p.causal && key0 > wpos + 16 * QT - 1)) {
            f32x4 s[QT][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    const float at = from_less<T> ? less[t] : 0.f;
                    s[t][k] = f32x4{at, at, at, at};
                }
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    piece<T> a;
                    K.rows(a, 16 * k, 32 * c);
#pragma unroll
                    for (int t = 0; t < QT; ++t) mma(s[t][k], a, qf[t][c]);
                }
            }
            settle();
            // element r of s[t][k]: query row wrow + 16 t + j, key key0 + 16 k + 4 g + r
            const int nearest = wpos - (key0 + kTile - 1), furthest = wpos + 16 * QT - 1 - key0;
            if (nearest >= bias.high || furthest <= bias.low) {
                const float b = bias.at[bias.zero + (nearest >= bias.high ? bias.high : bias.low)];
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[t][k][r] = s[t][k][r] * scale2 + (from_less<T> ? b : b - m[t]);
            } else {
                const float *b = bias.at + bias.zero + nearest + (j - 4 * g) + 12;
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float x = b[51 + 16 * t - 16 * k - r];
                            s[t][k][r] = s[t][k][r] * scale2 + (from_less<T> ? x : x - m[t]);
                        }
            }
            if (first_edge < 0) {
                // a hidden pair's product may be no number, and -inf added to that is none: its score is -inf all the same
                const int near = min(max(nearest, bias.low - (62 + 16 * QT)), bias.high);
                const float *b = bias.at + bias.zero + near + (j - 4 * g) + 12;
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        __builtin_amdgcn_sched_barrier(0);           // registers for four biases at a time
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (b[51 + 16 * t - 16 * k - r] == neg_inf()) s[t][k][r] = neg_inf();
                    }
            }
            if ((p.causal && key0 + kTile - 1 > wpos) || key0 + kTile > u.nk) {
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    const int pos = wpos + 16 * t + j;
                    const int seen = p.causal && pos + 1 < u.nk ? pos + 1 : u.nk;      // keys that the row sees
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (key0 + 16 * k + 4 * g + r >= seen) s[t][k][r] = neg_inf();
                }
            }
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                float top = s[t][0][0];
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = fmaxf(top, s[t][k][r]);
                top = column_max(top);
                const bool behind = top > ahead[t];
                if (__any(behind)) {
                    // at first, where top may be anything, there is nothing to shrink yet
                    const float step = behind ? top : 0.f, shrink = __builtin_amdgcn_exp2f(-fmaxf(step, 0.f));
                    m[t] += step;
                    less[t] = -m[t] / scale2;
                    ahead[t] = behind ? 8.f : ahead[t];
                    l[t] *= shrink;
#pragma unroll
                    for (int c = 0; c < MT; ++c)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            acc[t][c][r] *= shrink;
                            if constexpr (EXACT) acc_rest[t][c][r] *= shrink;
                        }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[t][k][r] -= step;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[t][k][r] = __builtin_amdgcn_exp2f(s[t][k][r]);
                        l[t] += s[t][k][r];
                    }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                piece<T> pf[QT], rest[EXACT ? QT : 1][2];
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    if constexpr (EXACT) {
                        take_operand(pf[t], s[t][2 * c], s[t][2 * c + 1]);
                        take_operand(rest[t][0], s[t][2 * c], s[t][2 * c + 1]);
                        as_operand(rest[t][1], s[t][2 * c], s[t][2 * c + 1]);
                    } else {
                        as_operand(pf[t], s[t][2 * c], s[t][2 * c + 1]);
                    }
                }
#pragma unroll
                for (int d = 0; d < MT; ++d) {
                    piece<T> a;
                    V.cols(a, 32 * c, 16 * d);
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        mma(acc[t][d], a, pf[t]);
                        if constexpr (EXACT) {
                            mma(acc_rest[t][d], a, rest[t][0]);
                            mma(acc_rest[t][d], a, rest[t][1]);
                        }
                    }
                }
            }
            settle();
            if (edge(n)) {
                uint32_t any = 0;
                for (int x = 0; x < kAttnWaves; ++x) any |= odd[x];
                if (any) {
                    // the values left out of the product, key by key, for the rows that see them
                    const int keys = u.nk - key0 < kTile ? u.nk - key0 : kTile;
                    for (int k = 0; k < keys; ++k) {
                        const T *v = vbase + (int64_t)(key0 + k) * p.v_stride;
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
                            const int d = wpos + 16 * t + j - key0 - k;
                            const int dc = d > bias.high ? bias.high : d < bias.low ? bias.low : d;
                            const bool sees = !(p.causal && d < 0) && bias.at[bias.zero + dc] != neg_inf();
#pragma unroll
                            for (int c = 0; c < MT; ++c)
#pragma unroll
                                for (int r = 0; r < 4; ++r) {
                                    const int col = 16 * c + 4 * g + r;
                                    const float x = col < p.width ? load1(v + col) : 0.f;
                                    if (sees && !(fabsf(x) < __builtin_inff())) acc[t][c][r] += x;
                                }
                        }
                    }
                }
            }
        }
        if (n + 1 < tiles) {
            __syncthreads();
            stage(n + 1);
        }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const float sum = column_sum(l[t]);
        const int row = wrow + 16 * t + j;
        if (row >= u.nq) continue;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;              // a row that sees nothing: zeros
        const int64_t at = ((u.q0 + row) * p.heads + head) * p.width;
        if (p.lse && g == 0) p.lse[(int64_t)head * p.n_q + u.q0 + row] = sum == 0.f ? neg_inf() : (m[t] + __log2f(sum)) * kLn2;
#pragma unroll
        for (int c = 0; c < MT; ++c) {
            const int col = 16 * c + 4 * g;
            f32x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float x = acc[t][c][r];
                if constexpr (EXACT) x += fabsf(x) < __builtin_inff() ? acc_rest[t][c][r] : 0.f;
                o[r] = x * inv;
            }
            if (col < p.width) {
                store4(static_cast<T *>(p.out) + at + col, o);
                if (p.out_f32) store4(p.out_f32 + at + col, o);
            }
        }
    }
}

// ---- few query rows -----------------------------------------------------------------------------------------------------------
// Serving: a few new rows of each user against a long history.  What there is to do is to read k and v once, so the keys are
// cut up: a workgroup has a chunk of one user's keys for all query rows and heads that share a key head (at most sixteen
// columns of a product), its wavefronts take kSplitKeys keys each in turn, and what they have of m, l and o is put together, in
// the workgroup first, then, where a user has several chunks, by a second launch.  Bound by the waits of one chunk, one behind
// the other, more than by memory: 256 users with 93 k keys, 8 heads of 64 columns over 2, 47 MB: 20.6 us (2.3 TB/s) and 6.  Here
// P is three terms of bf16 always, as the matrix units have the time for it (19.5 us with one term).
constexpr int kSplitCols = 16;
constexpr int kSplitKeys = 32;                        // keys of a wavefront at a time
constexpr int kSplitStep = kAttnWaves * kSplitKeys;   // keys of a workgroup at a time

// bytes of LDS for the wavefronts' rows of v, and afterwards for what they have of the result: m, l and rows of DH + 4
template <typename T, int DH>
constexpr int split_rows_lds = kAttnWaves * (sizeof(tile<T, DH, kSplitKeys>) > 4 * kSplitCols * (DH + 6)
                                                 ? (int)sizeof(tile<T, DH, kSplitKeys>) : 4 * kSplitCols * (DH + 6));
// Wavefronts of a SIMD: all of a serving batch's workgroups want to be under way at once, since each is one chain of waits
template <typename T, int DH>
constexpr int split_waves = sizeof(T) * DH <= 64 ? 5 : sizeof(T) * DH <= 128 ? 4 : sizeof(T) * DH <= 256 ? 2 : 1;

template <typename T, int DH>
__global__ __launch_bounds__(kAttnThreads, (split_waves<T, DH>)) void attn_split_kernel(attn_params p) {
    const int shift = p.split_shift, max_q = p.max_q;
    constexpr int KC = DH / 32, MT = DH / 16;
    extern __shared__ __align__(16) char lds[];
    using vtile = tile<T, DH, kSplitKeys>;
    vtile *vt = reinterpret_cast<vtile *>(lds);                                               // [wavefronts]
    float *merge = reinterpret_cast<float *>(lds);                                            // the same memory, afterwards
    float *bias_lds = reinterpret_cast<float *>(lds + split_rows_lds<T, DH>);
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15, w = wave_id();
    const int kv_heads = p.heads / p.group, kvh = blockIdx.x % kv_heads;
    const int slot = (int)(blockIdx.x / kv_heads);
    if (kvh == 0) check_layout(p, slot, (int)(gridDim.x / kv_heads));
    user u;
    int index;
    if (!find_user(p, p.kv_offsets, slot, shift, u, index)) return;
    const int chunk = 1 << shift, cols = u.nq * p.group;
    const bool none = u.nk == 0 && index == 0;         // nobody else writes the rows of a user without keys
    if (u.nq > max_q) {
        if (threadIdx.x == 0 && index == 0) atomicOr(p.flags, kFlagOffsets);
        return;
    }
    if (u.nq == 0 || (!none && (int64_t)index * chunk >= u.nk)) return;
    const int begin = index * chunk, stop = u.nk - begin < chunk ? u.nk : begin + chunk;
    const T *kbase = static_cast<const T *>(p.k) + u.k0 * p.k_stride + kvh * p.width;
    const T *vbase = static_cast<const T *>(p.v) + u.k0 * p.v_stride + kvh * p.width;

    const bool live = j < cols;
    const int row = live ? j / p.group : 0, head = kvh * p.group + j % p.group, pos = u.first + row;     // of the lane's column
    piece<T> qf[KC];
#pragma unroll
    for (int c = 0; c < KC; ++c)
        global_rows(qf[c], static_cast<const T *>(p.q) + u.q0 * p.q_stride + head * p.width, p.q_stride, row, live, 32 * c, p.width);
    const float scale2 = p.scale * kLog2e;
    const int high = p.distances - 1, low = p.causal ? 0 : -high;

    // further terms of P in bf16, with a sum of their own as in attn_forward_kernel
    constexpr int kMore = sizeof(T) == 2 ? 2 : 0;
    f32x4 acc[MT] = {}, acc_rest[kMore ? MT : 1] = {};
    float m = neg_inf(), l = 0.f;
    const int met = kSplitStep + u.nq - 1;                // distances of a step's keys from the query rows
    for (int step = begin; step < stop; step += kSplitStep) {
        const int key0 = step + kSplitKeys * w, keys = stop - key0 < kSplitKeys ? stop - key0 : kSplitKeys;   // of the wavefront; may be none
        // from the last key's distance to the first's: their buckets on the way first, the biases behind the rows of k and v
        const int from = u.first - (step + kSplitStep - 1);
        const int bucket = p.bias ? p.bucket_of[min(max(from + (int)threadIdx.x, low), high) - low] : 0;
        piece<T> kf[kSplitKeys / 16][KC];
#pragma unroll
        for (int k = 0; k < kSplitKeys / 16; ++k)
#pragma unroll
            for (int c = 0; c < KC; ++c)
                global_rows(kf[k][c], kbase + (int64_t)key0 * p.k_stride, p.k_stride, 16 * k + j, 16 * k + j < keys, 32 * c, p.width);
        // the wavefront's rows of v: the lanes take the chunks of 16 bytes one after the other
        constexpr int kMine = vtile::kChunks * kSplitKeys / kWave;
        u32x4 vv[kMine];
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int k = lane + 64 * x, r = k / vtile::kChunks, c = (k % vtile::kChunks) * vtile::kPer;
            const u32x4 zero = {0u, 0u, 0u, 0u};
            vv[x] = r < keys && c < p.width ? *reinterpret_cast<const u32x4 *>(vbase + (int64_t)(key0 + r) * p.v_stride + c) : zero;
        }
        if (step > begin) __syncthreads();
        bool hides = false;
        if ((int)threadIdx.x < met) {                      // a thread each: kSplitStep + 15 of them at most
            const bool none = bucket < 0 || bucket >= p.buckets;
            if (p.bias && none) atomicOr(p.flags, kFlagRowRange);
            for (int h = 0; h < p.group; ++h) {
                const float b = none ? 0.f : bias_power(p.bias[(int64_t)bucket * p.heads + kvh * p.group + h]);
                bias_lds[threadIdx.x * p.group + h] = b;
                hides |= b == neg_inf();
            }
        }
        hides = __syncthreads_or(hides) != 0;
        if (keys > 0) {
            const bool edge = hides || (p.causal && key0 + keys - 1 > u.first);
            bool odd = false;
#pragma unroll
            for (int x = 0; x < kMine; ++x) {
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) vv[x][i] = clean_word<T>(vv[x][i], odd);
                }
                const int k = lane + 64 * x, r = k / vtile::kChunks, c = (k % vtile::kChunks) * vtile::kPer;
                *reinterpret_cast<u32x4 *>(vt[w].at + r * vtile::kLd + c) = vv[x];
            }
            odd = __any(odd) != 0;
            wave_lds_order();
            f32x4 s[kSplitKeys / 16];
            float top = neg_inf();
            const int seen = !live ? 0 : p.causal && pos + 1 < stop ? pos + 1 : stop;
            const float *b = bias_lds + ((pos - key0) - from) * p.group + head - kvh * p.group;
#pragma unroll
            for (int k = 0; k < kSplitKeys / 16; ++k) {
                s[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KC; ++c) mma(s[k], kf[k][c], qf[c]);
            }
            settle();
#pragma unroll
            for (int k = 0; k < kSplitKeys / 16; ++k) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = 16 * k + 4 * g + r;
                    const float x = b[-key * p.group];                         // in the strip for every key of the step
                    // a hidden pair's product may be no number: -inf is not added to it but put in its place
                    s[k][r] = key0 + key < seen && x != neg_inf() ? s[k][r] * scale2 + x : neg_inf();
                    top = fmaxf(top, s[k][r]);
                }
            }
            const float next = fmaxf(m, column_max(top)), base = next == neg_inf() ? 0.f : next;
            const float shrink = __builtin_amdgcn_exp2f(m - base);
            m = next;
            l *= shrink;
#pragma unroll
            for (int d = 0; d < MT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    acc[d][r] *= shrink;
                    if constexpr (kMore > 0) acc_rest[d][r] *= shrink;
                }
#pragma unroll
            for (int k = 0; k < kSplitKeys / 16; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[k][r] = __builtin_amdgcn_exp2f(s[k][r] - base);
                    l += s[k][r];
                }
#pragma unroll
            for (int c = 0; c < kSplitKeys / 32; ++c) {
                piece<T> pf, rest[kMore ? kMore : 1];
                if constexpr (kMore > 0) {
                    take_operand(pf, s[2 * c], s[2 * c + 1]);
#pragma unroll
                    for (int i = 0; i < kMore; ++i) take_operand(rest[i], s[2 * c], s[2 * c + 1]);
                } else {
                    as_operand(pf, s[2 * c], s[2 * c + 1]);
                }
#pragma unroll
                for (int d = 0; d < MT; ++d) {
                    piece<T> a;
                    vt[w].cols(a, 32 * c, 16 * d);
                    mma(acc[d], a, pf);
#pragma unroll
                    for (int i = 0; i < kMore; ++i) mma(acc_rest[d], a, rest[i]);
                }
            }
            settle();
            if (odd) {                                  // the values left out of the product, for the rows that see them
                for (int k = 0; k < keys; ++k) {
                    const bool sees = key0 + k < seen && b[-k * p.group] != neg_inf();
#pragma unroll
                    for (int d = 0; d < MT; ++d)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int col = 16 * d + 4 * g + r;
                            const float x = col < p.width ? load1(vbase + (int64_t)(key0 + k) * p.v_stride + col) : 0.f;
                            if (sees && !(fabsf(x) < __builtin_inff())) acc[d][r] += x;
                        }
                }
            }
        }
    }
    // across the wavefronts: merge[w][column] = {m, l}, then [w][column][DH + 4] of o
    __syncthreads();
    constexpr int kLd = DH + 4;
    float *ml = merge, *os = merge + 2 * kAttnWaves * kSplitCols;
    l = column_sum(l);
    if (g == 0) {
        ml[2 * (w * kSplitCols + j)] = m;
        ml[2 * (w * kSplitCols + j) + 1] = l;
    }
#pragma unroll
    for (int d = 0; d < MT; ++d) {
        if constexpr (kMore > 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[d][r] += fabsf(acc[d][r]) < __builtin_inff() ? acc_rest[d][r] : 0.f;
        }
        *reinterpret_cast<f32x4 *>(os + (w * kSplitCols + j) * kLd + 16 * d + 4 * g) = acc[d];
    }
    __syncthreads();
    const bool whole = u.nk <= chunk;
    for (int x = threadIdx.x; x < cols * (DH / 4); x += kAttnThreads) {
        const int c = x / (DH / 4), col = 4 * (x % (DH / 4));
        float top = neg_inf();
#pragma unroll
        for (int v = 0; v < kAttnWaves; ++v) top = fmaxf(top, ml[2 * (v * kSplitCols + c)]);
        const float base = top == neg_inf() ? 0.f : top;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < kAttnWaves; ++v) {
            const float part = __builtin_amdgcn_exp2f(ml[2 * (v * kSplitCols + c)] - base);
            const f32x4 a = *reinterpret_cast<const f32x4 *>(os + (v * kSplitCols + c) * kLd + col);
            sum += part * ml[2 * (v * kSplitCols + c) + 1];
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] += part * a[r];
        }
        const int crow = c / p.group, chead = kvh * p.group + c % p.group;
        if (whole) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] *= inv;
            if (p.lse && col == 0)
                p.lse[(int64_t)chead * p.n_q + u.q0 + crow] = sum == 0.f ? neg_inf() : (top + __log2f(sum)) * kLn2;
            if (col < p.width) {
                const int64_t at = ((u.q0 + crow) * p.heads + chead) * p.width + col;
                store4(static_cast<T *>(p.out) + at, o);
                if (p.out_f32) store4(p.out_f32 + at, o);
            }
        } else {
            const int64_t at = ((int64_t)slot * kv_heads + kvh) * (max_q * p.group) + c;
            if (col == 0) {
                p.split_ml[2 * at] = top;
                p.split_ml[2 * at + 1] = sum;
            }
            store4(p.split_acc + at * DH + col, o);
        }
    }
}

// The chunks of a user put together: a wavefront has one query row of one head at a time.
template <typename T, int DH>
__global__ __launch_bounds__(kAttnThreads) void attn_join_kernel(attn_params p) {
    const int shift = p.split_shift, max_q = p.max_q;
    const int lane = threadIdx.x & 63;
    for (int64_t item = (int64_t)blockIdx.x * kAttnWaves + wave_id(); item < p.n_q * p.heads; item += (int64_t)gridDim.x * kAttnWaves) {
        const int head = (int)(item % p.heads);
        const int64_t at_row = item / p.heads;
        // users without query rows begin where their successor does; the last one at or before a row is the row's
        const int b = last_user(p.q_offsets, (int)p.batch, 0, 0, at_row);
        const int64_t qa = p.q_offsets[b], qb = p.q_offsets[b + 1], ka = p.kv_offsets[b], kb = p.kv_offsets[b + 1];
        if (qa < 0 || qb > p.n_q || ka < 0 || kb < ka || kb > p.n_kv || at_row < qa || at_row >= qb || qb - qa > max_q ||
            kb - ka > 0x3fffffff)
            continue;
        const int nk = rows_in_use(p.kv_lengths ? p.kv_lengths[b] : kb - ka, (int)(kb - ka));
        const int chunk = 1 << shift;
        if (nk <= chunk) continue;                           // written by the workgroup that had them all
        const int row = (int)(at_row - qa);
        const int kv_heads = p.heads / p.group, kvh = head / p.group, chunks = (nk + chunk - 1) >> shift;
        const int64_t slot0 = (ka >> shift) + b;
        const int64_t first = (slot0 * kv_heads + kvh) * (max_q * p.group) + row * p.group + head % p.group;
        const int64_t apart = (int64_t)kv_heads * max_q * p.group;
        float top = neg_inf();
        for (int c = lane; c < chunks; c += 64) top = fmaxf(top, p.split_ml[2 * (first + c * apart)]);
#pragma unroll
        for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, kWave));
        const float base = top == neg_inf() ? 0.f : top;
        constexpr int kMine = DH < kWave ? 1 : DH / kWave, kAtOnce = 8;
        float o[kMine] = {}, sum = 0.f;
        for (int c0 = 0; c0 < chunks; c0 += kAtOnce) {          // eight chunks asked for before the first is used
            float part[kAtOnce], l[kAtOnce], a[kAtOnce][kMine];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int64_t at = first + min(c0 + i, chunks - 1) * apart;
                part[i] = p.split_ml[2 * at];
                l[i] = p.split_ml[2 * at + 1];
#pragma unroll
                for (int x = 0; x < kMine; ++x) a[i][x] = p.split_acc[at * DH + min(lane + 64 * x, DH - 1)];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (c0 + i < chunks) {
                    const float weight = __builtin_amdgcn_exp2f(part[i] - base);
                    sum += weight * l[i];
#pragma unroll
                    for (int x = 0; x < kMine; ++x) o[x] += weight * a[i][x];
                }
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (p.lse && lane == 0) p.lse[(int64_t)head * p.n_q + at_row] = sum == 0.f ? neg_inf() : (top + __log2f(sum)) * kLn2;
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int col = lane + 64 * x;
            if (col >= p.width) continue;
            const int64_t at = (at_row * p.heads + head) * p.width + col;
            const float v = o[x] * inv;
            if constexpr (sizeof(T) == 4) static_cast<T *>(p.out)[at] = v;
            else static_cast<T *>(p.out)[at].bits = (uint16_t)f32_to_bf16_bits(v);
            if (p.out_f32) p.out_f32[at] = v;
        }
    }
}

// ---- host side --------------------------------------------------------------------------------------------------------------
#define FS_NEED(cond, msg)                                   \
    do {                                                     \
        if (!(cond)) return set_err(ctx, FS_EINVAL, msg);    \
    } while (0)

constexpr int64_t kMaxGroups = 1 << 24;       // a launch has fewer than 2^32 threads

// Whether the rows are few enough for the split form: max_q of them, times the heads that share a key head, fit the sixteen
// columns of a product.
bool splits(const fs_attention_args &a) { return a.max_q > 0 && a.max_q * (int64_t)(a.heads / a.kv_heads) <= kSplitCols; }
// Keys of a workgroup of the split form, as a power of two: two turns of it while that makes up to sixteen workgroups a CU, more
// in larger caches.  us with both launches, for 128 / 256 keys at least: 28.8 / 27.1 (256 users with 93 k keys, 8 heads of 64
// columns over 2), 41.9 / 34.4 (64 with 98 k, 128 columns), 15.2 / 15.8 (32 with up to 8192 keys, 64 columns).  For up to 8 / 16 /
// 32 workgroups a CU: 201 / 184 / 186 (256 users with 1.6 M keys, 64 columns).
int split_shift(const fs_attention_args &a) {
    int shift = 8;
    while (shift < 16 && (a.n_kv >> shift) * a.kv_heads > 16 * 256) ++shift;
    return shift;
}
int padded(int width) { return width <= 32 ? 32 : width <= 64 ? 64 : 128; }

int attn_check(fs_ctx *ctx, const fs_attention_args &a) {
    FS_NEED(a.dt == FS_F32 || a.dt == FS_BF16, "jagged attention: unknown dtype");
    FS_NEED(a.n_q >= 0 && a.n_kv >= 0 && a.batch >= 0 && a.max_q >= 0, "jagged attention: negative size");
    FS_NEED(a.batch > 0 || (a.n_q == 0 && a.n_kv == 0), "jagged attention: rows without users");
    FS_NEED(a.heads > 0 && a.kv_heads > 0 && a.heads % a.kv_heads == 0 && a.heads <= 1024,
            "jagged attention: heads must be a multiple of kv_heads, at most 1024");
    const int unit = 16 / elem_size(a.dt);
    FS_NEED(a.head_dim > 0 && a.head_dim <= FS_MAX_HEAD_DIM && a.head_dim % unit == 0,
            "jagged attention: head_dim must be a multiple of 4 (fp32) / 8 (bf16), at most FS_MAX_HEAD_DIM");
    FS_NEED(a.scale > 1e-30f && a.scale < 1e30f, "jagged attention: scale must be a positive number");
    FS_NEED(a.causal == 0 || a.causal == 1, "jagged attention: causal must be 0 or 1");
    if (a.bias) {
        FS_NEED(a.bucket_of, "jagged attention: a bias without bucket_of");
        FS_NEED(a.num_buckets > 0 && a.num_buckets <= FS_MAX_BIAS_BUCKETS && a.num_distances > 0 &&
                    a.num_distances <= FS_MAX_BIAS_DISTANCES,
                "jagged attention: num_buckets or num_distances out of range");
    }
    const int64_t rows = a.n_q > a.n_kv ? a.n_q : a.n_kv;
    FS_NEED(rows < (1ll << 40) && a.batch < (1ll << 31) && attn_slots(rows, a.batch, 6) * a.heads < kMaxGroups,
            "jagged attention: (rows / 64 + batch) * heads must stay below 2^24");
    if (a.batch == 0) return FS_OK;
    FS_NEED(a.q_offsets && a.kv_offsets, "jagged attention: null pointer");
    const int64_t wide = (int64_t)a.heads * a.head_dim, narrow = (int64_t)a.kv_heads * a.head_dim;
    FS_NEED(a.q_stride <= FS_MAX_ROW_STRIDE && a.k_stride <= FS_MAX_ROW_STRIDE && a.v_stride <= FS_MAX_ROW_STRIDE,
            "jagged attention: a stride beyond FS_MAX_ROW_STRIDE");
    FS_NEED(a.q_stride >= wide && a.k_stride >= narrow && a.v_stride >= narrow && a.q_stride % unit == 0 && a.k_stride % unit == 0 &&
                a.v_stride % unit == 0,
            "jagged attention: a stride is less than its row or not a multiple of 16 bytes");
    if (a.n_q > 0) FS_NEED(a.q && a.out, "jagged attention: null pointer");
    if (a.n_kv > 0) FS_NEED(a.k && a.v, "jagged attention: null pointer");
    FS_NEED(aligned16(a.q) && aligned16(a.k) && aligned16(a.v) && aligned16(a.out) && (a.dt == FS_F32 || aligned16(a.out_f32)),
            "jagged attention: pointer not 16-byte aligned");
    return FS_OK;
}

attn_params params_of(fs_ctx *ctx, const fs_attention_args &a) {
    attn_params p;
    memset(&p, 0, sizeof(p));
    p.q = a.q;
    p.k = a.k;
    p.v = a.v;
    p.q_stride = a.q_stride;
    p.k_stride = a.k_stride;
    p.v_stride = a.v_stride;
    p.n_q = a.n_q;
    p.n_kv = a.n_kv;
    p.batch = a.batch;
    p.q_offsets = a.q_offsets;
    p.kv_offsets = a.kv_offsets;
    p.kv_lengths = a.kv_lengths;
    p.heads = a.heads;
    p.group = a.heads / a.kv_heads;
    p.width = a.head_dim;
    p.causal = a.causal;
    p.scale = a.scale;
    p.bias = a.bias;
    p.bucket_of = a.bucket_of;
    p.buckets = a.bias ? a.num_buckets : 0;
    p.distances = a.bias ? a.num_distances : 1;
    p.out = a.out;
    p.out_f32 = a.dt == FS_F32 ? nullptr : a.out_f32;
    p.lse = a.lse;
    p.dout = a.dout;
    p.dq = a.dq;
    p.dk = a.dk;
    p.dv = a.dv;
    p.dq_stride = a.dq_stride;
    p.dk_stride = a.dk_stride;
    p.dv_stride = a.dv_stride;
    p.dbias = a.bias ? a.dbias : nullptr;
    p.split_shift = split_shift(a);
    p.max_q = a.max_q;
    p.flags = ctx ? ctx->d_flags : nullptr;
    return p;
}

int64_t split_rows(const fs_attention_args &a) {       // rows of partial results: every slot's columns for every key head
    return attn_slots(a.n_kv, a.batch, split_shift(a)) * a.kv_heads * a.max_q * (a.heads / a.kv_heads);
}

}  // namespace

extern "C" {

size_t fs_jagged_attention_work_bytes(const fs_attention_args *args) {
    if (!args || attn_check(nullptr, *args) != FS_OK || !splits(*args)) return 0;
    return (size_t)split_rows(*args) * (padded(args->head_dim) + 2) * sizeof(float);
}

int fs_jagged_attention(fs_ctx *ctx, const fs_attention_args *args, fs_stream stream) {
    if (!ctx) return FS_EINVAL;
    FS_NEED(args, "jagged attention: null pointer");
    const fs_attention_args &a = *args;
    const int rc = attn_check(ctx, a);
    if (rc != FS_OK) return rc;
    const bool split = splits(a);
    if (split)
        FS_NEED(a.n_q == 0 || (a.work && aligned16(a.work) && a.work_bytes >= fs_jagged_attention_work_bytes(args)),
                "jagged attention: work is null, not 16-byte aligned or too small");
    if (a.n_q == 0) return FS_OK;
    device_scope on(ctx->device);
    if (!on.ok) return set_err(ctx, FS_EHIP, "jagged attention: the context's GPU cannot be made current");
    attn_params p = params_of(ctx, a);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return by_head(a.dt, a.head_dim, [&](auto *t, auto dh) -> int {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr int DH = dh();
        if (split) {
            p.split_acc = static_cast<float *>(a.work);
            p.split_ml = p.split_acc + split_rows(a) * DH;
            const size_t lds = split_rows_lds<T, DH> + (size_t)(kSplitStep + a.max_q) * p.group * sizeof(float);
            const int done = launch_attention(ctx, attn_split_kernel<T, DH>, attn_slots(a.n_kv, a.batch, p.split_shift) * a.kv_heads,
                                              lds, s, "attn_split", p);
            if (done != FS_OK || a.n_kv <= 1ll << p.split_shift) return done;     // nobody has several chunks
            const int64_t groups = ceil_div(a.n_q * a.heads, kAttnWaves);         // rows are not bounded by attn_check
            return launch_attention(ctx, attn_join_kernel<T, DH>, groups < kMaxGroups ? groups : kMaxGroups - 1, 0, s, "attn_join", p);
        }
        const auto run = [&](auto exact) {
            const size_t lds = 2 * sizeof(tile<T, DH>) + kAttnWaves * sizeof(uint32_t) +
                               strip<row_pad(QT)>::entries(p.distances, a.causal != 0) * sizeof(float);
            return launch_attention(ctx, attn_forward_kernel<T, DH, exact()>,
                                    attn_slots(a.n_q, a.batch, 6) * a.heads, lds, s, "attn_forward", p);
        };
        if constexpr (sizeof(T) == 2) {
            if (p.out_f32) return run(std::true_type());
        }
        return run(std::false_type());
    });
}

size_t fs_jagged_attention_backward_work_bytes(const fs_attention_args *args) {
    if (!args || attn_check(nullptr, *args) != FS_OK) return 0;
    return attention_backward_work(params_of(nullptr, *args), args->dt);
}

int fs_jagged_attention_backward(fs_ctx *ctx, const fs_attention_args *args, fs_stream stream) {
    if (!ctx) return FS_EINVAL;
    FS_NEED(args, "jagged attention backward: null pointer");
    const fs_attention_args &a = *args;
    const int rc = attn_check(ctx, a);
    if (rc != FS_OK) return rc;
    const int unit = 16 / elem_size(a.dt);
    const int64_t wide = (int64_t)a.heads * a.head_dim, narrow = (int64_t)a.kv_heads * a.head_dim;
    if (a.n_q > 0) FS_NEED(a.dout && a.dq && a.lse, "jagged attention backward: null pointer");
    if (a.n_kv > 0) FS_NEED(a.dk && a.dv, "jagged attention backward: null pointer");
    if (a.batch > 0)
        FS_NEED(a.dq_stride >= wide && a.dk_stride >= narrow && a.dv_stride >= narrow && a.dq_stride % unit == 0 &&
                    a.dk_stride % unit == 0 && a.dv_stride % unit == 0,
                "jagged attention backward: a stride is less than its row or not a multiple of 16 bytes");
    FS_NEED(aligned16(a.dout) && aligned16(a.dq) && aligned16(a.dk) && aligned16(a.dv),
            "jagged attention backward: pointer not 16-byte aligned");
    attn_params p = params_of(ctx, a);
    const size_t need = attention_backward_work(p, a.dt);
    FS_NEED(need == 0 || (a.work && aligned16(a.work) && a.work_bytes >= need),
            "jagged attention backward: work is null, not 16-byte aligned or too small");
    device_scope on(ctx->device);
    if (!on.ok) return set_err(ctx, FS_EHIP, "jagged attention backward: the context's GPU cannot be made current");
    return launch_attention_backward(ctx, p, a.dt, a.work, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
