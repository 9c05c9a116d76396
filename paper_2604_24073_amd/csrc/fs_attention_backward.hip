// Attention over a jagged batch with a learned relative position bias, backward.
//
// With P the softmax as the forward pass left it (its row sums are in lse) and D_i = dO_i . o_i:
//   dS = P (dO V^T - D),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T dO,  dbias[b, head] = sum of dS over the pairs in b
// Two launches recompute the scores, one that owns query rows (dq, D and the bias) and one that owns keys (dk, dv): seven
// products instead of the five of a single launch, and in exchange no sum crosses a workgroup but the bias's, so that nothing
// is added up in an order that changes.  Both keep the scores in registers from product to product, as the forward pass does.
//
// P and dS are rounded to the rows' type where they go into a product: half a step of bf16 of each, beside the same of dq, dk and
// dv themselves (2.4e-3 off in all against 1.7e-3).
//
// 160 histories with 150 k rows, 8 of them of 16384, 4 heads of 64 columns over 2 key heads: query rows 2.5 to 2.6 ms (660
// TFLOP/s of their three products), keys 3.4 to 3.6 (630 of their four).  1024 histories with 262 k rows, 4 heads of 32: 0.67 to
// 0.72 and 0.58 to 0.61 ms, a third of the former the bias's sums, which tell the buckets of a tile apart.  Of the time the
// vector units are busy 56 % (query rows, 64 columns; 8.9 instructions a score) and 71 % (32 columns; 18.5), and no unit of the keys'
// kernel is busy for long: vector 40 % (7.7 instructions a score), matrix 30 %, LDS 41 % with 64 columns, 60, 17 and 61 % with 32;
// its wavefronts wait 45 % of their time, and every turn fetches spilled scalars back.  Tiles that are partly seen, all there are
// in short histories, cost several times the others: their masks are branches for each score.  A second pair of tiles in LDS, to
// save a barrier a tile, was slower: fewer workgroups fit (0.81 and 0.60).
#include "fs_attention.h"

using namespace fs;

namespace {

// ---- the bias's gradient ------------------------------------------------------------------------------------------------------
// A wavefront's sums by bucket, in LDS that only it writes.
struct bucket_sums {
    float *bins;            // [buckets]
    float run = 0.f;        // a lane's share of the bucket below, not yet in its bin
    int now = -1;

    // a neighbour's value, without a trip through LDS: CTRL is one of the vector units' lane patterns
    template <int CTRL, int ROWS = 0xf>
    static __device__ __forceinline__ float from(float x) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, ROWS, 0xf, false));
    }
    static __device__ __forceinline__ float wave_sum(float x) {          // in every lane
        x += from<0x128>(x);                                             // row_ror: 8, 4, 2, 1
        x += from<0x124>(x);
        x += from<0x122>(x);
        x += from<0x121>(x);
        return column_sum(x);
    }
    // A single lane's addition to a bin of its wavefront's own: nothing else is added to it at the same time, and LDS keeps a
    // wavefront's order, so this is an addition that nobody waits for, not one whose order is open.
    __device__ __forceinline__ void put(int bucket, float x) {
        __hip_atomic_fetch_add(bins + bucket, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    __device__ __forceinline__ void add(int bucket, float total) {       // of the whole wavefront
        if (bucket >= 0 && (threadIdx.x & 63) == 0) put(bucket, total);
    }
    __device__ __forceinline__ void flush() {
        add(now, wave_sum(run));
        run = 0.f;
    }
    // every lane's share of one bucket
    __device__ __forceinline__ void one(int bucket, float share) {
        if (bucket != now) {
            flush();
            now = bucket;
        }
        run += share;
    }
    // Every lane's value of a bucket of its own, the lanes' distances ascending.  Runs of a bucket are added up by a scan that
    // starts anew where the bucket changes, and each run's last lane has its sum; buckets that come back after another one
    // (no table of distances needs them to) are taken one after the other.
    __device__ __forceinline__ void each(int bucket, float value) {
        const int lane = threadIdx.x & 63;
        const int before = __builtin_amdgcn_update_dpp(bucket, bucket, 0x138, 0xf, 0xf, false);        // wave_shr:1
        const uint64_t heads = __ballot(bucket != before) | 1;
        if (__ballot(bucket > before) && __ballot(bucket < before)) {
            uint64_t left = __ballot(bucket >= 0);
            while (left) {
                const int b = __builtin_amdgcn_readlane(bucket, __ffsll((unsigned long long)left) - 1);
                const bool mine = bucket == b;
                add(b, wave_sum(mine ? value : 0.f));
                left &= ~__ballot(mine);
            }
            return;
        }
        const int start = 63 - __clzll((long long)(heads & (~0ull >> (63 - lane)))), in_row = lane & 15;
        float x = value, y;
        y = from<0x111>(x);                                              // row_shr: 1, 2, 4, 8
        x += in_row >= 1 && lane - 1 >= start ? y : 0.f;
        y = from<0x112>(x);
        x += in_row >= 2 && lane - 2 >= start ? y : 0.f;
        y = from<0x114>(x);
        x += in_row >= 4 && lane - 4 >= start ? y : 0.f;
        y = from<0x118>(x);
        x += in_row >= 8 && lane - 8 >= start ? y : 0.f;
        y = from<0x142, 0xa>(x);                                         // a row's last lane to the next row: rows 1 and 3
        x += (lane & 16) && (lane & 32) + 15 >= start ? y : 0.f;
        y = from<0x143, 0xc>(x);                                         // a half's last lane to the other half
        x += (lane & 32) && 31 >= start ? y : 0.f;
        const bool last = lane == 63 || ((heads >> 1) >> lane & 1);
        if (last && bucket >= 0) put(bucket, x);                         // a bucket each
    }
};

// Sixteen query rows x 64 keys, summed along their diagonals: value (q, key) belongs to distance q - key + 63 of the 79.
// Each is written where its distance's row has column q, and a lane adds up a row.  A row's sixteen columns are four pieces of
// 16 bytes, at places that turn with the row, so that sixteen lanes read their rows' pieces from different banks.  The columns
// that a row has no value for are zeros from the start (clear_skew) and never written.
constexpr int kSpan = kTile + 15;
constexpr int kSkew = kSpan * 16;
__device__ __forceinline__ void clear_skew(float *skew) {
    for (int i = threadIdx.x & 63; i < kSkew; i += kWave) skew[i] = 0.f;
}
__device__ __forceinline__ float row_total(const float *skew, int row) {
    const float *at = skew + 16 * row;
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(at + 4 * (c ^ ((row >> 2) & 3)));
        sum += (x[0] + x[1]) + (x[2] + x[3]);
    }
    return sum;
}
// near: the sum of distance `lane`; far: of distance 64 + lane, where there is one.  live: the lane's row exists
__device__ __forceinline__ void diagonal_sums(float *skew, const f32x4 (&s)[4], bool live, float &near, float &far) {
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int d = j + 63 - 4 * g - r;                  // of key 4 g + r; sixteen keys further on the places turn alike
        float *at = skew + 16 * d + 4 * ((j >> 2) ^ ((d >> 2) & 3)) + (j & 3);
#pragma unroll
        for (int k = 0; k < 4; ++k) at[-256 * k] = live ? s[k][r] : 0.f;
    }
    wave_lds_order();
    near = row_total(skew, lane);
    far = lane < 15 ? row_total(skew, 64 + lane) : 0.f;
    wave_lds_order();
}

// a lane's values, those of the first `rows` rows
template <int QT>
__device__ __forceinline__ float lane_sum(const f32x4 (&s)[QT][4], int rows) {
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        float row = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) row += (s[t][k][0] + s[t][k][1]) + (s[t][k][2] + s[t][k][3]);
        sum += 16 * t + (int)(threadIdx.x & 15) < rows ? row : 0.f;
    }
    return sum;
}

// The 16 QT x 64 values s of a wavefront added to the sums of their buckets; b0: the bucket of the lane's of the first 64
// distances, b1: of those behind them, the last one's in the lanes that have none.  Tables of distances have few buckets in so
// many distances but near zero: one bucket takes every lane's sum as it is, two are told apart by comparing distances, and only
// more are brought into the order of the distances.  Further distances come first: the tiles go from far to near, and a
// bucket's lanes are added up when the next bucket begins.  The first `rows` rows exist (any number); the others have whatever the
// keys made of them, a NaN if one of those is none, and are left out where a lane, which has one row, has its sum.
template <int QT>
__device__ __forceinline__ void add_by_bucket(bucket_sums &sums, float *skew, const f32x4 (&s)[QT][4], int rows, int b0, int b1) {
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
    const int last0 = __builtin_amdgcn_readlane(b0, 63), before0 = __builtin_amdgcn_update_dpp(b0, b0, 0x138, 0xf, 0xf, false);
    int before1 = __builtin_amdgcn_update_dpp(b1, b1, 0x138, 0xf, 0xf, false);
    before1 = lane == 0 ? last0 : before1;
    const uint64_t h0 = __ballot(b0 != before0), h1 = __ballot(b1 != before1);    // where a bucket begins
    const int changes = __popcll(h0) + __popcll(h1);
    if (changes == 0) {
        sums.one(__builtin_amdgcn_readfirstlane(b0), lane_sum<QT>(s, rows));
    } else if (changes == 1) {
        // the distances from `at` on have another bucket than those before
        const int at = h0 ? 63 - __clzll((long long)h0) : 127 - __clzll((long long)h1);
        const int mine = j + 63 - 4 * g;                   // element r of s[t][k] has distance mine + 16 t - 16 k - r
        float near = 0.f, far = 0.f;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float near_t = 0.f, far_t = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool beyond = mine >= at + 16 * k + r - 16 * t;
                    far_t += beyond ? s[t][k][r] : 0.f;
                    near_t += beyond ? 0.f : s[t][k][r];
                }
            far += 16 * t + j < rows ? far_t : 0.f;
            near += 16 * t + j < rows ? near_t : 0.f;
        }
        sums.one(__builtin_amdgcn_readlane(b1, 63), far);    // the last distance's
        sums.one(__builtin_amdgcn_readfirstlane(b0), near);
    } else {
        float near, far;
        diagonal_sums(skew, s[0], j < rows, near, far);
        if constexpr (QT == 2) {
            // the second sixteen rows' distances are sixteen further on
            float near2, far2;
            diagonal_sums(skew, s[1], 16 + j < rows, near2, far2);
            const float y = __shfl(near2, (lane + 48) & 63, kWave), z = __shfl(far2, (lane + 48) & 63, kWave);
            near += lane >= 16 ? y : 0.f;
            far += lane < 16 ? y : z;                      // z: zeros from distance 95 on
        }
        sums.each(b0, near);
        sums.each(b1, far);
    }
}

// ---- query rows ---------------------------------------------------------------------------------------------------------------
// QT: sixteens of query rows of a wavefront
template <typename T, int DH, int QT>
__global__ __launch_bounds__(kAttnThreads, (attn_waves<T, DH>)) void attn_dq_kernel(attn_params p) {
    constexpr int kRows = 16 * kAttnWaves * QT, kShift = QT == 1 ? 6 : 7, kPad = row_pad(QT);
    constexpr int KC = DH / 32, MT = DH / 16;
    extern __shared__ __align__(16) char lds[];
    tile<T, DH> &K = *reinterpret_cast<tile<T, DH> *>(lds), &V = (&K)[1];
    float *mark = reinterpret_cast<float *>(&V + 1);                              // [kTile]
    float *skew = mark + kTile;                                                   // [wavefronts][kSkew]
    float *bias_lds = skew + kAttnWaves * kSkew;
    const int entries = strip<kPad>::entries(p.distances, p.causal != 0);
    float *bins = bias_lds + entries;                                             // [wavefronts][buckets]

    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15, w = wave_id();
    const int head = blockIdx.x % p.heads;
    const int slot = (int)(blockIdx.x / p.heads);
    if (head == 0) check_layout(p, slot, (int)(gridDim.x / p.heads));
    user u;
    int index;
    float *part = p.dbias ? p.bias_part + ((int64_t)slot * p.heads + head) * p.buckets : nullptr;
    if (!find_user(p, p.q_offsets, slot, kShift, u, index) || (int64_t)index * kRows >= u.nq) {
        if (part)
            for (int b = threadIdx.x; b < p.buckets; b += kAttnThreads) part[b] = 0.f;
        return;
    }
    index = (u.nq - 1) / kRows - index;                                           // the last rows, which see most, begin first
    const int row0 = index * kRows;
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

    const int wrow = row0 + 16 * QT * w, wpos = u.first + wrow;
    piece<T> qf[QT][KC], of[QT][KC];
    // What a row's scores are less by, as from_less has it, and its D.  D is taken from a finished dO V^T: a sum that began at -D
    // would be cut off at D's size, always downwards, and the bias's gradient adds up millions of them (16384 rows: 7e-6 of it
    // off in place of 1e-6).
    float less_s[QT], delta[QT];
    const int64_t orow = p.heads * (int64_t)p.width;                              // out and dout are packed
    const int64_t obase = u.q0 * orow + head * p.width;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int row = wrow + 16 * t + j;
        const bool live = row < u.nq;
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            global_rows(qf[t][c], static_cast<const T *>(p.q) + u.q0 * p.q_stride + head * p.width, p.q_stride, row, live, 32 * c,
                        p.width);
            global_rows(of[t][c], static_cast<const T *>(p.dout) + obase, orow, row, live, 32 * c, p.width);
            const int col = 32 * c + 8 * g, left = live ? p.width - col : 0;
            const int64_t at = obase + row * orow + col;
            float o[8], d[8];
            if (p.out_f32) load8(p.out_f32 + at, left, o);
            else load8(static_cast<const T *>(p.out) + at, left, o);
            load8(static_cast<const T *>(p.dout) + at, left, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += o[i] * d[i];
        }
        sum = column_sum(sum);
        delta[t] = sum;
        less_s[t] = neg_inf();                                                    // a row that sees nothing: P = 0
        if (live) {
            const int64_t at = (int64_t)head * p.n_q + u.q0 + row;
            const float x = p.lse[at];
            if (x != neg_inf()) less_s[t] = from_less<T> ? -x / p.scale : -x * kLog2e;
            if (g == 0) p.delta[at] = sum;
        }
    }
    strip<kPad> bias;
    bucket_sums sums;
    sums.bins = bins + w * p.buckets;
    if (part) {
        for (int b = lane; b < p.buckets; b += kWave) sums.bins[b] = 0.f;
        clear_skew(skew + w * kSkew);
    }
    const bool hides = bias.fill(p, head, bias_lds, pos0 - (end > 0 ? end - 1 : 0), pos_last);
    const float scale2 = p.scale * kLog2e;

    f32x4 acc[QT][MT] = {};
    // some rows do not see all keys of the tile, or some of those are none
    const auto edge = [&](int n) { return hides || (n + 1) * kTile > u.nk || (p.causal && (n + 1) * kTile - 1 > pos0); };
    const auto stage = [&](int n) {
        // what a row does not see must not reach it, not even as 0 * NaN: the keys' infinities and NaN are taken out of the
        // product and put into the scores, where they are masked like any other
        if (edge(n)) kr.clean(mark);
        kr.store(K);
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
            const int nearest = wpos - (key0 + kTile - 1), furthest = wpos + 16 * QT - 1 - key0;
            const bool all_far = nearest >= bias.high || furthest <= bias.low;
            const float far = bias.at[bias.zero + (nearest >= bias.high ? bias.high : bias.low)];
            // of a tile beyond the table, the distances nearest to it have the same bias
            const int near = min(max(nearest, bias.low - (62 + 16 * QT)), bias.high);
            const float *bb = bias.at + bias.zero + near + (j - 4 * g) + 12;
            // the table's entries for the distances, on their way while the scores are made (and not looked at before)
            int buckets[2];
            if (part) {
                buckets[0] = bias.entry(p, near + lane);
                buckets[1] = bias.entry(p, near + min(64 + lane, 62 + 16 * QT));
            }
            // element r of s[t][k]: query row wrow + 16 t + j, key key0 + 16 k + 4 g + r
            f32x4 s[QT][4];
            // A tile has one form from its first product to its last, so that products run beside powers: mask - some pairs are
            // not seen (whatever their product is, their score is -inf), or are none; away - all distances are beyond the table.
            const auto work = [&](auto mask, auto away) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    f32x4 dp[QT] = {};
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        const float at = from_less<T> ? less_s[t] : 0.f;
                        s[t][k] = f32x4{at, at, at, at};
                    }
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        piece<T> a;
                        K.rows(a, 16 * k, 32 * c);
#pragma unroll
                        for (int t = 0; t < QT; ++t) mma(s[t][k], a, qf[t][c]);
                        V.rows(a, 16 * k, 32 * c);
#pragma unroll
                        for (int t = 0; t < QT; ++t) mma(dp[t], a, of[t][c]);
                    }
                    f32x4 x;
                    if constexpr (mask()) settle();                                // what follows may be branches
                    if constexpr (mask()) x = *reinterpret_cast<const f32x4 *>(mark + 16 * k + 4 * g);
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        const int seen = p.causal ? min(wpos + 16 * t + j + 1, u.nk) : u.nk;     // keys that the row sees
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float b = away() ? far : bb[51 + 16 * t - 16 * k - r];
                            float power = s[t][k][r] * scale2 + (from_less<T> ? b : b + less_s[t]), d = dp[t][r] - delta[t];
                            if constexpr (mask()) power = key0 + 16 * k + 4 * g + r < seen && b != neg_inf() ? power + x[r] : neg_inf();
                            const float e = __builtin_amdgcn_exp2f(power);
                            if constexpr (mask()) d = e == 0.f ? 0.f : d;
                            s[t][k][r] = e * d;
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    piece<T> sf[QT];
#pragma unroll
                    for (int t = 0; t < QT; ++t) as_operand(sf[t], s[t][2 * c], s[t][2 * c + 1]);
#pragma unroll
                    for (int d = 0; d < MT; ++d) {
                        piece<T> a;
                        K.cols(a, 32 * c, 16 * d);
#pragma unroll
                        for (int t = 0; t < QT; ++t) mma(acc[t][d], a, sf[t]);
                    }
                }
                settle();
            };
            if (edge(n)) work(std::true_type(), std::false_type());
            else if (all_far) work(std::false_type(), std::true_type());
            else work(std::false_type(), std::false_type());
            if (part) {
                if (all_far) {
                    sums.one(__builtin_amdgcn_readfirstlane(bias.bucket(p, buckets[0])), lane_sum<QT>(s, u.nq - wrow));
                } else {
                    add_by_bucket<QT>(sums, skew + w * kSkew, s, u.nq - wrow, bias.bucket(p, buckets[0]), bias.bucket(p, buckets[1]));
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
        const int row = wrow + 16 * t + j;
        if (row >= u.nq) continue;
#pragma unroll
        for (int c = 0; c < MT; ++c) {
            const int col = 16 * c + 4 * g;
            f32x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = acc[t][c][r] * p.scale;
            if (col < p.width) store4(static_cast<T *>(p.dq) + (u.q0 + row) * p.dq_stride + head * p.width + col, o);
        }
    }
    if (part) {
        sums.flush();
        __syncthreads();
        for (int b = threadIdx.x; b < p.buckets; b += kAttnThreads) {
            float x = 0.f;
#pragma unroll
            for (int v = 0; v < kAttnWaves; ++v) x += bins[v * p.buckets + b];
            part[b] = x;
        }
    }
}

// ---- keys ------------------------------------------------------------------------------------------------------------------------
// KT: sixteens of keys of a wavefront; with one, narrow rows have room for three wavefronts a SIMD if that is asked for (1000
// histories of up to 400 rows of 64 columns: 435 us to 357)
template <typename T, int DH, int KT>
__global__ __launch_bounds__(kAttnThreads, (KT == 1 && sizeof(T) * DH <= 128 ? 3 : attn_waves<T, DH>))
void attn_dkv_kernel(attn_params p) {
    constexpr int kKeys = 16 * kAttnWaves * KT, kShift = KT == 1 ? 6 : 7, kPad = kKeys + kTile;
    constexpr int KC = DH / 32, MT = DH / 16;
    extern __shared__ __align__(16) char lds[];
    tile<T, DH> &Q = *reinterpret_cast<tile<T, DH> *>(lds), &O = (&Q)[1];
    float *stats = reinterpret_cast<float *>(&O + 1);                             // [what scores are less by, -D][kTile]
    float *mark = stats + 2 * kTile;                                              // [q, dout][kTile]
    uint32_t *odd = reinterpret_cast<uint32_t *>(mark + 2 * kTile);               // [wavefronts]
    float *bias_lds = reinterpret_cast<float *>(odd + kAttnWaves);

    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15, w = wave_id();
    const int kv_heads = p.heads / p.group, kvh = blockIdx.x % kv_heads;
    user u;
    int index;
    if (!find_user(p, p.kv_offsets, (int)(blockIdx.x / kv_heads), kShift, u, index) || (int64_t)index * kKeys >= u.room) return;
    const int key_first = index * kKeys;
    const int wkey = key_first + 16 * KT * w;
    // query rows at or behind the first key; every tile of 64 of them, for every head that shares the keys
    const int from = p.causal && key_first > u.first ? (key_first - u.first) / kTile * kTile : 0;
    const int tiles = key_first >= u.nk || from >= u.nq ? 0 : (u.nq - from + kTile - 1) / kTile;
    const int turns = tiles * p.group;

    piece<T> kf[KT][KC], vf[KT][KC];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        const int key = wkey + 16 * t + j;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            global_rows(kf[t][c], static_cast<const T *>(p.k) + u.k0 * p.k_stride + kvh * p.width, p.k_stride, key, key < u.nk, 32 * c,
                        p.width);
            global_rows(vf[t][c], static_cast<const T *>(p.v) + u.k0 * p.v_stride + kvh * p.width, p.v_stride, key, key < u.nk, 32 * c,
                        p.width);
        }
    }
    f32x4 dk[KT][MT] = {}, dv[KT][MT] = {};
    const int64_t orow = p.heads * (int64_t)p.width;
    const float scale2 = p.scale * kLog2e, inv_scale = 1.f / p.scale;
    tile_regs<T, DH> qr, dr;
    qr.place(p.q_stride, p.width);
    dr.place(orow, p.width);
    float stat = 0.f;
    // The tile that is fetched next: its first row among the user's, its head, and where its rows begin.
    int next_row = from, next_head = kvh * p.group;
    const T *next_q, *next_o;
    const float *next_stat;                   // of wavefront 0: lse, of wavefront 1: D
    const auto begin_head = [&]() {
        next_row = from;
        next_q = static_cast<const T *>(p.q) + (u.q0 + from) * p.q_stride + next_head * p.width;
        next_o = static_cast<const T *>(p.dout) + (u.q0 + from) * orow + next_head * p.width;
        next_stat = (w == 0 ? p.lse : p.delta) + (int64_t)next_head * p.n_q + u.q0 + from;
    };
    const auto fetch = [&]() {
        const int rows = min(u.nq - next_row, kTile);
        qr.load(next_q, p.q_stride, rows);
        dr.load(next_o, orow, rows);
        // a row's lse or D, as it is: whatever is made of it here would wait for it here
        if (w < 2) stat = window(next_stat, 4 * rows).load1(4 * lane);
    };
    const auto advance = [&]() {
        next_row += kTile;
        next_q += kTile * p.q_stride;
        next_o += kTile * orow;
        next_stat += kTile;
        if (next_row >= u.nq) {
            ++next_head;
            begin_head();
        }
    };
    strip<kPad> bias;
    bool hides = false;
    // some of the tile's rows do not see all keys of the workgroup, or some of either are none
    const auto edge = [&](int r0) {
        return key_first + kKeys > u.nk || r0 + kTile > u.nq || (p.causal && u.first + r0 < key_first + kKeys - 1);
    };
    const auto stage = [&](int r0, bool clean) {
        if (clean) {
            qr.clean(mark);
            const bool any = __any(dr.clean(mark + kTile));
            if (lane == 0) odd[w] = any;
        }
        qr.store(Q);
        dr.store(O);
        if (w < 2) {
            const bool lse = w == 0, row = r0 + lane < u.nq;
            const float less = lse ? (stat == neg_inf() ? neg_inf() : -stat * (from_less<T> ? inv_scale : kLog2e)) : -stat;
            // rows that see nothing and rows that are none
            stats[threadIdx.x] = row ? less : lse ? neg_inf() : 0.f;
        }
    };
    const auto fill = [&](int head) {
        return bias.fill(p, head, bias_lds, u.first + from - (key_first + kKeys - 1), u.first + u.nq - 1 - key_first);
    };
    bool masked = false;                      // the tile at hand was cleaned, and is worked on with its marks and masks
    if (turns > 0) {
        begin_head();
        fetch();
        hides = fill(next_head);
        stage(from, masked = edge(from) || hides);
    }
    for (int n = 0; n < turns; ++n) {
        __syncthreads();
        const int r0 = next_row, pos0 = u.first + r0, head = next_head;
        if (r0 == from && n > 0) hides = fill(head);
        advance();
        if (n + 1 < turns) fetch();
        // A tile has one form from its first product to its last, so that the products of one half run beside the powers of the
        // other: mask - some pairs are not seen, or are none; away - all distances are beyond the table.
        const auto work = [&](auto mask, auto away) {
            const int nearest = pos0 - (wkey + 16 * KT - 1);
            const float far = bias.at[bias.zero + (nearest >= bias.high ? bias.high : bias.low)];
#pragma unroll
            for (int c2 = 0; c2 < 2; ++c2) {                                      // 32 query rows at a time
                // element r of s[h][t]: query row r0 + 32 c2 + 16 h + 4 g + r, key wkey + 16 t + j
                f32x4 s[2][KT], dp[2][KT];
                // of a tile beyond the table, the distances nearest to it have the same bias
                const int near = min(max(nearest + 32 * c2, bias.low - (30 + 16 * KT)), bias.high);
                const float *bb = bias.at + bias.zero + near + (4 * g - j + 15);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // dO V^T less D goes only into a product of such factors: it begins where the scores do, at -D
                    const int at = 32 * c2 + 16 * h + 4 * g;
                    const f32x4 less_s = *reinterpret_cast<const f32x4 *>(stats + at);
                    const f32x4 less_dp = *reinterpret_cast<const f32x4 *>(stats + kTile + at);
#pragma unroll
                    for (int t = 0; t < KT; ++t) {
                        s[h][t] = from_less<T> ? less_s : f32x4{0.f, 0.f, 0.f, 0.f};
                        dp[h][t] = from_less<T> ? less_dp : f32x4{0.f, 0.f, 0.f, 0.f};
                    }
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        piece<T> a;
                        Q.rows(a, 32 * c2 + 16 * h, 32 * c);
#pragma unroll
                        for (int t = 0; t < KT; ++t) mma(s[h][t], a, kf[t][c]);
                        O.rows(a, 32 * c2 + 16 * h, 32 * c);
#pragma unroll
                        for (int t = 0; t < KT; ++t) mma(dp[h][t], a, vf[t][c]);
                    }
                    f32x4 mq, mo;
                    if constexpr (mask()) {
                        settle();                                                 // what follows may be branches
                        mq = *reinterpret_cast<const f32x4 *>(mark + at);
                        mo = *reinterpret_cast<const f32x4 *>(mark + kTile + at);
                    }
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float x = away() ? far : bb[16 * (KT - 1) + 16 * h + r - 16 * t];
                            float power = s[h][t][r] * scale2 + (from_less<T> ? x : x + less_s[r]), d = from_less<T> ? dp[h][t][r] : dp[h][t][r] + less_dp[r];
                            if constexpr (mask()) {
                                // a key that the row does not see, a hidden pair (whatever its product is), the keys behind
                                // the last, the rows behind the last
                                const int key = wkey + 16 * t + j, row = r0 + 32 * c2 + 16 * h + 4 * g + r;
                                int seen = p.causal ? min(u.first + row + 1, u.nk) : u.nk;
                                seen = row < u.nq ? seen : 0;
                                power = key < seen && x != neg_inf() ? power + mq[r] : neg_inf();
                                d += mo[r];
                            }
                            const float e = __builtin_amdgcn_exp2f(power);
                            if constexpr (mask()) d = e == 0.f ? 0.f : d;
                            s[h][t][r] = e;
                            dp[h][t][r] = e * d;
                        }
                }
                piece<T> pf[KT], sf[KT];
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    as_operand(pf[t], s[0][t], s[1][t]);
                    as_operand(sf[t], dp[0][t], dp[1][t]);
                }
#pragma unroll
                for (int d = 0; d < MT; ++d) {
                    piece<T> a;
                    O.cols(a, 32 * c2, 16 * d);
#pragma unroll
                    for (int t = 0; t < KT; ++t) mma(dv[t][d], a, pf[t]);
                    Q.cols(a, 32 * c2, 16 * d);
#pragma unroll
                    for (int t = 0; t < KT; ++t) mma(dk[t][d], a, sf[t]);
                }
                settle();
            }
        };
        if (wkey < u.nk && !(p.causal && pos0 + kTile - 1 < wkey)) {
            const int nearest = pos0 - (wkey + 16 * KT - 1), furthest = pos0 + kTile - 1 - wkey;
            if (masked) work(std::true_type(), std::false_type());
            else if (nearest >= bias.high || furthest <= bias.low) work(std::false_type(), std::true_type());
            else work(std::false_type(), std::false_type());
            if (masked) {
                uint32_t any = 0;
                for (int x = 0; x < kAttnWaves; ++x) any |= odd[x];
                if (any) {
                    // the elements of dout left out of the product, row by row, for the keys that are seen
                    const int count = u.nq - r0 < kTile ? u.nq - r0 : kTile;
                    for (int q = 0; q < count; ++q) {
                        const T *o = static_cast<const T *>(p.dout) + (u.q0 + r0 + q) * orow + head * p.width;
#pragma unroll
                        for (int t = 0; t < KT; ++t) {
                            const int key = wkey + 16 * t + j, d = pos0 + q - key;
                            const int dc = d > bias.high ? bias.high : d < bias.low ? bias.low : d;
                            const bool sees = key < u.nk && !(p.causal && d < 0) && bias.at[bias.zero + dc] != neg_inf();
#pragma unroll
                            for (int c = 0; c < MT; ++c)
#pragma unroll
                                for (int r = 0; r < 4; ++r) {
                                    const int col = 16 * c + 4 * g + r;
                                    const float x = col < p.width ? load1(o + col) : 0.f;
                                    if (sees && !(fabsf(x) < __builtin_inff())) dv[t][c][r] += x;
                                }
                        }
                    }
                }
            }
        }
        if (n + 1 < turns) {
            // a head's first tile is put down before its bias is known to hide nothing
            masked = edge(next_row) || hides || next_row == from;
            __syncthreads();
            stage(next_row, masked);
        }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        const int key = wkey + 16 * t + j;
        if (key >= u.room) continue;
#pragma unroll
        for (int c = 0; c < MT; ++c) {
            const int col = 16 * c + 4 * g;
            if (col >= p.width) continue;
            f32x4 o;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = dk[t][c][r] * p.scale;
            store4(static_cast<T *>(p.dk) + (u.k0 + key) * p.dk_stride + kvh * p.width + col, o);
            store4(static_cast<T *>(p.dv) + (u.k0 + key) * p.dv_stride + kvh * p.width + col, dv[t][c]);
        }
    }
}

// ---- the bias's gradient, added up over the workgroups ---------------------------------------------------------------------------
// [slots, columns] in two launches, 64 columns a workgroup: kBiasCuts cuts of the slots into sums of 64 bits, then those.
constexpr int kBiasCuts = 64;
__global__ __launch_bounds__(256) void attn_bias_cut_kernel(const float *__restrict__ part, int64_t slots, int columns,
                                                            double *__restrict__ cut) {
    __shared__ double sh[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
    const int64_t per = (slots + kBiasCuts - 1) / kBiasCuts, a = blockIdx.y * per, b = a + per < slots ? a + per : slots;
    double s = 0.0;
    if (c < columns)
        for (int64_t k = a + w; k < b; k += 4) s += (double)part[k * columns + c];
    sh[w][threadIdx.x & 63] = s;
    __syncthreads();
    if (w == 0 && c < columns) cut[(int64_t)blockIdx.y * columns + c] = (sh[0][c & 63] + sh[1][c & 63]) + (sh[2][c & 63] + sh[3][c & 63]);
}
// sixteen columns a workgroup, sixteen threads a column
__global__ __launch_bounds__(256) void attn_bias_sum_kernel(const double *__restrict__ cut, int heads, int buckets, int cuts,
                                                            float *__restrict__ dbias) {
    __shared__ double sh[16][17];
    const int c = threadIdx.x & 15, w = threadIdx.x >> 4, k = blockIdx.x * 16 + c, columns = heads * buckets;
    double s = 0.0;
    if (k < columns)
#pragma unroll
        for (int i = 0; i < kBiasCuts / 16; ++i) s += w + 16 * i < cuts ? cut[(int64_t)(w + 16 * i) * columns + k] : 0.0;
    sh[w][c] = s;
    __syncthreads();
    if (w != 0 || k >= columns) return;
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sh[i][c];
    dbias[(k % buckets) * heads + k / buckets] = (float)s;
}

// Whether a wavefront may have 32 query rows, or 32 keys: they halve what a score reads from LDS.  Narrower rows read less of it,
// fp32 and wider rows have no registers for twice as many.
template <typename T, int DH>
constexpr bool two_sixteens = sizeof(T) == 2 && DH == 64;

}  // namespace

namespace fs {

// Query rows of a workgroup of attn_dq_kernel and keys of one of attn_dkv_kernel, as powers of two: with 32 a wavefront there are
// fewer wavefronts, and more rows that are none in short histories.  us with 16 / 32, bf16 rows of 64 columns:
//   query rows: 334 / 410 (2000 histories of up to 200), 361 / 413 (1000 of up to 400), 1006 / 1008 (1024 of 256 on average),
//   316 / 311 (300 of 400 up), 1883 / 1724 (64 of 4000 up), 3422 / 2460 (8 of 16384);  keys, the same: 332 / 381, 357 / 385,
//   1019 / 981, -, -, 4002 / 3524.  Query rows of 32 columns: 718 / 882 (1024 of 256 on average), 1342 / 1488 (64 of 4000 up).
static bool may_have_two(const attn_params &p, int dt) { return dt == FS_BF16 && p.width > 32 && p.width <= 64; }
static int dq_shift(const attn_params &p, int dt) { return may_have_two(p, dt) && p.n_q >= 512 * p.batch ? 7 : 6; }
static int dkv_shift(const attn_params &p, int dt) { return may_have_two(p, dt) && p.n_kv >= 256 * p.batch ? 7 : 6; }

// scratch: delta, then the bias's sums of every workgroup, then those of the cuts
static size_t delta_bytes(const attn_params &p) { return ((size_t)p.heads * p.n_q * sizeof(float) + 255) / 256 * 256; }
static size_t part_bytes(const attn_params &p, int dt) {
    if (!p.dbias) return 0;
    return ((size_t)attn_slots(p.n_q, p.batch, dq_shift(p, dt)) * p.heads * p.buckets * sizeof(float) + 255) / 256 * 256;
}

size_t attention_backward_work(const attn_params &p, int dt) {
    return delta_bytes(p) + part_bytes(p, dt) + (p.dbias ? (size_t)kBiasCuts * p.heads * p.buckets * sizeof(double) : 0);
}

int launch_attention_backward(fs_ctx *ctx, const attn_params &args, int dt, void *work, hipStream_t s) {
    attn_params p = args;
    p.delta = static_cast<float *>(work);
    p.bias_part = reinterpret_cast<float *>(static_cast<char *>(work) + delta_bytes(p));
    double *cut = reinterpret_cast<double *>(static_cast<char *>(work) + delta_bytes(p) + part_bytes(p, dt));
    const int shift = dq_shift(p, dt);
    const int64_t slots = attn_slots(p.n_q, p.batch, shift);
    const bool causal = p.causal != 0;
    if (p.batch > 0) {
        const int rc = by_head(dt, p.width, [&](auto *t, auto dh) -> int {
            using T = std::remove_pointer_t<decltype(t)>;
            constexpr int DH = dh();
            const auto query_rows = [&](auto qt) {
                constexpr int QT = qt();
                const size_t bias = strip<row_pad(QT)>::entries(p.distances, causal);
                const size_t lds = 2 * sizeof(tile<T, DH>) + (kTile + kAttnWaves * kSkew + bias + kAttnWaves * p.buckets) * sizeof(float);
                return launch_attention(ctx, attn_dq_kernel<T, DH, QT>, slots * p.heads, lds, s, "attn_dq", p);
            };
            int done = FS_OK;
            if constexpr (two_sixteens<T, DH>)
                done = shift == 7 ? query_rows(std::integral_constant<int, 2>()) : query_rows(std::integral_constant<int, 1>());
            else
                done = query_rows(std::integral_constant<int, 1>());
            if (done != FS_OK) return done;
            const auto keys = [&](auto kt) {
                constexpr int KT = kt();
                const size_t lds = 2 * sizeof(tile<T, DH>) + (4 * kTile + kAttnWaves) * sizeof(float) +
                                   strip<16 * kAttnWaves * KT + kTile>::entries(p.distances, causal) * sizeof(float);
                return launch_attention(ctx, attn_dkv_kernel<T, DH, KT>,
                                        attn_slots(p.n_kv, p.batch, KT == 1 ? 6 : 7) * (p.heads / p.group), lds, s, "attn_dkv", p);
            };
            if constexpr (two_sixteens<T, DH>) {
                if (dkv_shift(p, dt) == 7) return keys(std::integral_constant<int, 2>());
            }
            return keys(std::integral_constant<int, 1>());
        });
        if (rc != FS_OK) return rc;
    }
    if (!p.dbias) return FS_OK;
    const int columns = p.heads * p.buckets;
    if (p.batch > 0) {
        attn_bias_cut_kernel<<<dim3((unsigned)ceil_div(columns, 64), kBiasCuts), 256, 0, s>>>(p.bias_part, slots, columns, cut);
        FS_LAUNCH_CHECK(ctx, "attn_bias_cut");
    }
    attn_bias_sum_kernel<<<(unsigned)ceil_div(columns, 16), 256, 0, s>>>(cut, p.heads, p.buckets, p.batch > 0 ? kBiasCuts : 0, p.dbias);
    FS_LAUNCH_CHECK(ctx, "attn_bias_sum");
    return FS_OK;
}

}  // namespace fs
