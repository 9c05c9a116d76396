// What the kernels of the jagged attention share: the shapes of their tiles, how a matrix product is fed, where a workgroup
// finds its rows, and the bias by distance.
//
// Products are made of 16 x 16 pieces over 32 terms.  With lane l = 16 g + j an operand piece holds, for its row (or column)
// j, eight of the 32 terms, and which eight belong to g is a free choice as long as both operands make the same one; a result
// piece holds column j, rows 4 g .. 4 g + 3.  Two result pieces of 16 rows each are therefore, as they lie in the registers, an
// operand piece over their 32 rows: g has rows 4 g + i of the first and of the second.  So the scores go from the product that
// makes them into the products that use them without a trip through LDS, in bf16 (one v_mfma_f32_16x16x32_bf16) as in fp32
// (eight v_mfma_f32_16x16x4_f32, the i-th over element i of every g).
#pragma once

#include <type_traits>

#include "fs_rowvec.h"

namespace fs {

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / kWave;
constexpr int kTile = 64;                 // keys (or query rows) of a tile in LDS
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// ---- operand pieces -------------------------------------------------------------------------------------------------------
template <typename T>
struct piece;
template <>
struct piece<bf16_t> {
    bf16x8 v;
};
template <>
struct piece<float> {
    float v[8];
};

__device__ __forceinline__ void mma(f32x4 &c, const piece<bf16_t> &a, const piece<bf16_t> &b) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x4 &c, const piece<float> &a, const piece<float> &b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
}

// Behind the last products of a block that ends in a branch: nothing reads a result before it is there.  A matrix instruction's
// result takes up to 10 wait states, and this compiler, which counts them out within a block, has left a copy of an accumulator
// 3 states behind its product where a branch stood between them (fp32 rows of 32 and 64 columns: the last row of a result came
// out one product short; 13 such reads in the backward pass's kernels without this, none in the forward pass's).  The tests follow
// every way through the compiler's output from each product to what reads it.
__device__ __forceinline__ void settle() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 11");
}

// two result pieces as the operand over their rows
__device__ __forceinline__ void as_operand(piece<bf16_t> &p, const f32x4 &lo, const f32x4 &hi) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 a = {lo[2 * i], lo[2 * i + 1]}, b = {hi[2 * i], hi[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2));
        w[2 + i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2));
    }
    p.v = __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ void as_operand(piece<float> &p, const f32x4 &lo, const f32x4 &hi) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p.v[i] = lo[i];
        p.v[4 + i] = hi[i];
    }
}

// The same, leaving in lo and hi what the rounding took off: of bf16 three such terms hold a value to its 24 bits.
__device__ __forceinline__ void take_operand(piece<bf16_t> &p, f32x4 &lo, f32x4 &hi) {
    as_operand(p, lo, hi);
    const u32x4 w = __builtin_bit_cast(u32x4, p.v);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        lo[2 * i] -= bf16_lo(w[i]);
        lo[2 * i + 1] -= bf16_hi(w[i]);
        hi[2 * i] -= bf16_lo(w[2 + i]);
        hi[2 * i + 1] -= bf16_hi(w[2 + i]);
    }
}

// ---- tiles in LDS -------------------------------------------------------------------------------------------------------------
// kTile rows of DH columns (the head's width rounded up to 32, 64 or 128; zeros behind it), rows 16 bytes further apart than
// they are long: sixteen lanes that read 16 bytes each of neighbouring rows find them in different banks.
template <typename T, int DH, int ROWS = kTile>
struct tile {
    static constexpr int kLd = DH + 16 / (int)sizeof(T);
    static constexpr int kPer = 16 / (int)sizeof(T);              // elements of a 16-byte chunk
    static constexpr int kChunks = DH / kPer;                     // chunks of a row
    static constexpr int kMine = ROWS * kChunks / kAttnThreads;   // chunks of a thread of a workgroup
    T at[ROWS * kLd];

    // A over columns: rows row0 + j, columns col0 + 8 g + i
    __device__ __forceinline__ void rows(piece<T> &p, int row0, int col0) const {
        const int lane = threadIdx.x & 63;
        const T *s = at + (row0 + (lane & 15)) * kLd + col0 + 8 * (lane >> 4);
        if constexpr (sizeof(T) == 2) {
            p.v = *reinterpret_cast<const bf16x8 *>(s);
        } else {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(s), b = *reinterpret_cast<const f32x4 *>(s + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p.v[i] = a[i];
                p.v[4 + i] = b[i];
            }
        }
    }
    // A over rows (the tile transposed): columns col0 + j, rows row0 + 4 g + i and row0 + 16 + 4 g + i, i < 4
    __device__ __forceinline__ void cols(piece<T> &p, int row0, int col0) const {
        const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
        if constexpr (sizeof(T) == 2) {
            // the sixteen lanes of a g name four rows, four columns each, and get a column of the four rows each
            const T *s = at + (row0 + 4 * g + (j >> 2)) * kLd + col0 + 4 * (j & 3);
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)s);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(s + 16 * kLd));
            const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
            const u32x4 w = {x[0], x[1], y[0], y[1]};
            p.v = __builtin_bit_cast(bf16x8, w);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) p.v[i] = at[(row0 + 16 * (i / 4) + 4 * g + (i & 3)) * kLd + col0 + j];
        }
    }
};

// a word with zeros in place of the elements that are no numbers; says whether there were any
template <typename T>
__device__ __forceinline__ uint32_t clean_word(uint32_t w, bool &any) {
    const bool hi = (w & 0x7F800000u) == 0x7F800000u;
    if constexpr (sizeof(T) == 4) {
        any |= hi;
        return hi ? 0u : w;
    } else {
        const bool lo = (w & 0x7F80u) == 0x7F80u;
        any |= lo | hi;
        return (lo ? 0u : w & 0xFFFFu) | (hi ? 0u : w & 0xFFFF0000u);
    }
}

// Rows of a head as the memory unit sees them: what it reads behind the last byte is zeros, and nothing there is touched.
typedef int i32x4 __attribute__((ext_vector_type(4)));
struct window {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ window(const void *base, int64_t bytes)
        : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00027000)) {}
    __device__ __forceinline__ u32x4 load(int offset) const {
        return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, offset, 0, 0));
    }
    __device__ __forceinline__ float load1(int offset) const {
        return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, offset, 0, 0));
    }
};

// A thread's chunks of the next tile on their way from memory to LDS.
template <typename T, int DH>
struct tile_regs {
    static_assert(tile<T, DH>::kMine >= 1, "a tile has at least one chunk for every thread");
    u32x4 v[tile<T, DH>::kMine];
    int offset[tile<T, DH>::kMine];          // of the thread's chunks from the tile's first row, in bytes; beyond every tile
                                             // for the columns behind the head's last
    __device__ __forceinline__ void place(int64_t stride, int width) {
        using t = tile<T, DH>;
#pragma unroll
        for (int m = 0; m < t::kMine; ++m) {
            const int k = threadIdx.x + kAttnThreads * m, r = k / t::kChunks, c = (k % t::kChunks) * t::kPer;
            offset[m] = c < width ? (r * (int)stride + c) * (int)sizeof(T) : 0x7FFFFFF0;
        }
    }
    // the first `rows` rows from base on exist (any number)
    __device__ __forceinline__ void load(const T *__restrict__ base, int64_t stride, int rows) {
        const window w(base, (int64_t)min(max(rows, 0), kTile) * stride * (int)sizeof(T));
#pragma unroll
        for (int m = 0; m < tile<T, DH>::kMine; ++m) v[m] = w.load(offset[m]);
    }
    __device__ __forceinline__ void store(tile<T, DH> &to) const {
        using t = tile<T, DH>;
#pragma unroll
        for (int m = 0; m < t::kMine; ++m) {
            const int k = threadIdx.x + kAttnThreads * m, r = k / t::kChunks, c = (k % t::kChunks) * t::kPer;
            *reinterpret_cast<u32x4 *>(to.at + r * t::kLd + c) = v[m];
        }
    }
    // Zeros in place of infinities and NaN; says whether this thread had any.  mark, where it is given, gets a NaN for every
    // row that had one and a zero for every other: a row's chunks are neighbouring lanes of one wavefront.
    __device__ __forceinline__ bool clean(float *mark = nullptr) {
        using t = tile<T, DH>;
        bool any = false;
#pragma unroll
        for (int m = 0; m < t::kMine; ++m) {
            bool mine = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[m][i] = clean_word<T>(v[m][i], mine);
            any |= mine;
            if (mark) {
                const int k = threadIdx.x + kAttnThreads * m, lane = threadIdx.x & 63;
                const uint64_t row = (__ballot(mine) >> (lane & ~(t::kChunks - 1))) & ((1ull << t::kChunks) - 1);
                if (k % t::kChunks == 0) mark[k / t::kChunks] = row ? __builtin_nanf("") : 0.f;
            }
        }
        return any;
    }
};

__device__ __forceinline__ float load1(const float *p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t *p) { return __uint_as_float((uint32_t)p->bits << 16); }

// An operand over columns straight from memory: rows j of base (rows [0, rows) exist), columns col0 + 8 g + i below width.
template <typename T>
__device__ __forceinline__ void global_rows(piece<T> &p, const T *__restrict__ base, int64_t stride, int row, bool live, int col0,
                                            int width) {
    const int col = col0 + 8 * ((threadIdx.x & 63) >> 4);
    const T *s = base + row * stride + col;
    const u32x4 zero = {0u, 0u, 0u, 0u};
    if constexpr (sizeof(T) == 2) {
        p.v = __builtin_bit_cast(bf16x8, live && col < width ? *reinterpret_cast<const u32x4 *>(s) : zero);
    } else {
        const u32x4 a = live && col < width ? *reinterpret_cast<const u32x4 *>(s) : zero;
        const u32x4 b = live && col + 4 < width ? *reinterpret_cast<const u32x4 *>(s + 4) : zero;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p.v[i] = __uint_as_float(a[i]);
            p.v[4 + i] = __uint_as_float(b[i]);
        }
    }
}

// Four neighbouring columns of a result row (result pieces hold rows of the transposed product).
__device__ __forceinline__ void store4(float *p, const f32x4 &v) { *reinterpret_cast<f32x4 *>(p) = v; }
__device__ __forceinline__ void store4(bf16_t *p, const f32x4 &v) {
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 a = {v[2 * i], v[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2));
    }
    *reinterpret_cast<u32x2 *>(p) = w;
}

// sum and maximum over the four g of a column, in every one of them
__device__ __forceinline__ float column_sum(float x) {
    const unsigned u = __float_as_uint(x);
    const u32x2 a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const unsigned v = __float_as_uint(y);
    const u32x2 b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float column_max(float x) {
    const unsigned u = __float_as_uint(x);
    const u32x2 a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const unsigned v = __float_as_uint(y);
    const u32x2 b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// ---- where the rows are -----------------------------------------------------------------------------------------------------
struct attn_params {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    int64_t n_q, n_kv, batch;
    const int64_t *q_offsets, *kv_offsets, *kv_lengths;
    int heads, group, width, causal;         // group: query heads that share a key head
    float scale;
    const float *bias;                       // [buckets, heads], or NULL
    const int32_t *bucket_of;
    int buckets, distances;                  // distances behind the last are the last
    void *out;
    float *out_f32, *lse;                    // lse [heads, n_q]
    const void *dout;
    void *dq, *dk, *dv;
    int64_t dq_stride, dk_stride, dv_stride;
    float *dbias;
    float *delta;                            // scratch [heads, n_q]
    float *bias_part;                        // scratch [slots, heads, buckets]
    float *split_acc, *split_ml;             // scratch of the split form
    int split_shift, max_q;
    int *flags;
};

// the wavefront's number in its workgroup, known to be the same in every lane
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

struct user {
    int64_t q0, k0;                          // first row of its queries, of its keys
    int64_t b;
    int nq, nk;                              // how many of each
    int room;                                // rows of k and v that are the user's, the unused ones among them
    int first;                               // position of its first query row among its keys: nk - nq, may be negative
};

// The last of the users [0, count) whose offsets[b] / 2^shift + step b is at most `value`, 0 if there is none; a 64-ary search by
// the whole wavefront, which stays among the users whatever the offsets hold.  In 32 bits: for 64-bit bounds, which are the same
// in every lane, this compiler has made two selections of one comparison's outcome.
__device__ __forceinline__ int last_user(const int64_t *__restrict__ offsets, int count, int shift, int per_user, int64_t value) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int step = (int)((unsigned)(hi - lo + 63) / 64u), left = hi - lo, ahead = left / step;      // probes that exist
        bool le = false;
        if (lane < ahead) {
            const int probe = lo + (lane + 1) * step;
            le = (offsets[probe] >> shift) + (int64_t)per_user * probe <= value;
        }
        const int cnt = __popcll(__ballot(le));
        const int span = min((cnt + 1) * step - 1, left);
        hi = lo + span;
        lo = lo + cnt * step;
    }
    return lo;
}

// The rows in use of a user with so many rows, brought into [0, room].
__device__ __forceinline__ int rows_in_use(int64_t used, int room) {
    const int high = (int)(used >> 32), low = (int)used;
    const int some = high > 0 ? room : low < 0 ? room : min(low, room);
    return high < 0 ? 0 : some;
}

// Slots: tiles of 2^shift rows of one user, numbered so that a user's begin at offsets[b] / 2^shift + b, which leaves room for
// one that is cut off at each end and needs nobody to add up the tiles before.  Finds the user of a slot and which of its tiles
// the slot is; false where there is none.  Boundaries that do not fit leave their user out; every access stays inside the rows
// whatever the offsets hold.
__device__ __forceinline__ bool find_user(const attn_params &p, const int64_t *__restrict__ offsets, int slot, int shift, user &u,
                                          int &index) {
    const int lo = last_user(offsets, (int)p.batch, shift, 1, slot);
    u.b = lo;
    const int64_t qa = p.q_offsets[lo], qb = p.q_offsets[lo + 1], ka = p.kv_offsets[lo], kb = p.kv_offsets[lo + 1];
    const int64_t used = p.kv_lengths ? p.kv_lengths[lo] : kb - ka;                // asked for with the boundaries
    if (qa < 0 || qb < qa || qb > p.n_q || ka < 0 || kb < ka || kb > p.n_kv || qb - qa > 0x3fffffff || kb - ka > 0x3fffffff)
        return false;
    u.q0 = qa;
    u.k0 = ka;
    u.nq = (int)(qb - qa);
    u.room = (int)(kb - ka);
    u.nk = rows_in_use(used, u.room);
    u.first = u.nk - u.nq;
    const int64_t k = slot - ((offsets[lo] >> shift) + lo);
    index = (int)k;
    return k >= 0 && k < 0x3fffffff;
}

// Thread by thread over the slots, the last slots first, which often have no tile to work on: offsets that do not ascend from 0
// to the number of rows, lengths beyond their room.
__device__ __forceinline__ void check_layout(const attn_params &p, int slot, int slots) {
    for (int64_t b = (int64_t)(slots - 1 - slot) * kAttnThreads + threadIdx.x; b < p.batch; b += (int64_t)slots * kAttnThreads) {
        const int64_t qa = p.q_offsets[b], qb = p.q_offsets[b + 1], ka = p.kv_offsets[b], kb = p.kv_offsets[b + 1];
        bool bad = qa < 0 || qb < qa || qb > p.n_q || ka < 0 || kb < ka || kb > p.n_kv;
        bad |= b == 0 && (qa != 0 || ka != 0);
        bad |= b == p.batch - 1 && (qb != p.n_q || kb != p.n_kv);
        bad |= qb - qa > 0x3fffffff || kb - ka > 0x3fffffff;
        if (p.kv_lengths) bad |= p.kv_lengths[b] < 0 || p.kv_lengths[b] > kb - ka;
        if (bad) atomicOr(p.flags, kFlagOffsets);
    }
}

// ---- the bias by distance -----------------------------------------------------------------------------------------------------
// A bias as the kernels add it, times log2 e.  One so low that 24 bits have no room for a score beside it hides its pairs like
// -inf: what a row that met nothing else would get of it is the roundings of sums of that size, not a softmax.
constexpr float kHidden = FS_HIDDEN_BIAS;
__device__ __forceinline__ float bias_power(float b) { return b <= kHidden ? neg_inf() : b * kLog2e; }

// What a strip needs beside the distances that count, for workgroups of 64 QT query rows: a wavefront's tile reaches 62 + 16 QT
// distances beyond one of them, and there may be up to 64 QT - 1 rows behind the last.
constexpr int row_pad(int qt) { return 64 * qt > kTile + 16 * qt ? 64 * qt : kTile + 16 * qt; }

// at[zero + d] is the bias of distance d (times log2 e) for the distances a workgroup meets, kPad further on either side: the
// distances of a tile lie within kPad of one that counts, so that nobody has to bring a distance into range.
template <int kPad>
struct strip {
    float *at;              // LDS
    int zero, low, high;    // distances below low are low, above high are high; at[] begins at distance low - kPad

    static __host__ __device__ int entries(int distances, bool causal) {
        return (causal ? distances : 2 * distances - 1) + 2 * kPad;
    }
    // what the table has for a distance, and the bucket that is: -1 where it is none
    __device__ __forceinline__ int entry(const attn_params &p, int d) const { return p.bucket_of[min(max(d, low), high) - low]; }
    static __device__ __forceinline__ int bucket(const attn_params &p, int k) { return k < p.buckets ? max(k, -1) : -1; }
    // Distances from `from` to `to` (and kPad around) are met.  Returns whether any bias of them hides (is -inf then); has a barrier.
    __device__ __forceinline__ bool fill(const attn_params &p, int head, float *lds, int from, int to) {
        at = lds;
        high = p.distances - 1;
        low = p.causal ? 0 : -high;
        zero = kPad - low;
        int a = (from < low ? low : from > high ? high : from) - kPad, b = (to > high ? high : to < low ? low : to) + kPad;
        bool hides = false;
        for (int d = a + (int)threadIdx.x; d <= b; d += kAttnThreads) {
            float x = 0.f;
            if (p.bias) {
                const int k = bucket(p, entry(p, d));
                if (k < 0) atomicOr(p.flags, kFlagRowRange);
                else x = bias_power(p.bias[(int64_t)k * p.heads + head]);
            }
            at[zero + d] = x;
            hides |= x == neg_inf();
        }
        return __syncthreads_or(hides) != 0;
    }
};

// Whether the sums of a row's scores begin at what the scores are less by, -lse / scale, which saves an addition for every score.
// A matrix product keeps 24 bits of its running sum, which are then spent on the size of lse / scale: enough where the factors
// have 8 bits, not where they have 24.
template <typename T>
constexpr bool from_less = sizeof(T) == 2;

// Wavefronts of a SIMD that a kernel is compiled for.  With two or more of them asked for, all of a wavefront's registers can be
// named by every instruction, and the accumulators stay where the vector units can read them.  One / two, backward: rows of 256
// bytes (64 histories of 2000 up, bf16) keys 2.40 ms / 1.33; of 512 bytes (32 of 2000 up, fp32), which spill then, query rows 2.68 /
// 4.44.  Scalar registers spill in all of them, 65 to 164 of the keys' kernels up to 64 columns and 340 to 370 at 128, and 3 to 5
// vector registers of the keys' kernels with 256 of them.
template <typename T, int DH>
constexpr int attn_waves = sizeof(T) * DH <= 256 ? 2 : 1;

// ---- host side --------------------------------------------------------------------------------------------------------------
// The compiler's reduction behind __syncthreads_or has 512 bytes of a workgroup's LDS.  Every kernel is allowed all of the rest
// (the largest asks for 135 KB) and not what one call needs: threads of the host whose tables differ share that allowance.
constexpr int kStaticLds = 512;
constexpr int kMaxLds = 160 * 1024 - kStaticLds;
constexpr int kFreeLds = 64 * 1024 - kStaticLds;           // what a kernel may ask for without saying so beforehand

template <typename F>
int launch_attention(fs_ctx *ctx, F *kernel, int64_t groups, size_t lds, hipStream_t s, const char *name, const attn_params &p) {
    if (lds > (size_t)kMaxLds) return set_err(ctx, FS_EINVAL, "jagged attention: head_dim, buckets and distances do not fit together");
    if (lds > (size_t)kFreeLds)
        FS_HIP(ctx, hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxLds));
    kernel<<<(unsigned)groups, kAttnThreads, lds, s>>>(p);
    FS_LAUNCH_CHECK(ctx, name);
    return FS_OK;
}

// f(T *, DH) for a type and a head's width rounded up
template <typename F>
int by_head(int dt, int width, F &&f) {
    const auto widths = [&](auto *t) {
        if (width <= 32) return f(t, std::integral_constant<int, 32>());
        if (width <= 64) return f(t, std::integral_constant<int, 64>());
        return f(t, std::integral_constant<int, 128>());
    };
    return dt == FS_F32 ? widths((float *)nullptr) : widths((bf16_t *)nullptr);
}

// slots of tiles of 2^shift rows (find_user)
inline int64_t attn_slots(int64_t rows, int64_t batch, int shift) { return (rows >> shift) + batch; }

int launch_attention_backward(fs_ctx *ctx, const attn_params &p, int dt, void *work, hipStream_t s);
size_t attention_backward_work(const attn_params &p, int dt);

}  // namespace fs
