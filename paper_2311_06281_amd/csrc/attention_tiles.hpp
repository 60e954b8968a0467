// Tiles of the linear attention kernels: matrix products of 16 x 16 blocks over 32 steps of the contraction, the operands'
// layouts in registers and LDS, and the decays within a chunk of tokens.
//
// A fragment holds, in each lane, eight entries along the contraction: lane l = 16 g + r has row (or column) r and the steps
// 4g..4g+3 and 16+4g..16+4g+3.  That is how two neighbouring accumulator blocks of a product lie in the lanes (a block has
// column r and rows 4g..4g+3 in lane l), so an accumulated state is an operand of the next product as it is, without a way
// through LDS.  In float32 the same entries go through eight products of four steps each.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hs {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Vec;
template <> struct Vec<float> {
    typedef f32x4 x4;
    typedef f32x8 x8;
};
template <> struct Vec<__bf16> {
    typedef bf16x4 x4;
    typedef bf16x8 x8;
};
template <typename T> using x4 = typename Vec<T>::x4;
template <typename T> using Frag = typename Vec<T>::x8;

// acc += A^T B for two fragments: acc has A's rows as its rows and B's as its columns.
__device__ static inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 acc) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0); }
__device__ static inline f32x4 mma(f32x8 a, f32x8 b, f32x4 acc)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    return acc;
}

template <typename T> __device__ static inline Frag<T> join(x4<T> a, x4<T> b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
template <typename T> __device__ static inline Frag<T> to_frag(f32x4 a, f32x4 b)
{
    return join<T>(__builtin_convertvector(a, x4<T>), __builtin_convertvector(b, x4<T>));
}

// Rows of tiles in LDS are padded by 16 bytes.
template <typename T> __host__ __device__ constexpr int pitch(int d) { return d + 16 / (int)sizeof(T); }

// Fragment of rows row0.. of a tile, contraction along the row from k0 on.
template <typename T> __device__ static inline Frag<T> load_rows(const T *tile, int pitch, int row0, int k0, int lane)
{
    const T *p = tile + (row0 + (lane & 15)) * pitch + k0 + 4 * (lane >> 4);
    return join<T>(*reinterpret_cast<const x4<T> *>(p), *reinterpret_cast<const x4<T> *>(p + 16));
}

// Fragment of columns col0.. of a tile, contraction down the rows from k0 on.
__device__ static inline bf16x4 transposed4(const __bf16 *p)
{
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                          (__attribute__((address_space(3))) i16x4 *)(const_cast<__bf16 *>(p))));
}
__device__ static inline bf16x8 load_cols(const __bf16 *tile, int pitch, int col0, int k0, int lane)
{
    // sixteen lanes read four rows of sixteen entries, four entries each, and get a column each
    const __bf16 *p = tile + (k0 + 4 * (lane >> 4) + ((lane & 15) >> 2)) * pitch + col0 + 4 * (lane & 3);
    return join<__bf16>(transposed4(p), transposed4(p + 16 * pitch));
}
__device__ static inline f32x8 load_cols(const float *tile, int pitch, int col0, int k0, int lane)
{
    const float *p = tile + (k0 + 4 * (lane >> 4)) * pitch + col0 + (lane & 15);
    f32x8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = p[((i >> 2) * 16 + (i & 3)) * pitch];
    return f;
}

// ---- tiles of rows from global memory ---------------------------------------------------------------------

// 16 bytes of a row of d entries from entry `col` on, zeros after its end.  `whole`: rows start on 16-byte boundaries and
// d is a whole number of vectors.
template <typename T> __device__ static inline u32x4 load16(const T *row, int col, int d, bool whole)
{
    constexpr int N = 16 / (int)sizeof(T);
    u32x4 v = {0, 0, 0, 0};
    if (whole) {
        if (col < d) v = *reinterpret_cast<const u32x4 *>(row + col);
        return v;
    }
    typedef T vec __attribute__((ext_vector_type(N)));
    vec e;
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = col + i < d ? row[col + i] : (T)0.0f;
    return __builtin_bit_cast(u32x4, e);
}

// A tile of C rows of D entries on its way from global memory to LDS, in registers.
template <typename T, int C, int D, int THREADS> struct TileLoad {
    static constexpr int N = 16 / (int)sizeof(T);
    static constexpr int PER_ROW = D / N;
    static constexpr int COUNT = C * PER_ROW / THREADS;
    static_assert(C * PER_ROW % THREADS == 0, "whole rounds");
    u32x4 v[COUNT];
    // rows 0..rows-1 start at base + row * stride and have d entries; the others are zeros
    __device__ void load(const T *base, int64_t stride, int rows, int d, bool whole)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int at = threadIdx.x + i * THREADS, row = at / PER_ROW, col = at % PER_ROW * N;
            v[i] = row < rows ? load16(base + row * stride, col, d, whole) : u32x4{0, 0, 0, 0};
        }
    }
    __device__ void store(T *tile) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int at = threadIdx.x + i * THREADS, row = at / PER_ROW, col = at % PER_ROW * N;
            *reinterpret_cast<u32x4 *>(tile + row * pitch<T>(D) + col) = v[i];
        }
    }
    // whether an entry is infinite or NaN
    __device__ bool not_finite() const
    {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (sizeof(T) == 4) bad |= (v[i][j] & 0x7f800000u) == 0x7f800000u;
                else bad |= (uint32_t)((v[i][j] & 0x7f800000u) == 0x7f800000u) | (uint32_t)((v[i][j] & 0x7f80u) == 0x7f80u);
            }
        return bad != 0;
    }
};

// four entries from `col` on of a row of d entries
template <typename T> __device__ static inline void store4(T *row, int col, int d, bool whole, f32x4 v)
{
    const x4<T> e = __builtin_convertvector(v, x4<T>);
    if (whole) {
        if (col < d) *reinterpret_cast<x4<T> *>(row + col) = e;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < d) row[col + i] = e[i];
}

// ---- decays within a chunk ------------------------------------------------------------------------------------
//
// G_t, the sum of log2 a up to token t of the chunk, as a whole number and a fraction, so that the difference of two of
// them keeps 24 bits behind the point wherever the two stand.  An a that is zero in float32 counts as 2^-4096: whatever
// spans it has weight zero.  A NaN spreads to the tokens after it.
template <int C> struct Decays {
    float whole[C], part[C]; // G_t
    float from_start[C];     // 2^G_t
    float to_end[C];         // 2^(G_C - G_t)
    float total;             // 2^G_C
};

__device__ static inline double lane_up(double x, int by)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __shfl_up((uint32_t)u, by), hi = __shfl_up((uint32_t)(u >> 32), by);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ static inline double lane_at(double x, int lane)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __shfl((uint32_t)u, lane), hi = __shfl((uint32_t)(u >> 32), lane);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

// One wave: lane t has log a_t (natural), zero after the last token.  Returns log2 of the chunk's decay.
template <int C> __device__ static inline double write_decays(Decays<C> &d, float log_a, int lane)
{
    double g = (double)log_a * 1.4426950408889634;
    if (log_a <= -104.0f) g = -4096.0; // exp(-104) is zero in float32, subnormal numbers included
    if (log_a >= 2840.0f) g = 4096.0;
    if (lane >= C) g = 0.0;
#pragma unroll
    for (int by = 1; by < C; by *= 2) {
        const double other = lane_up(g, by);
        if (lane >= by) g += other;
    }
    const double end = lane_at(g, C - 1);
    if (lane < C) {
        const double w = floor(g);
        d.whole[lane] = (float)w;
        d.part[lane] = (float)(g - w);
        d.from_start[lane] = __builtin_amdgcn_exp2f((float)g);
        d.to_end[lane] = __builtin_amdgcn_exp2f((float)(end - g));
        if (lane == 0) d.total = __builtin_amdgcn_exp2f((float)end);
    }
    return end;
}

template <typename T> __device__ static inline float to_float(T x) { return (float)x; }

// The tokens of sequence b: the first one's place, and how many there are (at most n).
__device__ static inline int64_t sequence(const int64_t *starts, int64_t n, int b, int64_t &first)
{
    if (starts == nullptr) {
        first = b * n;
        return n;
    }
    first = starts[b];
    const int64_t len = starts[b + 1] - first;
    return len < 0 ? 0 : len < n ? len : n;
}

} // namespace hs
