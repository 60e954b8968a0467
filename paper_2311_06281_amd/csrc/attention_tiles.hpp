// Tiles of the linear attention kernels: matrix products of 16 x 16 blocks over 32 steps of the contraction, the operands'
// layouts in registers and LDS, and the decays within a chunk of tokens.
//
// A fragment holds, in each lane l = 16 g + r, the entries of row (or column) r at eight steps of the contraction: 8g..8g+7 in
// bfloat16, 4g..4g+3 and 16+4g..16+4g+3 in float32, where they go through eight products of four steps.  An accumulator block
// has column r and rows 4g..4g+3 in lane l.  Two neighbouring blocks of a state are such a fragment as they are, without a way
// through LDS, if their rows stand for the right entries: paired() says which.
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

// Step of the contraction that entry e of a fragment stands for, and the index that row r of block `tile` of a state has.
template <typename T> __device__ static inline int step_of(int g, int e) { return sizeof(T) == 2 ? 8 * g + e : (e >> 2) * 16 + 4 * g + (e & 3); }
template <typename T> __device__ static inline int paired(int tile, int r)
{
    return sizeof(T) == 2 ? 32 * (tile >> 1) + 8 * (r >> 2) + 4 * (tile & 1) + (r & 3) : 16 * tile + r;
}

// Tiles of rows of D entries in LDS.  The 16-byte pieces of a row change places with the row's number, so that the accesses
// below, sixteen lanes at a time, each touch all banks once: a piece of sixteen rows, four neighbouring or every second piece
// of four rows (bfloat16), four neighbouring pieces of every fourth row (float32).
template <typename T, int D> __device__ static inline int at(int row, int col)
{
    constexpr int N = 16 / (int)sizeof(T), PIECES = D / N;
    static_assert(PIECES >= 8, "eight pieces to a row at least");
    int swap;
    if (PIECES >= 16) swap = sizeof(T) == 2 ? ((row & 3) << 2) | ((row >> 2) & 3) : row & 15;
    else swap = sizeof(T) == 2 ? ((row & 2) << 1) | ((row >> 2) & 3) : (row >> 1) & 7;
    return row * D + (((col / N) ^ swap) * N) + col % N;
}

// Fragment of rows row0.. of a tile, contraction along the row from k0 on.
template <int D> __device__ static inline bf16x8 load_rows(const __bf16 *tile, int row0, int k0, int lane)
{
    return *reinterpret_cast<const bf16x8 *>(tile + at<__bf16, D>(row0 + (lane & 15), k0 + 8 * (lane >> 4)));
}
template <int D> __device__ static inline f32x8 load_rows(const float *tile, int row0, int k0, int lane)
{
    const int row = row0 + (lane & 15), col = k0 + 4 * (lane >> 4);
    return join<float>(*reinterpret_cast<const f32x4 *>(tile + at<float, D>(row, col)), *reinterpret_cast<const f32x4 *>(tile + at<float, D>(row, col + 16)));
}

// Fragment of columns of a tile, contraction down the rows from k0 on.
__device__ static inline bf16x4 transposed4(const __bf16 *p)
{
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                          (__attribute__((address_space(3))) i16x4 *)(const_cast<__bf16 *>(p))));
}
// sixteen lanes read four entries each of four rows, `apart` entries from one lane's to the next one's, and get a column each
template <int D> __device__ static inline bf16x8 columns(const __bf16 *tile, int col0, int apart, int k0, int lane)
{
    const int row = k0 + 8 * (lane >> 4) + ((lane & 15) >> 2), col = col0 + apart * (lane & 3);
    return join<__bf16>(transposed4(tile + at<__bf16, D>(row, col)), transposed4(tile + at<__bf16, D>(row + 4, col)));
}
template <int D> __device__ static inline f32x8 columns(const float *tile, int col0, int, int k0, int lane)
{
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = tile[at<float, D>(k0 + step_of<float>(lane >> 4, e), col0 + (lane & 15))];
    return f;
}
// columns 16 * tile.., or those that the rows of block `tile` of a state stand for
template <int D, typename T> __device__ static inline Frag<T> load_cols(const T *tile, int col0, int k0, int lane)
{
    return columns<D>(tile, col0, 4, k0, lane);
}
template <int D, typename T> __device__ static inline Frag<T> load_paired(const T *tile, int block, int k0, int lane)
{
    return columns<D>(tile, paired<T>(block, 0), sizeof(T) == 2 ? 8 : 4, k0, lane);
}

// ---- rows in global memory --------------------------------------------------------------------------------
//
// Rows start wherever their type may: the accesses are of 16 (stores: 8 or 16) bytes all the same, which the memory pipeline
// takes at any address.  No branches around loads, so that all of a tile's are under way at once.

template <typename T> struct Unaligned;
template <> struct Unaligned<float> {
    typedef u32x4 __attribute__((aligned(4))) vec16;
    typedef f32x4 __attribute__((aligned(4))) vec4;
};
template <> struct Unaligned<__bf16> {
    typedef u32x4 __attribute__((aligned(2))) vec16;
    typedef bf16x4 __attribute__((aligned(2))) vec4;
};

// A tile of C rows of D entries on its way from global memory to LDS, in registers.
template <typename T, int C, int D, int THREADS> struct TileLoad {
    static constexpr int N = 16 / (int)sizeof(T);
    static constexpr int PER_ROW = D / N;
    static constexpr int COUNT = C * PER_ROW / THREADS;
    static_assert(C * PER_ROW % THREADS == 0 && THREADS % PER_ROW == 0, "whole rounds of whole rows");
    u32x4 v[COUNT];

    __device__ static int col() { return threadIdx.x % PER_ROW * N; }
    __device__ static int row(int i) { return threadIdx.x / PER_ROW + i * (THREADS / PER_ROW); }

    // rows 0..rows-1 start at base + row * stride and have d entries: the others and the rest of each are read from where
    // there are some
    __device__ void load(const T *base, int64_t stride, int rows, int d)
    {
        if (d < N) { // too few for a vector
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                typedef T vec __attribute__((ext_vector_type(N)));
                const T *const from = base + (row(i) < rows ? row(i) : rows - 1) * stride;
                vec e;
#pragma unroll
                for (int j = 0; j < N; ++j) e[j] = from[j < d ? j : 0];
                v[i] = __builtin_bit_cast(u32x4, e);
            }
            return;
        }
        const uint32_t first = (col() < d - N ? col() : d - N) * (uint32_t)sizeof(T), step = (uint32_t)stride * (uint32_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const uint32_t offset = (uint32_t)(row(i) < rows ? row(i) : rows - 1) * step + first;
            v[i] = *reinterpret_cast<const typename Unaligned<T>::vec16 *>(reinterpret_cast<const char *>(base) + offset);
        }
    }
    // puts what was read in place: entries from the d-th on and rows from `rows` on are zero
    __device__ void settle(int rows, int d)
    {
        if (d < D) {
            const int from = d < N ? 0 : col() < d - N ? col() : d - N; // the first entry read
            const int shift = (col() - from) * 8 * (int)sizeof(T), keep = d - col() < N ? d - col() : N;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const uint64_t lo = ((uint64_t)v[i][1] << 32) | v[i][0], hi = ((uint64_t)v[i][3] << 32) | v[i][2];
                uint64_t a = shift >= 64 ? hi : lo, b = shift >= 64 ? 0 : hi;
                a = (a >> (shift & 63)) | ((b << 1) << (63 - (shift & 63)));
                b >>= shift & 63;
                if (d < N && keep > 0) { // entries read in the place of others
                    const int bits = keep * 8 * (int)sizeof(T);
                    a = bits >= 64 ? a : a & (((uint64_t)1 << bits) - 1);
                    b = bits > 64 ? b & (((uint64_t)1 << (bits - 64)) - 1) : 0;
                }
                if (keep <= 0) a = b = 0;
                v[i] = u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
            }
        }
        if (rows < C)
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
                if (row(i) >= rows) v[i] = u32x4{0, 0, 0, 0};
    }
    __device__ void store(T *tile) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) *reinterpret_cast<u32x4 *>(tile + at<T, D>(row(i), col())) = v[i];
    }
    // whether an entry is infinite or NaN
    __device__ bool not_finite() const
    {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bad |= (uint32_t)((v[i][j] & 0x7f800000u) == 0x7f800000u);
                if (sizeof(T) == 2) bad |= (uint32_t)((v[i][j] & 0x7f80u) == 0x7f80u);
            }
        return bad != 0;
    }
};

// four entries of a row of d float32 from `col` on, zeros after its end
__device__ static inline f32x4 load4(const float *row, int col, int d)
{
    f32x4 v = {0, 0, 0, 0};
    if (col + 4 <= d) v = *reinterpret_cast<const Unaligned<float>::vec4 *>(row + col);
    else
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (col + i < d) v[i] = row[col + i];
    return v;
}

// four entries from `col` on of a row of d entries
template <typename T> __device__ static inline void store4(T *row, int col, int d, f32x4 v)
{
    const x4<T> e = __builtin_convertvector(v, x4<T>);
    if (col + 4 <= d) *reinterpret_cast<typename Unaligned<T>::vec4 *>(row + col) = e;
    else
#pragma unroll
        for (int i = 0; i < 3; ++i)
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

// x, of which the compiler does not know that it is: what is formed from it is formed here, not ahead of the loop, where the
// addresses of all the accesses of a chunk would fill the registers.
__device__ static inline int fresh(int x)
{
    asm volatile("" : "+v"(x));
    return x;
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
