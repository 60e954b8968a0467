// The norms before and after a block, fused with its gate, residual scale and residual, and their gradients.
//
//     z = u                                     or  u r w_post,   r = (mean u^2 + eps)^(-1/2)    the norm after the block
//     h = residual + scale (act(gate) z)        act(x) = x sigmoid(x), or sigmoid(x)             the residual stream
//     y = h r' w_pre,   r' = (mean h^2 + eps)^(-1/2)                                             the norm before the next block
// Gradients, with t = dy w_pre, n' = h r':
//     dh' = dh + r' (t - n' mean(t n'));  dresidual = dh';  dw_pre = sum dy n';  dscale = sum dh' act z
//     dz = dh' scale act;  dgate = dh' scale z act';  dw_post = sum dz u r;  du = r (dz w_post - u r mean(dz w_post u r))
// A row is read once and stays in registers; both passes are bound by memory where rows start on 16 bytes.  Measured, bytes read
// and written over time: 32768 rows of 1024 bfloat16 forward 66 us, 5.1 TB/s, backward 117 us, 4.6 TB/s; 131072 rows of 2048
// float32 997 us, 5.4 TB/s, and 1637 us, 5.2 TB/s; 126042 rows of 110 bfloat16 18 us, 4.7 TB/s, and 35 us, 4.0 TB/s.  Of rows of
// more than 8192 entries the backward pass keeps half in scratch memory (16384: 0.6 to 1 TB/s).
#include "operators.hpp"

namespace hs {
namespace {

struct NormArgs {
    const void *u, *gate, *residual;
    const float *scale, *w_post, *w_pre;
    void *h, *y;
    const void *grad_h, *grad_y;
    void *grad_u, *grad_gate, *grad_residual;
    float *sums; // [3, workgroups, D]: gradients of scale, w_post, w_pre summed over a workgroup's rows, or null
    int wanted;  // bit for each of these
    int64_t rows, u_stride, gate_stride;
    int D;
    float eps;
    bool sigmoid;
};

// A row's entries in the lanes: EPT entries to a thread in vectors of VEC, neighbouring vectors in neighbouring threads, at any
// alignment; TPR threads to a row.
// Where the row ends within a vector (RAGGED) the last one is moved back to end with it, and has some entries of the one before
// it again; threads past the end have the last vector's.  own() says which entries are a thread's own.
template <typename T, int VEC, int TPR, int EPT, bool RAGGED> struct Row {
    static constexpr int COUNT = EPT / VEC;
    typedef T vec __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
    typedef float weights __attribute__((ext_vector_type(VEC), aligned(sizeof(float))));
    vec v[COUNT] = {};

    __device__ static int place(int i) { return (int)(threadIdx.x % TPR + i * TPR) * VEC; }
    __device__ static int col(int i, int D) { return place(i) < D - VEC ? place(i) : D - VEC; }
    __device__ static bool own(int i, int e, int D) { return RAGGED ? col(i, D) + e >= place(i) : place(i) < D; }

    __device__ void load(const T *row, int D)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = *reinterpret_cast<const vec *>(row + col(i, D));
    }
    template <typename F> __device__ void get(F (&x)[EPT]) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[i * VEC + e] = (F)(float)v[i][e];
    }
    template <typename F> __device__ static void store(T *row, const F (&x)[EPT], int D)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            vec out;
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[e] = (T)(float)x[i * VEC + e];
            T *const to = row + col(i, D);
            // Entries that two threads have, both store: in one wave both have read theirs by then, also where an output
            // takes the place of an input.  Two waves are not in step; there only the own entries are stored.
            if (RAGGED && TPR > 64 && place(i) > D - VEC) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (own(i, e, D)) to[e] = out[e];
            } else if (place(i) < D) // outputs are not read here again (bfloat16, rows of 1024: 48 us against 63)
                __builtin_nontemporal_store(out, reinterpret_cast<vec *>(to));
        }
    }
    template <typename F> __device__ static void load_weights(F (&x)[EPT], const float *p, int D)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const weights w = *reinterpret_cast<const weights *>(p + col(i, D));
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[i * VEC + e] = w[e];
        }
    }
    // the sum over this thread's own entries; add(sum, i): the sum and the i-th entry's
    template <typename F, typename G> __device__ static F sum(int D, G add)
    {
        F sum = 0;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            F of = 0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) of = RAGGED && !own(i, e, D) ? of : add(of, i * VEC + e);
            sum += !RAGGED && !own(i, 0, D) ? 0 : of;
        }
        return sum;
    }
};

template <int CTRL> __device__ static inline uint32_t moved(uint32_t x) { return __builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false); }
template <int CTRL> __device__ static inline float moved(float x) { return __builtin_bit_cast(float, moved<CTRL>(__builtin_bit_cast(uint32_t, x))); }
template <int CTRL> __device__ static inline double moved(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, ((uint64_t)moved<CTRL>((uint32_t)(u >> 32)) << 32) | moved<CTRL>((uint32_t)u));
}
// x + the x of the other half of each 32 (HALF 16) or 64 (HALF 32) lanes
template <int HALF> __device__ static inline auto swapped(uint32_t x)
{
    if constexpr (HALF == 16) return __builtin_amdgcn_permlane16_swap(x, x, false, false);
    else return __builtin_amdgcn_permlane32_swap(x, x, false, false);
}
template <int HALF> __device__ static inline float add_half(float x)
{
    const auto s = swapped<HALF>(__builtin_bit_cast(uint32_t, x));
    return __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
}
template <int HALF> __device__ static inline double add_half(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const auto lo = swapped<HALF>((uint32_t)u), hi = swapped<HALF>((uint32_t)(u >> 32));
    return __builtin_bit_cast(double, ((uint64_t)(uint32_t)hi[0] << 32) | (uint32_t)lo[0]) + __builtin_bit_cast(double, ((uint64_t)(uint32_t)hi[1] << 32) | (uint32_t)lo[1]);
}

// the sum of x over sixteen lanes
template <typename F> __device__ static inline F ring(F x)
{
    x += moved<0x128>(x); // by 8, 4, 2, 1
    x += moved<0x124>(x);
    x += moved<0x122>(x);
    return x + moved<0x121>(x);
}

// Sums over the threads of a row.  With more than a wave to a row every thread of the workgroup has to come here, and the
// waves hand theirs over in one of two places in turn: before a place is written again there is the other one's barrier.
template <int TPR, typename F> struct RowSums {
    static constexpr int WAVES = TPR / 64;
    typedef F Places[2][2][16];
    Places &place;
    int turn = 0;
    __device__ explicit RowSums(Places &p) : place(p)
    {
        if (WAVES <= 4) return;
        if (threadIdx.x < 64) place[threadIdx.x / 32][threadIdx.x / 16 % 2][threadIdx.x % 16] = 0; // of waves that are not there
        __syncthreads();
    }
    template <int N> __device__ void operator()(F (&x)[N])
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            x[k] = ring(x[k]);
            if (TPR >= 32) x[k] = add_half<16>(x[k]);
            if (TPR >= 64) x[k] = add_half<32>(x[k]);
        }
        if (WAVES <= 1) return;
        turn ^= 1;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) place[turn][k][threadIdx.x / 64] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (WAVES > 4) {
                x[k] = ring(place[turn][k][threadIdx.x % 16]);
                continue;
            }
            x[k] = place[turn][k][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) x[k] += place[turn][k][i];
        }
    }
};

__device__ static inline float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)); }
__device__ static inline double logistic(double x) { return 1.0 / (1.0 + exp(-x)); }

// A thousand threads have 128 registers each: the backward pass has its weights in LDS there, which is slower where registers
// hold them (us of 4096 entries, 8192 rows, bfloat16: 161 against 125) and faster than spilling them (8192 entries: 198 against 344).
template <int TPR, int EPT> __host__ __device__ constexpr bool weights_in_lds() { return TPR == 1024 && EPT == 8; }

template <int TPR> __host__ __device__ constexpr int threads_of() { return TPR <= 64 ? 256 : TPR; }

// this thread's row of those that a workgroup begins with
template <int TPR> __device__ static inline int64_t first_row()
{
    constexpr int GROUPS = threads_of<TPR>() / TPR;
    const int group = TPR >= 64 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x / TPR)) : (int)(threadIdx.x / TPR);
    return (int64_t)blockIdx.x * GROUPS + group;
}

template <typename T, int VEC, int TPR, int EPT, bool RAGGED>
__global__ __launch_bounds__(threads_of<TPR>()) void heinsen_norm_forward(NormArgs p)
{
    typedef Row<T, VEC, TPR, EPT, RAGGED> R;
    constexpr int GROUPS = threads_of<TPR>() / TPR;
    __shared__ typename RowSums<TPR, float>::Places places;
    RowSums<TPR, float> row_sums(places);
    const float inverse = 1.0f / (float)p.D;
    float scale[EPT], w_post[EPT], w_pre[EPT];
    if (p.scale) R::load_weights(scale, p.scale, p.D);
    if (p.w_post) R::load_weights(w_post, p.w_post, p.D);
    if (p.w_pre) R::load_weights(w_pre, p.w_pre, p.D);
    // with several rows to a workgroup a row is within a wave, and waves may end before others
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = first_row<TPR>();
    for (; row < p.rows; row += step) {
        R in_u, in_gate, in_residual;
        in_u.load(static_cast<const T *>(p.u) + row * p.u_stride, p.D);
        if (p.gate) in_gate.load(static_cast<const T *>(p.gate) + row * p.gate_stride, p.D);
        if (p.residual) in_residual.load(static_cast<const T *>(p.residual) + row * p.D, p.D);
        float z[EPT], gate[EPT], h[EPT];
        in_u.get(z);
        in_gate.get(gate);
        in_residual.get(h);
        if (p.w_post) {
            float sum[1] = {R::template sum<float>(p.D, [&](float s, int i) { return s + z[i] * z[i]; })};
            row_sums(sum);
            const float r = rsqrtf(sum[0] * inverse + p.eps);
#pragma unroll
            for (int i = 0; i < EPT; ++i) z[i] = z[i] * r * w_post[i];
        }
        if (p.gate)
#pragma unroll
            for (int i = 0; i < EPT; ++i) z[i] *= p.sigmoid ? logistic(gate[i]) : gate[i] * logistic(gate[i]);
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            if (p.scale) z[i] *= scale[i];
            h[i] = p.residual ? h[i] + z[i] : z[i];
        }
        if (p.h) R::store(static_cast<T *>(p.h) + row * p.D, h, p.D);
        if (p.y) {
            float sum[1] = {R::template sum<float>(p.D, [&](float s, int i) { return s + h[i] * h[i]; })};
            row_sums(sum);
            const float r = rsqrtf(sum[0] * inverse + p.eps);
#pragma unroll
            for (int i = 0; i < EPT; ++i) h[i] = h[i] * r * w_pre[i];
            R::store(static_cast<T *>(p.y) + row * p.D, h, p.D);
        }
    }
}

// x, of which the compiler forgets what it is: wider copies made of it before are not kept for what comes after
template <typename F, int N> __device__ static inline void forget(F (&x)[N])
{
    if (N > 8) return; // there are no registers to keep either in
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// x - by * mean, rounded once: without rounding what is taken off
__device__ static inline double less(double x, double by, double mean) { return x - by * mean; }
__device__ static inline float less(float x, float by, double mean)
{
    const float high = (float)mean, low = (float)(mean - high);
    return __builtin_fmaf(-by, low, __builtin_fmaf(-by, high, x));
}

// F: the type of what is done to an entry.  A norm's gradient is what is left of two terms that cancel where a row has few
// entries or one large one: statistics are in float64 whatever F is (its multiply-adds are as fast here as float32's), and so is
// the mean that is taken off.  With few entries all of it is in float64: there h itself may be a small rest, by which the
// gradient is divided.
//
// Registers hold the row's five inputs, the weights and the three sums over rows, eight entries a thread, and leave two waves to
// a SIMD unit; the three reductions of a row are what a wave waits for.  So bfloat16 rows are loaded one ahead (1024 entries, 32768
// rows: 117 us against 129); float32 rows, which take twice the registers for that, are not (2048 entries, 131072 rows: 1790 with,
// 1630 without).
template <typename T, int VEC, int TPR, int EPT, bool RAGGED, typename F>
__global__ __launch_bounds__(threads_of<TPR>()) void heinsen_norm_backward(NormArgs p)
{
    typedef Row<T, VEC, TPR, EPT, RAGGED> R;
    constexpr int THREADS = threads_of<TPR>(), GROUPS = THREADS / TPR;
    constexpr bool AHEAD = sizeof(T) == 2 && TPR < 1024;   // a row's loads begin before the row before it is worked on
    constexpr bool SHARED = weights_in_lds<TPR, EPT>();
    __shared__ typename RowSums<TPR, double>::Places places;
    __shared__ float columns[GROUPS > 1 ? GROUPS * TPR * EPT : 1];
    extern __shared__ float shared[]; // [3, D]
    RowSums<TPR, double> row_sums(places);
    const double inverse = 1.0 / p.D;
    const float *const given[3] = {p.scale, p.w_post, p.w_pre};
    enum { kScale, kPost, kPre };
    F own_weights[3][EPT];
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (given[k]) {
            if (SHARED)
                for (int c = threadIdx.x; c < p.D; c += THREADS) shared[k * p.D + c] = given[k][c];
            else R::load_weights(own_weights[k], given[k], p.D);
        }
    if (SHARED) __syncthreads();
    auto weights = [&](F (&w)[EPT], int k) {
        if (SHARED) R::load_weights(w, shared + k * p.D, p.D);
        else
#pragma unroll
            for (int i = 0; i < EPT; ++i) w[i] = own_weights[k][i];
    };
    float sums[3][EPT] = {};
    struct Inputs {
        R u, gate, residual, dh, dy; // zeros where there is none
        __device__ void load(const NormArgs &p, int64_t row)
        {
            u.load(static_cast<const T *>(p.u) + row * p.u_stride, p.D);
            if (p.gate) gate.load(static_cast<const T *>(p.gate) + row * p.gate_stride, p.D);
            if (p.residual) residual.load(static_cast<const T *>(p.residual) + row * p.D, p.D);
            if (p.grad_h) dh.load(static_cast<const T *>(p.grad_h) + row * p.D, p.D);
            if (p.grad_y) dy.load(static_cast<const T *>(p.grad_y) + row * p.D, p.D);
        }
    } next;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = first_row<TPR>();
    if (AHEAD && row < p.rows) next.load(p, row);
    for (; row < p.rows; row += step) {
        if (!AHEAD) {
            next = Inputs();
            next.load(p, row);
        }
        F u[EPT], act[EPT], slope[EPT], h[EPT], dh[EPT], dy[EPT], w_post[EPT], scale[EPT], w_pre[EPT]; // slope: act'
        next.u.get(u);
        next.gate.get(slope);
        next.residual.get(h);
        next.dh.get(dh);
        next.dy.get(dy);
        if (AHEAD && row + step < p.rows) next.load(p, row + step);
        double r = 1.0, rr = 1.0; // rr: r^2
        if (p.w_post) {
            double sum[1] = {R::template sum<double>(p.D, [&](double s, int i) { return s + (double)u[i] * u[i]; })};
            forget(u);
            row_sums(sum);
            rr = 1.0 / (sum[0] * inverse + p.eps);
            r = sqrt(rr);
            weights(w_post, kPost);
        }
        if (p.scale) weights(scale, kScale);
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            act[i] = 1;
            if (p.gate) {
                const F gate = slope[i], s = logistic(gate);
                act[i] = p.sigmoid ? s : gate * s;
                slope[i] = p.sigmoid ? s * (1 - s) : s * (1 + gate * (1 - s));
            }
            F z = u[i] * (F)r * act[i];
            if (p.w_post) z *= w_post[i];
            if (p.scale) z *= scale[i];
            h[i] = p.residual ? h[i] + z : z;
        }
        if (p.grad_y) {
            weights(w_pre, kPre);
            double sum[2] = {R::template sum<double>(p.D, [&](double s, int i) { return s + (double)h[i] * h[i]; }),
                             R::template sum<double>(p.D, [&](double s, int i) { return s + (double)(dy[i] * w_pre[i]) * h[i]; })};
            forget(h);
            forget(dy);
            row_sums(sum);
            const double rrh = 1.0 / (sum[0] * inverse + p.eps), rh = sqrt(rrh), mean = sum[1] * inverse * rrh;
            weights(w_pre, kPre);
#pragma unroll
            for (int i = 0; i < EPT; ++i) {
                sums[kPre][i] += (float)(dy[i] * (h[i] * (F)rh));
                dh[i] += (F)rh * less(dy[i] * w_pre[i], h[i], mean);
            }
        }
        if (p.grad_residual) R::store(static_cast<T *>(p.grad_residual) + row * p.D, dh, p.D);
        if (p.w_post) weights(w_post, kPost);
        if (p.scale) weights(scale, kScale);
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            const F unit = u[i] * (F)r, z = p.w_post ? unit * w_post[i] : unit;
            sums[kScale][i] += (float)(dh[i] * act[i] * z);
            if (p.scale) dh[i] *= scale[i];
            slope[i] = dh[i] * z * slope[i];
            dh[i] *= act[i];
            if (p.w_post) {
                sums[kPost][i] += (float)(dh[i] * unit);
                dh[i] *= w_post[i];
            }
        }
        if (p.gate && p.grad_gate) R::store(static_cast<T *>(p.grad_gate) + row * p.D, slope, p.D);
        if (p.w_post) {
            double sum[1] = {R::template sum<double>(p.D, [&](double s, int i) { return s + (double)dh[i] * u[i]; })};
            forget(u);
            forget(dh);
            row_sums(sum);
            const double mean = sum[0] * inverse * rr;
#pragma unroll
            for (int i = 0; i < EPT; ++i) dh[i] = (F)r * less(dh[i], u[i], mean);
        }
        R::store(static_cast<T *>(p.grad_u) + row * p.D, dh, p.D);
    }
    if (p.sums == nullptr) return;
    // the workgroup's sums: over its rows side by side in a fixed order
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (!(p.wanted & 1 << k)) continue;
        float *const to = p.sums + ((int64_t)k * gridDim.x + blockIdx.x) * p.D;
        if (GROUPS > 1) __syncthreads();
        float *const at = GROUPS > 1 ? columns + threadIdx.x / TPR * (TPR * EPT) : to;
#pragma unroll
        for (int i = 0; i < R::COUNT; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (R::own(i, e, p.D)) at[R::col(i, p.D) + e] = sums[k][i * VEC + e];
        if (GROUPS == 1) continue;
        __syncthreads();
        for (int c = threadIdx.x; c < p.D; c += THREADS) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) sum += columns[i * (TPR * EPT) + c];
            to[c] = sum;
        }
    }
}

// Sums of the workgroups' sums: sixteen columns to a workgroup, a 64th of the rows to a thread.
__global__ __launch_bounds__(1024) void heinsen_norm_columns(const float *sums, float *scale, float *w_post, float *w_pre, int D, int count)
{
    __shared__ float part[64][17];
    const int lane = threadIdx.x % 16, group = threadIdx.x / 16, which = blockIdx.y, c = blockIdx.x * 16 + lane;
    float *const to = which == 0 ? scale : which == 1 ? w_post : w_pre;
    if (to == nullptr) return;
    float sum = 0.0f;
    if (c < D)
#pragma unroll 8
        for (int i = group; i < count; i += 64) sum += sums[((int64_t)which * count + i) * D + c];
    part[group][lane] = sum;
    for (int by = 32; by > 0; by /= 2) {
        __syncthreads();
        if (group < by) part[group][lane] += part[group + by][lane];
    }
    if (group == 0 && c < D) to[c] = part[0][lane];
}

// ---- host -----------------------------------------------------------------------------------------------------

// The backward pass's workgroups walk over the rows, so that weights are read and sums written once for several of them: at most
// so many waves of them to a compute unit.
constexpr int kForwardWaves = 512, kBackwardWaves = 8;

// threads: of a workgroup, groups: rows that one has side by side
int64_t workgroups(const NormCall &c, int threads, int groups, int waves)
{
    const int64_t all = (c.rows + groups - 1) / groups, most = (int64_t)(waves > threads / 64 ? waves / (threads / 64) : 1) * compute_units();
    return all < most ? all : most;
}

template <typename T, int VEC, int TPR, int EPT, bool RAGGED> hipError_t forward(const NormCall &c, const NormArgs &a)
{
    constexpr int threads = threads_of<TPR>();
    const unsigned count = (unsigned)workgroups(c, threads, threads / TPR, kForwardWaves);
    heinsen_norm_forward<T, VEC, TPR, EPT, RAGGED><<<dim3(count), threads, 0, c.stream>>>(a);
    return hipGetLastError();
}

template <typename T, int VEC, int TPR, int EPT, bool RAGGED, typename F = float> hipError_t backward(const NormCall &c, const NormArgs &a)
{
    constexpr int threads = threads_of<TPR>();
    const unsigned count = (unsigned)workgroups(c, threads, threads / TPR, kBackwardWaves);
    heinsen_norm_backward<T, VEC, TPR, EPT, RAGGED, F><<<dim3(count), threads, weights_in_lds<TPR, EPT>() ? 3 * c.D * sizeof(float) : 0, c.stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.sums == nullptr) return e;
    heinsen_norm_columns<<<dim3((c.D + 15) / 16, 3), 1024, 0, c.stream>>>(a.sums, c.grad_scale, c.grad_w_post, c.grad_w_pre, c.D, (int)count);
    return hipGetLastError();
}

template <typename T, int VEC, bool RAGGED> hipError_t sized(const NormCall &c, const NormArgs &a, bool back)
{
    if (c.D <= 16 && back) return backward<T, VEC, 16, 8, RAGGED, double>(c, a);
    if (c.D <= 128) return back ? backward<T, VEC, 16, 8, RAGGED>(c, a) : forward<T, VEC, 16, 8, RAGGED>(c, a);
    if (c.D <= 256) return back ? backward<T, VEC, 32, 8, RAGGED>(c, a) : forward<T, VEC, 32, 8, RAGGED>(c, a);
    if (c.D <= 512) return back ? backward<T, VEC, 64, 8, RAGGED>(c, a) : forward<T, VEC, 64, 8, RAGGED>(c, a);
    if (c.D <= 1024) return back ? backward<T, VEC, 128, 8, RAGGED>(c, a) : forward<T, VEC, 128, 8, RAGGED>(c, a);
    if (c.D <= 1536) return back ? backward<T, VEC, 192, 8, RAGGED>(c, a) : forward<T, VEC, 192, 8, RAGGED>(c, a);
    if (c.D <= 2048) return back ? backward<T, VEC, 256, 8, RAGGED>(c, a) : forward<T, VEC, 256, 8, RAGGED>(c, a);
    if (c.D <= 3072) return back ? backward<T, VEC, 384, 8, RAGGED>(c, a) : forward<T, VEC, 384, 8, RAGGED>(c, a);
    if (c.D <= 4096) return back ? backward<T, VEC, 512, 8, RAGGED>(c, a) : forward<T, VEC, 512, 8, RAGGED>(c, a);
    if (c.D <= 6144) return back ? backward<T, VEC, 768, 8, RAGGED>(c, a) : forward<T, VEC, 768, 8, RAGGED>(c, a);
    if (c.D <= 8192) return back ? backward<T, VEC, 1024, 8, RAGGED>(c, a) : forward<T, VEC, 1024, 8, RAGGED>(c, a);
    return back ? backward<T, VEC, 1024, 16, RAGGED>(c, a) : forward<T, VEC, 1024, 16, RAGGED>(c, a);
}

template <typename T> hipError_t typed(const NormCall &c, const NormArgs &a, bool back)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    if (c.D % VEC == 0) return sized<T, VEC, false>(c, a, back);
    if (c.D > VEC) return sized<T, VEC, true>(c, a, back);
    return back ? backward<T, 1, 16, 8, false, double>(c, a) : forward<T, 1, 16, 8, false>(c, a); // shorter than a vector
}

hipError_t run(const NormCall &c, float *sums, bool back)
{
    NormArgs a = {};
    a.u = c.u, a.gate = c.gate, a.residual = c.residual, a.scale = c.scale, a.w_post = c.w_post, a.w_pre = c.w_pre, a.h = c.h, a.y = c.y;
    a.grad_h = c.grad_h, a.grad_y = c.grad_y, a.grad_u = c.grad_u, a.grad_gate = c.grad_gate, a.grad_residual = c.grad_residual;
    a.wanted = (c.grad_scale ? 1 : 0) | (c.grad_w_post ? 2 : 0) | (c.grad_w_pre ? 4 : 0);
    a.sums = a.wanted ? sums : nullptr, a.rows = c.rows, a.u_stride = c.u_stride, a.gate_stride = c.gate_stride, a.D = c.D, a.eps = c.eps, a.sigmoid = c.sigmoid;
    return c.bf16 ? typed<__bf16>(c, a, back) : typed<float>(c, a, back);
}

} // namespace

hipError_t norm_launch(const NormCall &c) { return run(c, nullptr, false); }

size_t norm_backward_scratch(const NormCall &c)
{
    if (!c.grad_scale && !c.grad_w_post && !c.grad_w_pre) return 0;
    return (size_t)(kBackwardWaves / 2) * compute_units() * 3 * c.D * sizeof(float); // workgroups of two waves at least
}

hipError_t norm_backward_launch(const NormCall &c, void *scratch) { return run(c, static_cast<float *>(scratch), true); }

} // namespace hs
