// The norms before and after a block, fused with its gate, residual scale and residual, and their gradients.
//
//     z = u                                     or  u r w_post,   r = (mean u^2 + eps)^(-1/2)    the norm after the block
//     h = residual + scale (act(gate) z)        act(x) = x sigmoid(x), or sigmoid(x)             the residual stream
//     y = h r' w_pre,   r' = (mean h^2 + eps)^(-1/2)                                             the norm before the next block
// Gradients, with t = dy w_pre, n' = h r':
//     dh' = dh + r' (t - n' mean(t n'));  dresidual = dh';  dw_pre = sum dy n';  dscale = sum dh' act z
//     dz = dh' scale act;  dgate = dh' scale z act';  dw_post = sum dz u r;  du = r (dz w_post - u r mean(dz w_post u r))
// A row is read once and stays in registers; both passes are bound by memory.
#include "operators.hpp"

namespace hs {
namespace {

struct NormArgs {
    const void *u, *gate, *residual;
    const float *scale, *w_post, *w_pre;
    void *h, *y;
    const void *grad_h, *grad_y;
    void *grad_u, *grad_gate, *grad_residual;
    float *sums; // [workgroups, 3, D]: gradients of scale, w_post, w_pre summed over a workgroup's rows
    int64_t rows, u_stride, gate_stride;
    int D;
    float eps;
    bool sigmoid;
};

// A row's entries in the lanes: TPR threads to a row, EPT entries to a thread in vectors of VEC, neighbouring vectors in
// neighbouring threads.
template <typename T, int VEC, int TPR, int EPT, typename F = float> struct Row {
    static constexpr int COUNT = EPT / VEC;
    typedef T vec __attribute__((ext_vector_type(VEC)));
    __device__ static int col(int i) { return ((threadIdx.x % TPR) + i * TPR) * VEC; }
    __device__ static void load(F (&x)[EPT], const T *row, int D)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            vec v = (vec)(T)0.0f;
            if (col(i) < D) v = *reinterpret_cast<const vec *>(row + col(i));
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[i * VEC + e] = (F)v[e];
        }
    }
    __device__ static void load_vector(F (&x)[EPT], const float *p, int D)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[i * VEC + e] = col(i) + e < D ? p[col(i) + e] : 0.0f;
    }
    __device__ static void store(T *row, const F (&x)[EPT], int D)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            vec v;
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = (T)(float)x[i * VEC + e];
            if (col(i) < D) *reinterpret_cast<vec *>(row + col(i)) = v;
        }
    }
};

// Sum over the threads of a row.  With more than a wave to a row every thread of the workgroup has to come here.
template <int TPR, typename F> __device__ static inline F row_sum(F x, F *shared)
{
#pragma unroll
    for (int by = 1; by < (TPR < 64 ? TPR : 64); by *= 2) x += __shfl_xor(x, by);
    if (TPR > 64) {
        __syncthreads();
        if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) x += shared[i];
    }
    return x;
}

__device__ static inline float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)); }

__device__ static inline double logistic(double x) { return 1.0 / (1.0 + exp(-x)); }

template <int TPR> __host__ __device__ constexpr int threads_of() { return TPR < 256 ? 256 : TPR; }

template <typename T, int VEC, int TPR, int EPT>
__global__ __launch_bounds__(threads_of<TPR>()) void heinsen_norm_forward(NormArgs p)
{
    typedef Row<T, VEC, TPR, EPT> R;
    constexpr int GROUPS = threads_of<TPR>() / TPR;
    __shared__ float shared[TPR > 64 ? TPR / 64 : 1];
    const float inverse = 1.0f / (float)p.D;
    float scale[EPT], w_post[EPT], w_pre[EPT];
    if (p.scale) R::load_vector(scale, p.scale, p.D);
    if (p.w_post) R::load_vector(w_post, p.w_post, p.D);
    if (p.w_pre) R::load_vector(w_pre, p.w_pre, p.D);
    // with several rows to a workgroup a row is within a wave, and waves may end before others
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * GROUPS) {
        float z[EPT], gate[EPT], h[EPT];
        R::load(z, static_cast<const T *>(p.u) + row * p.u_stride, p.D);
        if (p.gate) R::load(gate, static_cast<const T *>(p.gate) + row * p.gate_stride, p.D);
        if (p.residual) R::load(h, static_cast<const T *>(p.residual) + row * p.D, p.D);
        if (p.w_post) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < EPT; ++i) sum += z[i] * z[i];
            const float r = rsqrtf(row_sum<TPR>(sum, shared) * inverse + p.eps);
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
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < EPT; ++i) sum += h[i] * h[i];
            const float r = rsqrtf(row_sum<TPR>(sum, shared) * inverse + p.eps);
#pragma unroll
            for (int i = 0; i < EPT; ++i) h[i] = h[i] * r * w_pre[i];
            R::store(static_cast<T *>(p.y) + row * p.D, h, p.D);
        }
    }
}

// F: the type of what is done to an entry.  A norm's gradient is what is left of two terms that cancel where a row has few
// entries or one large one: statistics and that difference are in float64 whatever F is, which costs no more instructions
// here than float32.  With few entries all of it is: there h itself may be a small rest, by which the gradient is divided.
template <typename T, int VEC, int TPR, int EPT, typename F>
__global__ __launch_bounds__(threads_of<TPR>()) void heinsen_norm_backward(NormArgs p)
{
    typedef Row<T, VEC, TPR, EPT, F> R;
    constexpr int THREADS = threads_of<TPR>(), GROUPS = THREADS / TPR;
    __shared__ double shared[TPR > 64 ? TPR / 64 : 1];
    __shared__ float columns[GROUPS > 1 ? GROUPS * TPR * EPT : 1];
    const double inverse = 1.0 / p.D;
    F scale[EPT], w_post[EPT], w_pre[EPT];
    if (p.scale) R::load_vector(scale, p.scale, p.D);
    if (p.w_post) R::load_vector(w_post, p.w_post, p.D);
    if (p.w_pre) R::load_vector(w_pre, p.w_pre, p.D);
    float sums[3][EPT] = {};
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * GROUPS) {
        F u[EPT], gate[EPT], h[EPT], dh[EPT], dy[EPT];
        R::load(u, static_cast<const T *>(p.u) + row * p.u_stride, p.D);
        if (p.gate) R::load(gate, static_cast<const T *>(p.gate) + row * p.gate_stride, p.D);
        if (p.residual) R::load(h, static_cast<const T *>(p.residual) + row * p.D, p.D);
        if (p.grad_h) R::load(dh, static_cast<const T *>(p.grad_h) + row * p.D, p.D);
        if (p.grad_y) R::load(dy, static_cast<const T *>(p.grad_y) + row * p.D, p.D);
        double r = 1.0, rr = 1.0; // rr: r^2
        if (p.w_post) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) sum += (double)u[i] * u[i];
            rr = 1.0 / (row_sum<TPR>(sum, shared) * inverse + p.eps);
            r = sqrt(rr);
        }
        F act[EPT];
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            if (!p.grad_h) dh[i] = 0;
            act[i] = 1;
            if (p.gate) {
                const F s = logistic(gate[i]);
                act[i] = p.sigmoid ? s : gate[i] * s;
                gate[i] = p.sigmoid ? s * (1 - s) : s * (1 + gate[i] * (1 - s)); // act'
            }
        }
        if (p.grad_y) {
            double sum = 0.0, dot = 0.0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) {
                F z = u[i] * (F)r * act[i];
                if (p.w_post) z *= w_post[i];
                if (p.scale) z *= scale[i];
                h[i] = p.residual ? h[i] + z : z;
                sum += (double)h[i] * h[i];
                dot += (double)(dy[i] * w_pre[i]) * h[i];
            }
            const double rrh = 1.0 / (row_sum<TPR>(sum, shared) * inverse + p.eps), rh = sqrt(rrh);
            const double mean = row_sum<TPR>(dot, shared) * inverse * rrh;
#pragma unroll
            for (int i = 0; i < EPT; ++i) {
                sums[2][i] += (float)(dy[i] * (h[i] * (F)rh));
                dh[i] += (F)(rh * ((double)(dy[i] * w_pre[i]) - h[i] * mean));
            }
        }
        if (p.grad_residual) R::store(static_cast<T *>(p.grad_residual) + row * p.D, dh, p.D);
        double dot = 0.0;
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            const F unit = u[i] * (F)r, z = p.w_post ? unit * w_post[i] : unit;
            sums[0][i] += (float)(dh[i] * act[i] * z);
            if (p.scale) dh[i] *= scale[i];
            gate[i] = dh[i] * z * gate[i];
            dh[i] *= act[i];
            if (p.w_post) {
                sums[1][i] += (float)(dh[i] * unit);
                dh[i] *= w_post[i];
                dot += (double)dh[i] * u[i];
            }
        }
        if (p.gate && p.grad_gate) R::store(static_cast<T *>(p.grad_gate) + row * p.D, gate, p.D);
        if (p.w_post) {
            const double mean = row_sum<TPR>(dot, shared) * inverse * rr;
#pragma unroll
            for (int i = 0; i < EPT; ++i) dh[i] = (F)(r * ((double)dh[i] - u[i] * mean));
        }
        R::store(static_cast<T *>(p.grad_u) + row * p.D, dh, p.D);
    }
    if (p.sums == nullptr) return;
    // the workgroup's sums: over its rows side by side in a fixed order
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        float *const to = p.sums + ((int64_t)blockIdx.x * 3 + k) * p.D;
        if (GROUPS == 1) {
#pragma unroll
            for (int i = 0; i < R::COUNT; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (R::col(i) + e < p.D) to[R::col(i) + e] = sums[k][i * VEC + e];
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R::COUNT; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) columns[threadIdx.x / TPR * (TPR * EPT) + R::col(i) + e] = sums[k][i * VEC + e];
        __syncthreads();
        for (int c = threadIdx.x; c < p.D; c += THREADS) {
            float sum = 0.0f;
            for (int i = 0; i < GROUPS; ++i) sum += columns[i * (TPR * EPT) + c];
            to[c] = sum;
        }
    }
}

// Sums of the workgroups' sums: 64 columns to a workgroup, its four waves a quarter of the rows each.
__global__ __launch_bounds__(256) void heinsen_norm_columns(const float *sums, float *scale, float *w_post, float *w_pre, int D, int count)
{
    __shared__ float part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = blockIdx.y, c = blockIdx.x * 64 + lane;
    float *const to = which == 0 ? scale : which == 1 ? w_post : w_pre;
    if (to == nullptr) return;
    float sum = 0.0f;
    if (c < D)
        for (int i = wave; i < count; i += 4) sum += sums[((int64_t)i * 3 + which) * D + c];
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < D) to[c] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

// ---- host -----------------------------------------------------------------------------------------------------

constexpr int kBackwardPerUnit = 4; // workgroups of the backward pass to a compute unit, at most (of 256 threads)

int64_t workgroups(const NormCall &c, int groups, int per_unit)
{
    const int64_t all = (c.rows + groups - 1) / groups, most = (int64_t)per_unit * compute_units();
    return all < most ? all : most;
}

template <typename T, int VEC, int TPR, int EPT, typename F = float> hipError_t launch(const NormCall &c, NormArgs &a, bool back)
{
    constexpr int THREADS = threads_of<TPR>(), GROUPS = THREADS / TPR;
    if (!back) {
        heinsen_norm_forward<T, VEC, TPR, EPT><<<dim3((unsigned)workgroups(c, GROUPS, 32)), THREADS, 0, c.stream>>>(a);
        return hipGetLastError();
    }
    const unsigned count = (unsigned)workgroups(c, GROUPS, kBackwardPerUnit);
    heinsen_norm_backward<T, VEC, TPR, EPT, F><<<dim3(count), THREADS, 0, c.stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.sums == nullptr) return e;
    heinsen_norm_columns<<<dim3((c.D + 63) / 64, 3), 256, 0, c.stream>>>(a.sums, c.grad_scale, c.grad_w_post, c.grad_w_pre, c.D, (int)count);
    return hipGetLastError();
}

template <typename T, int VEC> hipError_t sized(const NormCall &c, NormArgs &a, bool back)
{
    if (c.D <= 16 && back) return launch<T, VEC, 16, 8, double>(c, a, true);
    if (c.D <= 128) return launch<T, VEC, 16, 8>(c, a, back);
    if (c.D <= 256) return launch<T, VEC, 32, 8>(c, a, back);
    if (c.D <= 512) return launch<T, VEC, 64, 8>(c, a, back);
    if (c.D <= 1024) return launch<T, VEC, 64, 16>(c, a, back);
    if (c.D <= 2048) return launch<T, VEC, 256, 8>(c, a, back);
    if (c.D <= 4096) return launch<T, VEC, 256, 16>(c, a, back);
    if (c.D <= 8192) return launch<T, VEC, 1024, 8>(c, a, back);
    return launch<T, VEC, 1024, 16>(c, a, back);
}

// The widest vectors that every row of every array starts on a boundary of.
template <typename T> bool rows_on(const NormCall &c, size_t bytes)
{
    const void *const arrays[] = {c.u, c.gate, c.residual, c.h, c.y, c.grad_h, c.grad_y, c.grad_u, c.grad_gate, c.grad_residual};
    for (const void *p : arrays)
        if (reinterpret_cast<uintptr_t>(p) % bytes != 0) return false;
    return c.D * sizeof(T) % bytes == 0 && c.u_stride * sizeof(T) % bytes == 0 && c.gate_stride * sizeof(T) % bytes == 0;
}

hipError_t run(const NormCall &c, float *sums, bool back)
{
    NormArgs a = {};
    a.u = c.u, a.gate = c.gate, a.residual = c.residual, a.scale = c.scale, a.w_post = c.w_post, a.w_pre = c.w_pre, a.h = c.h, a.y = c.y;
    a.grad_h = c.grad_h, a.grad_y = c.grad_y, a.grad_u = c.grad_u, a.grad_gate = c.grad_gate, a.grad_residual = c.grad_residual;
    a.sums = sums, a.rows = c.rows, a.u_stride = c.u_stride, a.gate_stride = c.gate_stride, a.D = c.D, a.eps = c.eps, a.sigmoid = c.sigmoid;
    if (c.bf16) {
        if (rows_on<__bf16>(c, 16)) return sized<__bf16, 8>(c, a, back);
        if (rows_on<__bf16>(c, 4)) return sized<__bf16, 2>(c, a, back);
        return sized<__bf16, 1>(c, a, back);
    }
    return rows_on<float>(c, 16) ? sized<float, 4>(c, a, back) : sized<float, 1>(c, a, back);
}

} // namespace

hipError_t norm_launch(const NormCall &c) { return run(c, nullptr, false); }

size_t norm_backward_scratch(const NormCall &c)
{
    if (!c.grad_scale && !c.grad_w_post && !c.grad_w_pre) return 0;
    return (size_t)kBackwardPerUnit * compute_units() * 3 * c.D * sizeof(float);
}

hipError_t norm_backward_launch(const NormCall &c, void *scratch) { return run(c, static_cast<float *>(scratch), true); }

} // namespace hs
