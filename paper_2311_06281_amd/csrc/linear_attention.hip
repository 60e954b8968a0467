// Linear attention with a decay for each head: prompts (chunks of tokens), single tokens, and the sweeps over the states that
// prompts cut into segments and the gradients need.
//
//     S_t = a_t S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t            (S: K x V, float32)
//
// Chunked: with S the state at the start of a chunk of C tokens and G_t the sum of log a up to token t in it,
//     o_t = scale (e^{G_t} S^T q_t + sum_{s<=t} e^{G_t-G_s} (q_t . k_s) v_s),   S' = e^{G_C} S + sum_s e^{G_C-G_s} k_s v_s^T.
#include "attention_tiles.hpp"
#include "operators.hpp"

namespace hs {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

enum Sweep { kOutput, kSegmentState, kSegmentGradient, kChunkStates };

struct SweepArgs {
    const void *q, *k, *v, *log_a;
    const float *s0;
    const int64_t *starts;
    void *out;               // kOutput: out; kChunkStates: the state at each chunk's start, [B, H, chunks, DK, DV] in T
    float *sn;
    int64_t n, q_stride, k_stride, v_stride;
    int64_t segment;         // tokens of a segment, a whole number of chunks
    float *segment_state;    // [B, H, segments, K, V]: kSegment...: written; else, where there are several: the state at its start
    float *segment_decay;    // [B, H, segments]: written by kSegment...
    int H, share, K, V, segments, chunks;
    float scale;
    bool per_head, q_whole, k_whole, v_whole, out_whole;
};

// The fragment with zeros in the place of infinite and NaN entries.
template <typename F> __device__ static inline F finite(F f)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(__builtin_fabsf(to_float(f[i])) < __builtin_inff())) f[i] = 0.0f;
    return f;
}

// A workgroup takes one segment of one head's tokens and goes through its chunks, the state in registers: each wave has a
// slice of DV / 4 columns.  kSegmentGradient goes from the last chunk to the first over (scale q, grad_out) in place of
// (k, v) and gives the segment's own part of the gradient of the state it starts from.
template <typename T, int C, int DK, int DV, int SWEEP>
__global__ __launch_bounds__(kThreads, 2) void heinsen_attention_sweep(SweepArgs p)
{
    constexpr int KT = DK / 16, NT = DV / 16 / kWaves, TT = C / 16, PK = pitch<T>(DK), PV = pitch<T>(DV), PP = pitch<T>(C);
    constexpr bool BACK = SWEEP == kSegmentGradient;
    // v scaled by its decay is summed into the state as the sum of this many bfloat16 numbers: three hold 24 bits
    constexpr int PLANES = sizeof(T) == 4 ? 1 : 3;
    __shared__ __align__(16) T ks[C * PK];
    __shared__ __align__(16) T vs[C * PV];
    __shared__ __align__(16) T qs[SWEEP == kOutput ? C * PK : 16];
    __shared__ __align__(16) T ps[SWEEP == kOutput ? C * PP : 16];
    __shared__ Decays<C> decays;
    __shared__ int not_finite[2]; // of even and odd chunks

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int seg = blockIdx.x % p.segments, bh = blockIdx.x / p.segments, h = bh % p.H, b = bh / p.H;
    int64_t first;
    const int64_t len = sequence(p.starts, p.n, b, first);
    const int64_t begin = seg * p.segment, end = begin + p.segment < len ? begin + p.segment : len;
    if (begin >= len && (seg > 0 || SWEEP != kOutput)) return;

    const T *const k = static_cast<const T *>(p.k) + first * p.k_stride + (int64_t)(h / p.share) * p.K;
    const T *const q = static_cast<const T *>(p.q) + first * p.q_stride + (int64_t)(h / p.share) * p.K;
    const T *const v = static_cast<const T *>(p.v) + first * p.v_stride + (int64_t)h * p.V;
    const T *const log_a = static_cast<const T *>(p.log_a);
    const int col = wave * (DV / kWaves) + r; // of this lane's first column

    f32x4 state[KT][NT];
    const bool segment_start = (SWEEP == kOutput || SWEEP == kChunkStates) && p.segments > 1 && begin < len;
    const float *const from = segment_start ? p.segment_state + ((int64_t)bh * p.segments + seg) * p.K * p.V
                              : (SWEEP == kOutput || SWEEP == kChunkStates) && p.s0 ? p.s0 + (int64_t)bh * p.K * p.V : nullptr;
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 16 * i + 4 * g + e, c = col + 16 * j;
                state[i][j][e] = from && row < p.K && c < p.V ? from[(int64_t)row * p.V + c] : 0.0f;
            }
    double total = 0.0; // log2 of the decay so far (wave 0)

    const int chunks = (int)((end - begin + C - 1) / C);
    auto chunk_start = [&](int i) { return begin + (int64_t)(BACK ? chunks - 1 - i : i) * C; };
    TileLoad<T, C, DK, kThreads> next_q, next_k;
    TileLoad<T, C, DV, kThreads> next_v;
    float next_log_a = 0.0f;
    auto request = [&](int64_t t0) {
        const int rows = (int)(end - t0 < C ? end - t0 : C);
        next_k.load(k + t0 * p.k_stride, p.k_stride, rows, p.K, p.k_whole);
        next_v.load(v + t0 * p.v_stride, p.v_stride, rows, p.V, p.v_whole);
        if (SWEEP == kOutput) next_q.load(q + t0 * p.q_stride, p.q_stride, rows, p.K, p.q_whole);
        if (wave == 0)
            next_log_a = log_a == nullptr || lane >= rows ? 0.0f
                         : p.per_head ? to_float(log_a[h]) : to_float(log_a[(first + t0 + lane) * p.H + h]);
    };
    if (threadIdx.x < 2) not_finite[threadIdx.x] = 0;
    if (chunks > 0) request(chunk_start(0));
    __syncthreads();

    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int64_t t0 = chunk_start(chunk);
        const int rows = (int)(end - t0 < C ? end - t0 : C);
        next_k.store(ks);
        next_v.store(vs);
        if (SWEEP == kOutput) next_q.store(qs);
        if (next_v.not_finite()) atomicOr(&not_finite[chunk & 1], 1);
        if (wave == 0) total += write_decays<C>(decays, next_log_a, lane);
        __syncthreads();
        const bool odd_values = not_finite[chunk & 1] != 0;
        if (threadIdx.x == 0) not_finite[(chunk + 1) & 1] = 0;
        if (chunk + 1 < chunks) request(chunk_start(chunk + 1));

        if (SWEEP == kOutput) {
            // the weights of the chunk's tokens for one another, scale e^{G_t-G_s} q_t . k_s, in tiles of 16 x 16: this wave's
            // are those of tokens t in one row of tiles
            const int tt = wave % TT;
            Frag<T> qf[DK / 32];
#pragma unroll
            for (int i = 0; i < DK / 32; ++i) qf[i] = load_rows(qs, PK, 16 * tt, 32 * i, lane);
            const float whole_t = decays.whole[16 * tt + r], part_t = decays.part[16 * tt + r];
            for (int st = wave / TT; st <= (tt | 1); st += kWaves / TT) {
                f32x4 acc = {0, 0, 0, 0};
                if (st <= tt) {
#pragma unroll
                    for (int i = 0; i < DK / 32; ++i) acc = mma(load_rows(ks, PK, 16 * st, 32 * i, lane), qf[i], acc);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int s = 16 * st + 4 * g + e;
                        const float w = __builtin_amdgcn_exp2f((whole_t - decays.whole[s]) + (part_t - decays.part[s])) * p.scale;
                        acc[e] = s <= 16 * tt + r ? acc[e] * w : 0.0f;
                    }
                }
                *reinterpret_cast<x4<T> *>(ps + (16 * tt + r) * PP + 16 * st + 4 * g) = __builtin_convertvector(acc, x4<T>);
            }
            __syncthreads();
        }
        if (SWEEP == kChunkStates) {
            T *const to = static_cast<T *>(p.out) + ((int64_t)bh * p.chunks + t0 / C) * (DK * DV);
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) to[(16 * i + 4 * g + e) * DV + col + 16 * j] = (T)state[i][j][e];
        }

        Frag<T> vf[C / 32][NT];
#pragma unroll
        for (int i = 0; i < C / 32; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) vf[i][j] = load_cols(vs, PV, wave * (DV / kWaves) + 16 * j, 32 * i, lane);

        if (SWEEP == kOutput) {
            f32x4 o[TT][NT]; // rows: columns of v, columns: tokens
#pragma unroll
            for (int i = 0; i < TT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) o[i][j] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < DK / 32; ++i) {
                Frag<T> sf[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j) sf[j] = to_frag<T>(state[2 * i][j], state[2 * i + 1][j]);
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const Frag<T> qf = load_rows(qs, PK, 16 * t, 32 * i, lane);
#pragma unroll
                    for (int j = 0; j < NT; ++j) o[t][j] = mma(sf[j], qf, o[t][j]);
                }
            }
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const float w = decays.from_start[16 * t + r] * p.scale;
#pragma unroll
                for (int j = 0; j < NT; ++j) o[t][j] *= w;
#pragma unroll
                for (int i = 0; i <= t / 2; ++i) {
                    const Frag<T> pf = load_rows(ps, PP, 16 * t, 32 * i, lane);
#pragma unroll
                    for (int j = 0; j < NT; ++j) o[t][j] = mma(odd_values ? finite(vf[i][j]) : vf[i][j], pf, o[t][j]);
                }
                // an infinite or NaN v_s has no part in the tokens before it, where its zero weight would make it NaN: such
                // values were left out above and are added to the tokens that see them
                if (odd_values)
                    for (int s = 0; s <= 16 * t + r; ++s) {
                        const float w = to_float(ps[(16 * t + r) * PP + s]);
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float x = to_float(vs[s * PV + wave * (DV / kWaves) + 16 * j + 4 * g + e]);
                                if (!(__builtin_fabsf(x) < __builtin_inff())) o[t][j][e] += w * x;
                            }
                    }
                if (16 * t + r < rows) {
                    T *const row = static_cast<T *>(p.out) + ((first + t0 + 16 * t + r) * p.H + h) * (int64_t)p.V;
#pragma unroll
                    for (int j = 0; j < NT; ++j) store4(row, wave * (DV / kWaves) + 16 * j + 4 * g, p.V, p.out_whole, o[t][j]);
                }
            }
        }

        // the state after the chunk
        const float decay = decays.total;
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) state[i][j] *= decay;
#pragma unroll
        for (int i = 0; i < C / 32; ++i) {
            const float *const w = (BACK ? decays.from_start : decays.to_end) + 32 * i + 4 * g;
            Frag<T> vw[NT][PLANES];
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = to_float(vf[i][j][e]) * w[(e >> 2) * 16 + (e & 3)];
                    if (BACK) x *= p.scale;
#pragma unroll
                    for (int plane = 0; plane < PLANES; ++plane) {
                        const T part = (T)x;
                        vw[j][plane][e] = part;
                        x -= to_float(part);
                        if (PLANES > 1 && odd_values && !(__builtin_fabsf(to_float(part)) < __builtin_inff())) x = 0.0f;
                    }
                }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const Frag<T> kf = load_cols(ks, PK, 16 * kt, 32 * i, lane);
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int plane = 0; plane < PLANES; ++plane) state[kt][j] = mma(kf, vw[j][plane], state[kt][j]);
            }
        }
        // rows past the K-th stay zero, also where zero was multiplied by infinity
        if (odd_values || !(__builtin_fabsf(decay) < __builtin_inff()))
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (16 * i + 4 * g + e >= p.K) state[i][j][e] = 0.0f;
        __syncthreads();
    }

    float *to = nullptr;
    if (SWEEP == kSegmentState || SWEEP == kSegmentGradient) {
        to = p.segment_state + ((int64_t)bh * p.segments + seg) * p.K * p.V;
        if (threadIdx.x == 0) p.segment_decay[(int64_t)bh * p.segments + seg] = __builtin_amdgcn_exp2f((float)total);
    } else if (SWEEP == kOutput && p.sn && end == len) {
        to = p.sn + (int64_t)bh * p.K * p.V;
    }
    if (to)
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = 16 * i + 4 * g + e, c = col + 16 * j;
                    if (row < p.K && c < p.V) to[(int64_t)row * p.V + c] = state[i][j][e];
                }
}

// Chains the segments: each one's own sum is replaced by the state it starts from (BACK: the gradient it ends with).
template <bool BACK>
__global__ __launch_bounds__(256) void heinsen_attention_chain(float *segment_state, const float *segment_decay, const float *init,
                                                               const int64_t *starts, int64_t n, int64_t segment, int H, int segments,
                                                               int size)
{
    const int blocks = (size + 255) / 256, bh = blockIdx.x / blocks, at = blockIdx.x % blocks * 256 + threadIdx.x;
    int64_t first;
    const int64_t len = sequence(starts, n, bh / H, first);
    const int used = (int)((len + segment - 1) / segment);
    if (at >= size) return;
    float s = init ? init[(int64_t)bh * size + at] : 0.0f;
    for (int i = 0; i < used; ++i) {
        const int64_t j = (int64_t)bh * segments + (BACK ? used - 1 - i : i);
        const float own = segment_state[j * size + at];
        segment_state[j * size + at] = s;
        s = s * segment_decay[j] + own;
    }
}

// ---- few tokens -----------------------------------------------------------------------------------------------
//
// The recurrence itself, a token at a time: the state is read once, stays in registers and is written once, which is all
// the memory traffic there is.  A workgroup has COLS columns of a head's state; a thread has VEC neighbouring columns of
// every ROWS-th row.
struct StepArgs {
    const void *q, *k, *v, *log_a;
    const float *s0;
    const int64_t *starts;
    void *out;
    float *sn;
    int64_t n, q_stride, k_stride, v_stride;
    int H, share, K, V, slices;
    float scale;
    bool per_head;
};

template <typename T, int COLS, int VEC>
__global__ __launch_bounds__(256) void heinsen_attention_step(StepArgs p)
{
    constexpr int ACROSS = COLS / VEC, ROWS = 256 / ACROSS, PER = (128 + ROWS - 1) / ROWS, IN_WAVE = 64 / ACROSS > 1 ? 64 / ACROSS : 1;
    constexpr int PARTS = ROWS / IN_WAVE; // partial sums of an output
    typedef float vec __attribute__((ext_vector_type(VEC)));
    __shared__ float qk[2][128];
    __shared__ float sums[PARTS][COLS];
    const int slice = blockIdx.x % p.slices, bh = blockIdx.x / p.slices, h = bh % p.H, b = bh / p.H;
    const int row0 = threadIdx.x / ACROSS, local = threadIdx.x % ACROSS * VEC, col = slice * COLS + local;
    const bool inside = col < p.V;
    int64_t first;
    const int64_t len = sequence(p.starts, p.n, b, first);
    const int64_t at = (int64_t)bh * p.K * p.V + col;

    vec state[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = row0 + i * ROWS;
        state[i] = (vec)0.0f;
        if (p.s0 && inside && row < p.K) state[i] = *reinterpret_cast<const vec *>(p.s0 + at + (int64_t)row * p.V);
    }
    for (int64_t t = 0; t < len; ++t) {
        const int64_t token = first + t;
        if (threadIdx.x < 128) {
            const int i = threadIdx.x;
            const int64_t head = (int64_t)(h / p.share) * p.K + i;
            qk[0][i] = i < p.K ? to_float(static_cast<const T *>(p.q)[token * p.q_stride + head]) * p.scale : 0.0f;
            qk[1][i] = i < p.K ? to_float(static_cast<const T *>(p.k)[token * p.k_stride + head]) : 0.0f;
        }
        const T *const log_a = static_cast<const T *>(p.log_a);
        const float la = log_a == nullptr ? 0.0f : to_float(log_a[p.per_head ? h : token * p.H + h]);
        const float a = la <= -104.0f ? 0.0f : expf(la);
        vec value = (vec)0.0f;
        if (inside) {
            const T *const v = static_cast<const T *>(p.v) + token * p.v_stride + (int64_t)h * p.V + col;
#pragma unroll
            for (int e = 0; e < VEC; ++e) value[e] = to_float(v[e]);
        }
        __syncthreads();
        vec o = (vec)0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int row = row0 + i * ROWS;
            if (row < p.K) {
                state[i] = state[i] * a + qk[1][row] * value;
                o += qk[0][row] * state[i];
            }
        }
#pragma unroll
        for (int by = ACROSS; by < 64; by *= 2)
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] += __shfl_xor(o[e], by);
        if (threadIdx.x % 64 < ACROSS || ACROSS > 64) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) sums[row0 / IN_WAVE][local + e] = o[e];
        }
        __syncthreads();
        if (threadIdx.x < COLS && slice * COLS + threadIdx.x < p.V) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < PARTS; ++i) sum += sums[i][threadIdx.x];
            static_cast<T *>(p.out)[(token * p.H + h) * p.V + slice * COLS + threadIdx.x] = (T)sum;
        }
        __syncthreads();
    }
    if (p.sn && inside)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int row = row0 + i * ROWS;
            if (row < p.K) *reinterpret_cast<vec *>(p.sn + at + (int64_t)row * p.V) = state[i];
        }
}

// ---- host -----------------------------------------------------------------------------------------------------

template <typename T> constexpr int chunk_tokens() { return sizeof(T) == 2 ? 64 : 32; }

bool rows16(const void *p, int64_t stride, int d, size_t size)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && d * size % 16 == 0;
}

template <typename T, int SWEEP, int DK, int DV> hipError_t sweep_sized(const SweepArgs &a, int64_t blocks, hipStream_t stream)
{
    heinsen_attention_sweep<T, chunk_tokens<T>(), DK, DV, SWEEP><<<dim3((unsigned)blocks), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T, int SWEEP> hipError_t sweep(const SweepArgs &a, int64_t blocks, hipStream_t stream)
{
    if (a.K <= 64) return a.V <= 64 ? sweep_sized<T, SWEEP, 64, 64>(a, blocks, stream) : sweep_sized<T, SWEEP, 64, 128>(a, blocks, stream);
    return a.V <= 64 ? sweep_sized<T, SWEEP, 128, 64>(a, blocks, stream) : sweep_sized<T, SWEEP, 128, 128>(a, blocks, stream);
}

SweepArgs sweep_args(const AttentionCall &c)
{
    const size_t size = c.bf16 ? 2 : 4;
    SweepArgs a = {};
    a.q = c.q, a.k = c.k, a.v = c.v, a.log_a = c.log_a, a.s0 = c.s0, a.starts = c.starts, a.out = c.out, a.sn = c.sn;
    a.n = c.n, a.q_stride = c.q_stride, a.k_stride = c.k_stride, a.v_stride = c.v_stride;
    a.H = c.H, a.share = c.share, a.K = c.K, a.V = c.V, a.scale = c.scale, a.per_head = c.per_head;
    a.q_whole = rows16(c.q, c.q_stride, c.K, size), a.k_whole = rows16(c.k, c.k_stride, c.K, size), a.v_whole = rows16(c.v, c.v_stride, c.V, size);
    a.out_whole = reinterpret_cast<uintptr_t>(c.out) % (4 * size) == 0 && c.V % 4 == 0;
    return a;
}

hipError_t chain(bool back, float *state, const float *decay, const float *init, const AttentionCall &c, const Segments &s)
{
    const int size = c.K * c.V;
    const dim3 grid((unsigned)((size + 255) / 256 * c.B * c.H));
    if (back) heinsen_attention_chain<true><<<grid, 256, 0, c.stream>>>(state, decay, init, c.starts, c.n, s.tokens, c.H, s.count, size);
    else heinsen_attention_chain<false><<<grid, 256, 0, c.stream>>>(state, decay, init, c.starts, c.n, s.tokens, c.H, s.count, size);
    return hipGetLastError();
}

template <typename T, int COLS, int VEC> hipError_t step_sized(StepArgs &a, const AttentionCall &c)
{
    a.slices = (c.V + COLS - 1) / COLS;
    heinsen_attention_step<T, COLS, VEC><<<dim3((unsigned)((int64_t)c.B * c.H * a.slices)), 256, 0, c.stream>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t step(const AttentionCall &c)
{
    StepArgs a = {};
    a.q = c.q, a.k = c.k, a.v = c.v, a.log_a = c.log_a, a.s0 = c.s0, a.starts = c.starts, a.out = c.out, a.sn = c.sn;
    a.n = c.n, a.q_stride = c.q_stride, a.k_stride = c.k_stride, a.v_stride = c.v_stride;
    a.H = c.H, a.share = c.share, a.K = c.K, a.V = c.V, a.scale = c.scale, a.per_head = c.per_head;
    const bool whole = c.V % 4 == 0 && reinterpret_cast<uintptr_t>(c.s0) % 16 == 0 && reinterpret_cast<uintptr_t>(c.sn) % 16 == 0;
    if (!whole) return step_sized<T, 64, 1>(a, c);
    // narrow slices where heads alone do not fill the chip
    if ((int64_t)c.B * c.H * 2 <= compute_units() && c.V > 32) return step_sized<T, 32, 4>(a, c);
    return step_sized<T, 128, 4>(a, c);
}

} // namespace

Segments attention_segments(const AttentionCall &c)
{
    // two workgroups to a compute unit at least, while a segment stays long against the states it adds
    const int64_t heads = (int64_t)c.B * c.H, want = 2 * compute_units();
    int64_t count = heads >= want ? 1 : (want + heads - 1) / heads;
    const int64_t most = (c.n + 511) / 512;
    if (count > most) count = most;
    Segments s;
    s.tokens = ((c.n + count - 1) / count + 63) / 64 * 64;
    s.count = (int)((c.n + s.tokens - 1) / s.tokens);
    return s;
}

size_t segment_scratch(const AttentionCall &c, const Segments &s)
{
    if (s.count == 1) return 0;
    const size_t count = (size_t)c.B * c.H * s.count;
    return align_up(count * c.K * c.V * sizeof(float), 256) + align_up(count * sizeof(float), 256);
}

// The states at the segments' starts (BACK: the gradients at their ends) from the segments' own sums.
hipError_t attention_segment_states(const AttentionCall &c, const Segments &s, bool back, void *scratch)
{
    SweepArgs a = sweep_args(c);
    a.segment = s.tokens, a.segments = s.count;
    a.segment_state = static_cast<float *>(scratch);
    a.segment_decay = a.segment_state + align_up((size_t)c.B * c.H * s.count * c.K * c.V * sizeof(float), 256) / sizeof(float);
    const int64_t blocks = (int64_t)c.B * c.H * s.count;
    hipError_t e;
    if (back) {
        const size_t size = c.bf16 ? 2 : 4;
        a.k = c.q, a.k_stride = c.q_stride, a.k_whole = a.q_whole;
        a.v = c.grad_out, a.v_stride = (int64_t)c.H * c.V, a.v_whole = rows16(c.grad_out, a.v_stride, c.V, size);
        e = c.bf16 ? sweep<__bf16, kSegmentGradient>(a, blocks, c.stream) : sweep<float, kSegmentGradient>(a, blocks, c.stream);
    } else {
        e = c.bf16 ? sweep<__bf16, kSegmentState>(a, blocks, c.stream) : sweep<float, kSegmentState>(a, blocks, c.stream);
    }
    if (e != hipSuccess) return e;
    return chain(back, a.segment_state, a.segment_decay, back ? c.grad_sn : c.s0, c, s);
}

hipError_t attention_chunk_states(const AttentionCall &c, const Segments &s, float *segment_state, void *states, int chunks)
{
    SweepArgs a = sweep_args(c);
    a.segment = s.tokens, a.segments = s.count, a.segment_state = segment_state;
    a.out = states, a.chunks = chunks;
    const int64_t blocks = (int64_t)c.B * c.H * s.count;
    return c.bf16 ? sweep<__bf16, kChunkStates>(a, blocks, c.stream) : sweep<float, kChunkStates>(a, blocks, c.stream);
}

int attention_chunk_tokens(bool bf16) { return bf16 ? chunk_tokens<__bf16>() : chunk_tokens<float>(); }

size_t attention_scratch(const AttentionCall &c) { return c.n <= kFewTokens ? 0 : segment_scratch(c, attention_segments(c)); }

hipError_t attention_launch(const AttentionCall &c, void *scratch)
{
    if (c.n <= kFewTokens) return c.bf16 ? step<__bf16>(c) : step<float>(c);
    const Segments s = attention_segments(c);
    if (s.count > 1) {
        const hipError_t e = attention_segment_states(c, s, false, scratch);
        if (e != hipSuccess) return e;
    }
    SweepArgs a = sweep_args(c);
    a.segment = s.tokens, a.segments = s.count, a.segment_state = static_cast<float *>(scratch);
    const int64_t blocks = (int64_t)c.B * c.H * s.count;
    return c.bf16 ? sweep<__bf16, kOutput>(a, blocks, c.stream) : sweep<float, kOutput>(a, blocks, c.stream);
}

} // namespace hs
