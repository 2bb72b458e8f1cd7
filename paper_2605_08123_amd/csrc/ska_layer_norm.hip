// Layer norm of rows, its gradient, and the reduction of the weight's gradient (sinkhorn_attn_layer.h).
//
//   forward   mean and variance of a row held in registers (two passes over registers, none over memory), Y from them
//   backward  dX = rstd (g - mean(g) - h mean(g h)) + dS  with h = (S - mean) rstd, g = dY weight: both sums in one exchange;
//             a thread's features are the same in every row it takes, so dweight = sum dY h and dbias = sum dY stay in
//             registers until the block's last row, go to memory once per block and are added up by a second launch
// Both are bound by memory (MI355X, where a copy of 4 GB reaches 4.8 TB/s): forward with a residual, 262144 rows of 512, bf16,
// 190 us, 5.7 TB/s; backward, 30011 rows of 1283, fp32, 88 + 5 us, 5.3 TB/s in the first launch; 16384 rows of 512, bf16,
// 16.5 + 3.9 us, 4.1 TB/s; 48828 rows of 4096, bf16, 221 us in all, 5.4 TB/s.  Rows that leave the registers: 20000 of 20000, bf16,
// forward 426 us, 3.8 TB/s; backward, whose two launches read S and dY three times, 951 us, 2.5 TB/s of what it cannot do without.
// A row is dealt to TPR threads (a power of two) in NV pieces of 16 bytes, piece t + k TPR to thread t.  Rows of up to 256
// pieces (backward: 128) are a wavefront's or several in one, so that their sums need no barrier; wider ones are a block's.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "sinkhorn_attn_layer.h"

namespace {

constexpr int NT = 256;          // threads of a block whose rows stay in registers
constexpr int NT_LOOP = 1024;    // threads of a block whose row does not
constexpr int MAX_BLOCKS = 1024; // blocks (of partial sums) of the backward: four a CU

struct NormArgs {
    const void *x, *r, *w, *b;   // backward: x = dY, r = dS
    void *s, *y;                 // backward: s = S (read), y = dX
    long ldx, ldr, lds, ldy;
    float *stats;
    long N;
    long first;                  // row of the launch's first block (kernels with blocks for all rows)
    int D;
    float eps;
    int tpr;                     // threads per row
    float *part;                 // backward: [blocks][2][D] partial sums, or null
};

// 16 bytes of adjacent features, which may start on any element
template <typename T> constexpr int VEC = 16 / (int)sizeof(T);
template <typename T> using Vec = T __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));

// n: features of the row from this piece on (<= 0: none)
template <int V, typename T> __device__ __forceinline__ void load_piece(const T *p, int n, float (&f)[V])
{
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (n >= V) {
        vec v = *reinterpret_cast<const vec *>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < n ? (float)p[i] : 0.f;
    }
}
// the same, as it lies in memory
template <typename T> __device__ __forceinline__ void load_piece(const T *p, int n, Vec<T> &v)
{
    if (n >= VEC<T>) v = *reinterpret_cast<const Vec<T> *>(p);
    else {
#pragma unroll
        for (int i = 0; i < VEC<T>; ++i) v[i] = i < n ? p[i] : (T)0.f;
    }
}
template <int V, typename T> __device__ __forceinline__ void store_piece(T *p, int n, const float (&f)[V])
{
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (n >= V) {
        vec v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)f[i];
        *reinterpret_cast<vec *>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = (T)f[i];
    }
}

// Sums over the tpr threads of a row, the same bits in each of them.  red: one slot per wavefront and value, not used twice
// without a barrier in between.
template <int K> __device__ __forceinline__ void row_sums(float (&x)[K], int tpr, float (*red)[K])
{
    const int n = min(tpr, 64);
    for (int s = 1; s < n; s <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] += __shfl_xor(x[k], s);
    if (tpr > 64) {
        const int wv = threadIdx.x >> 6, per = tpr >> 6, first = wv & ~(per - 1);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) red[wv][k] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            x[k] = 0.f;
            for (int i = 0; i < per; ++i) x[k] += red[first + i][k];
        }
    }
}

template <typename T, typename TW, int NV> __global__ __launch_bounds__(NT) void norm_fwd_kernel(const NormArgs a)
{
    constexpr int V = VEC<T>;
    __shared__ float red[2][NT / 64][1];
    const int t = threadIdx.x & (a.tpr - 1);
    const long row = a.first + (long)blockIdx.x * (NT / a.tpr) + threadIdx.x / a.tpr;
    const bool have = row < a.N;
    const long at = have ? row : a.N - 1;
    float x[NV][V];
    const T *xp = reinterpret_cast<const T *>(a.x) + at * a.ldx;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (t + k * a.tpr) * V;
        load_piece<V>(xp + c, a.D - c, x[k]);
    }
    if (a.r) {
        const T *rp = reinterpret_cast<const T *>(a.r) + at * a.ldr;
        T *sp = reinterpret_cast<T *>(a.s) + at * a.lds;
        float r[NV][V];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (t + k * a.tpr) * V;
            load_piece<V>(rp + c, a.D - c, r[k]);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (t + k * a.tpr) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) x[k][i] = (float)(T)(x[k][i] + r[k][i]);   // the sum as it is stored, which the backward reads
            if (have) store_piece<V>(sp + c, a.D - c, x[k]);
        }
    }
    float sum[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[0] += x[k][i];
    row_sums<1>(sum, a.tpr, red[0]);
    const float mean = sum[0] / (float)a.D;
    float var[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int n = a.D - (t + k * a.tpr) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float e = i < n ? x[k][i] - mean : 0.f;
            var[0] = fmaf(e, e, var[0]);
        }
    }
    row_sums<1>(var, a.tpr, red[1]);
    const float rstd = 1.f / sqrtf(var[0] / (float)a.D + a.eps);
    if (!have) return;
    if (a.stats && t == 0) {
        a.stats[row] = mean;
        a.stats[a.N + row] = rstd;
    }
    T *yp = reinterpret_cast<T *>(a.y) + row * a.ldy;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (t + k * a.tpr) * V;
        float w[V], b[V], y[V];
        if (a.w) load_piece<V>(reinterpret_cast<const TW *>(a.w) + c, a.D - c, w);
        if (a.b) load_piece<V>(reinterpret_cast<const TW *>(a.b) + c, a.D - c, b);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = fmaf((x[k][i] - mean) * rstd, a.w ? w[i] : 1.f, a.b ? b[i] : 0.f);
        store_piece<V>(yp + c, a.D - c, y);
    }
}

// Rows that do not fit the registers of a block: a block per row, which reads it again (from its XCD's L2) for each sum.
template <typename T, typename TW> __global__ __launch_bounds__(NT_LOOP) void norm_fwd_loop_kernel(const NormArgs a)
{
    constexpr int V = VEC<T>;
    __shared__ float red[2][NT_LOOP / 64][1];
    const long row = a.first + blockIdx.x;
    const T *xp = reinterpret_cast<const T *>(a.x) + row * a.ldx;
    const int first = threadIdx.x * V;
    constexpr int step = NT_LOOP * V;
    float sum[1] = {0.f}, var[1] = {0.f}, x[V];
    if (a.r) {
        const T *rp = reinterpret_cast<const T *>(a.r) + row * a.ldr;
        T *sp = reinterpret_cast<T *>(a.s) + row * a.lds;
        for (int c = first; c < a.D; c += step) {
            float r[V];
            load_piece<V>(xp + c, a.D - c, x);
            load_piece<V>(rp + c, a.D - c, r);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = (float)(T)(x[i] + r[i]);
            store_piece<V>(sp + c, a.D - c, x);
        }
        xp = sp;   // (a thread reads what it has written itself)
    }
    for (int c = first; c < a.D; c += step) {
        load_piece<V>(xp + c, a.D - c, x);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[0] += x[i];
    }
    row_sums<1>(sum, NT_LOOP, red[0]);
    const float mean = sum[0] / (float)a.D;
    for (int c = first; c < a.D; c += step) {
        load_piece<V>(xp + c, a.D - c, x);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float e = c + i < a.D ? x[i] - mean : 0.f;
            var[0] = fmaf(e, e, var[0]);
        }
    }
    row_sums<1>(var, NT_LOOP, red[1]);
    const float rstd = 1.f / sqrtf(var[0] / (float)a.D + a.eps);
    if (a.stats && threadIdx.x == 0) {
        a.stats[row] = mean;
        a.stats[a.N + row] = rstd;
    }
    T *yp = reinterpret_cast<T *>(a.y) + row * a.ldy;
    for (int c = first; c < a.D; c += step) {
        float w[V], b[V], y[V];
        load_piece<V>(xp + c, a.D - c, x);
        if (a.w) load_piece<V>(reinterpret_cast<const TW *>(a.w) + c, a.D - c, w);
        if (a.b) load_piece<V>(reinterpret_cast<const TW *>(a.b) + c, a.D - c, b);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = fmaf((x[i] - mean) * rstd, a.w ? w[i] : 1.f, a.b ? b[i] : 0.f);
        store_piece<V>(yp + c, a.D - c, y);
    }
}

template <typename T, typename TW, int NV> __global__ __launch_bounds__(NT) void norm_bwd_kernel(const NormArgs a)
{
    constexpr int V = VEC<T>;
    // Rows asked for one ahead in bf16 where the registers hold another (both launches for 110926 rows of 1803 368 us, without 403;
    // 59808 of 3344 273, 299; with NV = 4, 33333 of 6000, 576, 329).  Rows of a wavefront, which no barrier holds up, are the other
    // way about, by less: 262144 of 512 162, 152; 195312 of 1024 233, 232.  fp32 rows are twice as long: 77942 of 1283 238, 225.
    constexpr bool AHEAD = sizeof(T) == 2 && NV <= 2;
    __shared__ float red[2][NT / 64][2];
    extern __shared__ float sums[];   // with partial sums and rows of at most 64 threads: [wavefronts][tpr NV V]
    const int t = threadIdx.x & (a.tpr - 1), rows = NT / a.tpr;
    const float inv = 1.f / (float)a.D;
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (t + k * a.tpr) * V;
        if (a.w) load_piece<V>(reinterpret_cast<const TW *>(a.w) + c, a.D - c, w[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!a.w) w[k][i] = 1.f;
            dw[k][i] = db[k][i] = 0.f;
        }
    }
    const long stride = (long)gridDim.x * rows;
    Vec<T> ng[NV], nh[NV];   // the row at hand, or with AHEAD the next one
    float mean, rstd;
    auto ask = [&](long first) __attribute__((always_inline)) {
        const long at = min(first + threadIdx.x / a.tpr, a.N - 1);
        mean = a.stats[at];
        rstd = a.stats[a.N + at];
        const T *gp = reinterpret_cast<const T *>(a.x) + at * a.ldx, *sp = reinterpret_cast<const T *>(a.s) + at * a.lds;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (t + k * a.tpr) * V;
            load_piece(gp + c, a.D - c, ng[k]);
            load_piece(sp + c, a.D - c, nh[k]);
        }
    };
    if (AHEAD) ask((long)blockIdx.x * rows);
    int turn = 0;
    for (long first = (long)blockIdx.x * rows; first < a.N; first += stride, turn ^= 1) {
        const long row = first + threadIdx.x / a.tpr;
        const bool have = row < a.N;
        if (!AHEAD) ask(first);
        const float mu = mean, rs = rstd;
        float g[NV][V], h[NV][V], sum[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                g[k][i] = (float)ng[k][i];
                h[k][i] = (float)nh[k][i];
            }
        if (AHEAD && first + stride < a.N) ask(first + stride);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int n = a.D - (t + k * a.tpr) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                h[k][i] = i < n ? (h[k][i] - mu) * rs : 0.f;
                if (have) {
                    dw[k][i] = fmaf(g[k][i], h[k][i], dw[k][i]);
                    db[k][i] += g[k][i];
                }
                g[k][i] *= w[k][i];
                sum[0] += g[k][i];
                sum[1] = fmaf(g[k][i], h[k][i], sum[1]);
            }
        }
        row_sums<2>(sum, a.tpr, red[turn]);
        if (!have) continue;   // (the last round of a block; barriers are in row_sums alone, where one row is a block's)
        const float m0 = sum[0] * inv, m1 = sum[1] * inv;
        T *yp = reinterpret_cast<T *>(a.y) + row * a.ldy;
        const T *rp = reinterpret_cast<const T *>(a.r) + row * a.ldr;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (t + k * a.tpr) * V;
            float r[V], y[V];
            if (a.r) load_piece<V>(rp + c, a.D - c, r);
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = fmaf(rs, g[k][i] - m0 - h[k][i] * m1, a.r ? r[i] : 0.f);
            store_piece<V>(yp + c, a.D - c, y);
        }
    }
    if (!a.part) return;
    // the block's sums: over the rows of a wavefront by exchanges, over the wavefronts by LDS, in the order of the wavefronts
    float *out = a.part + (long)blockIdx.x * 2 * a.D;
    if (a.tpr <= 64) {
        const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, width = a.tpr * NV * V;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float(&v)[NV][V] = which ? db : dw;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    for (int s = a.tpr; s < 64; s <<= 1) v[k][i] += __shfl_xor(v[k][i], s);
                    if (lane < a.tpr) sums[wv * width + (t + k * a.tpr) * V + i] = v[k][i];
                }
            __syncthreads();
            for (int c = threadIdx.x; c < a.D; c += NT) {
                float x = sums[c];
#pragma unroll
                for (int i = 1; i < NT / 64; ++i) x += sums[i * width + c];
                out[which * a.D + c] = x;
            }
            __syncthreads();
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (t + k * a.tpr) * V;
            store_piece<V>(out + c, a.D - c, dw[k]);
            store_piece<V>(out + a.D + c, a.D - c, db[k]);
        }
    }
}

// Rows that do not fit registers: dX with a block per row, which is read twice, and the partial sums by columns.
template <typename T, typename TW> __global__ __launch_bounds__(NT_LOOP) void norm_bwd_loop_kernel(const NormArgs a)
{
    constexpr int V = VEC<T>;
    __shared__ float red[NT_LOOP / 64][2];
    const long row = a.first + blockIdx.x;
    const T *gp = reinterpret_cast<const T *>(a.x) + row * a.ldx, *sp = reinterpret_cast<const T *>(a.s) + row * a.lds;
    const float mean = a.stats[row], rstd = a.stats[a.N + row];
    const int first = threadIdx.x * V;
    constexpr int step = NT_LOOP * V;
    float sum[2] = {0.f, 0.f}, g[V], h[V], w[V];
    auto take = [&](int c) {
        load_piece<V>(gp + c, a.D - c, g);
        load_piece<V>(sp + c, a.D - c, h);
        if (a.w) load_piece<V>(reinterpret_cast<const TW *>(a.w) + c, a.D - c, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[i] = c + i < a.D ? (h[i] - mean) * rstd : 0.f;
            if (a.w) g[i] *= w[i];
        }
    };
    for (int c = first; c < a.D; c += step) {
        take(c);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sum[0] += g[i];
            sum[1] = fmaf(g[i], h[i], sum[1]);
        }
    }
    row_sums<2>(sum, NT_LOOP, red);
    const float m0 = sum[0] / (float)a.D, m1 = sum[1] / (float)a.D;
    T *yp = reinterpret_cast<T *>(a.y) + row * a.ldy;
    for (int c = first; c < a.D; c += step) {
        float r[V], y[V];
        take(c);
        if (a.r) load_piece<V>(reinterpret_cast<const T *>(a.r) + row * a.ldr + c, a.D - c, r);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = fmaf(rstd, g[i] - m0 - h[i] * m1, a.r ? r[i] : 0.f);
        store_piece<V>(yp + c, a.D - c, y);
    }
}
// partial sums of rows blockIdx.y, blockIdx.y + gridDim.y, ... of a block's columns
template <typename T> __global__ __launch_bounds__(NT) void norm_columns_kernel(const NormArgs a)
{
    constexpr int V = VEC<T>;
    const int c = (blockIdx.x * NT + threadIdx.x) * V;
    if (c >= a.D) return;
    float dw[V], db[V];
#pragma unroll
    for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.f;
    for (long row = blockIdx.y; row < a.N; row += gridDim.y) {
        const float mean = a.stats[row], rstd = a.stats[a.N + row];
        float g[V], s[V];
        load_piece<V>(reinterpret_cast<const T *>(a.x) + row * a.ldx + c, a.D - c, g);
        load_piece<V>(reinterpret_cast<const T *>(a.s) + row * a.lds + c, a.D - c, s);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            dw[i] = fmaf(g[i], (s[i] - mean) * rstd, dw[i]);
            db[i] += g[i];
        }
    }
    float *out = a.part + (long)blockIdx.y * 2 * a.D;
    store_piece<V>(out + c, a.D - c, dw);
    store_piece<V>(out + a.D + c, a.D - c, db);
}

// dweight, dbias = sums of the blocks' partial sums: 32 columns a block, every 32nd part a thread
constexpr int SUM_COLS = 32, SUM_THREADS = 1024;
template <typename TW> __global__ __launch_bounds__(SUM_THREADS) void norm_sum_kernel(const float *part, int parts, int D, TW *dw, TW *db)
{
    constexpr int SLICES = SUM_THREADS / SUM_COLS;
    __shared__ float red[SLICES][SUM_COLS + 1];
    const int col = threadIdx.x % SUM_COLS, slice = threadIdx.x / SUM_COLS, c = blockIdx.x * SUM_COLS + col;
    float x = 0.f;
    if (c < 2 * D) {
#pragma unroll 8
        for (int i = slice; i < parts; i += SLICES) x += part[(long)i * 2 * D + c];
    }
    red[slice][col] = x;
    __syncthreads();
    if (slice == 0 && c < 2 * D) {
        for (int i = 1; i < SLICES; ++i) x += red[i][col];
        TW *out = c < D ? dw : db;
        if (out) out[c < D ? c : c - D] = (TW)x;
    }
}

// ------------------------------------------------------------------ host side
inline int pow2_at_least(int n)
{
    int p = 1;
    while (p < n) p <<= 1;
    return p;
}
// Threads and pieces per thread of a row of `pieces`: a wavefront or less while that is at most wave_nv pieces a thread, else
// a block.  nv 0: the row does not fit (at most most_nv pieces a thread).
struct RowShape { int tpr, nv; };
inline RowShape row_shape(int pieces, int wave_nv, int most_nv)
{
    if (pieces <= 64 * wave_nv) {
        const int nv = pow2_at_least((pieces + 63) / 64);
        return {pow2_at_least((pieces + nv - 1) / nv), nv};
    }
    const int nv = pow2_at_least((pieces + NT - 1) / NT);
    return {NT, nv <= most_nv ? nv : 0};
}
constexpr int FWD_WAVE_NV = 4, FWD_NV = 8, BWD_WAVE_NV = 2;
template <typename T> constexpr int BWD_NV = 32 / VEC<T>;   // five arrays of 32 values in registers (fp32 rows of 6000: 237 us for 16666, by memory 420)

inline bool type_ok(int dtype) { return dtype == SKA_F32 || dtype == SKA_BF16; }
int check_rows(long long N, int D, int dtype, int wdtype)
{
    if (N < 0 || N > 0x7fffffffLL || D < 1) return SKA_EINVAL;
    if (D > 65536 || !type_ok(dtype) || !type_ok(wdtype)) return SKA_EUNSUPPORTED;
    return SKA_OK;
}
// row distance of an input (any, not negative) and of an output (rows apart)
inline bool in_ok(long long ld) { return ld >= 0; }
inline bool out_ok(long long ld, long long N, int D) { return ld >= 0 && (N <= 1 || ld >= D); }
inline int launched() { return hipGetLastError() == hipSuccess ? SKA_OK : SKA_EHIP; }
// Launches a kernel with `rows` rows to a block of `threads` for all rows, several times where that takes 2^32 threads or more: a
// launch is accepted with more, and runs their number modulo 2^32.
template <typename K> int for_all_rows(K kernel, NormArgs a, int rows, int threads, hipStream_t st)
{
    const long most = 0xffffffffL / threads;   // blocks of a launch
    for (long left = (a.N + rows - 1) / rows; left > 0; left -= most, a.first += most * rows) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(left < most ? left : most)), dim3(threads), 0, st, a);
        if (hipGetLastError() != hipSuccess) return SKA_EHIP;
    }
    return SKA_OK;
}

template <typename F> int with_types(int dtype, int wdtype, F f)
{
    if (dtype == SKA_F32) return wdtype == SKA_F32 ? f(0.f, 0.f) : f(0.f, __bf16{});
    return wdtype == SKA_F32 ? f(__bf16{}, 0.f) : f(__bf16{}, __bf16{});
}

template <typename T, typename TW> int norm_fwd(NormArgs a, hipStream_t st)
{
    const RowShape sh = row_shape((a.D + VEC<T> - 1) / VEC<T>, FWD_WAVE_NV, FWD_NV);
    if (!sh.nv) return for_all_rows(norm_fwd_loop_kernel<T, TW>, a, 1, NT_LOOP, st);
    a.tpr = sh.tpr;
    const int rows = NT / sh.tpr;
    switch (sh.nv) {
    case 1: return for_all_rows(norm_fwd_kernel<T, TW, 1>, a, rows, NT, st);
    case 2: return for_all_rows(norm_fwd_kernel<T, TW, 2>, a, rows, NT, st);
    case 4: return for_all_rows(norm_fwd_kernel<T, TW, 4>, a, rows, NT, st);
    default: return for_all_rows(norm_fwd_kernel<T, TW, 8>, a, rows, NT, st);
    }
}

template <typename T, typename TW> int norm_bwd(NormArgs a, TW *dw, TW *db, hipStream_t st)
{
    const RowShape sh = row_shape((a.D + VEC<T> - 1) / VEC<T>, BWD_WAVE_NV, BWD_NV<T>);
    int parts = 0;
    if (a.N && !sh.nv) {
        if (a.part) {
            const int cols = (a.D + NT * VEC<T> - 1) / (NT * VEC<T>);
            parts = (int)(a.N < MAX_BLOCKS / 4 ? a.N : MAX_BLOCKS / 4);
            hipLaunchKernelGGL((norm_columns_kernel<T>), dim3(cols, parts), dim3(NT), 0, st, a);   // (before dX, which may be dY)
        }
        const int rc = for_all_rows(norm_bwd_loop_kernel<T, TW>, a, 1, NT_LOOP, st);
        if (rc != SKA_OK) return rc;
    } else if (a.N) {
        a.tpr = sh.tpr;
        const int rows = NT / sh.tpr;
        const long blocks = (a.N + rows - 1) / rows;
        // as many as are there at a time, four a CU or what the registers allow (59808 rows of 3344, bf16, three a CU: 275 us, four:
        // 341; 39062 of 2560, fp32, 227, 267)
        const int values = sh.nv * VEC<T>, most = values <= 8 ? MAX_BLOCKS : values == 16 ? MAX_BLOCKS / 4 * 3 : MAX_BLOCKS / 2;
        parts = (int)(blocks < most ? blocks : most);
        const int lds = a.part && sh.tpr <= 64 ? NT / 64 * sh.tpr * sh.nv * VEC<T> * 4 : 0;
        switch (sh.nv) {
        case 1: hipLaunchKernelGGL((norm_bwd_kernel<T, TW, 1>), dim3(parts), dim3(NT), lds, st, a); break;
        case 2: hipLaunchKernelGGL((norm_bwd_kernel<T, TW, 2>), dim3(parts), dim3(NT), lds, st, a); break;
        case 4: hipLaunchKernelGGL((norm_bwd_kernel<T, TW, 4>), dim3(parts), dim3(NT), lds, st, a); break;
        default:
            if constexpr (BWD_NV<T> == 8) hipLaunchKernelGGL((norm_bwd_kernel<T, TW, 8>), dim3(parts), dim3(NT), lds, st, a);
        }
    }
    if (dw || db)
        hipLaunchKernelGGL((norm_sum_kernel<TW>), dim3((2 * a.D + SUM_COLS - 1) / SUM_COLS), dim3(SUM_THREADS), 0, st, a.part, parts, a.D, dw, db);
    return launched();
}

}  // namespace

extern "C" {

int ska_layer_norm_fwd(const void *X, long long ldx, const void *R, long long ldr, const void *weight, const void *bias, void *S,
                       long long lds, void *Y, long long ldy, float *stats, long long N, int D, float ln_eps, int dtype, int wdtype,
                       void *stream)
{
    if ((N > 0 && (!X || !Y || (R != nullptr) != (S != nullptr))) || !(ln_eps >= 0.f) || !isfinite(ln_eps)) return SKA_EINVAL;
    const int rc = check_rows(N, D, dtype, wdtype);
    if (rc != SKA_OK) return rc;
    if (!in_ok(ldx) || !out_ok(ldy, N, D) || (R && (!in_ok(ldr) || !out_ok(lds, N, D)))) return SKA_EINVAL;
    if (N == 0) return SKA_OK;
    const NormArgs a{X, R, weight, bias, S, Y, (long)ldx, (long)ldr, (long)lds, (long)ldy, stats, (long)N, 0, D, ln_eps, 0, nullptr};
    return with_types(dtype, wdtype, [&](auto t, auto w) { return norm_fwd<decltype(t), decltype(w)>(a, static_cast<hipStream_t>(stream)); });
}

size_t ska_layer_norm_workspace_bytes(long long N, int D)
{
    if (check_rows(N, D, SKA_F32, SKA_F32) != SKA_OK) return 0;
    return (size_t)(N < MAX_BLOCKS ? N : MAX_BLOCKS) * 2 * D * sizeof(float);
}

int ska_layer_norm_bwd(const void *dY, long long lddy, const void *S, long long lds, const void *weight, const float *stats,
                       const void *dS, long long ldds, void *dX, long long lddx, void *dweight, void *dbias, long long N, int D,
                       int dtype, int wdtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (N > 0 && (!dY || !S || !stats || !dX)) return SKA_EINVAL;
    const int rc = check_rows(N, D, dtype, wdtype);
    if (rc != SKA_OK) return rc;
    if (!in_ok(lddy) || !in_ok(lds) || (dS && !in_ok(ldds)) || !out_ok(lddx, N, D)) return SKA_EINVAL;
    const bool sums = dweight || dbias;
    if (sums && N > 0) {
        if (!workspace || workspace_bytes < ska_layer_norm_workspace_bytes(N, D)) return SKA_EWORKSPACE;
        if (reinterpret_cast<uintptr_t>(workspace) & 15) return SKA_EINVAL;
    }
    if (N == 0 && !sums) return SKA_OK;
    const NormArgs a{dY, dS, weight, nullptr, const_cast<void *>(S), dX, (long)lddy, (long)ldds, (long)lds, (long)lddx,
                     const_cast<float *>(stats), (long)N, 0, D, 0.f, 0, sums ? static_cast<float *>(workspace) : nullptr};
    return with_types(dtype, wdtype, [&](auto t, auto w) {
        using TW = decltype(w);
        return norm_bwd<decltype(t), TW>(a, static_cast<TW *>(dweight), static_cast<TW *>(dbias), static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
