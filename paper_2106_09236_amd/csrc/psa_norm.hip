// Layer norm over the rows of X [rows, cols] and its gradients.
//
//   Y = (X - mean) rstd gamma + beta,  rstd = 1 / sqrt(mean((X - mean)^2) + eps)
//   g = dY gamma,  xhat = (X - mean) rstd:
//   dX = rstd (g - mean(g) - xhat mean(g xhat)),  dgamma = sum_rows dY xhat,  dbeta = sum_rows dY
//
// Both are bound by memory: a row is read once, kept in registers while its sums are formed, and written once.  TPR
// threads share a row (a part of a wave, a wave, or a work-group of 256), each with NV vectors of 16 bytes, so that a
// short row does not leave lanes idle and a long one still fits; rows beyond that are read three times, the second and
// third out of the cache.
//
// Sums are float32.  The mean m0 of the first pass is off by its rounding, which for rows far from zero is not small
// against their spread, so the deviations d = x - m0 are summed beside their squares: mean = m0 + mean(d), var =
// mean(d^2) - mean(d)^2, where mean(d) is tiny and nothing cancels.  The backward does the same for the mean it is given.
#include "psa_vec.h"

namespace psa {

constexpr int kNormThreads = 256;
constexpr int kNormMaxCols = 8192;         // longest row that is kept: 32 elements to each of 256 threads

// Sums of N values over the TPR threads of a row, in all of them.  TPR = 256: through LDS, s holds 4 N floats.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* s)
{
#pragma unroll
    for (int k = 1; k < (TPR < 64 ? TPR : 64); k *= 2)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], k, 64);
    if (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();                   // the sums before these have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) s[wave * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (s[i] + s[N + i]) + (s[2 * N + i] + s[3 * N + i]);
    }
}

template <typename T, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads)
void norm_fwd_kernel(const T* X, const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                     T* Y, float* __restrict__ mean_out, float* __restrict__ rstd_out, int64_t rows, int cols)
{
    constexpr int VEC = kVec<T>;
    __shared__ float s[8];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (kNormThreads / TPR) + threadIdx.x / TPR;
    if (TPR <= 64 && row >= rows) return;              // (a whole group of TPR lanes; TPR = 256: one row to a work-group)
    const T* x = X + row * cols;
    float v[NV][VEC];
    float sum[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + t) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[k][i] = 0.f;
        if (c < cols) load_vec(v[k], x + c, cols - c);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[0] += v[k][i];
    }
    row_sum<TPR>(sum, s);
    const float inv = 1.f / (float)cols;
    const float m0 = sum[0] * inv;
    float dev[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + t) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float d = v[k][i] - m0;
            v[k][i] = d;
            if (c + i < cols) { dev[0] += d; dev[1] += d * d; }
        }
    }
    row_sum<TPR>(dev, s);
    const float off = dev[0] * inv;
    const float var = fmaxf(dev[1] * inv - off * off, 0.f);
    const float rstd = 1.f / sqrtf(var + eps);
    if (t == 0 && mean_out) { mean_out[row] = m0 + off; rstd_out[row] = rstd; }
    T* y = Y + row * cols;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + t) * VEC;
        if (c >= cols) continue;
        float g[VEC], b[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) { g[i] = 1.f; b[i] = 0.f; }
        if (gamma) load_vec(g, gamma + c, cols - c);
        if (beta) load_vec(b, beta + c, cols - c);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[k][i] = fmaf((v[k][i] - off) * rstd, g[i], b[i]);
        store_vec(y + c, v[k], cols - c);
    }
}

// Rows of any length, a work-group each: the row is read again for each step instead of kept.  kNormLongGroups work-groups at the most, which take
// several rows then: a launch has fewer than 2^32 threads.
constexpr int kNormLongGroups = 1 << 17;
template <typename T>
__global__ __launch_bounds__(kNormThreads)
void norm_fwd_long_kernel(const T* X, const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                          T* Y, float* __restrict__ mean_out, float* __restrict__ rstd_out, int64_t rows, int cols)
{
    constexpr int VEC = kVec<T>;
    __shared__ float s[8];
    const float inv = 1.f / (float)cols;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* x = X + row * cols;
        float v[VEC];
        float sum[1] = {0.f};
        for (int c = threadIdx.x * VEC; c < cols; c += kNormThreads * VEC) {
            load_vec(v, x + c, cols - c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[0] += v[i];
        }
        row_sum<kNormThreads>(sum, s);
        const float m0 = sum[0] * inv;
        float dev[2] = {0.f, 0.f};
        for (int c = threadIdx.x * VEC; c < cols; c += kNormThreads * VEC) {
            load_vec(v, x + c, cols - c);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (c + i < cols) { const float d = v[i] - m0; dev[0] += d; dev[1] += d * d; }
        }
        row_sum<kNormThreads>(dev, s);
        const float off = dev[0] * inv;
        const float rstd = 1.f / sqrtf(fmaxf(dev[1] * inv - off * off, 0.f) + eps);
        if (threadIdx.x == 0 && mean_out) { mean_out[row] = m0 + off; rstd_out[row] = rstd; }
        T* y = Y + row * cols;
        for (int c = threadIdx.x * VEC; c < cols; c += kNormThreads * VEC) {
            float g[VEC], b[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) { g[i] = 1.f; b[i] = 0.f; }
            load_vec(v, x + c, cols - c);              // (Y may be X: a thread reads what it writes)
            if (gamma) load_vec(g, gamma + c, cols - c);
            if (beta) load_vec(b, beta + c, cols - c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = fmaf((v[i] - m0 - off) * rstd, g[i], b[i]);
            store_vec(y + c, v, cols - c);
        }
    }
}

// ---- backward.  A work-group walks rows blockIdx.x * RPW, + gridDim.x * RPW, ... (RPW = 256 / TPR at a time); its
// threads keep the sums over those rows of dY xhat and dY for the columns they hold, and the work-group leaves one
// partial row of each in `part` [gridDim.x, 2, cols].  norm_sum_kernel adds the partial rows: two launches, no atomics,
// the same order every time.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads)
void norm_bwd_kernel(const T* __restrict__ dY, const T* __restrict__ X, const T* __restrict__ gamma, const float* __restrict__ mean,
                     const float* __restrict__ rstd_in, T* __restrict__ dX, float* __restrict__ part, int64_t rows, int cols)
{
    constexpr int VEC = kVec<T>, RPW = kNormThreads / TPR;
    constexpr int W = TPR * NV * VEC;                  // columns the threads of a row cover
    __shared__ float s[TPR > 64 ? 12 : 1];
    __shared__ float col[RPW > 1 ? RPW / 2 * W : 1];   // column sums of half of the work-group's rows
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float sg[NV][VEC], sb[NV][VEC], w[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TPR + t) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) { sg[k][i] = sb[k][i] = 0.f; w[k][i] = 1.f; }
        if (gamma && c < cols) load_vec(w[k], gamma + c, cols - c);
    }
    const float inv = 1.f / (float)cols;
    // the next row is asked for before this one is used (131072 x 512 bfloat16, without / with: 112 / 77 us, 5.2 TB/s)
    Chunk<T> xr[NV], gr[NV];
    float m_next = 0.f, r_next = 0.f;
    auto fetch = [&](int64_t row) {
        m_next = mean[row];
        r_next = rstd_in[row];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
            if (c < cols) {
                xr[k] = load_chunk(X + row * cols + c, cols - c);
                gr[k] = load_chunk(dY + row * cols + c, cols - c);
            }
        }
    };
    const int64_t step = (int64_t)gridDim.x * RPW;
    int64_t row = (int64_t)blockIdx.x * RPW + slot;
    if (row < rows) fetch(row);
    for (; row < rows; row += step) {
        const float m = m_next, rstd = r_next;
        float d[NV][VEC], g[NV][VEC];
        float sum[3] = {0.f, 0.f, 0.f};                // of d = x - mean, of g, of g d
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) { d[k][i] = 0.f; g[k][i] = 0.f; }
            if (c < cols) { unpack(xr[k].w, d[k], T{}); unpack(gr[k].w, g[k], T{}); }
        }
        if (row + step < rows) fetch(row + step);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                d[k][i] = c + i < cols ? d[k][i] - m : 0.f;
                sum[0] += d[k][i];
                const float gw = g[k][i] * w[k][i];
                sum[1] += gw;
                sum[2] = fmaf(gw, d[k][i], sum[2]);
            }
        }
        row_sum<TPR>(sum, s);
        const float off = sum[0] * inv;                // what the rounded mean is off by
        const float c1 = sum[1] * inv;
        const float c2 = (sum[2] - off * sum[1]) * rstd * inv;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float xhat = (d[k][i] - off) * rstd;
                sg[k][i] = fmaf(g[k][i], xhat, sg[k][i]);
                sb[k][i] += g[k][i];
                d[k][i] = rstd * (g[k][i] * w[k][i] - c1 - xhat * c2);
            }
            if (c < cols) store_vec(dX + row * cols + c, d[k], cols - c);
        }
    }
    if (!part) return;
    // sums over the slots of the work-group, halving: slot j + half hands its sums to slot j
    for (int half = RPW / 2; half > 0; half /= 2) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int e = ((k * VEC + i) * TPR) + t;       // a lane's elements TPR apart: no bank conflicts
                    float& mine = which ? sb[k][i] : sg[k][i];
                    if (slot >= half && slot < 2 * half) col[(slot - half) * W + e] = mine;
                }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int e = ((k * VEC + i) * TPR) + t;
                    float& mine = which ? sb[k][i] : sg[k][i];
                    if (slot < half) mine += col[slot * W + e];
                }
        }
    }
    if (slot == 0) {
        float* pg = part + (size_t)blockIdx.x * 2 * cols;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TPR + t) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (c + i < cols) { pg[c + i] = sg[k][i]; pg[cols + c + i] = sb[k][i]; }
        }
    }
}

// Rows of any length: dX as above with the row read again (work-groups as in the forward), and the column sums in a kernel of their own.
template <typename T>
__global__ __launch_bounds__(kNormThreads)
void norm_bwd_long_kernel(const T* __restrict__ dY, const T* __restrict__ X, const T* __restrict__ gamma, const float* __restrict__ mean,
                          float* __restrict__ off_out, const float* __restrict__ rstd_in, T* __restrict__ dX, int64_t rows, int cols)
{
    constexpr int VEC = kVec<T>;
    __shared__ float s[12];
    const float inv = 1.f / (float)cols;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* x = X + row * cols;
        const T* dy = dY + row * cols;
        const float m = mean[row], rstd = rstd_in[row];
        float sum[3] = {0.f, 0.f, 0.f};
        for (int c = threadIdx.x * VEC; c < cols; c += kNormThreads * VEC) {
            float d[VEC], g[VEC], w[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = 1.f;
            load_vec(d, x + c, cols - c);
            load_vec(g, dy + c, cols - c);
            if (gamma) load_vec(w, gamma + c, cols - c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float dev = c + i < cols ? d[i] - m : 0.f, gw = g[i] * w[i];
                sum[0] += dev;
                sum[1] += gw;
                sum[2] = fmaf(gw, dev, sum[2]);
            }
        }
        row_sum<kNormThreads>(sum, s);
        const float off = sum[0] * inv, c1 = sum[1] * inv, c2 = (sum[2] - off * sum[1]) * rstd * inv;
        if (threadIdx.x == 0 && off_out) off_out[row] = off;
        for (int c = threadIdx.x * VEC; c < cols; c += kNormThreads * VEC) {
            float d[VEC], g[VEC], w[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = 1.f;
            load_vec(d, x + c, cols - c);
            load_vec(g, dy + c, cols - c);
            if (gamma) load_vec(w, gamma + c, cols - c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) d[i] = rstd * (g[i] * w[i] - c1 - (d[i] - m - off) * rstd * c2);
            store_vec(dX + row * cols + c, d, cols - c);
        }
    }
}
// Column sums of the rows blockIdx.y * per .. + per, a vector of columns to a thread.
template <typename T>
__global__ __launch_bounds__(64)
void norm_cols_kernel(const T* __restrict__ dY, const T* __restrict__ X, const float* __restrict__ mean,
                      const float* __restrict__ off, const float* __restrict__ rstd, float* __restrict__ part,
                      int64_t rows, int cols, int64_t per)
{
    constexpr int VEC = kVec<T>;
    const int c = (blockIdx.x * 64 + threadIdx.x) * VEC;
    if (c >= cols) return;
    float sg[VEC], sb[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sg[i] = sb[i] = 0.f;
    const int64_t last = min(rows, (int64_t)(blockIdx.y + 1) * per);
    for (int64_t row = (int64_t)blockIdx.y * per; row < last; ++row) {
        float x[VEC], g[VEC];
        load_vec(x, X + row * cols + c, cols - c);
        load_vec(g, dY + row * cols + c, cols - c);
        const float m = mean[row], o = off[row], r = rstd[row];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            sg[i] = fmaf(g[i], (x[i] - m - o) * r, sg[i]);
            sb[i] += g[i];
        }
    }
    float* pg = part + (size_t)blockIdx.y * 2 * cols;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        if (c + i < cols) { pg[c + i] = sg[i]; pg[cols + c + i] = sb[i]; }
}

// dgamma and dbeta: the sums of n (at most 1024) partial rows of 2 cols floats; 16 columns to a work-group, every 64th row to a
// thread, so that all of its loads are in flight at once and there are enough work-groups for short rows (32 columns and every
// eighth row: 39 us for 1024 x 1024 floats; so: 5.0 us).
constexpr int kNormParts = 1024;
__global__ __launch_bounds__(1024)
void norm_sum_kernel(const float* __restrict__ part, int n, int cols, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    constexpr int PER = kNormParts / 64;
    __shared__ float s[64][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t width = 2 * (int64_t)cols, c = (int64_t)blockIdx.x * 16 + x;
    float v[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int r = y + 64 * k;
        v[k] = r < n && c < width ? part[(size_t)r * width + c] : 0.f;
    }
#pragma unroll
    for (int h = PER / 2; h > 0; h /= 2)
#pragma unroll
        for (int k = 0; k < h; ++k) v[k] += v[k + h];
    s[y][x] = v[0];
    __syncthreads();
    if (y < 8) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += s[y + 8 * k][x];
        s[y][x] = t;              // (row y belongs to this thread from here on)
    }
    __syncthreads();
    if (y == 0 && c < width) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += s[k][x];
        if (c < cols) dgamma[c] = t; else dbeta[c - cols] = t;
    }
}

// How a row of `cols` elements is shared: TPR threads with NV vectors each, or (nv = 0) the kernels for long rows.  One vector to a
// thread while a wave covers the row.  The forward takes two where there are many rows: the latency of a row's reductions is hidden by
// others and two rows to a wave keep more loads in flight.  1 | 2, a call among others: bfloat16 x 512, 16384 rows 9.9 | 10.0 us, 32768 16.1 | 14.8, 65536
// 28.6 | 24.2, 131072 60.1 | 53.0, 131072 x 300 71 | 51; float32 x 256, 18000 11.1 | 12.4, 32768 15.2 | 16.5, 65536 26.0 | 27.9, 131072 58.0 | 56.7, 262144
// 117 | 114.5; one row 2.3 | 3.1.  The backward, which asks for the next row ahead, does not (131072 x 512 bfloat16 75 | 90 us).
struct NormShape { int tpr, nv; };
static NormShape norm_shape(int64_t rows, int cols, int dtype, bool forward)
{
    const int vec = dtype == PSA_F32 ? 4 : 8;
    const int chunks = (cols + vec - 1) / vec;
    int tpr = chunks <= 16 ? 16 : chunks <= 32 ? 32 : chunks <= 64 * 4 ? 64 : 256;
    if (forward && tpr == 64 && chunks <= 64 && rows >= (dtype == PSA_F32 ? 131072 : 32768)) tpr = 32;
    int nv = 1;
    while (nv * tpr < chunks) nv *= 2;
    return NormShape{tpr, cols <= kNormMaxCols ? nv : 0};
}

NormPlan make_norm_plan(int64_t rows, int cols, int dtype, bool forward)
{
    const NormShape sh = norm_shape(rows, cols, dtype, forward);
    NormPlan p{};
    p.tpr = sh.tpr; p.nv = sh.nv;
    if (sh.nv) {
        const int64_t groups = (rows + kNormThreads / sh.tpr - 1) / (kNormThreads / sh.tpr);
        p.n_part = (int)(groups < kNormParts ? groups : kNormParts);
    } else {
        p.n_part = (int)(rows < 64 ? rows : 64);
    }
    p.off_part = sh.nv ? 0 : ((size_t)rows * sizeof(float) + 255) & ~(size_t)255;
    p.total = p.off_part + (((size_t)p.n_part * 2 * (size_t)cols * sizeof(float) + 255) & ~(size_t)255);
    return p;
}

static unsigned norm_long_groups(int64_t rows) { return (unsigned)(rows < kNormLongGroups ? rows : kNormLongGroups); }

template <typename T, int TPR, int NV>
static void norm_fwd_go(const void* X, const void* gamma, const void* beta, float eps, void* Y, float* mean, float* rstd,
                        int64_t rows, int cols, hipStream_t stream)
{
    constexpr int64_t kMost = (int64_t)(1 << 23) * (kNormThreads / TPR);       // rows of a launch, which has fewer than 2^32 threads
    for (int64_t r0 = 0; r0 < rows; r0 += kMost) {
        const int64_t n = rows - r0 < kMost ? rows - r0 : kMost, grid = (n + kNormThreads / TPR - 1) / (kNormThreads / TPR);
        norm_fwd_kernel<T, TPR, NV><<<(unsigned)grid, kNormThreads, 0, stream>>>(
            static_cast<const T*>(X) + r0 * cols, static_cast<const T*>(gamma), static_cast<const T*>(beta), eps, static_cast<T*>(Y) + r0 * cols,
            mean ? mean + r0 : nullptr, rstd ? rstd + r0 : nullptr, n, cols);
    }
}
template <typename T>
static void norm_fwd_pick(const NormPlan& p, const void* X, const void* gamma, const void* beta, float eps, void* Y, float* mean,
                          float* rstd, int64_t rows, int cols, hipStream_t stream)
{
    switch (p.nv ? p.tpr * 16 + p.nv : 0) {
        case 16 * 16 + 1:  return norm_fwd_go<T, 16, 1>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 32 * 16 + 1:  return norm_fwd_go<T, 32, 1>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 32 * 16 + 2:  return norm_fwd_go<T, 32, 2>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 64 * 16 + 1:  return norm_fwd_go<T, 64, 1>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 64 * 16 + 2:  return norm_fwd_go<T, 64, 2>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 64 * 16 + 4:  return norm_fwd_go<T, 64, 4>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 256 * 16 + 2: return norm_fwd_go<T, 256, 2>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 256 * 16 + 4: return norm_fwd_go<T, 256, 4>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        case 256 * 16 + 8: return norm_fwd_go<T, 256, kVec<T> == 4 ? 8 : 4>(X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
        default:
            norm_fwd_long_kernel<T><<<norm_long_groups(rows), kNormThreads, 0, stream>>>(
                static_cast<const T*>(X), static_cast<const T*>(gamma), static_cast<const T*>(beta), eps, static_cast<T*>(Y), mean, rstd, rows, cols);
    }
}
hipError_t launch_norm_fwd(const NormPlan& p, const void* X, const void* gamma, const void* beta, float eps, void* Y, float* mean,
                           float* rstd, int64_t rows, int cols, int dtype, hipStream_t stream)
{
    if (dtype == PSA_F32) norm_fwd_pick<float>(p, X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
    else norm_fwd_pick<bf16_t>(p, X, gamma, beta, eps, Y, mean, rstd, rows, cols, stream);
    return hipGetLastError();
}

template <typename T, int TPR, int NV>
static void norm_bwd_go(const NormPlan& p, const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd,
                        void* dX, float* part, int64_t rows, int cols, hipStream_t stream)
{
    norm_bwd_kernel<T, TPR, NV><<<(unsigned)p.n_part, kNormThreads, 0, stream>>>(
        static_cast<const T*>(dY), static_cast<const T*>(X), static_cast<const T*>(gamma), mean, rstd, static_cast<T*>(dX), part, rows, cols);
}
template <typename T>
static void norm_bwd_pick(const NormPlan& p, const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd,
                          void* dX, float* part, float* off, int64_t rows, int cols, hipStream_t stream)
{
    switch (p.nv ? p.tpr * 16 + p.nv : 0) {
        case 16 * 16 + 1:  return norm_bwd_go<T, 16, 1>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        case 32 * 16 + 1:  return norm_bwd_go<T, 32, 1>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        case 64 * 16 + 1:  return norm_bwd_go<T, 64, 1>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        case 64 * 16 + 2:  return norm_bwd_go<T, 64, 2>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        case 64 * 16 + 4:  return norm_bwd_go<T, 64, 4>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        case 256 * 16 + 2: return norm_bwd_go<T, 256, 2>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        case 256 * 16 + 4: return norm_bwd_go<T, 256, 4>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        case 256 * 16 + 8: return norm_bwd_go<T, 256, kVec<T> == 4 ? 8 : 4>(p, dY, X, gamma, mean, rstd, dX, part, rows, cols, stream);
        default: {
            const T *dy = static_cast<const T*>(dY), *x = static_cast<const T*>(X);
            // (the row kernel leaves what the rounded means are off by for the column sums)
            norm_bwd_long_kernel<T><<<norm_long_groups(rows), kNormThreads, 0, stream>>>(dy, x, static_cast<const T*>(gamma), mean, part ? off : nullptr,
                                                                                         rstd, static_cast<T*>(dX), rows, cols);
            if (!part) return;
            const int64_t per = (rows + p.n_part - 1) / p.n_part;
            norm_cols_kernel<T><<<dim3((unsigned)((cols + 64 * kVec<T> - 1) / (64 * kVec<T>)), (unsigned)p.n_part), 64, 0, stream>>>(
                dy, x, mean, off, rstd, part, rows, cols, per);
        }
    }
}
hipError_t launch_norm_bwd(const NormPlan& p, const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd,
                           void* dX, float* dgamma, float* dbeta, int64_t rows, int cols, int dtype, void* workspace, hipStream_t stream)
{
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    float* off = reinterpret_cast<float*>(ws);
    float* part = dgamma ? reinterpret_cast<float*>(ws + p.off_part) : nullptr;
    if (dtype == PSA_F32) norm_bwd_pick<float>(p, dY, X, gamma, mean, rstd, dX, part, off, rows, cols, stream);
    else norm_bwd_pick<bf16_t>(p, dY, X, gamma, mean, rstd, dX, part, off, rows, cols, stream);
    if (part) norm_sum_kernel<<<(unsigned)((2 * (int64_t)cols + 15) / 16), 1024, 0, stream>>>(part, p.n_part, cols, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace psa
