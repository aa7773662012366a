// Rotary positions: the leading `dim` elements of each head as dim / 2 pairs, pair i of the row at position p turned by
// p f_i (or back, in the backward), all heads of Q and K in one launch.
//
// Bound by memory: every element is read and written once.  The angle does not depend on the head, so a work-group takes
// up to 16 rows of one batch item, forms their cosines and sines once in LDS (a product and a reduction in float64, which
// keeps angles up to 2^26 exact to float32, and one sine and cosine) and applies them to all heads.
#include "psa_vec.h"

namespace psa {

constexpr int kRotaryThreads = 256;
constexpr int kRotaryRows = 16;             // at the most

struct RotaryTurns { double f[32]; };          // turns (of 2 pi) per position of each pair

template <typename T>
struct RotaryHeads { const T* in; T* out; int64_t in_b, in_h, in_l, out_b, out_h, out_l; int H; };

// 8 x (8 + 8) x 2048, dim 64: bfloat16 12.4 us (5.4 TB/s), float32 23.5 (5.7).
//
// LAYOUT: psa_rotary_layout_t.  WIDE: dim / 2 is a multiple of the elements of 16 bytes (HALF), or dim of it (INTERLEAVED);
// else elements are taken one pair at a time, 2 or 4 bytes to an access (bfloat16, dim 62: 38 us, dim 24 by halves 37).
template <typename T, int LAYOUT, bool WIDE>
__global__ __launch_bounds__(kRotaryThreads)
void rotary_kernel(RotaryHeads<T> q, RotaryHeads<T> k, RotaryTurns turns, const int* __restrict__ positions, int64_t positions_stride,
                   int first, int dim, float magnitude, int L, int per)
{
    constexpr int VEC = kVec<T>;
    __shared__ float2 cs[kRotaryRows][32];
    const int b = blockIdx.y;
    const int l0 = blockIdx.x * per;
    const int rows = min(per, L - l0);
    const int half = dim / 2;
    for (int i = threadIdx.x; i < rows * 32; i += kRotaryThreads) {
        const int r = i >> 5, p = i & 31;
        if (p < half) {
            const int64_t pos = positions ? positions[b * positions_stride + l0 + r] : (int64_t)first + l0 + r;
            double t = (double)pos * turns.f[p];
            t -= rint(t);
            float sn, cn;
            sincospif(2.f * (float)t, &sn, &cn);
            cs[r][p] = make_float2(cn * magnitude, sn * magnitude);
        }
    }
    __syncthreads();
    const int H = q.H + k.H;
    // units of a head: VEC pairs (HALF: two vectors dim / 2 apart; INTERLEAVED: two vectors in a row) or one pair; then what is copied
    const int n_pair = WIDE ? (half + VEC - 1) / VEC : half;
    const int n_copy = 64 - dim;                               // elements, even
    const int n_unit = n_pair + (WIDE ? n_copy / VEC : n_copy / 2);
    const int n_item = H * rows * n_unit;
    for (int i = threadIdx.x; i < n_item; i += kRotaryThreads) {
        const int u = i % n_unit, hr = i / n_unit;
        const int r = hr % rows, hq = hr / rows;
        const bool is_q = hq < q.H;
        const int h = is_q ? hq : hq - q.H;
        const int64_t l = l0 + r;
        const T* in = is_q ? q.in + b * q.in_b + h * q.in_h + l * q.in_l : k.in + b * k.in_b + h * k.in_h + l * k.in_l;
        T* out = is_q ? q.out + b * q.out_b + h * q.out_h + l * q.out_l : k.out + b * k.out_b + h * k.out_h + l * k.out_l;
        if (WIDE) {
            if (u >= n_pair) {
                const int e = dim + (u - n_pair) * VEC;
                if (in + e != out + e) *reinterpret_cast<uint4*>(out + e) = *reinterpret_cast<const uint4*>(in + e);
            } else if (LAYOUT == PSA_ROTARY_HALF) {
                float a[VEC], c[VEC];
                load_vec(a, in + u * VEC, VEC);
                load_vec(c, in + half + u * VEC, VEC);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float2 w = cs[r][u * VEC + j];
                    const float x = a[j], y = c[j];
                    a[j] = x * w.x - y * w.y;
                    c[j] = x * w.y + y * w.x;
                }
                store_vec(out + u * VEC, a, VEC);
                store_vec(out + half + u * VEC, c, VEC);
            } else {
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const int e = (2 * u + v) * VEC;
                    if (e < dim) {
                        float a[VEC];
                        load_vec(a, in + e, VEC);
#pragma unroll
                        for (int j = 0; j < VEC; j += 2) {
                            const float2 w = cs[r][(e + j) / 2];
                            const float x = a[j], y = a[j + 1];
                            a[j] = x * w.x - y * w.y;
                            a[j + 1] = x * w.y + y * w.x;
                        }
                        store_vec(out + e, a, VEC);
                    }
                }
            }
        } else {
            if (u >= n_pair) {
                const int e = dim + (u - n_pair) * 2;
                const T x = in[e], y = in[e + 1];
                out[e] = x;
                out[e + 1] = y;
            } else {
                const int e0 = LAYOUT == PSA_ROTARY_HALF ? u : 2 * u, e1 = LAYOUT == PSA_ROTARY_HALF ? u + half : 2 * u + 1;
                const float x = to_f32(in[e0]), y = to_f32(in[e1]);
                const float2 w = cs[r][u];
                from_f32(out[e0], x * w.x - y * w.y);
                from_f32(out[e1], x * w.y + y * w.x);
            }
        }
    }
}

template <typename T>
static RotaryHeads<T> rotary_heads(const psa_heads_t* in, const psa_heads_t* out, int H)
{
    if (!in) return RotaryHeads<T>{nullptr, nullptr, 0, 0, 0, 0, 0, 0, 0};
    return RotaryHeads<T>{static_cast<const T*>(in->data), static_cast<T*>(out->data), in->batch_stride, in->head_stride, in->row_stride,
                          out->batch_stride, out->head_stride, out->row_stride, H};
}
template <typename T>
static void rotary_go(const psa_heads_t* Q, const psa_heads_t* K, int H_kv, const psa_rotary_t& o, const double* freq, bool back,
                      const int* positions, int64_t positions_stride, int first, const psa_heads_t* Qo, const psa_heads_t* Ko,
                      const psa_shape_t& s, hipStream_t stream)
{
    RotaryTurns turns{};
    for (int i = 0; i < o.dim / 2; ++i) turns.f[i] = (back ? -freq[i] : freq[i]) * 0.15915494309189533577;
    const auto q = rotary_heads<T>(Q, Qo, s.H);
    const auto k = rotary_heads<T>(K, Ko, H_kv);
    // rows to a work-group: 16, or fewer where there would not be two work-groups to a compute unit (B=1, L=333, 6 heads: 6.7 -> 3.7 us)
    int per = kRotaryRows;
    while (per > 1 && (int64_t)s.B * ((s.L_K + per - 1) / per) < 512) per /= 2;
    const dim3 grid((unsigned)((s.L_K + per - 1) / per), (unsigned)s.B);
    const bool half = o.layout == PSA_ROTARY_HALF;
    const bool wide = (half ? o.dim / 2 : o.dim) % kVec<T> == 0;
    const float mag = (float)o.magnitude;
    if (half && wide) rotary_kernel<T, PSA_ROTARY_HALF, true><<<grid, kRotaryThreads, 0, stream>>>(q, k, turns, positions, positions_stride, first, o.dim, mag, s.L_K, per);
    else if (half) rotary_kernel<T, PSA_ROTARY_HALF, false><<<grid, kRotaryThreads, 0, stream>>>(q, k, turns, positions, positions_stride, first, o.dim, mag, s.L_K, per);
    else if (wide) rotary_kernel<T, PSA_ROTARY_INTERLEAVED, true><<<grid, kRotaryThreads, 0, stream>>>(q, k, turns, positions, positions_stride, first, o.dim, mag, s.L_K, per);
    else rotary_kernel<T, PSA_ROTARY_INTERLEAVED, false><<<grid, kRotaryThreads, 0, stream>>>(q, k, turns, positions, positions_stride, first, o.dim, mag, s.L_K, per);
}
hipError_t launch_rotary(const psa_heads_t* Q, const psa_heads_t* K, int H_kv, const psa_rotary_t& o, const double* freq, bool back,
                         const int* positions, int64_t positions_stride, int first, const psa_heads_t* Qo, const psa_heads_t* Ko,
                         const psa_shape_t& s, hipStream_t stream)
{
    if (s.dtype == PSA_F32) rotary_go<float>(Q, K, H_kv, o, freq, back, positions, positions_stride, first, Qo, Ko, s, stream);
    else rotary_go<bf16_t>(Q, K, H_kv, o, freq, back, positions, positions_stride, first, Qo, Ko, s, stream);
    return hipGetLastError();
}

}  // namespace psa
