// Dense attention over packed sequences, forward: softmax(scale Q K^T) V row by row, the keys of a sequence in one pass with
// the running maximum and sum of online softmax.
//
// Bound by the matrix units and, in bfloat16, as much by the vector unit: a head of 64 elements has 256 flops of products
// to a weight, whose exponential, maximum, sum and rounding take as long.
#include "psa_packed.h"

namespace psa {

// What a wave keeps for 32 rows: running maximum (in base 2, scaled), sum and the output's accumulators.
struct Rows32 {
    float m, l;
    floatx16 o[2];                         // element 32 dt + acc_row(r, h) of row c in o[dt][r]
    __device__ __forceinline__ void init() { m = kMaxInit; l = 0.f; clear(o[0]); clear(o[1]); }
    // Scores of N x 32 keys to weights; the constant that is subtracted follows the maximum only when that has grown by
    // more than 2^8 (kLagLog2): weights up to 2^8 are as exact as weights up to 1, and a change scales 32 accumulators.
    template <int N>
    __device__ __forceinline__ void weights(floatx16 (&s)[N], float scale) {
        float t = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) t = fmaxf(t, s[n][r]);
        t = max_xor32(t) * scale;
        const float m_new = t > m + kLagLog2 ? t : m;
        const float alpha = fast_exp2(m - m_new);
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) { s[n][r] = fast_exp2(fmaf(s[n][r], scale, -m_new)); sum += s[n][r]; }
        l = l * alpha + sum;
        if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {
#pragma unroll
            for (int dt = 0; dt < 2; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
        }
        m = m_new;
    }
    // The infinities and NaN of V rows j0 .. j0 + n - 1 that were left out of the tile: to the rows that see them.
    template <typename T>
    __device__ __forceinline__ void add_nonfinite(const T* v, int64_t row_stride, int n, int n_vis, int h) {
        for (int j = 0; j < n; ++j)
#pragma unroll
            for (int dt = 0; dt < 2; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float x = to_f32(v[j * row_stride + 32 * dt + acc_row(r, h)]);
                    if (j < n_vis && !isfinite(x)) o[dt][r] += x;
                }
    }
};

// 4 waves of 32 rows each; tiles of KT keys and values go through LDS, the next tile's rows are on their way meanwhile.
template <typename T, int KT>
__global__ __launch_bounds__(256)
void packed_rows_kernel(Heads<const T> Q, Heads<const T> K, Heads<const T> V, Packing p, Heads<T> out, float* __restrict__ lse,
                        int H_kv, int causal, float scale, int n_tile)
{
    constexpr int CH = 64 * sizeof(T) / 16;            // 16-byte chunks of a row
    constexpr int NL = KT * CH / 256;                  // of a tile, to a thread
    constexpr int kTileBytes = KT * LdsTile<T>::kRowBytes;
    __shared__ __attribute__((aligned(16))) unsigned char sK[2][kTileBytes], sV[2][kTileBytes];
    __shared__ int s_bad[2][4];
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    zero_outside(out, p.qo, p.B, p.Tq, hk * p.G, p.G, x, n_tile, [&](int head, int row) { if (lse) lse[(int64_t)head * p.Tq + row] = -INFINITY; });
    const SeqTile f = find_tile<128, false>(p, x);
    if (f.tile < 0) return;

    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;                 // causal: query t sees the first t + shift keys
    auto visible = [&](int r) { const int t = r / p.G; return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int row = f.tile * 128 + wave * 32 + c, rc = min(row, n_rows - 1);
    const int t = rc / p.G, head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int n_all = __builtin_amdgcn_readfirstlane(visible(min(f.tile * 128 + 127, n_rows - 1)));         // keys any row of the work-group sees
    const int n_every = __builtin_amdgcn_readfirstlane(visible(f.tile * 128));                              // ... and those that all see
    const int row0 = f.tile * 128 + wave * 32;
    const int n_wave = __builtin_amdgcn_readfirstlane(row0 < n_rows ? visible(min(row0 + 31, n_rows - 1)) : 0);
    const int n_wave_every = __builtin_amdgcn_readfirstlane(visible(min(row0, n_rows - 1)));

    ColOperand<T> q;
    q.load(Q.at(head, f.q0 + t), h);
    const T* Kh = K.at(hk, f.k0);
    const T* Vh = V.at(hk, f.k0);
    int k_ofs[NL], v_ofs[NL], s_ofs[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int id = i * 256 + tid, r = id / CH, ch = id % CH;
        k_ofs[i] = (int)(r * K.row * (int64_t)sizeof(T)) + ch * 16;
        v_ofs[i] = (int)(r * V.row * (int64_t)sizeof(T)) + ch * 16;
        s_ofs[i] = LdsTile<T>::chunk_at(r, ch);
    }
    uint4 kr[NL], vr[NL];
    auto fetch = [&](int j0) {
        const int n = min(KT, f.nk - j0);
        const auto kb = tile_rows(Kh + j0 * K.row, K.row, n), vb = tile_rows(Vh + j0 * V.row, V.row, n);
#pragma unroll
        for (int i = 0; i < NL; ++i) { kr[i] = buffer_load16<uint4>(kb, k_ofs[i]); vr[i] = buffer_load16<uint4>(vb, v_ofs[i]); }
    };
    Rows32 acc;
    acc.init();
    if (n_all > 0) fetch(0);
    int buf = 0;
    for (int j0 = 0; j0 < n_all; j0 += KT, buf ^= 1) {
        // a weight of 0 does not keep an infinity or NaN of a value that a row does not see out of its sum: in tiles that
        // some row sees in part they are left out and added afterwards
        const bool part = j0 + KT > n_every;
        if (part) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < NL; ++i) bad |= nonfinite(vr[i], T{});
            const bool any = __builtin_amdgcn_ballot_w64(bad) != 0;
            if (lane == 0) s_bad[buf][wave] = any;
            if (any)
#pragma unroll
                for (int i = 0; i < NL; ++i) vr[i] = finite_only(vr[i], T{});
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            *reinterpret_cast<uint4*>(sK[buf] + s_ofs[i]) = kr[i];
            *reinterpret_cast<uint4*>(sV[buf] + s_ofs[i]) = vr[i];
        }
        if (j0 + KT < n_all) fetch(j0 + KT);
        lds_barrier();
        if (j0 < n_wave) {
            floatx16 s[KT / 32];
#pragma unroll
            for (int n = 0; n < KT / 32; ++n) {
                RowOperand<T> a;
                lds_rows(a, sK[buf], 32 * n, c, h);
                clear(s[n]);
                s[n] = product(a, q, s[n]);
            }
            if (j0 + KT > n_wave_every) {
#pragma unroll
                for (int n = 0; n < KT / 32; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[n][r] = j0 + 32 * n + acc_row(r, h) < n_vis ? s[n][r] : -INFINITY;
            }
            acc.weights(s, scale);
#pragma unroll
            for (int n = 0; n < KT / 32; ++n) accumulate(acc.o, sV[buf], 32 * n, s[n], c, h, T{});
            if (part && (s_bad[buf][0] | s_bad[buf][1] | s_bad[buf][2] | s_bad[buf][3]))
                acc.add_nonfinite(Vh + j0 * V.row, V.row, min(KT, f.nk - j0), n_vis - j0, h);
        }
    }
    if (row >= n_rows) return;
    float l = acc.l + swap_half(acc.l);
    if (n_vis == 0) { l = 0.f; clear(acc.o[0]); clear(acc.o[1]); }
    store_row(out.at(head, f.q0 + t), acc.o, l != 0.f ? 1.f / l : 0.f, h);
    if (lse && h == 0) lse[(int64_t)head * p.Tq + f.q0 + t] = n_vis > 0 ? acc.m * kLn2 + logf(l) : -INFINITY;
}

PackedPlan make_packed_plan(const psa_packed_shape_t& s)
{
    PackedPlan p{};
    const int64_t rows = (int64_t)s.T_q * (s.H / s.H_kv);
    p.rows = 128;
    p.n_tile = (int)(rows / p.rows) + s.B;
    p.n_split = 1;
    p.total = 256;
    return p;
}

template <typename T, int KT>
static void packed_go(const PackedPlan& p, const psa_packed_shape_t& s, const psa_heads_t& Q, const psa_heads_t& K, const psa_heads_t& V,
                      const Packing& pk, const psa_heads_t& out, float* lse, hipStream_t stream)
{
    packed_rows_kernel<T, KT><<<(unsigned)(p.n_tile * s.H_kv), 256, 0, stream>>>(
        heads_of<const T>(Q), heads_of<const T>(K), heads_of<const T>(V), pk, heads_of<T>(out), lse, s.H_kv, s.causal,
        (float)(s.scale * 1.4426950408889634), p.n_tile);
}
hipError_t launch_packed(const PackedPlan& p, const psa_packed_shape_t& s, const psa_heads_t& Q, const psa_heads_t& K, const psa_heads_t& V,
                         const int* q_offsets, const int* k_offsets, const psa_heads_t& out, float* lse, void* workspace, hipStream_t stream)
{
    (void)hipGetLastError();
    const Packing pk{q_offsets, k_offsets, s.B, s.T_q, s.T_k, s.H / s.H_kv};
    if (s.dtype == PSA_F32) packed_go<float, 32>(p, s, Q, K, V, pk, out, lse, stream);
    else packed_go<bf16_t, 64>(p, s, Q, K, V, pk, out, lse, stream);
    return hipGetLastError();
}

}  // namespace psa
