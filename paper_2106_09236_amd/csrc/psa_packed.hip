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
    // Takes the maximum of the scores of N x 32 keys; the constant that is subtracted follows it only when that has grown by
    // more than 2^8 (kLagLog2): weights up to 2^8 are as exact as weights up to 1, and a change scales 32 accumulators.
    template <int N>
    __device__ __forceinline__ void follow(const floatx16 (&s)[N], float scale) {
        float t = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) t = fmaxf(t, s[n][r]);
        t = max_xor32(t) * scale;
        const float m_new = t > m + kLagLog2 ? t : m;
        if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {
            const float alpha = fast_exp2(m - m_new);
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < 2; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
        }
        m = m_new;
    }
    // Scores to weights
    __device__ __forceinline__ void weights(floatx16& s, float scale) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) { s[r] = fast_exp2(fmaf(s[r], scale, -m)); sum += s[r]; }
        l += sum;
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
// bfloat16 is bound by the vector unit (131 instructions and 32 exponentials to 16 matrix instructions: 65 % of its issue
// cycles, the matrix unit 38 %) and, in long runs, by power: 16384 causal, 8 heads, 335 to 355 us a call in 200 of them (820 to 775 TFLOP/s,
// from card to card), 377 to 408 in 20 traced ones.  What helped: a step's LDS reads before the instructions that take them (8 x 2048 causal 56.8 -> 55.2 us, 32 clips 17.4 -> 17.0).  What
// did not: 64 rows to a wave (half the LDS reads, 2 waves to a SIMD: 530 us), 4 waves to a SIMD with 32 keys at a time
// (430), the scores of a step formed between the weights of the one before (440), priorities (no change).
//
// KW = 2 (float32): 8 waves, two to 32 rows, which take alternate tiles of KT keys and join their sums in LDS; see packed_halves().
//
// FINE: bfloat16 weights in two parts (packed_fine()).  Infinities of V are left out of every tile then: one times a part of the other sign is NaN.
template <typename T, int KT, int KW, bool FINE>
__global__ __launch_bounds__(256 * KW, sizeof(T) == 4 || FINE ? 2 : 3)
void packed_rows_kernel(Heads<const T> Q, Heads<const T> K, Heads<const T> V, Packing p, Heads<T> out, float* __restrict__ lse,
                        int H_kv, int causal, float scale, int n_tile)
{
    constexpr int CH = 64 * sizeof(T) / 16;            // 16-byte chunks of a row
    constexpr int NT = 256 * KW, TILE = KT * KW;       // threads; keys between barriers
    constexpr int NL = TILE * CH / NT;                 // chunks of a tile, to a thread
    constexpr int NS = KT / 32;
    constexpr int kBytes = kTileBytes<T, TILE>;
    static_assert(KW == 1 || 4 * kBytes >= 128 * (kJoinRow + 2) * 4, "the join of 128 rows does not fit the tiles");
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * kBytes];
    __shared__ int s_bad[2][4 * KW];
    unsigned char *const sK = lds, *const sV = lds + 2 * kBytes;
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const SeqTile f = find_tile<128, false>(p, x);
    auto outside = [&] { zero_outside(out, p.qo, p.B, p.Tq, hk * p.G, p.G, x, n_tile, [&](int head, int row) { if (lse) lse[(int64_t)head * p.Tq + row] = -INFINITY; }); };
    if (f.tile < 0) { outside(); return; }

    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;                 // causal: query t sees the first t + shift keys
    auto visible = [&](int r) { const int t = r / p.G; return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int rw = wave & 3, kg = KW == 1 ? 0 : wave >> 2;         // which rows, which keys
    const int row0 = f.tile * 128 + rw * 32;
    const int row = row0 + c, rc = min(row, n_rows - 1);
    const int t = rc / p.G, head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int n_all = __builtin_amdgcn_readfirstlane(visible(min(f.tile * 128 + 127, n_rows - 1)));         // keys any row of the work-group sees
    const int n_every = __builtin_amdgcn_readfirstlane(visible(f.tile * 128));                              // ... and those that all see
    const int n_wave = __builtin_amdgcn_readfirstlane(row0 < n_rows ? visible(min(row0 + 31, n_rows - 1)) : 0);
    const int n_wave_every = __builtin_amdgcn_readfirstlane(visible(min(row0, n_rows - 1)));

    HeadOperand<T> q;
    q.load(Q.at(head, f.q0 + t), h);
    const T* Kh = K.at(hk, f.k0);
    const T* Vh = V.at(hk, f.k0);
    int k_ofs[NL], v_ofs[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int id = i * NT + tid, r = id / CH, ch = id % CH;
        k_ofs[i] = (int)(r * K.row * (int64_t)sizeof(T)) + ch * 16;
        v_ofs[i] = (int)(r * V.row * (int64_t)sizeof(T)) + ch * 16;
    }
    uint4 kr[NL], vr[NL];
    auto fetch = [&](int j0) {
        const int n = min(TILE, f.nk - j0);
        const auto kb = tile_rows(Kh + j0 * K.row, K.row, n), vb = tile_rows(Vh + j0 * V.row, V.row, n);
#pragma unroll
        for (int i = 0; i < NL; ++i) { kr[i] = buffer_load16<uint4>(kb, k_ofs[i]); vr[i] = buffer_load16<uint4>(vb, v_ofs[i]); }
    };
    Rows32 acc;
    acc.init();
    if (n_all > 0) fetch(0);
    int buf = 0;
    for (int j0 = 0; j0 < n_all; j0 += TILE, buf ^= 1) {
        // a weight of 0 does not keep an infinity or NaN of a value that a row does not see out of its sum: in tiles that
        // some row sees in part they are left out and added afterwards (float32: in all, since an infinity has no parts)
        const bool look = sizeof(T) == 4 || FINE || j0 + TILE > n_every;
        if (look) {
            const bool any = __builtin_amdgcn_ballot_w64(nonfinite(vr, T{})) != 0;
            if (lane == 0) s_bad[buf][wave] = any;
            if (any)
#pragma unroll
                for (int i = 0; i < NL; ++i) vr[i] = finite_only(vr[i], T{});
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * NT + tid;
            put<TILE>(sK + buf * kBytes, id / CH, id % CH, kr[i], T{});
            put<TILE>(sV + buf * kBytes, id / CH, id % CH, vr[i], T{});
        }
        if (j0 + TILE < n_all) fetch(j0 + TILE);
        lds_barrier();
        const int j = j0 + kg * KT;
        if (j >= n_wave) continue;
        floatx16 s[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) s[n] = product<T, TILE>(sK + buf * kBytes, kg * KT + 32 * n, q, c, h);
        reads_first<4 * NS * kParts<T>, 4 * NS * (sizeof(T) == 4 ? 6 : 1)>();
        if (j + KT > n_wave_every) {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = j + 32 * n + acc_row(r, h) < n_vis ? s[n][r] : -INFINITY;
        }
        acc.follow(s, scale);
        Transposed<T> v[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) v[n] = transposed<T, TILE>(sV + buf * kBytes, kg * KT + 32 * n, c, h);
        reads_first<8 * NS * kParts<T>, 0>();
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            acc.weights(s[n], scale);
            accumulate<T, FINE>(acc.o, v[n], s[n]);
        }
        if (look) {
            int any = 0;
#pragma unroll
            for (int w = 0; w < 4 * KW; ++w) any |= s_bad[buf][w];
            if (any) acc.add_nonfinite(Vh + j * V.row, V.row, min(KT, f.nk - j), n_vis - j, h);
        }
    }
    outside();                                         // (last: its loads would delay the others)
    float l = acc.l + swap_half(acc.l);
    if (KW == 2) {
        float* join = reinterpret_cast<float*>(lds) + (rw * 32 + c) * kJoinRow;
        float* join_ml = reinterpret_cast<float*>(lds) + 128 * kJoinRow + (rw * 32 + c) * 2;
        __syncthreads();
        if (kg == 1) {
            store_row(join, acc.o, 1.f, h);
            if (h == 0) { join_ml[0] = acc.m; join_ml[1] = l; }
        }
        __syncthreads();
        if (kg == 1) return;
        const float m1 = join_ml[0], l1 = join_ml[1], m = fmaxf(acc.m, m1);
        const float a0 = fast_exp2(acc.m - m), a1 = fast_exp2(m1 - m);
        l = l * a0 + l1 * a1;
        acc.m = m;
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc.o[dt][r] = acc.o[dt][r] * a0 + join[32 * dt + acc_row(r, h)] * a1;
    }
    if (row >= n_rows) return;
    if (n_vis == 0) { l = 0.f; clear(acc.o[0]); clear(acc.o[1]); }
    store_row(out.at(head, f.q0 + t), acc.o, l != 0.f ? 1.f / l : 0.f, h);
    if (lse && h == 0) lse[(int64_t)head * p.Tq + f.q0 + t] = n_vis > 0 ? acc.m * kLn2 + logf(l) : -INFINITY;
}

// ---- few rows: 32 to a work-group, whose 4 waves divide the keys (of its split) among themselves, 32 at a time, and join their
// sums at the end.  Keys come straight from memory as the first product's operand, values through LDS of the wave's own;
// there is no barrier before the join.
template <typename T>
__global__ __launch_bounds__(256, 2)
void packed_few_kernel(Heads<const T> Q, Heads<const T> K, Heads<const T> V, Packing p, Heads<T> out, float* __restrict__ lse,
                       int H_kv, int causal, float scale, int n_tile, int n_split, float* __restrict__ part_o, float2* __restrict__ part_ml)
{
    constexpr int CH = 64 * sizeof(T) / 16;
    constexpr int NL = 32 * CH / 64;                   // chunks of a tile of 32 rows, to a lane
    constexpr int kBytes = kTileBytes<T, 32>;
    constexpr int kJoinBytes = 4 * 32 * kJoinRow * 4;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * kBytes > kJoinBytes ? 4 * kBytes : kJoinBytes];
    __shared__ float s_m[4][32], s_l[4][32];
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv, split = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const SeqTile f = find_tile<32, false>(p, x);
    auto outside = [&] {
        if (split == 0) zero_outside(out, p.qo, p.B, p.Tq, hk * p.G, p.G, x, n_tile, [&](int head, int row) { if (lse) lse[(int64_t)head * p.Tq + row] = -INFINITY; });
    };
    if (f.tile < 0) { outside(); return; }
    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;
    auto visible = [&](int r) { const int t = r / p.G; return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int row0 = f.tile * 32, row = row0 + c, rc = min(row, n_rows - 1);
    const int t = rc / p.G, head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int n_all = __builtin_amdgcn_readfirstlane(visible(min(row0 + 31, n_rows - 1)));
    const int n_every = __builtin_amdgcn_readfirstlane(visible(row0));
    // this split's tiles of 32 keys, every fourth of them this wave's
    const int tiles = (n_all + 31) / 32, per = (tiles + n_split - 1) / n_split;
    const int end = min(n_all, (split + 1) * per * 32);

    HeadOperand<T> q;
    q.load(Q.at(head, f.q0 + t), h);
    const T* Kh = K.at(hk, f.k0);
    const T* Vh = V.at(hk, f.k0);
    unsigned char* sV = lds + wave * kBytes;
    HeadRow<T> kn;
    uint4 vn[NL];
    auto fetch = [&](int j0) {
        const int n = min(32, f.nk - j0);
        const auto kb = tile_rows(Kh + j0 * K.row, K.row, n), vb = tile_rows(Vh + j0 * V.row, V.row, n);
        kn.load(kb, (int)(c * K.row * (int64_t)sizeof(T)), h);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 64 + lane;
            vn[i] = buffer_load16<uint4>(vb, (int)((id / CH) * V.row * (int64_t)sizeof(T)) + (id % CH) * 16);
        }
    };
    Rows32 acc;
    acc.init();
    int j0 = (split * per + wave) * 32;
    if (j0 < end) fetch(j0);
    for (; j0 < end; j0 += 128) {
        // infinities and NaN of V are left out of the product and added afterwards, in whole tiles too: the weights have parts of either
        // sign and of 0
        const bool any = __builtin_amdgcn_ballot_w64(nonfinite(vn, T{})) != 0;
        if (any)
#pragma unroll
            for (int i = 0; i < NL; ++i) vn[i] = finite_only(vn[i], T{});
        wave_lds_sync();
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 64 + lane;
            put<32>(sV, id / CH, id % CH, vn[i], T{});
        }
        floatx16 s[1];
        s[0] = product(kn, q);
        wave_lds_sync();
        if (j0 + 128 < end) fetch(j0 + 128);
        if (j0 + 32 > n_every) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] = j0 + acc_row(r, h) < n_vis ? s[0][r] : -INFINITY;
        }
        acc.follow(s, scale);
        acc.weights(s[0], scale);
        accumulate<T, 32, true>(acc.o, sV, 0, s[0], c, h);
        if (any) acc.add_nonfinite(Vh + j0 * V.row, V.row, min(32, f.nk - j0), n_vis - j0, h);
    }
    outside();                                         // (last: its loads would delay the others)
    // join: wave w's sums of row r at join[w][r]; a wave that saw no key has m = kMaxInit and sums of 0
    __syncthreads();
    float* join = reinterpret_cast<float*>(lds);
    const float l = acc.l + swap_half(acc.l);
    if (h == 0) { s_m[wave][c] = acc.m; s_l[wave][c] = l; }
    store_row(join + (wave * 32 + c) * kJoinRow, acc.o, 1.f, h);
    __syncthreads();
    // 8 threads of 8 elements to a row
    const int r = tid >> 3, e = (tid & 7) * 8;
    if (row0 + r >= n_rows) return;
    float m = s_m[0][r];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, s_m[w][r]);
    float sum = 0.f, o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (s_m[w][r] == kMaxInit && s_l[w][r] == 0.f) continue;       // (saw no key: its accumulators may hold 0 * NaN)
        const float a = fast_exp2(s_m[w][r] - m);
        sum = fmaf(s_l[w][r], a, sum);
        const float* src = join + (w * 32 + r) * kJoinRow + e;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = fmaf(src[i], a, o[i]);
    }
    const int rt = (row0 + r) / p.G, rh = hk * p.G + (row0 + r - rt * p.G);
    if (n_split > 1) {
        const int64_t rec = ((int64_t)split * H_kv + hk) * p.Tq * p.G + (int64_t)f.q0 * p.G + row0 + r;
        float4* dst = reinterpret_cast<float4*>(part_o + rec * 64 + e);
        dst[0] = make_float4(o[0], o[1], o[2], o[3]);
        dst[1] = make_float4(o[4], o[5], o[6], o[7]);
        if (e == 0) part_ml[rec] = make_float2(m, sum);
    } else {
        store_joined(out.at(rh, f.q0 + rt) + e, o, sum);
        if (lse && e == 0) lse[(int64_t)rh * p.Tq + f.q0 + rt] = sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
    }
}

// Joins the splits of each row that is in a sequence: a wave to a row, 16 lanes of 4 elements for every fourth split.  The loads of
// several splits are in flight at once (8 threads to a row and one split after the other: 10.2 us for 15 splits of 256 rows).
template <typename T>
__global__ __launch_bounds__(256, 2)
void packed_merge_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, int n_split, Packing p, int H_kv, Heads<T> out,
                         float* __restrict__ lse)
{
    const int64_t rows = (int64_t)p.Tq * p.G;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= rows * H_kv) return;
    const int lane = threadIdx.x & 63, e = (lane & 15) * 4, s0 = lane >> 4;
    const int hk = (int)(id / rows);
    const int r = (int)(id - hk * rows), t = r / p.G, head = hk * p.G + (r - t * p.G);
    if (p.qo && (t < p.qo[0] || t >= p.qo[p.B])) return;
    float m = kMaxInit, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int base = s0; base < n_split; base += 16) {
        float2 ml[4];
        float4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t rec = (int64_t)min(base + 4 * k, n_split - 1) * rows * H_kv + id;
            ml[k] = part_ml[rec];
            v[k] = *reinterpret_cast<const float4*>(part_o + rec * 64 + e);
            if (base + 4 * k >= n_split) { ml[k] = make_float2(kMaxInit, 0.f); v[k] = make_float4(0.f, 0.f, 0.f, 0.f); }
        }
        const float top = fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), m);
        const float a0 = fast_exp2(m - top);
        sum *= a0; o.x *= a0; o.y *= a0; o.z *= a0; o.w *= a0;
        m = top;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a = fast_exp2(ml[k].x - m);
            sum = fmaf(ml[k].y, a, sum);
            o.x = fmaf(v[k].x, a, o.x); o.y = fmaf(v[k].y, a, o.y); o.z = fmaf(v[k].z, a, o.z); o.w = fmaf(v[k].w, a, o.w);
        }
    }
#pragma unroll
    for (int k = 16; k < 64; k *= 2) {
        const float m2 = __shfl_xor(m, k, 64), top = fmaxf(m, m2);
        const float a = fast_exp2(m - top), b = fast_exp2(m2 - top);
        sum = sum * a + __shfl_xor(sum, k, 64) * b;
        o.x = o.x * a + __shfl_xor(o.x, k, 64) * b;
        o.y = o.y * a + __shfl_xor(o.y, k, 64) * b;
        o.z = o.z * a + __shfl_xor(o.z, k, 64) * b;
        o.w = o.w * a + __shfl_xor(o.w, k, 64) * b;
        m = top;
    }
    if (s0 != 0) return;
    const float f = sum != 0.f ? 1.f / sum : 0.f;
    store4(out.at(head, t) + e, sum != 0.f ? make_float4(o.x * f, o.y * f, o.z * f, o.w * f) : make_float4(0.f, 0.f, 0.f, 0.f));
    if (lse && e == 0) lse[(int64_t)head * p.Tq + t] = sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
}

// Tiles before each 64 sequences, counted from the last (find_tile): of rows in work-group 0, of keys in work-group 1.  16 waves with 64
// sequences each at a time.  A call has fewer than 2^28 tiles (2^31 rows in tiles of 32, and one more to a sequence), but where offsets
// decrease each sequence may claim all of its rows; sums stop at kMostTiles, so that they do not overflow and stay in order.
constexpr int kMostTiles = 1 << 29;
__global__ __launch_bounds__(1024)
void packed_before_kernel(Packing p, int per_q, int per_k, int* __restrict__ q_before, int* __restrict__ k_before)
{
    __shared__ int s[2][16];
    const bool keys = blockIdx.x == 1;
    int* out = keys ? k_before : q_before;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = (p.B + 63) / 64;
    int sum = 0;                                       // of all before these 16
    for (int g0 = 0, buf = 0; g0 < groups; g0 += 16, buf ^= 1) {
        const int g = g0 + wave;
        const int tiles = g < groups ? seq_tiles(seq_range(p, p.B - 1 - 64 * g - lane), p.G, keys ? per_k : per_q, keys) : 0;
        const int n = wave_sum(tiles >> 6) >= kMostTiles >> 6 ? kMostTiles : wave_sum(tiles);    // (64 x 2^26 may be; the second sum then is not)
        if (lane == 0) s[buf][wave] = n;
        __syncthreads();
        int mine = sum, all = sum;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) mine = min(mine + s[buf][w], kMostTiles);
            all = min(all + s[buf][w], kMostTiles);
        }
        if (g < groups && lane == 0) out[g] = mine;
        sum = all;
    }
}
Packing make_packing(const psa_packed_shape_t& s, const int* q_offsets, const int* k_offsets, int per_q, int per_k, void* room, bool keys, hipStream_t stream)
{
    Packing p{q_offsets, k_offsets, s.B, s.T_q, s.T_k, s.H / s.H_kv, nullptr, nullptr};
    if (const size_t bytes = packed_before_bytes(s.B)) {
        int* q = static_cast<int*>(room);
        int* k = reinterpret_cast<int*>(static_cast<unsigned char*>(room) + bytes);
        packed_before_kernel<<<keys ? 2 : 1, 1024, 0, stream>>>(p, per_q, per_k, q, k);
        p.q_before = q;
        p.k_before = keys ? k : nullptr;
    }
    return p;
}

// float32, two waves to 32 rows?  One work-group of them fills a compute unit, and a wave's chain of steps is half as long: for calls
// with few work-groups (`wide` of 128 rows) and long sequences.  1 | 2 waves, forward: 16 x 512 (4 heads, 320 work-groups) 41 | 35 us, 24
// ragged clips of 435 causal (374) 55 | 41, 8 x 1000 causal (8 heads, 531) 83 | 77; but 32 of 40 .. 500 (400) 50 | 54, 64 of 450 (1120)
// 135 | 154, 8 x 2048 causal (8 heads, 1088) 240 | 246.  dQ alike.  (bfloat16, which has two work-groups of 4 waves to a unit: 32 ragged
// clips 17.6 | 21.6, 8 x 2048 64 | 83.)
bool packed_halves(const psa_packed_shape_t& s, int64_t wide) { return s.dtype == PSA_F32 && wide < 640 && s.T_k / s.B >= 400; }

// Enough work-groups of 128 rows (`wide` of them)?  Causal tiles differ in length, so more of them.  32 | 128 rows, bfloat16: 7146 keys, 4
// heads to 2, 226 work-groups, 171 | 110 us, dQ 202 | 145; 5000, 158, 92 | 77 and 115 | 100 (float32 272 | 205, 361 | 263); 8 of 512, 160, 12.0 |
// 11.9; causal: 12 of 300 to 700, 234, 15.3 | 14.6 and 24.1 | 17.9; one of 3000, 8 heads, 192, 41 | 46 and 50 | 59 (float32 107 | 120, 130 | 155).
bool packed_enough(const psa_packed_shape_t& s, int64_t wide) { return wide >= (s.causal ? 224 : 152); }

// bfloat16 weights of rows: in two parts, 16 bits, unless the matrix and vector units are what the call waits for; rounded once they cost a
// result as much as its own rounding.  Once | two parts: 50 sequences of 1 to 60 rows, 4 heads, 7.0 | 6.8 us and with the backward 19.8 | 20.0, 100
// of them 7.3 | 7.5 and 22.0 | 23.7, one row and 20 keys 7.2 | 6.8, 20 of 20 to 100 7.3 | 7.5; but 5000 of 1 to 40 rows 150 | 217 and 594 | 684, 32 clips of 40 to 500 frames
// 17.7 | 24.7, 16384 causal 354 | 515, 8 x 2048 causal with the backward 234 | 302.
bool packed_fine(const psa_packed_shape_t& s, int64_t wide) { return !packed_enough(s, wide) || (wide <= 512 && s.T_k / s.B <= 64); }

// Few rows or many?  A wave owns 32 rows either way.  Work-groups of 128 rows read K and V a quarter as often but leave waves idle
// in sequences of fewer rows, and there must be enough of them, unless sequences are over in a step of 64 keys; those of 32 rows divide
// the keys among their waves, which pays for 32 rows and less with 100 keys and more.  32 | 128 rows, 4 or 8 heads: 256 sequences of 1 row and up to 4096 keys 50 | 61 us, 64 of 20 rows and 500
// to 2000 keys 26.7 | 32.5, 128 of 16 and 100 to 1000 float32 91 | 112; but 5000 of 1 to 40 rows, as many keys 181 | 140, 1000 of 20 to
// 60 float32 113 | 67, 2000 of 30 to 64 114 | 65, 64 of 64 rows and 500 to 2000 keys 52 | 45.  Calls with few
// work-groups: 50 sequences of 1 to 60 rows 7.1 | 5.9, one row and 20 keys 6.0 | 5.5, 4 of 30 float32 8.4 | 6.5, 20 of 20 to 100 7.5 | 7.2, but
// 8 of 60 to 130 6.4 | 7.2 and in float32 9.8 | 12.0.
PackedPlan make_packed_plan(const psa_packed_shape_t& s)
{
    PackedPlan p{};
    const int64_t rows = (int64_t)s.T_q * (s.H / s.H_kv);
    const int64_t wide = (rows / 128 + s.B) * s.H_kv;
    p.few = s.T_k / s.B > 64 && (!packed_enough(s, wide) || (rows / s.B <= 32 && s.T_k / s.B >= 100));
    p.halves = !p.few && packed_halves(s, wide);
    p.fine = p.few || packed_fine(s, wide);
    p.rows = p.few ? 32 : 128;
    p.n_tile = (int)(rows / p.rows) + s.B;
    p.n_split = 1;
    if (p.few) {
        // splits: towards 3 work-groups to a compute unit, each with a round of its 4 waves at the least (by the mean length); none
        // where every unit has a work-group or sequences are short, and joining them costs more (4 us and more with many rows).  32
        // streams of 1 .. 4096 keys, 256 | 512 | 768 | 1024 | 2048 work-groups: 15.2 | 13.3 | 11.9 | 12.2 | 12.8 us; 64 of 100 .. 500:
        // 8.6 unsplit, 8.8 and more with the join on top; 2000 causal, 8 heads, 512 work-groups: 2 splits 22.4 and 9.6 for the join
        const int64_t wgs = (int64_t)p.n_tile * s.H_kv, mean = (int64_t)s.T_k / s.B;
        int64_t split = wgs >= 256 ? 1 : 768 / wgs;
        const int64_t most = mean <= 768 ? 1 : (mean + 127) / 128;
        if (split > most) split = most;
        if (split > 64) split = 64;
        p.n_split = (int)(split < 1 ? 1 : split);
    }
    p.off_ml = packed_before_bytes(s.B);
    p.off_part = p.off_ml;
    if (p.n_split > 1) {
        p.off_part += ((size_t)p.n_split * (size_t)rows * s.H_kv * sizeof(float2) + 255) & ~(size_t)255;
        p.total = p.off_part + (size_t)p.n_split * (size_t)rows * s.H_kv * 64 * sizeof(float);
    } else {
        p.total = p.off_part > 256 ? p.off_part : 256;
    }
    return p;
}

template <typename T, int KT>
static void packed_go(const PackedPlan& p, const psa_packed_shape_t& s, const psa_heads_t& Q, const psa_heads_t& K, const psa_heads_t& V,
                      const Packing& pk, const psa_heads_t& out, float* lse, void* workspace, hipStream_t stream)
{
    const float scale = (float)(s.scale * 1.4426950408889634);
    const dim3 grid((unsigned)(p.n_tile * s.H_kv), (unsigned)p.n_split);
    if (!p.few) {
        constexpr int KW = sizeof(T) == 4 ? 2 : 1;
        constexpr bool FINE = sizeof(T) == 2;
        (p.halves ? packed_rows_kernel<T, KT, KW, false> : p.fine ? packed_rows_kernel<T, KT, 1, FINE> : packed_rows_kernel<T, KT, 1, false>)<<<grid, p.halves ? 512 : 256, 0, stream>>>(
            heads_of<const T>(Q), heads_of<const T>(K), heads_of<const T>(V), pk, heads_of<T>(out), lse, s.H_kv, s.causal, scale, p.n_tile);
        return;
    }
    float2* part_ml = reinterpret_cast<float2*>(static_cast<unsigned char*>(workspace) + p.off_ml);
    float* part_o = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + p.off_part);
    packed_few_kernel<T><<<grid, 256, 0, stream>>>(heads_of<const T>(Q), heads_of<const T>(K), heads_of<const T>(V), pk, heads_of<T>(out), lse,
                                                   s.H_kv, s.causal, scale, p.n_tile, p.n_split, part_o, part_ml);
    if (p.n_split > 1) {
        const int64_t rows = (int64_t)s.T_q * s.H;
        packed_merge_kernel<T><<<(unsigned)((rows + 3) / 4), 256, 0, stream>>>(part_o, part_ml, p.n_split, pk, s.H_kv, heads_of<T>(out), lse);
    }
}
hipError_t launch_packed(const PackedPlan& p, const psa_packed_shape_t& s, const psa_heads_t& Q, const psa_heads_t& K, const psa_heads_t& V,
                         const int* q_offsets, const int* k_offsets, const psa_heads_t& out, float* lse, void* workspace, hipStream_t stream)
{
    const Packing pk = make_packing(s, q_offsets, k_offsets, p.rows, 0, workspace, false, stream);
    if (s.dtype == PSA_F32) packed_go<float, 32>(p, s, Q, K, V, pk, out, lse, workspace, stream);
    else packed_go<bf16_t, 64>(p, s, Q, K, V, pk, out, lse, workspace, stream);
    return hipGetLastError();
}

}  // namespace psa
