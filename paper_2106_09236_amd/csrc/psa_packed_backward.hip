// Dense attention over packed sequences, backward.  With p the weights, recomputed from Q, K and the forward's lse, G = dOut
// and d_t = G[t].out[t]:
//   ds_tj = p_tj (G[t].V[j] - d_t),  dQ[t] = scale sum_j ds_tj K[j],  dK[j] = scale sum_t ds_tj Q[t],  dV[j] = sum_t p_tj G[t]
// Two launches: dQ with a work-group's rows held and the keys passing by, which also leaves d_t and lse where the other finds them;
// dK and dV with the keys held and the rows passing by.  (Small calls of float32 take one launch for both, and one before it for
// d_t; few keys that many rows read take one after them, which joins the parts of dK and dV.)  The scores and G.V are computed in both,
// seven products where five would do if dQ were added up in memory by atomics, whose order would change the result.
#include <type_traits>

#include "psa_packed.h"

namespace psa {

// lse in base 2; +infinity for a row that sees no key, whose weights then are 0
__device__ __forceinline__ float stat_of(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }
// Where a row's lse and d lie, [H_kv][T_q * G] each
struct Stats {
    float *l, *d;
    const float* lse;
    __device__ __forceinline__ static int64_t at(const Packing& p, int hk, int64_t row) { return (int64_t)hk * p.Tq * p.G + row; }
};
// Half of a row's d: a lane's 32 of its 64 products
template <typename T>
__device__ __forceinline__ float half_row_dot(const T* a, const T* b, int h)
{
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 32 / kVec<T>; ++k) {
        float x[kVec<T>], y[kVec<T>];
        load_vec(x, a + 32 * h + k * kVec<T>, kVec<T>);
        load_vec(y, b + 32 * h + k * kVec<T>, kVec<T>);
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) sum = fmaf(x[i], y[i], sum);
    }
    return sum;
}

// What a wave keeps of dQ for 32 rows.  out has been rounded, so d formed from it is off by 2^-8 of its terms for bfloat16 tensors, more than
// the rounding of dS where a few keys have the weight (dQ and dK then had twice the error of their own rounding).  But d is also
// sum_j p_j (G.V[j]): with d0 the value from out, e = sum_j p_j (G.V[j] - d0) is what d0 is off by, and
//     sum_j p_j (G.V[j] - d0 - e) K[j] = sum_j p_j (G.V[j] - d0) K[j] - e sum_j p_j K[j],
// one product more (of weights rounded once: e is small) and d = d0 + e for dK.  float32 tensors need none of it.
template <typename T> struct RowGradient;
template <> struct RowGradient<float> {
    floatx16 dq[2];
    __device__ __forceinline__ void init() { clear(dq[0]); clear(dq[1]); }
    static __device__ __forceinline__ void weights(floatx16& s, floatx16& w, float scale, float l, float d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) w[r] = fast_exp2(fmaf(s[r], scale, -l)) * (w[r] - d);
    }
    template <int ROWS, bool FINE>
    __device__ __forceinline__ void add(const floatx16&, const floatx16& w, const unsigned char* k, int row0, int c, int h) { accumulate<float, ROWS, false>(dq, k, row0, w, c, h); }
    __device__ __forceinline__ float finish() { return 0.f; }
};
template <> struct RowGradient<bf16_t> {
    floatx16 dq[2], pk[2];
    float e;
    __device__ __forceinline__ void init() { clear(dq[0]); clear(dq[1]); clear(pk[0]); clear(pk[1]); e = 0.f; }
    // s: scores to weights; w: G.V to dS
    static __device__ __forceinline__ void weights(floatx16& s, floatx16& w, float scale, float l, float d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) { s[r] = fast_exp2(fmaf(s[r], scale, -l)); w[r] = s[r] * (w[r] - d); }
    }
    template <int ROWS, bool FINE>
    __device__ __forceinline__ void add(const floatx16& s, const floatx16& w, const unsigned char* k, int row0, int c, int h) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += w[r];
        e += sum;
        accumulate_two<bf16_t, ROWS, FINE>(dq, w, pk, s, k, row0, c, h);
    }
    __device__ __forceinline__ float finish() {
        e += swap_half(e);
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) dq[dt][r] = fmaf(-e, pk[dt][r], dq[dt][r]);
        return e;
    }
};

// Both of every row, for calls whose two kernels run at once (float32).
template <typename T>
__global__ __launch_bounds__(256, 2)
void packed_stats_kernel(Heads<const T> out, Heads<const T> dOut, const float* __restrict__ lse, Packing p, int H,
                         float* __restrict__ stat_l, float* __restrict__ stat_d)
{
    constexpr int VEC = kVec<T>, CH = 64 / VEC;        // lanes of a row
    const int64_t id = (int64_t)blockIdx.x * (256 / CH) + threadIdx.x / CH;
    if (id >= (int64_t)p.Tq * H) return;
    const int head = (int)(id / p.Tq), t = (int)(id % p.Tq), ch = threadIdx.x % CH;
    float a[VEC], b[VEC], sum = 0.f;
    load_vec(a, out.at(head, t) + ch * VEC, VEC);
    load_vec(b, dOut.at(head, t) + ch * VEC, VEC);
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum = fmaf(a[i], b[i], sum);
#pragma unroll
    for (int k = 1; k < CH; k *= 2) sum += __shfl_xor(sum, k, 64);
    if (ch == 0) {
        const float l = lse[(int64_t)head * p.Tq + t];
        const int64_t o = Stats::at(p, head / p.G, (int64_t)t * p.G + head % p.G);
        stat_l[o] = stat_of(l);
        stat_d[o] = sum;
    }
}

// dK and dV of 128 keys: 4 waves of 32, tiles of QT rows of Q and dOut through LDS.  Where few work-groups would pass many rows each (the
// rows of all query heads of a group), blockIdx.y takes a part of the rows and leaves its sums in `part` [n_split, H_kv, T_k, 2, 64].
// FINE: bfloat16 weights in two parts.
template <typename T, int QT, bool FINE>
__global__ __launch_bounds__(256, 2)
void packed_dkv_kernel(Heads<const T> Q, Heads<const T> K, Heads<const T> V, Heads<const T> dOut, const float* __restrict__ stat_l,
                       const float* __restrict__ stat_d, Packing p, Heads<T> dK, Heads<T> dV, int H_kv, int causal, float scale,
                       float scale_log2, int n_tile, int n_split, float* __restrict__ part)
{
    constexpr int CH = 64 * sizeof(T) / 16, NL = QT * CH / 256;
    constexpr int kBytes = kTileBytes<T, QT>;
    __shared__ __attribute__((aligned(16))) unsigned char sQ[2][kBytes], sG[2][kBytes];
    __shared__ __attribute__((aligned(16))) float sL[2][QT], sD[2][QT];
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const SeqTile f = find_tile<128, true>(p, x);
    auto outside = [&] {
        if (blockIdx.y != 0) return;
        zero_outside(dK, p.ko, p.B, p.Tk, hk, 1, x, n_tile, [](int, int) {});
        zero_outside(dV, p.ko, p.B, p.Tk, hk, 1, x, n_tile, [](int, int) {});
    };
    if (f.tile < 0) { outside(); return; }
    const int shift = f.nk - f.nq + 1;
    // the first row that sees key j (rows are in the order of their queries)
    auto first_row = [&](int j) { return causal ? max(j - shift + 1, 0) * p.G : 0; };
    const int key = f.tile * 128 + wave * 32 + c, kc = min(key, f.nk - 1);
    const int first = first_row(kc);
    const int first_all = __builtin_amdgcn_readfirstlane(first_row(f.tile * 128));
    const int wave_key = min(f.tile * 128 + wave * 32, f.nk - 1);
    const int first_wave = __builtin_amdgcn_readfirstlane(first_row(wave_key));
    const int first_every = __builtin_amdgcn_readfirstlane(first_row(min(wave_key + 31, f.nk - 1)));

    HeadOperand<T> k, v;
    k.load(K.at(hk, f.k0 + kc), h);
    v.load(V.at(hk, f.k0 + kc), h);
    floatx16 dk[2], dv[2];
    clear(dk[0]); clear(dk[1]); clear(dv[0]); clear(dv[1]);

    const int64_t stat0 = ((int64_t)hk * p.Tq + f.q0) * p.G;
    uint4 qr[NL], gr[NL];
    float lr = INFINITY, dr = 0.f;
    int r0 = first_all / QT * QT, n_rows = f.nq * p.G;
    if (n_split > 1) {                                 // this part's rows
        const int steps = max((n_rows - r0 + QT - 1) / QT, 0), per = (steps + n_split - 1) / n_split * QT;
        r0 = (int)min((int64_t)r0 + (int64_t)blockIdx.y * per, (int64_t)n_rows);
        n_rows = (int)min((int64_t)r0 + per, (int64_t)n_rows);
    }
    const int ch = tid % CH, dt = 256 / CH / p.G, dg = 256 / CH - dt * p.G;     // (the thread's next chunk is 256 / CH rows on)
    RowAt at(r0 + tid / CH, p.G);
    auto fetch = [&](int r0) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            qr[i] = gr[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r0 + i * (256 / CH) + tid / CH < n_rows) {
                qr[i] = reinterpret_cast<const uint4*>(Q.at(hk * p.G + at.g, f.q0 + at.t))[ch];
                gr[i] = reinterpret_cast<const uint4*>(dOut.at(hk * p.G + at.g, f.q0 + at.t))[ch];
            }
            at.add(dt, dg, p.G);
        }
        if (tid < QT) {
            const bool in = r0 + tid < n_rows;
            lr = in ? stat_l[stat0 + r0 + tid] : INFINITY;
            dr = in ? stat_d[stat0 + r0 + tid] : 0.f;
        }
    };
    if (r0 < n_rows) fetch(r0);
    // (bfloat16: two steps to a round.  With the buffer known, LDS addresses are constants beside the lane's: 106.7 -> 102.8 us for 8 x 2048
    // causal.  float32 has no registers for it.)
    auto step = [&](auto which) {
        const int buf = which;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 256 + tid;
            put<QT>(sQ[buf], id / CH, id % CH, qr[i], T{});
            put<QT>(sG[buf], id / CH, id % CH, gr[i], T{});
        }
        if (tid < QT) { sL[buf][tid] = lr; sD[buf][tid] = dr; }
        if (r0 + QT < n_rows) fetch(r0 + QT);
        lds_barrier();
#pragma unroll
        for (int n = 0; n < QT / 32; ++n) {
            const int r = r0 + 32 * n;
            if (r + 32 <= first_wave || r >= n_rows) continue;
            floatx16 s = product<T, QT>(sQ[buf], 32 * n, k, c, h), w = product<T, QT>(sG[buf], 32 * n, v, c, h);
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const float4 l4 = *reinterpret_cast<const float4*>(&sL[buf][32 * n + 8 * r4 + 4 * h]), d4 = *reinterpret_cast<const float4*>(&sD[buf][32 * n + 8 * r4 + 4 * h]);
                const float l[4] = {l4.x, l4.y, l4.z, l4.w}, d[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[4 * r4 + e] = fast_exp2(fmaf(s[4 * r4 + e], scale_log2, -l[e]));
                    w[4 * r4 + e] = s[4 * r4 + e] * (w[4 * r4 + e] - d[e]);
                }
            }
            if (r < first_every) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (r + acc_row(i, h) < first) s[i] = w[i] = 0.f;
            }
            accumulate<T, QT, FINE>(dv, sG[buf], 32 * n, s, c, h);
            accumulate<T, QT, FINE>(dk, sQ[buf], 32 * n, w, c, h);
        }
    };
    int parity = 0;
    while (r0 < n_rows) {
        if constexpr (sizeof(T) == 2) {
            step(std::integral_constant<int, 0>{});
            r0 += QT;
            if (r0 >= n_rows) break;
            step(std::integral_constant<int, 1>{});
        } else {
            step(parity);
            parity ^= 1;
        }
        r0 += QT;
    }
    outside();
    if (key >= f.nk) return;
    if (n_split > 1) {
        float* sums = part + (((int64_t)blockIdx.y * H_kv + hk) * p.Tk + f.k0 + key) * 128;
        store_row(sums, dk, f.nk == 1 ? 0.f : 1.f, h);
        store_row(sums + 64, dv, 1.f, h);
        return;
    }
    store_row(dK.at(hk, f.k0 + key), dk, f.nk == 1 ? 0.f : scale, h);       // (the weight of an only key is 1 whatever the scores are)
    store_row(dV.at(hk, f.k0 + key), dv, 1.f, h);
}

// The parts' sums, 4 elements to a thread, in the order of the parts; 8 keys to a work-group.  (Keys in no sequence have been cleared.)
template <typename T>
__global__ __launch_bounds__(256)
void packed_join_keys_kernel(const float* __restrict__ part, int n_split, Packing p, Heads<T> dK, Heads<T> dV, int H_kv, float scale)
{
    const int64_t id = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int e = threadIdx.x % 32 * 4;                // of dK's 64 elements, then dV's
    if (id >= (int64_t)p.Tk * H_kv) return;
    const int hk = (int)(id / p.Tk), key = (int)(id % p.Tk);
    if (p.ko && (key < p.ko[0] || key >= p.ko[p.B])) return;
    const float* src = part + id * 128 + e;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < n_split; ++s) {
        const float4 x = *reinterpret_cast<const float4*>(src + (int64_t)s * H_kv * p.Tk * 128);
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
    }
    if (e < 64) store4(dK.at(hk, key) + e, make_float4(sum.x * scale, sum.y * scale, sum.z * scale, sum.w * scale));
    else store4(dV.at(hk, key) + e - 64, sum);
}

// dQ of 128 rows: 4 waves of 32, tiles of KT keys and values (64, float32: 32 to each of the KW) through LDS.
template <typename T, int KT, int KW, bool FINE>
__global__ __launch_bounds__(256 * KW, 2)
void packed_dq_kernel(Heads<const T> Q, Heads<const T> K, Heads<const T> V, Heads<const T> dOut, Heads<const T> out, Stats stats, Packing p,
                      Heads<T> dQ, int H_kv, int causal, float scale, float scale_log2, int n_tile)
{
    constexpr int NT = 256 * KW, TILE = KT * KW;       // KW = 2: 8 waves, two to 32 rows, with alternate tiles of KT keys (as in the forward)
    constexpr int CH = 64 * sizeof(T) / 16, NL = TILE * CH / NT;
    constexpr int kBytes = kTileBytes<T, TILE>;
    static_assert(KW == 1 || 4 * kBytes >= 128 * kJoinRow * 4, "the join of 128 rows does not fit the tiles");
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * kBytes];
    unsigned char *const sK = lds, *const sV = lds + 2 * kBytes;
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const SeqTile f = find_tile<128, false>(p, x);
    auto outside = [&] { zero_outside(dQ, p.qo, p.B, p.Tq, hk * p.G, p.G, x, n_tile, [](int, int) {}); };
    if (f.tile < 0) { outside(); return; }
    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;
    auto visible = [&](int r) { const int t = r / p.G; return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int rw = wave & 3, kg = KW == 1 ? 0 : wave >> 2;
    const int row0 = f.tile * 128 + rw * 32;
    const int row = row0 + c, rc = min(row, n_rows - 1);
    const int t = rc / p.G, head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int n_all = __builtin_amdgcn_readfirstlane(visible(min(f.tile * 128 + 127, n_rows - 1)));
    const int n_wave = __builtin_amdgcn_readfirstlane(row0 < n_rows ? visible(min(row0 + 31, n_rows - 1)) : 0);
    const int n_every = __builtin_amdgcn_readfirstlane(visible(min(row0, n_rows - 1)));
    HeadOperand<T> q, g;
    q.load(Q.at(head, f.q0 + t), h);
    g.load(dOut.at(head, f.q0 + t), h);
    const float l = stat_of(stats.lse[(int64_t)head * p.Tq + f.q0 + t]);
    float d = half_row_dot(out.at(head, f.q0 + t), dOut.at(head, f.q0 + t), h);
    d += swap_half(d);
    RowGradient<T> grad;
    grad.init();
    const T* Kh = K.at(hk, f.k0);
    const T* Vh = V.at(hk, f.k0);
    uint4 kr[NL], vr[NL];
    auto fetch = [&](int j0) {
        const int n = min(TILE, f.nk - j0);
        const auto kb = tile_rows(Kh + j0 * K.row, K.row, n), vb = tile_rows(Vh + j0 * V.row, V.row, n);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * NT + tid, r = id / CH, ch = id % CH;
            kr[i] = buffer_load16<uint4>(kb, (int)(r * K.row * (int64_t)sizeof(T)) + ch * 16);
            vr[i] = buffer_load16<uint4>(vb, (int)(r * V.row * (int64_t)sizeof(T)) + ch * 16);
        }
    };
    if (n_all > 0) fetch(0);
    int buf = 0;
    for (int j0 = 0; j0 < n_all; j0 += TILE, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * NT + tid;
            put<TILE>(sK + buf * kBytes, id / CH, id % CH, kr[i], T{});
            put<TILE>(sV + buf * kBytes, id / CH, id % CH, vr[i], T{});
        }
        if (j0 + TILE < n_all) fetch(j0 + TILE);
        lds_barrier();
#pragma unroll
        for (int n = 0; n < KT / 32; ++n) {
            const int in = kg * KT + 32 * n, j = j0 + in;
            if (j >= n_wave) break;
            floatx16 s = product<T, TILE>(sK + buf * kBytes, in, q, c, h);
            floatx16 w = product<T, TILE>(sV + buf * kBytes, in, g, c, h);
            if (sizeof(T) == 2) reads_first<8, 8>();   // (16 x 512: 18.6 -> 17.2 us; dK and dV, with more of its own to keep, lose 3 %)
            grad.weights(s, w, scale_log2, l, d);
            if (j + 32 > n_every) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j + acc_row(r, h) >= n_vis) s[r] = w[r] = 0.f;
            }
            grad.template add<TILE, FINE>(s, w, sK + buf * kBytes, in, c, h);
        }
    }
    outside();                                         // (last: its loads would delay the others)
    if (KW == 2) {
        float* join = reinterpret_cast<float*>(lds) + (rw * 32 + c) * kJoinRow;
        __syncthreads();
        if (kg == 1) store_row(join, grad.dq, 1.f, h);
        __syncthreads();
        if (kg == 1) return;
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) grad.dq[dt][r] += join[32 * dt + acc_row(r, h)];
    }
    if (row >= n_rows) return;
    d += grad.finish();
    store_row(dQ.at(head, f.q0 + t), grad.dq, n_vis == 1 ? 0.f : scale, h); // (the weight of an only key is 1 whatever the scores are)
    if (h == 0) {
        const int64_t so = Stats::at(p, hk, (int64_t)f.q0 * p.G + row);
        stats.l[so] = l;
        stats.d[so] = d;
    }
}

// ---- the same with 32 keys (rows) to a work-group, whose 4 waves divide the rows (keys) among themselves and join their sums in LDS at
// the end.  Four times as many work-groups, each a quarter as long, no barrier before the join; a tile of rows is read by one wave
// only, and 4 times as often.
constexpr int kJoinBytes = 4 * 32 * kJoinRow * 4;
// float32 tiles are 12 KB.  With K and V in registers and a tile of Q and one of dOut to each wave, a compute unit held one work-group, a wave
// to a SIMD; so K and V lie in LDS, and one tile of a wave holds Q, then dOut, then Q again (24 ragged clips of 435: 101 -> 73 us).
template <typename T> constexpr int kDkvTiles = sizeof(T) == 4 ? 6 : 8;
template <typename T> constexpr int kDkvLds = (kDkvTiles<T> * kTileBytes<T, 32> > kJoinBytes ? kDkvTiles<T> * kTileBytes<T, 32> : kJoinBytes) + 4 * 2 * 32 * 4;
template <typename T> constexpr int kDqLds = 4 * kTileBytes<T, 32> > kJoinBytes + 4 * 32 * 4 ? 4 * kTileBytes<T, 32> : kJoinBytes + 4 * 32 * 4;

template <typename T>
__device__ __forceinline__
void dkv_few(unsigned char* lds, int hk, int x, Heads<const T> Q, Heads<const T> K, Heads<const T> V, Heads<const T> dOut, const float* __restrict__ stat_l,
                           const float* __restrict__ stat_d, const Packing& p, Heads<T> dK, Heads<T> dV, int causal, float scale,
                           float scale_log2, int n_tile)
{
    constexpr int CH = 64 * sizeof(T) / 16, NL = 32 * CH / 64, RL = 64 / CH;       // lanes of a row, chunks of a lane, rows of one load
    constexpr int kBytes = kTileBytes<T, 32>;
    float(*const sL)[32] = reinterpret_cast<float(*)[32]>(lds + kDkvLds<T> - 4 * 2 * 32 * 4), (*const sD)[32] = sL + 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const SeqTile f = find_tile<32, true>(p, x);
    auto outside = [&] {
        zero_outside(dK, p.ko, p.B, p.Tk, hk, 1, x, n_tile, [](int, int) {});
        zero_outside(dV, p.ko, p.B, p.Tk, hk, 1, x, n_tile, [](int, int) {});
    };
    if (f.tile < 0) { outside(); return; }
    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;
    auto first_row = [&](int j) { return causal ? max(j - shift + 1, 0) * p.G : 0; };
    const int key0 = f.tile * 32, kc = min(key0 + c, f.nk - 1);
    const int first = first_row(kc);
    const int first_any = __builtin_amdgcn_readfirstlane(first_row(key0));
    const int first_every = __builtin_amdgcn_readfirstlane(first_row(min(key0 + 31, f.nk - 1)));

    constexpr bool kOneTile = sizeof(T) == 4;
    floatx16 dk[2], dv[2];
    clear(dk[0]); clear(dk[1]); clear(dv[0]); clear(dv[1]);
    unsigned char *sK = lds, *sV = lds + kBytes;
    unsigned char *sQ = lds + (kOneTile ? 2 + wave : 2 * wave) * kBytes, *sG = kOneTile ? sQ : sQ + kBytes;
    const int64_t stat0 = ((int64_t)hk * p.Tq + f.q0) * p.G;
    const int lr = lane / CH, ch = lane % CH;
    HeadOperand<T> k, v;
    if constexpr (kOneTile) {
        const int n = min(32, f.nk - key0);
        const auto kb = tile_rows(K.at(hk, f.k0 + key0), K.row, n), vb = tile_rows(V.at(hk, f.k0 + key0), V.row, n);
#pragma unroll
        for (int i = 0; i < 32 * CH / 256; ++i) {
            const int r = (i * 256 + tid) / CH, kc4 = (i * 256 + tid) % CH;
            put<32>(sK, r, kc4, buffer_load16<uint4>(kb, (int)(r * K.row * (int64_t)sizeof(T)) + kc4 * 16), T{});
            put<32>(sV, r, kc4, buffer_load16<uint4>(vb, (int)(r * V.row * (int64_t)sizeof(T)) + kc4 * 16), T{});
        }
        __syncthreads();
    } else {
        k.load(K.at(hk, f.k0 + kc), h);
        v.load(V.at(hk, f.k0 + kc), h);
    }

    // one set of registers carries a tile of Q, then the tile of dOut, then the next tile of Q (float32: one of Q, one of dOut)
    uint4 x4[NL], g4[NL];
    float l_next = INFINITY, d_next = 0.f;
    int r0 = first_any / 32 * 32 + wave * 32;
    const int dt = RL / p.G, dg = RL - dt * p.G, dt128 = 128 / p.G, dg128 = 128 - dt128 * p.G;
    RowAt base(r0 + lr, p.G);                          // of the tile that is fetched
    auto fetch = [&](const Heads<const T>& t, uint4 (&x4)[NL], int r0) {
        RowAt at = base;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            x4[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r0 + lr + i * RL < n_rows) x4[i] = reinterpret_cast<const uint4*>(t.at(hk * p.G + at.g, f.q0 + at.t))[ch];
            at.add(dt, dg, p.G);
        }
    };
    auto keep = [&](unsigned char* s, const uint4 (&x4)[NL]) {
#pragma unroll
        for (int i = 0; i < NL; ++i) put<32>(s, lr + i * RL, ch, x4[i], T{});
    };
    auto fetch_stats = [&](int r0) {
        const bool in = r0 + c < n_rows;
        l_next = in ? stat_l[stat0 + r0 + c] : INFINITY;
        d_next = in ? stat_d[stat0 + r0 + c] : 0.f;
    };
    if (r0 < n_rows) { fetch(Q, x4, r0); fetch_stats(r0); }
    for (; r0 < n_rows; r0 += 128) {
        wave_lds_sync();
        keep(sQ, x4);
        if (h == 0) { sL[wave][c] = l_next; sD[wave][c] = d_next; }
        fetch(dOut, kOneTile ? g4 : x4, r0);
        wave_lds_sync();
        floatx16 s, w;
        if constexpr (kOneTile) s = product<T, 32>(sQ, 0, sK, c, h); else s = product<T, 32>(sQ, 0, k, c, h);
        wave_lds_sync();
        keep(sG, kOneTile ? g4 : x4);
        base.add(dt128, dg128, p.G);
        if (r0 + 128 < n_rows) {
            if (!kOneTile) fetch(Q, x4, r0 + 128);
            fetch_stats(r0 + 128);
        }
        wave_lds_sync();
        if constexpr (kOneTile) w = product<T, 32>(sG, 0, sV, c, h); else w = product<T, 32>(sG, 0, v, c, h);
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const float4 l4 = *reinterpret_cast<const float4*>(&sL[wave][8 * r4 + 4 * h]), d4 = *reinterpret_cast<const float4*>(&sD[wave][8 * r4 + 4 * h]);
            const float l[4] = {l4.x, l4.y, l4.z, l4.w}, d[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[4 * r4 + e] = fast_exp2(fmaf(s[4 * r4 + e], scale_log2, -l[e]));
                w[4 * r4 + e] = s[4 * r4 + e] * (w[4 * r4 + e] - d[e]);
            }
        }
        if (r0 < first_every) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (r0 + acc_row(r, h) < first) s[r] = w[r] = 0.f;
        }
        accumulate<T, 32, true>(dv, sG, 0, s, c, h);
        if (kOneTile) {
            wave_lds_sync();
            keep(sQ, x4);
            if (r0 + 128 < n_rows) fetch(Q, x4, r0 + 128);
            wave_lds_sync();
        }
        accumulate<T, 32, true>(dk, sQ, 0, w, c, h);
    }
    outside();
    float* join = reinterpret_cast<float*>(lds);
    const int key = key0 + (tid >> 3), e = (tid & 7) * 8;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        store_row(join + (wave * 32 + c) * kJoinRow, which ? dv : dk, 1.f, h);
        __syncthreads();
        float sum[8];
        join_columns(sum, join, tid);
        if (key < f.nk) store8((which ? dV : dK).at(hk, f.k0 + key) + e, sum, which ? 1.f : f.nk == 1 ? 0.f : scale);
    }
}

template <typename T, bool FIND_STATS>
__device__ __forceinline__
void dq_few(unsigned char* lds, int hk, int x, Heads<const T> Q, Heads<const T> K, Heads<const T> V, Heads<const T> dOut, Heads<const T> out,
            const Stats& stats, const Packing& p, Heads<T> dQ, int causal, float scale, float scale_log2, int n_tile)
{
    constexpr int CH = 64 * sizeof(T) / 16, NL = 32 * CH / 64;
    constexpr int kBytes = kTileBytes<T, 32>;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const SeqTile f = find_tile<32, false>(p, x);
    auto outside = [&] { zero_outside(dQ, p.qo, p.B, p.Tq, hk * p.G, p.G, x, n_tile, [](int, int) {}); };
    if (f.tile < 0) { outside(); return; }
    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;
    auto visible = [&](int r) { const int t = r / p.G; return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int row0 = f.tile * 32, rc = min(row0 + c, n_rows - 1);
    const int t = rc / p.G, head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int n_all = __builtin_amdgcn_readfirstlane(visible(min(row0 + 31, n_rows - 1)));
    const int n_every = __builtin_amdgcn_readfirstlane(visible(row0));
    HeadOperand<T> q, g;
    q.load(Q.at(head, f.q0 + t), h);
    g.load(dOut.at(head, f.q0 + t), h);
    const int64_t so = Stats::at(p, hk, (int64_t)f.q0 * p.G + rc);
    float l, d;
    if (FIND_STATS) {
        l = stat_of(stats.lse[(int64_t)head * p.Tq + f.q0 + t]);
        d = half_row_dot(out.at(head, f.q0 + t), dOut.at(head, f.q0 + t), h);
        d += swap_half(d);
    } else {
        l = stats.l[so];
        d = stats.d[so];
    }
    RowGradient<T> grad;
    grad.init();
    const T* Kh = K.at(hk, f.k0);
    const T* Vh = V.at(hk, f.k0);
    unsigned char* sK = lds + wave * kBytes;
    uint4 kn[NL];
    HeadRow<T> vn;
    auto fetch = [&](int j0) {
        const int n = min(32, f.nk - j0);
        const auto kb = tile_rows(Kh + j0 * K.row, K.row, n), vb = tile_rows(Vh + j0 * V.row, V.row, n);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 64 + lane;
            kn[i] = buffer_load16<uint4>(kb, (int)((id / CH) * K.row * (int64_t)sizeof(T)) + (id % CH) * 16);
        }
        vn.load(vb, (int)(c * V.row * (int64_t)sizeof(T)), h);
    };
    int j0 = wave * 32;
    if (j0 < n_all) fetch(j0);
    for (; j0 < n_all; j0 += 128) {
        wave_lds_sync();
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 64 + lane;
            put<32>(sK, id / CH, id % CH, kn[i], T{});
        }
        floatx16 w = product(vn, g);
        wave_lds_sync();
        if (j0 + 128 < n_all) fetch(j0 + 128);
        floatx16 s = product<T, 32>(sK, 0, q, c, h);
        grad.weights(s, w, scale_log2, l, d);
        if (j0 + 32 > n_every) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (j0 + acc_row(r, h) >= n_vis) s[r] = w[r] = 0.f;
        }
        grad.template add<32, true>(s, w, sK, 0, c, h);
    }
    outside();
    __syncthreads();
    float* join = reinterpret_cast<float*>(lds);
    const int jr = tid >> 3, row = row0 + jr, rt = min(row, n_rows - 1) / p.G;
    store_row(join + (wave * 32 + c) * kJoinRow, grad.dq, 1.f, h);
    __syncthreads();
    float sum[8];
    join_columns(sum, join, tid);
    if constexpr (sizeof(T) == 2) {
        // e is the sum of the waves' parts, then d and sum_j p_j K[j] as in RowGradient::finish()
        float* join_e = reinterpret_cast<float*>(lds + kJoinBytes);
        const float e = grad.e + swap_half(grad.e);
        __syncthreads();
        store_row(join + (wave * 32 + c) * kJoinRow, grad.pk, 1.f, h);
        if (h == 0) join_e[wave * 32 + c] = e;
        __syncthreads();
        float pk[8];
        join_columns(pk, join, tid);
        auto whole = [&](int r) { return ((join_e[r] + join_e[32 + r]) + join_e[64 + r]) + join_e[96 + r]; };
        const float er = whole(jr);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(-er, pk[i], sum[i]);
        d += whole(c);
    }
    if (FIND_STATS && wave == 0 && h == 0 && row0 + c < n_rows) { stats.l[so] = l; stats.d[so] = d; }
    if (row >= n_rows) return;
    store8(dQ.at(hk * p.G + (row - rt * p.G), f.q0 + rt) + (tid & 7) * 8, sum, visible(row) == 1 ? 0.f : scale);
}

// The first n_k work-groups form dK and dV, the others dQ: both or (n_k = 0, or as many as there are) one of them.  One launch where both take
// few keys and rows of float32: such calls leave the card idle, and with d from a launch of its own the two do not depend on each other (2 clips
// of 400: 43.7 | 24.4 us).
template <typename T, bool DKV, bool DQ>
__global__ __launch_bounds__(256, 2)
void packed_grads_few_kernel(Heads<const T> Q, Heads<const T> K, Heads<const T> V, Heads<const T> dOut, Heads<const T> out, Stats stats, Packing p,
                             Heads<T> dQ, Heads<T> dK, Heads<T> dV, int H_kv, int causal, float scale, float scale_log2, int n_ktile, int n_qtile)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[DKV ? kDkvLds<T> : kDqLds<T>];
    const int n_k = DKV ? n_ktile * H_kv : 0, id = (int)blockIdx.x;
    if (DKV && (!DQ || id < n_k))
        dkv_few<T>(lds, id % H_kv, id / H_kv, Q, K, V, dOut, stats.l, stats.d, p, dK, dV, causal, scale, scale_log2, n_ktile);
    else if (DQ)
        dq_few<T, !DKV>(lds, (id - n_k) % H_kv, (id - n_k) / H_kv, Q, K, V, dOut, out, stats, p, dQ, causal, scale, scale_log2, n_qtile);
}

PackedBwdPlan make_packed_bwd_plan(const psa_packed_shape_t& s)
{
    PackedBwdPlan p{};
    const int64_t rows = (int64_t)s.T_q * (s.H / s.H_kv);
    // dQ: enough work-groups of 128 rows, as in the forward.  (24 ragged clips of 435 frames, 374 work-groups, 128 | 32: 20.5 | 25.3 us, 2 clips,
    // 32 of them, 15 | 7.5.)  dK and dV, whose work-groups differ more in length: at 210 of them 48 | 26 us, at 280 36.9 | 31.4, at 320
    // 23.6 | 28.9, float32 at 210 168 | 107.
    // 32 not in bfloat16 where the other axis is over in a step of 64: 50 sequences of 1 to 60 frames, 4 heads, 32 | 128: dQ 8.8 | 6.5, dK and dV
    // 7.4 | 6.1 us; 8 of 60 to 130: 7.9 | 8.9 and 6.6 | 8.0.  (float32, one launch for both: 17.0 and 3.1 for d | 22.6)
    const int64_t wide = (rows / 128 + s.B) * s.H_kv;
    const bool one = s.dtype == PSA_F32;               // (may take one launch for both)
    p.fine_q = packed_fine(s, wide);
    // 16 bits to the weights of dK and dV in small calls, as in the forward, and wherever few keys are read by many rows: once | two parts, with the
    // rest of the call, 13 of 539 to 1079 below 85 | 92 us, 8 of 1000 to 2000 171 | 193, one of 16000 957 | 1135.
    const int64_t wide_k = (int64_t)(s.T_k / 128 + s.B) * s.H_kv;
    p.fine_k = wide_k < 300 || (wide_k <= 512 && rows / s.B <= 64);
    p.few_k = wide_k < 300 && (one || rows / s.B > 64);
    // Many rows to a key head (several heads, long sequences): 128 keys and a part of the rows each, towards two work-groups to a compute unit.
    // 32 keys | so, with the join: 13 sequences of 539 to 1079, 4 heads to a key head, 57 | 38 us (towards three: 44), 8 of 1000 to 2000, 2 times
    // 4, 116 | 92, one of 16000 838 | 450; float32 173 | 122.  But one of 1863, a head each, 31 | 34, 9 of 280, 2 to a key head, 11.6 | 20.
    p.n_split = 1;
    if (p.few_k && rows / s.B >= 2048) {
        const int64_t wgs = (int64_t)(s.T_k / 128 + s.B) * s.H_kv, split = (511 + wgs) / wgs;
        p.n_split = (int)(split < 16 ? split : 16);
        p.few_k = 0;
    }
    p.few_q = one && p.few_k ? wide < 256 : !packed_enough(s, wide) && s.T_k / s.B > 64;
    p.halves_q = !p.few_q && packed_halves(s, wide);
    p.n_qtile = (int)(rows / (p.few_q ? 32 : 128)) + s.B;
    p.n_ktile = s.T_k / (p.few_k ? 32 : 128) + s.B;
    p.stat_bytes = ((size_t)s.T_q * s.H * sizeof(float) + 255) & ~(size_t)255;
    p.off_part = 2 * (p.stat_bytes + packed_before_bytes(s.B));
    p.total = p.off_part + (p.n_split > 1 ? (size_t)p.n_split * s.H_kv * s.T_k * 128 * sizeof(float) : 0);
    return p;
}

template <typename T>
static void packed_bwd_go(const PackedBwdPlan& p, const psa_packed_shape_t& s, const psa_heads_t& Q, const psa_heads_t& K, const psa_heads_t& V,
                          const Packing& pk, const psa_heads_t& out, const float* lse, const psa_heads_t& dOut, const psa_heads_t& dQ,
                          const psa_heads_t& dK, const psa_heads_t& dV, void* workspace, hipStream_t stream)
{
    const Stats st{static_cast<float*>(workspace), reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + p.stat_bytes), lse};
    const float scale = (float)s.scale, scale_log2 = (float)(s.scale * 1.4426950408889634);
    const auto q = heads_of<const T>(Q), k = heads_of<const T>(K), v = heads_of<const T>(V), g = heads_of<const T>(dOut), o = heads_of<const T>(out);
    const auto dq = heads_of<T>(dQ), dk = heads_of<T>(dK), dv = heads_of<T>(dV);
    const unsigned n_k = (unsigned)(p.n_ktile * s.H_kv), n_q = (unsigned)(p.n_qtile * s.H_kv);
    constexpr int KT = sizeof(T) == 4 ? 32 : 64, KW = sizeof(T) == 4 ? 2 : 1;
    constexpr bool FINE = sizeof(T) == 2;
    if constexpr (sizeof(T) == 4) {
        if (p.few_k && p.few_q) {
            constexpr int rows = 256 / (64 / kVec<T>);
            packed_stats_kernel<T><<<(unsigned)(((int64_t)s.T_q * s.H + rows - 1) / rows), 256, 0, stream>>>(o, g, lse, pk, s.H, st.l, st.d);
            packed_grads_few_kernel<T, true, true><<<n_k + n_q, 256, 0, stream>>>(q, k, v, g, o, st, pk, dq, dk, dv, s.H_kv, s.causal, scale, scale_log2, p.n_ktile, p.n_qtile);
            return;
        }
    }
    if (p.few_q)
        packed_grads_few_kernel<T, false, true><<<n_q, 256, 0, stream>>>(q, k, v, g, o, st, pk, dq, dk, dv, s.H_kv, s.causal, scale, scale_log2, p.n_ktile, p.n_qtile);
    else
        (p.halves_q ? packed_dq_kernel<T, KT, KW, false> : p.fine_q ? packed_dq_kernel<T, KT, 1, FINE> : packed_dq_kernel<T, KT, 1, false>)<<<n_q, p.halves_q ? 512 : 256, 0, stream>>>(
            q, k, v, g, o, st, pk, dq, s.H_kv, s.causal, scale, scale_log2, p.n_qtile);
    if (p.few_k)
        packed_grads_few_kernel<T, true, false><<<n_k, 256, 0, stream>>>(q, k, v, g, o, st, pk, dq, dk, dv, s.H_kv, s.causal, scale, scale_log2, p.n_ktile, p.n_qtile);
    else {
        float* part = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + p.off_part);
        (p.fine_k ? packed_dkv_kernel<T, KT, FINE> : packed_dkv_kernel<T, KT, false>)<<<dim3(n_k, p.n_split), 256, 0, stream>>>(q, k, v, g, st.l, st.d, pk, dk, dv, s.H_kv, s.causal, scale, scale_log2, p.n_ktile,
                                                                          p.n_split, part);
        if (p.n_split > 1)
            packed_join_keys_kernel<T><<<(unsigned)(((int64_t)s.T_k * s.H_kv + 7) / 8), 256, 0, stream>>>(part, p.n_split, pk, dk, dv, s.H_kv, scale);
    }
}
hipError_t launch_packed_bwd(const PackedBwdPlan& p, const psa_packed_shape_t& s, const psa_heads_t& Q, const psa_heads_t& K, const psa_heads_t& V,
                             const int* q_offsets, const int* k_offsets, const psa_heads_t& out, const float* lse, const psa_heads_t& dOut,
                             const psa_heads_t& dQ, const psa_heads_t& dK, const psa_heads_t& dV, void* workspace, hipStream_t stream)
{
    const Packing pk = make_packing(s, q_offsets, k_offsets, p.few_q ? 32 : 128, p.few_k ? 32 : 128, static_cast<unsigned char*>(workspace) + 2 * p.stat_bytes,
                                    true, stream);
    if (s.dtype == PSA_F32) packed_bwd_go<float>(p, s, Q, K, V, pk, out, lse, dOut, dQ, dK, dV, workspace, stream);
    else packed_bwd_go<bf16_t>(p, s, Q, K, V, pk, out, lse, dOut, dQ, dK, dV, workspace, stream);
    return hipGetLastError();
}

}  // namespace psa
