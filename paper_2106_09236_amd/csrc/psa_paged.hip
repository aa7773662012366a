// Dense attention over a cache in pages: softmax(scale Q K^T) V of the newest rows of each sequence, whose keys and values
// lie in pages named by a table.  The arithmetic is that of the packed kernels (psa_packed.h): rows are (query, head of the
// group) pairs, 32 to a wave, on the columns of the matrix instruction; keys in one pass with online softmax.
//
// Work.  The rows of a sequence are tiles of ROWS, and its keys are cut into splits of `chunk` keys, the same number
// for all its tiles.  `chunk` is found on the device from all lengths (find_part), so that the work-groups of a call are
// about `target` whatever the lengths are, and equal: a call that was captured serves as its sequences grow.  Sequences
// cut in several splits leave partial sums in the workspace, joined by a second kernel.
#include "psa_paged.h"

namespace psa {

__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

// Sequence s as the call has it: rows q0 .. q0 + nq - 1, nk keys
struct PagedSeq { int q0, nq, nk; };
__device__ __forceinline__ PagedSeq paged_seq(const PagedSeqs& p, int s)
{
    PagedSeq r{0, 0, 0};
    if (s < p.B) {
        if (p.offsets) {
            r.q0 = min(max(p.offsets[s], 0), p.T);
            r.nq = min(max(p.offsets[s + 1], r.q0), p.T) - r.q0;
        } else {
            r.q0 = s * p.uniform;
            r.nq = p.uniform;
        }
        r.nk = min(max(p.lengths[s], 0), p.capacity);
    }
    return r;
}
__device__ __forceinline__ int units_of(int nk) { return (nk + kUnit - 1) / kUnit; }
// tiles of a sequence of nq rows, and the splits of its keys, `chunk` units each
__device__ __forceinline__ int tiles_of(int nq, int G, int rows) { return (nq * G + rows - 1) / rows; }
__device__ __forceinline__ int splits_of(int nk, int chunk) { return max(1, (units_of(nk) + chunk - 1) / chunk); }

// Units of keys to a split: the work of all tiles (units times tiles) in about p.per_head shares, kLeastUnits at the least.  Every
// work-group of a call and of its join finds the same.  Summed in float64: offsets that decrease may claim 2^67.
__device__ __forceinline__ double wave_sum64(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ __forceinline__ int chunk_for(const PagedSeqs& p, double work) { return (int)fmin(fmax(ceil(work / p.per_head), (double)kLeastUnits), (double)(1 << 23)); }
__device__ __forceinline__ double work_of(const PagedSeqs& p, int s)
{
    const PagedSeq r = paged_seq(p, s);
    return (double)units_of(r.nk) * tiles_of(r.nq, p.G, p.rows);
}

// What a work-group takes: tile `tile` of sequence `seq`, split `split` of `splits`; `slot`: where the partial sums of its sequence
// begin (tile t, split i at slot + i * tiles + t); seq < 0: nothing.  JOIN: the pieces are the 32-row parts of the sequences with
// more than one split, and `tile` counts those.
struct Part { int seq, q0, nq, nk, tiles, tile, split, splits, chunk, slot; };
template <bool JOIN>
__device__ __forceinline__ Part find_part(const PagedSeqs& p, int x)
{
    Part f{};
    f.seq = -1;
    const int lane = threadIdx.x & 63;
    int s0 = 0, end = p.B, slot = 0;
    if (p.before) {
        // many sequences: the chunk and the parts, slots and joined pieces before each 64 of them have been summed up; the last 64
        // with at most x before them
        f.chunk = p.before[0];
        const int groups = (p.B + 63) / 64;
        const int* before = p.before + 1 + (JOIN ? 2 * groups : 0);
        int lo = 0, n = groups;
        while (n > 1) {
            const int step = (n + 63) / 64, i = lane * step;
            const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < n && before[min(lo + i, groups - 1)] <= x)) - 1;
            lo += k * step;
            n = min(step, n - k * step);
        }
        x -= before[lo];
        slot = p.before[1 + groups + lo];
        s0 = lo * 64;
        end = min(end, s0 + 64);
    } else {
        double work = 0.0;
        for (int s = lane; s < p.B; s += 64) work += work_of(p, s);
        f.chunk = chunk_for(p, wave_sum64(work));
    }
    for (; s0 < end; s0 += 64) {
        const PagedSeq r = paged_seq(p, s0 + lane);
        const int tiles = tiles_of(r.nq, p.G, p.rows), splits = splits_of(r.nk, f.chunk);
        // (a call has fewer than 2^24 parts, but where offsets decrease each sequence may claim all of its rows; there are never more
        // slots than twice p.per_head, since a sequence's parts are at most twice its work over the chunk)
        const int parts = tiles * splits, slots = splits > 1 ? parts : 0;
        const int n = min(JOIN ? (splits > 1 ? tiles_of(r.nq, p.G, 32) : 0) : parts, 1 << 24);
        const int sum = wave_scan(n), all = last_lane(sum);
        const int slot_sum = wave_scan(slots);
        if (x < all) {
            const int l = __builtin_popcountll(__builtin_amdgcn_ballot_w64(sum <= x));
            f.seq = s0 + l;
            f.q0 = __builtin_amdgcn_readlane(r.q0, l); f.nq = __builtin_amdgcn_readlane(r.nq, l); f.nk = __builtin_amdgcn_readlane(r.nk, l);
            f.tiles = __builtin_amdgcn_readlane(tiles, l); f.splits = __builtin_amdgcn_readlane(splits, l);
            f.slot = slot + __builtin_amdgcn_readlane(slot_sum - slots, l);
            const int y = x - __builtin_amdgcn_readlane(sum - n, l);
            if (JOIN) {
                f.tile = y;
            } else {
                f.split = y / f.tiles;                 // (the tiles of one split after each other: they read the same keys)
                f.tile = f.tiles - 1 - (y - f.split * f.tiles);
            }
            return f;
        }
        x -= all;
        slot += last_lane(slot_sum);
    }
    return f;
}
// The sums that find_part reads where there are many sequences.  They stop at 2^29, so that they do not overflow (where offsets
// decrease each sequence may claim all rows) and stay in order.
constexpr int kMostParts = 1 << 29;
__global__ __launch_bounds__(1024)
void paged_before_kernel(PagedSeqs p, int* __restrict__ before)
{
    __shared__ double s_work[16];
    __shared__ int s[2][3][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = (p.B + 63) / 64;
    double work = 0.0;
    for (int i = threadIdx.x; i < p.B; i += 1024) work += work_of(p, i);
    work = wave_sum64(work);
    if (lane == 0) s_work[wave] = work;
    __syncthreads();
    work = 0.0;
    for (int w = 0; w < 16; ++w) work += s_work[w];
    const int chunk = chunk_for(p, work);
    if (threadIdx.x == 0) before[0] = chunk;
    int sum[3] = {0, 0, 0};
    for (int g0 = 0, buf = 0; g0 < groups; g0 += 16, buf ^= 1) {
        const int g = g0 + wave;
        const PagedSeq r = paged_seq(p, g < groups ? g * 64 + lane : p.B);
        const int splits = splits_of(r.nk, chunk);
        const int64_t parts = (int64_t)tiles_of(r.nq, p.G, p.rows) * splits;
        const int64_t n[3] = {parts, splits > 1 ? parts : 0, splits > 1 ? tiles_of(r.nq, p.G, 32) : 0};
        for (int k = 0; k < 3; ++k) {
            const double all = wave_sum64((double)n[k]);
            if (lane == 0) s[buf][k][wave] = (int)fmin(all, (double)kMostParts);
        }
        __syncthreads();
        for (int k = 0; k < 3; ++k) {
            int mine = sum[k], all = sum[k];
            for (int w = 0; w < 16; ++w) {
                if (w < wave) mine = min(mine + s[buf][k][w], kMostParts);
                all = min(all + s[buf][k][w], kMostParts);
            }
            if (g < groups && lane == 0) before[1 + k * groups + g] = mine;
            sum[k] = all;
        }
    }
}

// ---- rows of the cache on their way
// Row j of a sequence: where it lies, in rows of its head's pages; < 0: on no page or behind the last.
struct PageTable {
    const int* row; int shift, n_pages, nk;
    __device__ __forceinline__ int page(int j) const {
        const int p = j < nk ? row[j >> shift] : -1;
        return (unsigned)p < (unsigned)n_pages ? p : -1;
    }
};
template <typename C>
__device__ __forceinline__ const C* row_at(const PageHeads<const C>& t, int hk, int page, int slot) { return t.data + hk * t.head + page * t.page + slot * t.row; }

template <typename V> __device__ __forceinline__ V load_or_zero(const void* p, bool valid)
{
    V v = {};
    if (valid) v = *static_cast<const V*>(p);
    return v;
}

// 8-bit elements: pairs of codes to pairs of bfloat16, times their power of two, exactly
__device__ __forceinline__ float mx_power(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ uint4 mx_codes(uint32_t a, uint32_t b, float power)
{
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, power, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, power, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, power, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, power, true)));
}

// What a tile of the cache is multiplied as: 8-bit elements as bfloat16
template <typename C> struct TileOf { typedef C type; };
template <> struct TileOf<mx8_t> { typedef bf16_t type; };

// Half a key's row, elements 32 h .., as the first operand of the product with the queries
template <typename C> struct KeyRow : HeadRow<C> {
    __device__ __forceinline__ void load(const C* row, const uint8_t*, bool valid, int h) {
#pragma unroll
        for (int i = 0; i < HeadRow<C>::N; ++i) this->x[i] = load_or_zero<uint4>(row + 32 * h + i * (16 / (int)sizeof(C)), valid);
    }
};
template <> struct KeyRow<mx8_t> {
    uint4 x[2];
    uint32_t power;
    __device__ __forceinline__ void load(const mx8_t* row, const uint8_t* scales, bool valid, int h) {
        x[0] = load_or_zero<uint4>(row + 32 * h, valid);
        x[1] = load_or_zero<uint4>(row + 32 * h + 16, valid);
        power = load_or_zero<uint8_t>(scales + h, valid);
    }
    __device__ __forceinline__ Operand<bf16_t> step(int k) const {
        const uint4& y = x[k >> 1];
        return operand(k & 1 ? mx_codes(y.z, y.w, mx_power(power)) : mx_codes(y.x, y.y, mx_power(power)), bf16_t{});
    }
};
// 16 bytes of a row, chunk ch of it, on their way into a tile
template <typename C> struct RowChunk {
    static constexpr int N = 1;                        // chunks of the tile's type
    uint4 x;
    __device__ __forceinline__ void load(const C* row, const uint8_t*, bool valid, int ch) { x = load_or_zero<uint4>(row + ch * (16 / (int)sizeof(C)), valid); }
    __device__ __forceinline__ void unpack(uint4* to) const { to[0] = x; }
};
template <> struct RowChunk<mx8_t> {
    static constexpr int N = 2;
    uint4 x;
    uint32_t power;
    __device__ __forceinline__ void load(const mx8_t* row, const uint8_t* scales, bool valid, int ch) {
        x = load_or_zero<uint4>(row + ch * 16, valid);
        power = load_or_zero<uint8_t>(scales + (ch >> 1), valid);
    }
    __device__ __forceinline__ void unpack(uint4* to) const {
        to[0] = mx_codes(x.x, x.y, mx_power(power));
        to[1] = mx_codes(x.z, x.w, mx_power(power));
    }
};

__device__ __forceinline__ floatx16 mfma(const Operand<bf16_t>& a, const Operand<float>& b, floatx16 d)
{
    d = mfma(a.v[0], b.v[2], d);           // a product with a bfloat16 number is that of three parts, exactly
    d = mfma(a.v[0], b.v[1], d);
    return mfma(a.v[0], b.v[0], d);
}

// Element e of a value's row, for the sums of infinities and NaN
template <typename C> __device__ __forceinline__ float value_at(const C* row, const uint8_t*, int e) { return to_f32(row[e]); }
template <> __device__ __forceinline__ float value_at<mx8_t>(const mx8_t* row, const uint8_t* scales, int e)
{
    return (row[e].x & 0x7F) == 0x7F ? __uint_as_float(0x7FC00000u) : 0.f;       // (no infinities, and nothing else is asked for)
}
// The infinities and NaN of values j0 .. j0 + n - 1 that were left out of the tile: to the rows that see them
template <typename C>
__device__ __forceinline__ void add_nonfinite(Rows32& acc, const PageHeads<const C>& V, const PageScales& vs, const PageTable& pt, int hk, int j0, int n, int n_vis, int h)
{
    for (int j = j0; j < j0 + n; ++j) {
        const int page = pt.page(j);
        if (page < 0) continue;
        const int slot = j & ((1 << pt.shift) - 1);
        const C* row = row_at(V, hk, page, slot);
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float x = value_at(row, vs.at(hk, page, slot), 32 * dt + acc_row(r, h));
                if (j < n_vis && !isfinite(x)) acc.o[dt][r] += x;
            }
    }
}

// D^T[e][col] += sum over 32 values of V[value][e] w[value] as accumulate() of the packed kernels, the values' tile of another type
template <typename T, typename TC, int ROWS, bool FINE>
__device__ __forceinline__ void accumulate_rows(floatx16 (&d)[2], const unsigned char* s, int row0, const floatx16& w, int c, int h)
{
    constexpr int N = kWeightParts<T, FINE>;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        Operand<T> b[N];
        weight_operand(b, w, st);
#pragma unroll
        for (int dt = 0; dt < 2; ++dt) {
            const Operand<TC> a = tile_transposed<TC, ROWS>(s, row0, st, dt, c, h);
#pragma unroll
            for (int n = 0; n < N; ++n) d[dt] = mfma(a, b[n], d[dt]);
        }
    }
}
template <typename T, typename TC, int ROWS>
__device__ __forceinline__ floatx16 product_rows(const unsigned char* s, int row0, const HeadOperand<T>& b, int c, int h)
{
    floatx16 d;
    clear(d);
#pragma unroll
    for (int k = 0; k < 4; ++k) d = mfma(tile_operand<TC, ROWS>(s, row0, k, c, h), b.v[k], d);
    return d;
}

// Zeros and -infinity in the rows of Q that are in no sequence
template <typename T>
__device__ __forceinline__ void outside_rows(const PagedSeqs& p, const Heads<T>& out, float* lse, int hk, int x, int n_part)
{
    zero_outside(out, p.offsets, p.B, p.T, hk * p.G, p.G, x, n_part, [&](int head, int row) { if (lse) lse[(int64_t)head * p.T + row] = -INFINITY; });
}

// ---- many rows: 4 waves of 32 rows each; tiles of KT keys and values go through LDS, the next tile's rows are on their way meanwhile.
template <typename T, typename C, int KT, bool FINE>
__global__ __launch_bounds__(256, sizeof(T) == 4 || FINE ? 2 : 3)
void paged_rows_kernel(Heads<const T> Q, PageHeads<const C> K, PageHeads<const C> V, PageScales ks, PageScales vs, PagedSeqs p, Heads<T> out,
                       float* __restrict__ lse, int H_kv, int causal, float scale, int n_part, float* __restrict__ part_o, float2* __restrict__ part_ml)
{
    typedef typename TileOf<C>::type TC;
    constexpr int CH = 64 * sizeof(C) / 16;            // 16-byte chunks of a row in the cache
    constexpr int NL = KT * CH / 256;                  // chunks of a tile, to a thread
    constexpr int NS = KT / 32;
    constexpr int NU = RowChunk<C>::N;
    constexpr int kBytes = kTileBytes<TC, KT>;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * kBytes];
    __shared__ int s_bad[2][4];
    unsigned char *const sK = lds, *const sV = lds + 2 * kBytes;
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const Part f = find_part<false>(p, x);
    if (f.seq < 0) { outside_rows(p, out, lse, hk, x, n_part); return; }

    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;                 // causal: query t sees the first t + shift keys
    auto visible = [&](int r) { const int t = r / p.G; return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int row0 = f.tile * 128 + wave * 32;
    const int row = row0 + c, rc = min(row, n_rows - 1);
    const int t = rc / p.G, head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int begin = f.split * f.chunk * kUnit;
    const int cut = f.split + 1 < f.splits ? begin + f.chunk * kUnit : f.nk;
    const int n_all = min(cut, __builtin_amdgcn_readfirstlane(visible(min(f.tile * 128 + 127, n_rows - 1))));
    const int n_every = __builtin_amdgcn_readfirstlane(visible(f.tile * 128));
    const int n_wave = min(cut, __builtin_amdgcn_readfirstlane(row0 < n_rows ? visible(min(row0 + 31, n_rows - 1)) : 0));
    const int n_wave_every = __builtin_amdgcn_readfirstlane(visible(min(row0, n_rows - 1)));

    HeadOperand<T> q;
    q.load(Q.at(head, f.q0 + t), h);
    const PageTable pt{p.table + (int64_t)f.seq * p.max_pages, p.shift, p.n_pages, f.nk};
    const int slot_mask = (1 << p.shift) - 1;
    RowChunk<C> kr[NL], vr[NL];
    uint32_t held[NS], held_next[NS];
    auto fetch = [&](int j0) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 256 + tid, j = j0 + id / CH, page = pt.page(j), slot = j & slot_mask;
            kr[i].load(row_at(K, hk, page, slot), ks.at(hk, page, slot), page >= 0, id % CH);
            vr[i].load(row_at(V, hk, page, slot), vs.at(hk, page, slot), page >= 0, id % CH);
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) held_next[n] = (uint32_t)__builtin_amdgcn_ballot_w64(pt.page(j0 + 32 * n + c) >= 0);
    };
    Rows32 acc;
    acc.init();
    if (begin < n_all) fetch(begin);
    int buf = 0;
    for (int j0 = begin; j0 < n_all; j0 += KT, buf ^= 1) {
        // a weight of 0 does not keep an infinity or NaN of a value that a row does not see out of its sum: in tiles that
        // some row sees in part they are left out and added afterwards (float32: in all, since an infinity has no parts)
        const bool look = sizeof(T) == 4 || FINE || j0 + KT > n_every;
        uint4 v[NL * NU];
#pragma unroll
        for (int i = 0; i < NL; ++i) vr[i].unpack(v + i * NU);
        if (look) {
            const bool any = __builtin_amdgcn_ballot_w64(nonfinite(v, TC{})) != 0;
            if (lane == 0) s_bad[buf][wave] = any;
            if (any)
#pragma unroll
                for (int i = 0; i < NL * NU; ++i) v[i] = finite_only(v[i], TC{});
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 256 + tid;
            uint4 k[NU];
            kr[i].unpack(k);
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                put<KT>(sK + buf * kBytes, id / CH, id % CH * NU + u, k[u], TC{});
                put<KT>(sV + buf * kBytes, id / CH, id % CH * NU + u, v[i * NU + u], TC{});
            }
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) held[n] = held_next[n];
        if (j0 + KT < n_all) fetch(j0 + KT);
        lds_barrier();
        if (j0 >= n_wave) continue;
        floatx16 s[NS];
        uint32_t all = ~0u;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            s[n] = product_rows<T, TC, KT>(sK + buf * kBytes, 32 * n, q, c, h);
            all &= held[n];
        }
        if (j0 + KT > n_wave_every || all != ~0u) {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = j0 + 32 * n + acc_row(r, h) < n_vis && (held[n] >> acc_row(r, h) & 1) ? s[n][r] : -INFINITY;
        }
        acc.follow(s, scale);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            acc.weights(s[n], scale);
            accumulate_rows<T, TC, KT, FINE>(acc.o, sV + buf * kBytes, 32 * n, s[n], c, h);
        }
        if (look) {
            int any = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) any |= s_bad[buf][w];
            if (any) add_nonfinite(acc, V, vs, pt, hk, j0, min(KT, f.nk - j0), n_vis, h);
        }
    }
    outside_rows(p, out, lse, hk, x, n_part);          // (last: its loads would delay the others)
    if (row >= n_rows) return;
    const float l = acc.l + swap_half(acc.l);
    if (f.splits > 1) {
        const int64_t rec = ((int64_t)(f.slot + f.split * f.tiles + f.tile) * H_kv + hk) * 128 + wave * 32 + c;
        store_row(part_o + rec * 64, acc.o, 1.f, h);
        if (h == 0) part_ml[rec] = make_float2(acc.m, l);
        return;
    }
    if (l == 0.f) { clear(acc.o[0]); clear(acc.o[1]); }
    store_row(out.at(head, f.q0 + t), acc.o, l != 0.f ? 1.f / l : 0.f, h);
    if (lse && h == 0) lse[(int64_t)head * p.T + f.q0 + t] = l != 0.f ? acc.m * kLn2 + logf(l) : -INFINITY;
}

// ---- few rows: 32 to a work-group, whose 4 waves divide the keys (of its split) among themselves, 32 at a time, and join their
// sums at the end.  Keys come straight from memory as the first product's operand, values through LDS of the wave's own;
// there is no barrier before the join.
template <typename T, typename C>
__global__ __launch_bounds__(256, 2)
void paged_few_kernel(Heads<const T> Q, PageHeads<const C> K, PageHeads<const C> V, PageScales ks, PageScales vs, PagedSeqs p, Heads<T> out,
                      float* __restrict__ lse, int H_kv, int causal, float scale, int n_part, float* __restrict__ part_o, float2* __restrict__ part_ml)
{
    typedef typename TileOf<C>::type TC;
    constexpr int CH = 64 * sizeof(C) / 16;
    constexpr int NL = 32 * CH / 64;                   // chunks of a tile of 32 rows, to a lane
    constexpr int NU = RowChunk<C>::N;
    constexpr int kBytes = kTileBytes<TC, 32>;
    constexpr int kJoinBytes = 4 * 32 * kJoinRow * 4;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * kBytes > kJoinBytes ? 4 * kBytes : kJoinBytes];
    __shared__ float s_m[4][32], s_l[4][32];
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const Part f = find_part<false>(p, x);
    if (f.seq < 0) { outside_rows(p, out, lse, hk, x, n_part); return; }
    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;
    auto visible = [&](int r) { const int t = r / p.G; return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int row0 = f.tile * 32, row = row0 + c, rc = min(row, n_rows - 1);
    const int t = rc / p.G, head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int begin = f.split * f.chunk * kUnit;
    const int cut = f.split + 1 < f.splits ? begin + f.chunk * kUnit : f.nk;
    const int end = min(cut, __builtin_amdgcn_readfirstlane(visible(min(row0 + 31, n_rows - 1))));
    const int n_every = __builtin_amdgcn_readfirstlane(visible(row0));

    HeadOperand<T> q;
    q.load(Q.at(head, f.q0 + t), h);
    const PageTable pt{p.table + (int64_t)f.seq * p.max_pages, p.shift, p.n_pages, f.nk};
    const int slot_mask = (1 << p.shift) - 1;
    unsigned char* sV = lds + wave * kBytes;
    KeyRow<C> kn;
    RowChunk<C> vn[NL];
    uint32_t held_next = 0;
    auto fetch = [&](int j0) {
        const int j = j0 + c, page = pt.page(j), slot = j & slot_mask;
        kn.load(row_at(K, hk, page, slot), ks.at(hk, page, slot), page >= 0, h);
        held_next = (uint32_t)__builtin_amdgcn_ballot_w64(page >= 0);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 64 + lane, jv = j0 + id / CH, pv = pt.page(jv), sv = jv & slot_mask;
            vn[i].load(row_at(V, hk, pv, sv), vs.at(hk, pv, sv), pv >= 0, id % CH);
        }
    };
    Rows32 acc;
    acc.init();
    int j0 = begin + wave * 32;
    if (j0 < end) fetch(j0);
    for (; j0 < end; j0 += 128) {
        // infinities and NaN of V are left out of the product and added afterwards, in whole tiles too: the weights have parts of either
        // sign and of 0
        uint4 v[NL * NU];
#pragma unroll
        for (int i = 0; i < NL; ++i) vn[i].unpack(v + i * NU);
        const bool any = __builtin_amdgcn_ballot_w64(nonfinite(v, TC{})) != 0;
        if (any)
#pragma unroll
            for (int i = 0; i < NL * NU; ++i) v[i] = finite_only(v[i], TC{});
        wave_lds_sync();
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int id = i * 64 + lane;
#pragma unroll
            for (int u = 0; u < NU; ++u) put<32>(sV, id / CH, id % CH * NU + u, v[i * NU + u], TC{});
        }
        floatx16 s[1];
        clear(s[0]);
#pragma unroll
        for (int k = 0; k < 4; ++k) s[0] = mfma(kn.step(k), q.v[k], s[0]);
        wave_lds_sync();
        const uint32_t held = held_next;
        if (j0 + 128 < end) fetch(j0 + 128);
        if (j0 + 32 > n_every || held != ~0u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] = j0 + acc_row(r, h) < n_vis && (held >> acc_row(r, h) & 1) ? s[0][r] : -INFINITY;
        }
        acc.follow(s, scale);
        acc.weights(s[0], scale);
        accumulate_rows<T, TC, 32, true>(acc.o, sV, 0, s[0], c, h);
        if (any) add_nonfinite(acc, V, vs, pt, hk, j0, min(32, f.nk - j0), n_vis, h);
    }
    outside_rows(p, out, lse, hk, x, n_part);
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
    if (f.splits > 1) {
        const int64_t rec = ((int64_t)(f.slot + f.split * f.tiles + f.tile) * H_kv + hk) * 32 + r;
        float4* dst = reinterpret_cast<float4*>(part_o + rec * 64 + e);
        dst[0] = make_float4(o[0], o[1], o[2], o[3]);
        dst[1] = make_float4(o[4], o[5], o[6], o[7]);
        if (e == 0) part_ml[rec] = make_float2(m, sum);
    } else {
        store_joined(out.at(rh, f.q0 + rt) + e, o, sum);
        if (lse && e == 0) lse[(int64_t)rh * p.T + f.q0 + rt] = sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
    }
}

// Joins the splits of 32 rows of a sequence that has several: a wave to a row, 16 lanes of 4 elements for every fourth split.
template <typename T>
__global__ __launch_bounds__(256, 2)
void paged_join_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, PagedSeqs p, int H_kv, Heads<T> out, float* __restrict__ lse)
{
    const int hk = blockIdx.x % H_kv;
    const Part f = find_part<true>(p, blockIdx.x / H_kv);
    if (f.seq < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = (lane & 15) * 4, s0 = lane >> 4;
    for (int r = f.tile * 32 + wave; r < min(f.tile * 32 + 32, f.nq * p.G); r += 4) {
        const int t = r / p.G, head = hk * p.G + (r - t * p.G), tile = r / p.rows;
        const int64_t first = ((int64_t)(f.slot + tile) * H_kv + hk) * p.rows + r % p.rows, step = (int64_t)f.tiles * H_kv * p.rows;
        float m = kMaxInit, sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int base = s0; base < f.splits; base += 16) {
            float2 ml[4];
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t rec = first + min(base + 4 * k, f.splits - 1) * step;
                ml[k] = part_ml[rec];
                v[k] = *reinterpret_cast<const float4*>(part_o + rec * 64 + e);
                // (a split that saw no key may hold 0 * NaN)
                if (base + 4 * k >= f.splits || ml[k].y == 0.f) { ml[k] = make_float2(kMaxInit, 0.f); v[k] = make_float4(0.f, 0.f, 0.f, 0.f); }
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
        if (s0 != 0) continue;
        const float f1 = sum != 0.f ? 1.f / sum : 0.f;
        store4(out.at(head, f.q0 + t) + e, sum != 0.f ? make_float4(o.x * f1, o.y * f1, o.z * f1, o.w * f1) : make_float4(0.f, 0.f, 0.f, 0.f));
        if (lse && e == 0) lse[(int64_t)head * p.T + f.q0 + t] = sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
    }
}

PagedPlan make_paged_plan(const psa_cache_t& cache, const psa_paged_shape_t& s)
{
    PagedPlan p{};
    const int64_t rows = (int64_t)s.T * (s.H / s.H_kv);
    const int64_t wide = (rows / 128 + s.B) * s.H_kv;
    p.few = rows <= (int64_t)32 * s.B;
    p.fine = p.few || wide < (s.causal ? 224 : 152);
    p.rows = p.few ? 32 : 128;
    const int target = p.few ? 1024 : 768;
    p.per_head = (target + s.H_kv - 1) / s.H_kv;
    const int64_t tiles = rows / p.rows + s.B;         // at most
    // splits: sum of ceil(tiles units / chunk) is at most per_head more than the tiles
    p.n_part = tiles + p.per_head;
    p.join = (int64_t)cache.max_pages * cache.page_rows > kLeastUnits * kUnit;
    // of sequences with several splits the parts are at most twice their work over the chunk, and a row is joined in parts of 32
    const int64_t slots = p.join ? 2 * (int64_t)p.per_head : 0;
    p.n_join = slots * (p.rows / 32) / 2 + 1;
    size_t at = 0;
    if (s.B > kPagedMany) at += ((size_t)(3 * ((s.B + 63) / 64) + 1) * sizeof(int) + 255) & ~(size_t)255;
    p.off_ml = at;
    at += ((size_t)slots * s.H_kv * p.rows * sizeof(float2) + 255) & ~(size_t)255;
    p.off_part = at;
    at += (size_t)slots * s.H_kv * p.rows * 64 * sizeof(float);
    p.total = at > 256 ? at : 256;
    return p;
}

template <typename T, typename C>
static void paged_go(const PagedPlan& p, const psa_paged_shape_t& s, const psa_heads_t& Q, const psa_cache_t& cache, PagedSeqs seqs, const psa_heads_t& out,
                     float* lse, void* workspace, hipStream_t stream)
{
    const float scale = (float)(s.scale * 1.4426950408889634);
    unsigned char* room = static_cast<unsigned char*>(workspace);
    if (s.B > kPagedMany) {
        int* before = reinterpret_cast<int*>(room);
        paged_before_kernel<<<1, 1024, 0, stream>>>(seqs, before);
        seqs.before = before;
    }
    float2* part_ml = reinterpret_cast<float2*>(room + p.off_ml);
    float* part_o = reinterpret_cast<float*>(room + p.off_part);
    constexpr int KT = sizeof(C) == 4 ? 32 : 64;
    constexpr bool FINE = sizeof(T) == 2;
    const unsigned grid = (unsigned)(p.n_part * s.H_kv);
    (p.few ? paged_few_kernel<T, C> : p.fine ? paged_rows_kernel<T, C, KT, FINE> : paged_rows_kernel<T, C, KT, false>)<<<grid, 256, 0, stream>>>(
        heads_of<const T>(Q), page_heads_of<const C>(cache.K), page_heads_of<const C>(cache.V), page_scales_of(cache.K_scales), page_scales_of(cache.V_scales), seqs,
        heads_of<T>(out), lse, s.H_kv, s.causal, scale, (int)p.n_part, part_o, part_ml);
    if (p.join) paged_join_kernel<T><<<(unsigned)(p.n_join * s.H_kv), 256, 0, stream>>>(part_o, part_ml, seqs, s.H_kv, heads_of<T>(out), lse);
}
hipError_t launch_paged(const PagedPlan& p, const psa_paged_shape_t& s, const psa_heads_t& Q, const int* offsets, const psa_cache_t& cache, const psa_heads_t& out,
                        float* lse, void* workspace, hipStream_t stream)
{
    const PagedSeqs seqs{offsets, cache.lengths, cache.table, s.B, s.T, s.T / s.B, s.H / s.H_kv, cache.max_pages * cache.page_rows, page_shift(cache.page_rows), cache.n_pages,
                         cache.max_pages, p.rows, (int)p.per_head, nullptr};
    const bool mx = cache.format == PSA_CACHE_MX;
    if (s.dtype == PSA_F32) {
        if (mx) paged_go<float, mx8_t>(p, s, Q, cache, seqs, out, lse, workspace, stream);
        else paged_go<float, float>(p, s, Q, cache, seqs, out, lse, workspace, stream);
    } else {
        if (mx) paged_go<bf16_t, mx8_t>(p, s, Q, cache, seqs, out, lse, workspace, stream);
        else paged_go<bf16_t, bf16_t>(p, s, Q, cache, seqs, out, lse, workspace, stream);
    }
    return hipGetLastError();
}

}  // namespace psa
