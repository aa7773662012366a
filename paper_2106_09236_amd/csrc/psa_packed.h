// Dense attention over packed sequences: what the forward and backward kernels share.
//
// A key head's rows.  The query heads of a group read the same keys, so the rows of a tile are (query, head of the group)
// pairs: row r of a sequence is query r / G of head r % G of the group (G = H / H_kv), and a tile of keys that is in LDS
// serves the whole group.  With one head to a group rows are queries.
//
// Products are taken with the queries (or keys) that a wave owns on the column axis of the matrix instruction
// (D[i][j], i = 8 (r / 4) + 4 h + r % 4 for accumulator register r, j = c; lane (c, h) = (lane % 32, lane / 32)): a lane
// owns one column, so everything softmax keeps per row is a scalar of the lane, and the accumulator registers of the first
// product are the second operand of the next as they are (their row order taken as its order of summation).
#pragma once

#include "psa_tile.h"
#include "psa_vec.h"

namespace psa {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kMaxInit = -3.0e38f;       // below every finite score; finite, so that exp2(-inf - it) is 0 and not NaN

// One tensor's heads as a kernel takes them (strides in elements).
template <typename T>
struct Heads {
    T* data; int64_t head, row;
    __device__ __forceinline__ T* at(int h, int64_t l) const { return data + h * head + l * row; }
};
template <typename T>
inline Heads<T> heads_of(const psa_heads_t& t) { return Heads<T>{static_cast<T*>(t.data), t.head_stride, t.row_stride}; }

// The sequences of a call: offsets and what they are clamped to; of calls with many, the tiles before each 64 of them (see below).
struct Packing { const int* qo; const int* ko; int B, Tq, Tk, G; const int* q_before; const int* k_before; };

// Sequence s's rows and keys
struct SeqRange { int q0, q1, k0, k1; };
__device__ __forceinline__ SeqRange seq_range(const Packing& p, int s)
{
    SeqRange r{0, 0, 0, 0};
    if (s >= 0) {
        r.q0 = min(max(p.qo[s], 0), p.Tq); r.q1 = min(max(p.qo[s + 1], r.q0), p.Tq);
        r.k0 = min(max(p.ko[s], 0), p.Tk); r.k1 = min(max(p.ko[s + 1], r.k0), p.Tk);
    }
    return r;
}
__device__ __forceinline__ int seq_tiles(const SeqRange& r, int G, int per, bool keys) { return ((keys ? r.k1 - r.k0 : (r.q1 - r.q0) * G) + per - 1) / per; }

constexpr int kManySequences = 256;
inline size_t packed_before_bytes(int B) { return B > kManySequences ? (((size_t)(B + 63) / 64 * sizeof(int)) + 255) & ~(size_t)255 : 0; }

// The tile a work-group takes: rows (or keys) tile * PER .. of the sequence; tile < 0: there is none.
struct SeqTile { int q0, nq, k0, nk, tile; };

// Sum over the lanes of a wave, in scalar registers
__device__ __forceinline__ int wave_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, false);       // lanes 1, 2, 4 (mirrored), 8 apart
    x += __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x140, 0xF, 0xF, false);
    return __builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16) + __builtin_amdgcn_readlane(x, 32) + __builtin_amdgcn_readlane(x, 48);
}

// Tile x of the call.  Sequences are taken in groups of 16, last group first, and of a group's tiles those with the highest index in
// their sequence come first (of tiles of keys the lowest: the index counts from the end): under a causal mask they have the most
// work, and what starts last should be short.  Groups, not all sequences, so that work-groups that run at one time share their keys in
// L2.  (In the order of the sequences: 8 x 2048 causal, forward 92 | 75 us, dK and dV 164 | 147, dQ 104 | 88.)  Every wave finds its
// tile for itself: 64 sequences at a time, a prefix sum over the lanes for the group and a search for the index.  Beyond
// kManySequences a kernel of its own has summed up the tiles before each 64 of them (packed_before_kernel): work-groups that each
// walk all of them would take a time that grows with the square of their number.
template <int PER, bool KEYS>
__device__ __forceinline__ SeqTile find_tile(const Packing& p, int x)
{
    SeqTile f{0, 0, 0, 0, -1};
    if (!p.qo) {
        f.nq = p.Tq; f.nk = p.Tk;
        const int n = ((KEYS ? p.Tk : p.Tq * p.G) + PER - 1) / PER;
        f.tile = x >= n ? -1 : KEYS ? x : n - 1 - x;
        return f;
    }
    const int lane = threadIdx.x & 63;
    int base = 0, end = p.B;
    if (const int* before = KEYS ? p.k_before : p.q_before) {
        // the last 64 sequences with at most x tiles before them: 64 candidates at a time
        int lo = 0, n = (p.B + 63) / 64;
        while (n > 1) {
            const int step = (n + 63) / 64, i = lane * step;
            const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < n && before[min(lo + i, (p.B + 63) / 64 - 1)] <= x)) - 1;      // (before[0] is 0, so that k >= 0)
            lo += k * step;
            n = min(step, n - k * step);
        }
        x -= before[lo];
        base = lo * 64;
        end = min(end, base + 64);
    }
    for (; base < end; base += 64) {
        const SeqRange r = seq_range(p, p.B - 1 - base - lane);
        const int q0 = r.q0, q1 = r.q1, k0 = r.k0, k1 = r.k1;
        int n = seq_tiles(r, p.G, PER, KEYS);
        int sum = n;                                   // of this lane's group of 16, up to this lane
#pragma unroll
        for (int d = 1; d < 16; d *= 2) {
            const int y = __shfl_up(sum, d, 16);
            if ((lane & 15) >= d) sum += y;
        }
        int group = -1;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int all = __builtin_amdgcn_readlane(sum, 16 * g + 15);
            if (group < 0) {
                if (x < all) group = g;
                else x -= all;
            }
        }
        if (group < 0) continue;
        if ((lane >> 4) != group) n = 0;
        // tiles of index >= t: sum of max(n - t, 0).  The t with more than x of them, of t + 1 at most x
        int lo = 0, hi = 1;
        while (wave_sum(max(n - hi, 0)) > x) { lo = hi; hi *= 2; }
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (wave_sum(max(n - mid, 0)) > x) lo = mid; else hi = mid;
        }
        const int k = x - wave_sum(max(n - hi, 0));    // of the sequences with more than lo tiles, which
        const uint64_t with = __builtin_amdgcn_ballot_w64(n > lo);
        const int rank = __builtin_popcountll(with & (((uint64_t)1 << lane) - 1));
        const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(n > lo && rank == k));
        f.q0 = __builtin_amdgcn_readlane(q0, l); f.nq = __builtin_amdgcn_readlane(q1, l) - f.q0;
        f.k0 = __builtin_amdgcn_readlane(k0, l); f.nk = __builtin_amdgcn_readlane(k1, l) - f.k0;
        f.tile = KEYS ? __builtin_amdgcn_readlane(n, l) - 1 - lo : lo;
        return f;
    }
    return f;
}

// The sequences of a call; where there are many, with a launch that sums up their tiles (of per_q rows and, `keys`, per_k keys) in `room`,
// 2 packed_before_bytes().
Packing make_packing(const psa_packed_shape_t& s, const int* q_offsets, const int* k_offsets, int per_q, int per_k, void* room, bool keys, hipStream_t stream);

// Zeros in the rows of `t` that belong to no sequence (before the first offset, from the last one on), the share `x` of
// `n` work-groups; `each(head, row)` is called by one thread of the work-group for each head.
template <typename T, typename F>
__device__ __forceinline__ void zero_outside(const Heads<T>& t, const int* offsets, int B, int rows, int head0, int heads, int x, int n, F each)
{
    if (!offsets) return;
    const int first = min(max(offsets[0], 0), rows), last = min(max(offsets[B], first), rows);
    const int per = (rows + n - 1) / n;
    const int64_t r0 = (int64_t)x * per;
    const int r1 = (int)min((int64_t)rows, r0 + per);
    if (r0 >= first && r1 <= last) return;
    constexpr int CH = 64 * sizeof(T) / 16;
    const int per_row = heads * CH;
    for (int64_t i = threadIdx.x; i < (int64_t)(r1 - r0) * per_row; i += blockDim.x) {
        const int row = (int)(r0 + i / per_row), k = (int)(i % per_row), h = head0 + k / CH;
        if (row >= first && row < last) continue;
        reinterpret_cast<uint4*>(t.at(h, row))[k % CH] = make_uint4(0u, 0u, 0u, 0u);
        if (k % CH == 0) each(h, row);
    }
}

// Row r = t G + g of a key head, moved on without divisions.
struct RowAt {
    int t, g;
    __device__ __forceinline__ RowAt(int r, int G) : t(r / G), g(r - (r / G) * G) {}
    // by n rows, given as n / G and n % G
    __device__ __forceinline__ void add(int dt, int dg, int G) {
        t += dt; g += dg;
        if (g >= G) { g -= G; ++t; }
    }
};

// Rows base .. base + n - 1 (n <= 128, and may be <= 0) of a head as a buffer: reads of rows behind them give zeros.  The base moves with
// the tile, so that offsets into a long tensor stay small: 127 rows of at most 2^22 elements are within 31 bits.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rows(const T* base, int64_t row_stride, int n)
{
    const int bytes = n > 0 ? (int)((n - 1) * row_stride * (int64_t)sizeof(T)) + 64 * (int)sizeof(T) : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, bytes, 0x00020000);
}

// Any infinity or NaN among the elements of N times 16 bytes?  (bfloat16: the largest of them without their signs, two at a time; 32 streams of one
// new frame, the test in every tile instead of the last, 16.5 -> 16.9 us, with a test of each element 17.7.)
template <int N>
__device__ __forceinline__ bool nonfinite(const uint4 (&x)[N], float)
{
    bool b = false;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) b |= (w[i] & 0x7F800000u) == 0x7F800000u;
    }
    return b;
}
template <int N>
__device__ __forceinline__ bool nonfinite(const uint4 (&x)[N], bf16_t)
{
    ushortx2 most = {0, 0};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(ushortx2, w[i] & 0x7FFF7FFFu));
    }
    return most.x >= 0x7F80 || most.y >= 0x7F80;
}
__device__ __forceinline__ uint4 finite_only(const uint4& x, float)
{
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] = 0u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 finite_only(const uint4& x, bf16_t)
{
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
        if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0x0000FFFFu;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Key (or row) of a tile of 32 that accumulator register r of half h holds.
__device__ __forceinline__ constexpr int acc_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

__device__ __forceinline__ void clear(floatx16& a)
{
#pragma unroll
    for (int r = 0; r < 16; ++r) a[r] = 0.f;
}

// ---- float32 on the bfloat16 matrix units.  A float32 number is the sum of three bfloat16 numbers (each the rounding of what
// the ones before it leave: 8 bits and a sign each), and a product of two is the six products of parts whose sizes are 2^-16 and
// more of it; the others together are below 2^-23 of |a||b| (2^-25 as a rule), as a float32 product's own rounding.  Six bfloat16
// products take 3/8 of the time of one on the float32 matrix unit (1024 against 64 flops a cycle of a SIMD).
template <typename T> constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

// x0, x1 into parts (pairs of bfloat16, low half first); the remainders are exact.  Finite numbers beyond the largest of bfloat16 would round to
// an infinity, whose remainders are an infinity and NaN: the first part is at most that largest and the others have the rest, 2^-8 of
// it at the most (24 ragged clips of 435, forward and backward, 152 -> 157 us).  (A two-term dot product of the pair with (-1, 0) and (0, -1)
// forms them in one instruction instead of two, on the matrix unit's time: 16 x 512 float32 35.6 | 34.4 us.)
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t (&part)[3])
{
    constexpr float kMost = 0x1.FEp127f;
    part[0] = cvt_pk_bf16(__builtin_amdgcn_fmed3f(x0, -kMost, kMost), __builtin_amdgcn_fmed3f(x1, -kMost, kMost));
    x0 -= bf16_lo(part[0]); x1 -= bf16_hi(part[0]);
    part[1] = cvt_pk_bf16(x0, x1);
    x0 -= bf16_lo(part[1]); x1 -= bf16_hi(part[1]);
    part[2] = cvt_pk_bf16(x0, x1);
}

// Operand of 8 elements of the order of summation to a lane, in its parts.
template <typename T> struct Operand { uint4 v[kParts<T>]; };
__device__ __forceinline__ Operand<bf16_t> operand(const uint4& x, bf16_t) { return Operand<bf16_t>{{x}}; }
__device__ __forceinline__ Operand<float> operand(const float (&x)[8])
{
    uint32_t p[4][3];
#pragma unroll
    for (int i = 0; i < 4; ++i) split_pair(x[2 * i], x[2 * i + 1], p[i]);
    Operand<float> o;
#pragma unroll
    for (int k = 0; k < 3; ++k) o.v[k] = make_uint4(p[0][k], p[1][k], p[2][k], p[3][k]);
    return o;
}
__device__ __forceinline__ floatx16 mfma(const uint4& a, const uint4& b, floatx16 d)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), d, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mfma(const Operand<bf16_t>& a, const Operand<bf16_t>& b, floatx16 d) { return mfma(a.v[0], b.v[0], d); }
__device__ __forceinline__ floatx16 mfma(const Operand<float>& a, const Operand<float>& b, floatx16 d)
{
    d = mfma(a.v[2], b.v[0], d);           // small ones first
    d = mfma(a.v[0], b.v[2], d);
    d = mfma(a.v[1], b.v[1], d);
    d = mfma(a.v[1], b.v[0], d);
    d = mfma(a.v[0], b.v[1], d);
    return mfma(a.v[0], b.v[0], d);
}

// ---- a tile of ROWS rows in LDS: a plane of bfloat16 for each part, row-major, its 16-byte chunks permuted inside a row.  256 bytes of
// banks are two rows, so the permutation comes from the row's bits 1 .. 3: one chunk of 16 rows in a row covers all banks (rows as first
// operand), and so do 64 bytes of 4 rows (the transposing read), for which rows 2 apart have to differ in the chunk's high bit.
constexpr int kTileRowBytes = 128;
template <typename T, int ROWS> constexpr int kTileBytes = ROWS * kTileRowBytes * kParts<T>;
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * kTileRowBytes + ((chunk ^ ((row & 2) << 1) ^ ((row >> 2) & 3)) & 7) * 16; }

// 16 bytes of a tensor's row (chunk `ch` of it) into the tile
template <int ROWS>
__device__ __forceinline__ void put(unsigned char* s, int row, int ch, const uint4& x, bf16_t) { *reinterpret_cast<uint4*>(s + chunk_at(row, ch)) = x; }
template <int ROWS>
__device__ __forceinline__ void put(unsigned char* s, int row, int ch, const uint4& x, float)
{
    uint32_t p[2][3];
    split_pair(__uint_as_float(x.x), __uint_as_float(x.y), p[0]);
    split_pair(__uint_as_float(x.z), __uint_as_float(x.w), p[1]);
    unsigned char* dst = s + chunk_at(row, ch >> 1) + (ch & 1) * 8;
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(dst + k * ROWS * kTileRowBytes) = make_uint2(p[0][k], p[1][k]);
}

// ---- operands over a head's 64 elements: lane (c, h) has elements 32 h + 8 k .. + 7 of row (or column) c in step k.
template <typename T> struct HeadOperand {
    Operand<T> v[4];
    __device__ __forceinline__ void load(const T* row, int h);
};
template <> __device__ __forceinline__ void HeadOperand<bf16_t>::load(const bf16_t* row, int h)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k].v[0] = reinterpret_cast<const uint4*>(row)[4 * h + k];
}
template <> __device__ __forceinline__ void HeadOperand<float>::load(const float* row, int h)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float x[8];
        load_vec(reinterpret_cast<float (&)[4]>(x[0]), row + 32 * h + 8 * k, 4);
        load_vec(reinterpret_cast<float (&)[4]>(x[4]), row + 32 * h + 8 * k + 4, 4);
        v[k] = operand(x);
    }
}
// A row on its way from memory to such an operand; `ofs` is the row's offset in the buffer.
template <typename T> struct HeadRow {
    static constexpr int N = 64 * sizeof(T) / 32;
    uint4 x[N];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t b, int ofs, int h) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = buffer_load16<uint4>(b, ofs + (16 * h * N) + 16 * i);
    }
    __device__ __forceinline__ Operand<T> step(int k) const;
};
template <> __device__ __forceinline__ Operand<bf16_t> HeadRow<bf16_t>::step(int k) const { return operand(x[k], bf16_t{}); }
template <> __device__ __forceinline__ Operand<float> HeadRow<float>::step(int k) const
{
    const uint4 &a = x[2 * k], &b = x[2 * k + 1];
    const float f[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                        __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
    return operand(f);
}

// D[row][col] = sum over the head's 64 elements, rows from memory
template <typename T>
__device__ __forceinline__ floatx16 product(const HeadRow<T>& a, const HeadOperand<T>& b)
{
    floatx16 d;
    clear(d);
#pragma unroll
    for (int k = 0; k < 4; ++k) d = mfma(a.step(k), b.v[k], d);
    return d;
}
// ... the operand of one step from 32 rows from row0 of a tile of ROWS in LDS
template <typename T, int ROWS>
__device__ __forceinline__ Operand<T> tile_operand(const unsigned char* s, int row0, int k, int c, int h)
{
    Operand<T> a;
#pragma unroll
    for (int i = 0; i < kParts<T>; ++i) a.v[i] = *reinterpret_cast<const uint4*>(s + i * ROWS * kTileRowBytes + chunk_at(row0 + c, 4 * h + k));
    return a;
}
template <typename T, int ROWS>
__device__ __forceinline__ floatx16 product(const unsigned char* s, int row0, const HeadOperand<T>& b, int c, int h)
{
    floatx16 d;
    clear(d);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        d = mfma(tile_operand<T, ROWS>(s, row0, k, c, h), b.v[k], d);
    }
    return d;
}

// ... both from LDS, the columns' tensor as a tile of 32 rows
template <typename T, int ROWS>
__device__ __forceinline__ floatx16 product(const unsigned char* s, int row0, const unsigned char* columns, int c, int h)
{
    floatx16 d;
    clear(d);
#pragma unroll
    for (int k = 0; k < 4; ++k) d = mfma(tile_operand<T, ROWS>(s, row0, k, c, h), tile_operand<T, 32>(columns, 0, k, c, h), d);
    return d;
}

// The column operands of a product over 16 rows (step st of 32), from what a lane has in accumulator order: w[8 st] .. w[8 st + 7].  bfloat16:
// rounded, or (N = 2) in two parts of 16 bits and a sign each.  Rounded weights cost a result as much as its own rounding (1.4 times the
// error with both); kernels that wait for memory or for each other rather than for the matrix unit take two parts.
template <int N>
__device__ __forceinline__ void weight_operand(Operand<bf16_t> (&b)[N], const floatx16& w, int st)
{
    if constexpr (N == 1) {
        b[0].v[0] = make_uint4(cvt_pk_bf16(w[8 * st], w[8 * st + 1]), cvt_pk_bf16(w[8 * st + 2], w[8 * st + 3]),
                               cvt_pk_bf16(w[8 * st + 4], w[8 * st + 5]), cvt_pk_bf16(w[8 * st + 6], w[8 * st + 7]));
    } else {
        uint32_t part[4][3];               // (the third parts are not used, and not computed)
#pragma unroll
        for (int i = 0; i < 4; ++i) split_pair(w[8 * st + 2 * i], w[8 * st + 2 * i + 1], part[i]);
#pragma unroll
        for (int n = 0; n < 2; ++n) b[n].v[0] = make_uint4(part[0][1 - n], part[1][1 - n], part[2][1 - n], part[3][1 - n]);      // the small one first
    }
}
template <int N>
__device__ __forceinline__ void weight_operand(Operand<float> (&b)[N], const floatx16& w, int st)
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = w[8 * st + i];
    b[0] = operand(x);
}
template <typename T, bool FINE> constexpr int kWeightParts = FINE && sizeof(T) == 2 ? 2 : 1;

// D^T[e][col] += sum over 32 rows of the tile from row0 of X[row][e] w[row], w in accumulator order (row acc_row(r, h) in w[r]); D in two
// accumulators of 32 elements e.  The tile's operand for 16 rows (step st) and 32 elements (dt) comes through the transposing LDS
// read: of each group of 16 lanes, lane s points at row s / 4 of four rows, columns 4 (s % 4) .., and lane i receives column i of
// the four rows.
template <typename T, int ROWS>
__device__ __forceinline__ Operand<T> tile_transposed(const unsigned char* s, int row0, int st, int dt, int c, int h)
{
    const int s16 = c & 15, row = row0 + 4 * h + (s16 >> 2), byte = ((c & 16) + 4 * (s16 & 3) + 32 * dt) * 2;
    Operand<T> a;
#pragma unroll
    for (int i = 0; i < kParts<T>; ++i) {
        uint2 part[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const unsigned char* p = s + i * ROWS * kTileRowBytes + chunk_at(row + 16 * st + 8 * e, byte >> 4) + (byte & 15);
            part[e] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((shortx4 __attribute__((address_space(3)))*)(p)));
        }
        a.v[i] = make_uint4(part[0].x, part[0].y, part[1].x, part[1].y);
    }
    return a;
}
template <typename T> struct Transposed { Operand<T> v[2][2]; };
template <typename T, int ROWS>
__device__ __forceinline__ Transposed<T> transposed(const unsigned char* s, int row0, int c, int h)
{
    Transposed<T> a;
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int dt = 0; dt < 2; ++dt) a.v[st][dt] = tile_transposed<T, ROWS>(s, row0, st, dt, c, h);
    return a;
}
template <typename T, bool FINE>
__device__ __forceinline__ void accumulate(floatx16 (&d)[2], const Transposed<T>& a, const floatx16& w)
{
    constexpr int N = kWeightParts<T, FINE>;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        Operand<T> b[N];
        weight_operand(b, w, st);
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int n = 0; n < N; ++n) d[dt] = mfma(a.v[st][dt], b[n], d[dt]);
    }
}
template <typename T, int ROWS, bool FINE>
__device__ __forceinline__ void accumulate(floatx16 (&d)[2], const unsigned char* s, int row0, const floatx16& w, int c, int h)
{
    constexpr int N = kWeightParts<T, FINE>;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        Operand<T> b[N];
        weight_operand(b, w, st);
#pragma unroll
        for (int dt = 0; dt < 2; ++dt) {
            const Operand<T> a = tile_transposed<T, ROWS>(s, row0, st, dt, c, h);
#pragma unroll
            for (int n = 0; n < N; ++n) d[dt] = mfma(a, b[n], d[dt]);
        }
    }
}
// Order of a step's instructions: N reads of LDS together, then M matrix instructions.  Left to itself the compiler asks for an operand
// right before the instruction that takes it, and each waits for its own.
template <int N, int M>
__device__ __forceinline__ void reads_first()
{
    __builtin_amdgcn_sched_group_barrier(0x100, N, 0);
    if (M > 0) __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
}

// The same for a second set of weights at once (rounded)
template <typename T, int ROWS, bool FINE>
__device__ __forceinline__ void accumulate_two(floatx16 (&d)[2], const floatx16& w, floatx16 (&d2)[2], const floatx16& w2, const unsigned char* s, int row0, int c, int h)
{
    constexpr int N = kWeightParts<T, FINE>;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        Operand<T> b[N], b2[1];
        weight_operand(b, w, st);
        weight_operand(b2, w2, st);
#pragma unroll
        for (int dt = 0; dt < 2; ++dt) {
            const Operand<T> a = tile_transposed<T, ROWS>(s, row0, st, dt, c, h);
#pragma unroll
            for (int n = 0; n < N; ++n) d[dt] = mfma(a, b[n], d[dt]);
            d2[dt] = mfma(a, b2[0], d2[dt]);
        }
    }
}

// Column c's 64 elements of D^T (elements 32 dt + acc_row(r, h) in d[dt][r]) times f, to its row of a tensor.
__device__ __forceinline__ void store_row(bf16_t* row, const floatx16 (&d)[2], float f, int h)
{
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *reinterpret_cast<uint2*>(row + 32 * dt + 8 * k + 4 * h) =
                make_uint2(cvt_pk_bf16(d[dt][4 * k] * f, d[dt][4 * k + 1] * f), cvt_pk_bf16(d[dt][4 * k + 2] * f, d[dt][4 * k + 3] * f));
}
__device__ __forceinline__ void store_row(float* row, const floatx16 (&d)[2], float f, int h)
{
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *reinterpret_cast<float4*>(row + 32 * dt + 8 * k + 4 * h) =
                make_float4(d[dt][4 * k] * f, d[dt][4 * k + 1] * f, d[dt][4 * k + 2] * f, d[dt][4 * k + 3] * f);
}

// The sums of a work-group's 4 waves over D^T (32 columns of 64 elements each), 8 threads of 8 elements to a column: column tid / 8, elements
// 8 (tid % 8) .. + 7, in the order of the waves.  `join` holds 4 * 32 * kJoinRow floats; barriers before and after belong to the caller.
constexpr int kJoinRow = 68;               // floats of a column in the join: 64, and 16 bytes against bank conflicts
__device__ __forceinline__ void join_columns(float (&v)[8], const float* join, int tid)
{
    const float* src = join + (tid >> 3) * kJoinRow + (tid & 7) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = ((src[i] + src[32 * kJoinRow + i]) + src[2 * 32 * kJoinRow + i]) + src[3 * 32 * kJoinRow + i];
}
template <typename T>
__device__ __forceinline__ void store8(T* dst, const float (&v)[8], float f)
{
#pragma unroll
    for (int k = 0; k < 8 / kVec<T>; ++k) {
        float part[kVec<T>];
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) part[i] = v[k * kVec<T> + i] * f;
        store_vec(dst + k * kVec<T>, part, kVec<T>);
    }
}
__device__ __forceinline__ void store4(float* dst, float4 v) { *reinterpret_cast<float4*>(dst) = v; }
__device__ __forceinline__ void store4(bf16_t* dst, float4 v) { *reinterpret_cast<uint2*>(dst) = make_uint2(cvt_pk_bf16(v.x, v.y), cvt_pk_bf16(v.z, v.w)); }
// 8 elements of a row's sums over its weights' sum, 0 where that is 0 (no key)
template <typename T>
__device__ __forceinline__ void store_joined(T* dst, const float (&o)[8], float sum)
{
    const float f = sum != 0.f ? 1.f / sum : 0.f;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = sum != 0.f ? o[i] * f : 0.f;
#pragma unroll
    for (int k = 0; k < 8 / kVec<T>; ++k) {
        float part[kVec<T>];
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) part[i] = v[k * kVec<T> + i];
        store_vec(dst + k * kVec<T>, part, kVec<T>);
    }
}

}  // namespace psa
