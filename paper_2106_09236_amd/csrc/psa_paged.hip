// Dense attention over a cache in pages: softmax(scale Q K^T) V of the newest rows of each sequence, whose keys and values
// lie in pages named by a table.  The arithmetic is that of the packed kernels (psa_packed.h): rows are (query, head of the
// group) pairs, 32 to a wave, on the columns of the matrix instruction; keys in one pass with online softmax.
//
// Work.  The rows of a sequence are tiles, and its keys are cut into equal splits, the same for all its tiles.  How many is found
// on the device from all lengths (find_part), so that a call has about as many work-groups as the card holds, of about one size, whatever
// the lengths are: a call that was captured serves as its sequences grow.  Sequences cut in several splits leave partial sums in
// the workspace, joined by a second kernel.
#include <algorithm>
#include <type_traits>

#include "psa_paged.h"

namespace psa {

__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

// Sequence s as the call has it: rows q0 .. q0 + nq - 1, nk keys
struct PagedSeq { int q0, nq, nk; };
// The query of row r of a key head (rows are G to a query)
__device__ __forceinline__ int query_of(int r, int G) { return G == 1 ? r : r / G; }
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
__device__ __forceinline__ int tiles_of(int nq, int G, int row_shift) { return (nq * G + (1 << row_shift) - 1) >> row_shift; }
// (at most 4 sqrt(units): a join takes 16 of them at a time, in about the time of a round of keys, so that more would take longer to join than they save: one sequence
// of 120000 keys, 8 heads to 2, one new row, 469 splits 36 us, 122 21)
// (p.per_head 0: nothing is divided)
__device__ __forceinline__ int splits_of(const PagedSeqs& p, int nk, int chunk)
{
    if (p.per_head == 0) return 1;
    const int units = units_of(nk);
    return max(1, min((units + chunk - 1) / chunk, (int)(4.f * __builtin_sqrtf((float)units))));
}

// Units of keys to a split: the work of all tiles (units times tiles) in about p.per_head shares, p.least at the least.  Every
// work-group of a call and of its join finds the same.  Summed in float32: a thread adds up to 1024 numbers (2^20 sequences in paged_before_kernel), and 22 more
// additions join them, so that the sum is off by less than 2^-13 of it.  p.per_head is at most 1024.  A divided sequence has u >= chunk + 1 units, hence at most 2 (u - 1) / chunk
// splits: the parts of all of them are fewer than 2 p.per_head (1 + 2^-13) <= 2 p.per_head + 1/4, a whole number, so at most twice p.per_head; in the same way all parts are
// at most p.per_head more than the tiles.  More than 4096 shares would need a more exact sum.
__device__ __forceinline__ float wave_sum(float x)
{
    auto add = [&](auto ctrl, auto rows) { x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl.value, rows.value, 0xF, false)); };
    using std::integral_constant;
    add(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});
    add(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
    add(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
    add(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
    add(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});
    add(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ int chunk_for(const PagedSeqs& p, float work) { return (int)fminf(fmaxf(ceilf(work / (float)max(p.per_head, 1)), (float)p.least), (float)(1 << 23)); }
__device__ __forceinline__ float work_of(const PagedSeqs& p, const PagedSeq& r)
{
    return (float)units_of(r.nk) * (float)tiles_of(r.nq, p.G, p.row_shift);
}

// What a work-group takes: tile `tile` of sequence `seq`, split `split` of `splits`, `per` units of keys each; `slot`: where the partial sums of its sequence
// begin (tile t, split i at slot + i * tiles + t); seq < 0: nothing.  JOIN: the pieces are the 32-row parts of the sequences with
// more than one split, and `tile` counts those.
struct Part { int seq, q0, nq, nk, tiles, tile, split, splits, per, slot; };
template <bool JOIN>
__device__ __forceinline__ Part find_part(const PagedSeqs& p, int x)
{
    Part f{};
    f.seq = -1;
    const int lane = threadIdx.x & 63;
    int s0 = 0, end = p.B, slot = 0, chunk;
    PagedSeq r = paged_seq(p, lane);
    if (p.before) {
        // many sequences: the chunk and the parts, slots and joined pieces before each 64 of them have been summed up; the last 64
        // with at most x before them
        chunk = p.before[0];
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
    } else if (p.per_head == 0) {
        chunk = 1 << 23;
    } else {
        float work = work_of(p, r);
        for (int s = lane + 64; s < p.B; s += 64) work += work_of(p, paged_seq(p, s));
        chunk = chunk_for(p, wave_sum(work));
    }
    for (; s0 < end; s0 += 64) {
        if (s0 > 0) r = paged_seq(p, s0 + lane);
        const int tiles = tiles_of(r.nq, p.G, p.row_shift), splits = splits_of(p, r.nk, chunk);
        // (a call has fewer than 2^24 parts, but where offsets decrease each sequence may claim all of its rows; there are never more
        // slots than twice p.per_head, since a sequence's parts are at most twice its work over the chunk)
        const int parts = tiles * splits, slots = splits > 1 ? parts : 0;
        const int n = min(JOIN ? (splits > 1 ? tiles_of(r.nq, p.G, 5) : 0) : parts, 1 << 24);
        const int sum = wave_scan(n), all = last_lane(sum);
        const int slot_sum = wave_scan(slots);
        if (x < all) {
            int l, y;
            // Undivided sequences with several tiles: of 16 sequences those with the highest index first, which have the most work under a causal mask;
            // what starts last should be short (8 x 2048 causal, 8 heads, 84 -> 60 us, 64 of 100 to 900 67 -> 58).
            const bool by_index = !JOIN && __builtin_amdgcn_ballot_w64(splits > 1) == 0 && __builtin_amdgcn_ballot_w64(tiles > 1) != 0;
            if (by_index) {
                int group = 0;
#pragma unroll
                for (int k = 0; k < 3; ++k) group += x >= __builtin_amdgcn_readlane(sum, 16 * k + 15);
                y = x - (group > 0 ? __builtin_amdgcn_readlane(sum, 16 * group - 1) : 0);
                const int mine = (lane >> 4) == group ? n : 0;
                // tiles of index >= t: sum of max(mine - t, 0).  The t with more than y of them, of t + 1 at most y
                int lo = 0, hi = 1;
                while (wave_sum(max(mine - hi, 0)) > y) { lo = hi; hi *= 2; }
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (wave_sum(max(mine - mid, 0)) > y) lo = mid; else hi = mid;
                }
                const int k = y - wave_sum(max(mine - hi, 0));         // of the sequences with more than lo tiles, which
                const uint64_t with = __builtin_amdgcn_ballot_w64(mine > lo);
                const int rank = __builtin_popcountll(with & (((uint64_t)1 << lane) - 1));
                l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine > lo && rank == k));
                y = lo;
            } else {
                l = __builtin_popcountll(__builtin_amdgcn_ballot_w64(sum <= x));
                y = x - __builtin_amdgcn_readlane(sum - n, l);
            }
            f.seq = s0 + l;
            f.q0 = __builtin_amdgcn_readlane(r.q0, l); f.nq = __builtin_amdgcn_readlane(r.nq, l); f.nk = __builtin_amdgcn_readlane(r.nk, l);
            f.tiles = __builtin_amdgcn_readlane(tiles, l); f.splits = __builtin_amdgcn_readlane(splits, l);
            f.per = f.splits > 1 ? (units_of(f.nk) + f.splits - 1) / f.splits : units_of(f.nk);
            f.slot = slot + __builtin_amdgcn_readlane(slot_sum - slots, l);
            if (JOIN || by_index) {
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
    __shared__ float s_work[16];
    __shared__ int s[2][3][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = (p.B + 63) / 64;
    float work = 0.f;
    for (int i = threadIdx.x; i < p.B; i += 1024) work += work_of(p, paged_seq(p, i));
    work = wave_sum(work);
    if (lane == 0) s_work[wave] = work;
    __syncthreads();
    work = 0.f;
    for (int w = 0; w < 16; ++w) work += s_work[w];
    const int chunk = chunk_for(p, work);
    if (threadIdx.x == 0) before[0] = chunk;
    int sum[3] = {0, 0, 0};
    for (int g0 = 0, buf = 0; g0 < groups; g0 += 16, buf ^= 1) {
        const int g = g0 + wave;
        const PagedSeq r = paged_seq(p, g < groups ? g * 64 + lane : p.B);
        const int splits = splits_of(p, r.nk, chunk);
        const int64_t parts = (int64_t)tiles_of(r.nq, p.G, p.row_shift) * splits;
        const int64_t n[3] = {parts, splits > 1 ? parts : 0, splits > 1 ? tiles_of(r.nq, p.G, 5) : 0};
        for (int k = 0; k < 3; ++k) {
            const float rough = wave_sum((float)n[k]);
            const int all = rough < (float)kMostParts ? last_lane(wave_scan((int)n[k])) : kMostParts;
            if (lane == 0) s[buf][k][wave] = min(all, kMostParts);
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
// 64 entries of a sequence's table, one to a lane: a tile's pages are read from a register and no load waits for another.  Entries that name no
// page are -1.  Pages of PG = 16 rows and more: rows that are asked for together lie on one page, whose addresses, of K and of V, the lanes hold as well
// (computed for every tile by every wave: 16384 keys, last 4096 rows, 182 -> 177 us).  PG = 0: smaller pages and irregular rows, each lane finds its row's.  A
// new window is waited for where it is asked for, so that the loads of rows in flight are waited for by nobody else.
template <typename C, int PG>
struct PageWindow {
    const int* row; int entries, n_pages, shift;
    const C *k, *v; int64_t k_page, v_page;            // of the key head
    int first, entry;
    bool whole;                                        // no entry of the window's is -1
    uint32_t lo[2], hi[2];                             // addresses; bit 31 of hi: no page
    __device__ __forceinline__ PageWindow(const PagedSeqs& p, int seq, int nk, const PageHeads<const C>& K, const PageHeads<const C>& V, int hk)
        : row(p.table + (int64_t)seq * p.max_pages), entries((nk + (1 << p.shift) - 1) >> p.shift), n_pages(p.n_pages), shift(p.shift),
          k(K.data + hk * K.head), v(V.data + hk * V.head), k_page(K.page), v_page(V.page), first(0), entry(-1), whole(false), lo{0, 0}, hi{0, 0} {}
    __device__ __forceinline__ void open(int from) {
        const int lane = threadIdx.x & 63, i = from + lane;
        int e = i < entries ? row[i] : -1;
        if ((unsigned)e >= (unsigned)n_pages) e = -1;
        first = from;
        entry = e;
        whole = __builtin_amdgcn_ballot_w64(e < 0 && i < entries) == 0;
        if constexpr (PG > 0) {
            const uint64_t a[2] = {reinterpret_cast<uint64_t>(k + max(e, 0) * k_page), reinterpret_cast<uint64_t>(v + max(e, 0) * v_page)};
#pragma unroll
            for (int x = 0; x < 2; ++x) { lo[x] = (uint32_t)a[x]; hi[x] = (uint32_t)(a[x] >> 32) | (e < 0 ? 0x80000000u : 0u); }
        }
    }
    // rows j0 .. j0 + n - 1 are about to be asked for: at most 64 pages
    __device__ __forceinline__ void reach(int j0, int n) { if (((j0 + n - 1) >> shift) - first >= 64) open(j0 >> shift); }
    __device__ __forceinline__ int lane(int j) const { return __shfl(entry, (j >> shift) - first, 64); }
    __device__ __forceinline__ bool held(int j) const { return __shfl(PG > 0 ? (int)hi[0] : entry, (j >> shift) - first, 64) >= 0; }
    __device__ __forceinline__ int slot(int j) const { return j & ((1 << shift) - 1); }
};
// Which of the 32 rows from j on exist: on a page, before row nk
template <typename W>
__device__ __forceinline__ uint32_t rows_held(const W& w, int j, int nk, int c)
{
    if (w.whole && j + 32 <= nk) return ~0u;
    const bool held = w.held(j + c);
    return (uint32_t)__builtin_amdgcn_ballot_w64(held && j + c < nk);
}

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

// 16 bytes of a row, on their way into a tile as N chunks of the tile's type
template <typename C> struct RowChunk {
    static constexpr int N = 1;
    uint4 x;
    __device__ __forceinline__ void unpack(uint4* to) const { to[0] = x; }
};
template <> struct RowChunk<mx8_t> {
    static constexpr int N = 2;
    uint4 x;
    uint32_t power;
    __device__ __forceinline__ void unpack(uint4* to) const {
        to[0] = mx_codes(x.x, x.y, mx_power(power));
        to[1] = mx_codes(x.z, x.w, mx_power(power));
    }
};

// Rows j .. of a sequence in K (0) or V (1) that are on one page: a buffer that ends with the sequence, so that rows behind it give zeros, as rows
// on no page do.  Scalars; what the host sees to (rows_regular): a row's stride is its width or more, and a page's span less than 2^31 bytes.
template <typename C>
struct PageRows {
    __amdgpu_buffer_rsrc_t rows, powers;
    int stride, power_stride;              // bytes
    template <int PG>
    __device__ __forceinline__ void open(const PageWindow<C, PG>& w, int which, const PageHeads<const C>& t, const PageScales& s, int hk, int j, int nk)
    {
        const int i = (j >> w.shift) - w.first, slot = w.slot(j);
        const uint32_t lo = __builtin_amdgcn_readlane(w.lo[which], i), hi = __builtin_amdgcn_readlane(w.hi[which], i);
        const int n = (int)hi < 0 ? 0 : min(PG, nk - j);
        stride = (int)(t.row * (int64_t)sizeof(C));
        const uint64_t base = ((uint64_t)(hi & 0x7FFFFFFFu) << 32 | lo) + (uint32_t)slot * (uint32_t)stride;
        rows = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, max(n * stride + (64 * (int)sizeof(C) - stride), 0), 0x00020000);
        if constexpr (sizeof(C) == 1) {
            power_stride = (int)s.row;
            powers = __builtin_amdgcn_make_buffer_rsrc(s.at(hk, max(__builtin_amdgcn_readlane(w.entry, i), 0), slot), 0, max(n * power_stride + (2 - power_stride), 0), 0x00020000);
        }
    }
    __device__ __forceinline__ uint4 bytes(int row, int at) const { return buffer_load16<uint4>(rows, row * stride + at); }
    __device__ __forceinline__ uint32_t power(int row, int half) const { return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(powers, row * power_stride + half, 0, 0); }
    __device__ __forceinline__ void load(RowChunk<C>& to, int row, int ch) const {
        to.x = bytes(row, ch * 16);
        if constexpr (sizeof(C) == 1) to.power = power(row, ch >> 1);
    }
};
// 16 bytes of row j, chunk ch of it, where each lane finds its row's page
template <typename C, typename W>
__device__ __forceinline__ void load_chunk(RowChunk<C>& to, const PageHeads<const C>& t, const PageScales& s, int hk, const W& w, int j, int ch, int nk)
{
    const int page = w.lane(j), slot = w.slot(j);
    const bool valid = page >= 0 && j < nk;
    to.x = load_or_zero<uint4>(row_at(t, hk, page, slot) + ch * (16 / (int)sizeof(C)), valid);
    if constexpr (sizeof(C) == 1) to.power = load_or_zero<uint8_t>(s.at(hk, page, slot) + (ch >> 1), valid);
}

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
template <typename C, typename W>
__device__ __forceinline__ void add_nonfinite(Rows32& acc, const PageHeads<const C>& V, const PageScales& vs, const W& w, int hk, int j0, int n, int n_vis, int h)
{
    for (int j = j0; j < j0 + n; ++j) {
        const int page = w.row[j >> w.shift], slot = w.slot(j);
        if ((unsigned)page >= (unsigned)w.n_pages) continue;
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

// -infinity in the scores of a tile of 32 keys that are not held, or not among the first n
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? ~0u : (1u << max(n, 0)) - 1; }
__device__ __forceinline__ void hide(floatx16& s, uint32_t held, int n, int h)
{
    const uint32_t seen = (held & first_bits(n)) >> (4 * h);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = seen >> acc_row(r, 0) & 1 ? s[r] : -INFINITY;
}
// accumulate() of the packed kernels with the values' tile of another type
template <typename T, typename TC, bool FINE>
__device__ __forceinline__ void accumulate_rows(floatx16 (&d)[2], const Transposed<TC>& a, const floatx16& w)
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

// ---- many rows: RW x KW waves, KW of them to the same 32 rows, which take alternate KT keys and join their sums in LDS; tiles of
// KT x KW keys and values go through LDS, the next tile's rows are on their way meanwhile.
//
// Infinities and NaN of V: a weight of 0 does not keep them out of a sum (and, in two parts, one times a part of the other sign is NaN).
// They always leave an infinity or NaN in the sums, so a work-group looks at those at its end, and only then takes its keys once
// more, with such values left out of the product and added afterwards to the rows that see them.
template <typename T, typename C, int PG, int KT, int RW, int KW, bool FINE>
__global__ __launch_bounds__(64 * RW * KW, sizeof(T) == 4 || FINE ? 2 : 3)
void paged_rows_kernel(Heads<const T> Q, PageHeads<const C> K, PageHeads<const C> V, PageScales ks, PageScales vs, PagedSeqs p, Heads<T> out,
                       float* __restrict__ lse, int H_kv, int causal, float scale, int n_part, float* __restrict__ part_o, float2* __restrict__ part_ml)
{
    typedef typename TileOf<C>::type TC;
    constexpr int ROWS = 32 * RW, NT = 64 * RW * KW, NWAVE = RW * KW, TILE = KT * KW;
    constexpr int CH = 64 * sizeof(C) / 16;            // 16-byte chunks of a row in the cache
    constexpr int NL = TILE * CH / NT;                 // chunks of a tile, to a thread
    constexpr int WR = TILE / NWAVE;                   // rows of a tile that a wave brings, 16 at most: on one page (8 rows here, 8 there, with pages of 16: clips of 40 to 500 20.3 -> 19.2 us)
    constexpr int NS = KT / 32;
    constexpr int NU = RowChunk<C>::N;
    constexpr int kBytes = kTileBytes<TC, TILE>;
    static_assert(WR <= 16 && (PG == 0 || PG == 16), "a wave's rows have to be on one page");
    static_assert(KW == 1 || 4 * kBytes >= ROWS * (kJoinRow + 2) * 4, "the join does not fit the tiles");
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * kBytes];
    __shared__ int s_bad[2][NWAVE];
    unsigned char *const sK = lds, *const sV = lds + 2 * kBytes;
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
    const Part f = find_part<false>(p, x);
    if (f.seq < 0) { outside_rows(p, out, lse, hk, x, n_part); return; }

    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;                 // causal: query t sees the first t + shift keys
    auto visible = [&](int r) { const int t = query_of(r, p.G); return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int rw = wave % RW, kg = wave / RW;          // which rows, which keys
    const int row0 = f.tile * ROWS + rw * 32;
    const int row = row0 + c, rc = min(row, n_rows - 1);
    const int t = query_of(rc, p.G), head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int begin = f.split * f.per * kUnit, cut = min(begin + f.per * kUnit, f.nk);
    const int n_all = min(cut, __builtin_amdgcn_readfirstlane(visible(min(f.tile * ROWS + ROWS - 1, n_rows - 1))));       // keys any row of the work-group sees
    const int n_wave = min(cut, __builtin_amdgcn_readfirstlane(row0 < n_rows ? visible(min(row0 + 31, n_rows - 1)) : 0));
    const int n_wave_every = __builtin_amdgcn_readfirstlane(visible(min(row0, n_rows - 1)));                              // ... and those that all of a wave's see

    HeadOperand<T> q;
    q.load(Q.at(head, f.q0 + t), h);
    PageWindow<C, PG> w(p, f.seq, f.nk, K, V, hk);
    RowChunk<C> kr[NL], vr[NL];
    uint32_t held_next[NS];
    auto row_of = [&](int i) { return wave * WR + i * (64 / CH) + lane / CH; };
    auto fetch = [&](int j0) {
        w.reach(j0, TILE);
        PageRows<C> pk, pv;
        if constexpr (PG > 0) {
            pk.open(w, 0, K, ks, hk, j0 + wave * WR, f.nk);
            pv.open(w, 1, V, vs, hk, j0 + wave * WR, f.nk);
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int r = row_of(i), ch = lane % CH;
            if constexpr (PG > 0) {
                pk.load(kr[i], r - wave * WR, ch);
                pv.load(vr[i], r - wave * WR, ch);
            } else {
                load_chunk(kr[i], K, ks, hk, w, j0 + r, ch, f.nk);
                load_chunk(vr[i], V, vs, hk, w, j0 + r, ch, f.nk);
            }
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) held_next[n] = rows_held(w, j0 + kg * KT + 32 * n, f.nk, c);
    };
    Rows32 acc;
    auto pass = [&](auto again) {
        constexpr bool careful = decltype(again)::value;
        acc.init();
        if (begin < n_all) { w.open(begin >> p.shift); fetch(begin); }
        auto tile = [&](int j0, auto which) {            // (the buffer known, its addresses are constants)
            constexpr int buf = decltype(which)::value;
            uint4 v[NL * NU];
#pragma unroll
            for (int i = 0; i < NL; ++i) vr[i].unpack(v + i * NU);
            if constexpr (careful) {
                const bool any = __builtin_amdgcn_ballot_w64(nonfinite(v, TC{})) != 0;
                if (lane == 0) s_bad[buf][wave] = any;
#pragma unroll
                for (int i = 0; i < NL * NU; ++i) v[i] = finite_only(v[i], TC{});
            }
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                uint4 k[NU];
                kr[i].unpack(k);
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    put<TILE>(sK + buf * kBytes, row_of(i), lane % CH * NU + u, k[u], TC{});
                    put<TILE>(sV + buf * kBytes, row_of(i), lane % CH * NU + u, v[i * NU + u], TC{});
                }
            }
            uint32_t held[NS], all = ~0u;
#pragma unroll
            for (int n = 0; n < NS; ++n) { held[n] = held_next[n]; all &= held[n]; }
            if (j0 + TILE < n_all) fetch(j0 + TILE);
            lds_barrier();
            const int j = j0 + kg * KT;
            if (j >= n_wave) return;
            floatx16 s[NS];
#pragma unroll
            for (int n = 0; n < NS; ++n) s[n] = product_rows<T, TC, TILE>(sK + buf * kBytes, kg * KT + 32 * n, q, c, h);
            reads_first<4 * NS * kParts<TC>, 4 * NS * (sizeof(T) == 2 ? 1 : sizeof(C) == 4 ? 6 : 3)>();
            if (j + KT > n_wave_every || all != ~0u) {
#pragma unroll
                for (int n = 0; n < NS; ++n) hide(s[n], held[n], n_vis - (j + 32 * n), h);
            }
            acc.follow(s, scale);
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const Transposed<TC> vt = transposed<TC, TILE>(sV + buf * kBytes, kg * KT + 32 * n, c, h);
                reads_first<8 * kParts<TC>, 0>();
                acc.weights(s[n], scale);
                accumulate_rows<T, TC, FINE>(acc.o, vt, s[n]);
            }
            if constexpr (careful) {
                int any = 0;
#pragma unroll
                for (int k = 0; k < NWAVE; ++k) any |= s_bad[buf][k];
                if (any) add_nonfinite(acc, V, vs, w, hk, j, min(KT, f.nk - j), n_vis, h);
            }
        };
        for (int j0 = begin; j0 < n_all; j0 += 2 * TILE) {
            tile(j0, std::integral_constant<int, 0>{});
            if (j0 + TILE < n_all) tile(j0 + TILE, std::integral_constant<int, 1>{});
        }
        bool bad = false;
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) bad |= !isfinite(acc.o[dt][r]);
        return __syncthreads_or(bad) != 0;
    };
    if (pass(std::false_type{})) pass(std::true_type{});
    outside_rows(p, out, lse, hk, x, n_part);          // (last: its loads would delay the others)
    float l = acc.l + swap_half(acc.l);
    if constexpr (KW == 2) {
        float* join = reinterpret_cast<float*>(lds) + (rw * 32 + c) * kJoinRow;
        float* join_ml = reinterpret_cast<float*>(lds) + ROWS * kJoinRow + (rw * 32 + c) * 2;
        if (kg == 1) {                                 // (a barrier lies behind the last reads of the tiles)
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
    if (f.splits > 1) {
        const int64_t rec = ((int64_t)(f.slot + f.split * f.tiles + f.tile) * H_kv + hk) * ROWS + rw * 32 + c;
        store_row(part_o + rec * 64, acc.o, 1.f, h);
        if (h == 0) part_ml[rec] = make_float2(acc.m, l);
        return;
    }
    if (l == 0.f) { clear(acc.o[0]); clear(acc.o[1]); }
    store_row(out.at(head, f.q0 + t), acc.o, l != 0.f ? 1.f / l : 0.f, h);
    if (lse && h == 0) lse[(int64_t)head * p.T + f.q0 + t] = l != 0.f ? acc.m * kLn2 + logf(l) : -INFINITY;
}

// ---- few rows, single tokens as a rule: 16 to a work-group, whose 4 waves divide the keys (of its split) among themselves, 32 at a time, and
// join their sums at the end.  Keys come straight from memory as the first product's operand, values through LDS of the wave's own; there
// is no barrier before the join.
//
// Bound by memory, and with few keys by the chain of loads before the first of them.  16 x 16 x 32 matrix instructions: for one row a tile of 32
// columns computes 31/32 of its scores, exponentials and products in vain and takes twice the registers, so that half the waves have rows on their
// way: 64 streams of 1 to 4096 keys, 8 heads to 2, bfloat16, 22.6 | 17.0 us, 16 of 4096 to 32768, 8 heads, 8-bit, 118 | 78; with up to 128 rows
// to a sequence it was never more than a tenth better.  A second tile on its way in registers (3 waves to a SIMD instead of 4): 20.3 -> 21.8 and 73.9 -> 78.3
// (whole calls).  8 waves to a work-group: 60 streams of 8000 keys 178 -> 162, but 8 of 1000 to 2000 11.8 -> 12.7, 64 of 300 to 2000 in float32 37.4 -> 42.3.
//   lane (c, g) = (lane % 16, lane / 16);  D[i][j]: i = 4 g + r, j = c;  A[i][k]: i = c, B[k][j]: j = c, 8 elements k to a lane, in an order of our own:
//   keys    element order of a step: those that make a wave read 64 bytes and more of a row at a time (head_element)
//   values  key 16 t + 4 g + r is element 4 t + r of a lane: the order that scores have in their accumulators
typedef float floatx4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ floatx4 mfma16(const uint4& a, const uint4& b, floatx4 d) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), d, 0, 0, 0); }
__device__ __forceinline__ floatx4 mfma16(const Operand<bf16_t>& a, const Operand<bf16_t>& b, floatx4 d) { return mfma16(a.v[0], b.v[0], d); }
__device__ __forceinline__ floatx4 mfma16(const Operand<bf16_t>& a, const Operand<float>& b, floatx4 d)
{
    d = mfma16(a.v[0], b.v[2], d);
    d = mfma16(a.v[0], b.v[1], d);
    return mfma16(a.v[0], b.v[0], d);
}
__device__ __forceinline__ floatx4 mfma16(const Operand<float>& a, const Operand<float>& b, floatx4 d)
{
    d = mfma16(a.v[2], b.v[0], d);         // small ones first
    d = mfma16(a.v[0], b.v[2], d);
    d = mfma16(a.v[1], b.v[1], d);
    d = mfma16(a.v[1], b.v[0], d);
    d = mfma16(a.v[0], b.v[1], d);
    return mfma16(a.v[0], b.v[0], d);
}
// First of the 4 elements that are floats 4 u .. of the 8 that lane g has in step k of a product over a head's 64 elements, keys of type C
template <typename C> __device__ __forceinline__ constexpr int head_element(int k, int u, int g) { return sizeof(C) == 4 ? 16 * (2 * k + u) + 4 * g : sizeof(C) == 2 ? 32 * k + 8 * g + 4 * u : 16 * g + 8 * k + 4 * u; }
template <typename T, typename C>
__device__ __forceinline__ void load_query(Operand<T> (&q)[2], const T* row, int g)
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if constexpr (sizeof(T) == 4) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) load_vec(reinterpret_cast<float (&)[4]>(x[4 * u]), row + head_element<C>(k, u, g), 4);
            q[k] = operand(x);
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(row + head_element<C>(k, 0, g)), b = *reinterpret_cast<const uint2*>(row + head_element<C>(k, 1, g));
            q[k].v[0] = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
}
// A lane's part of row c of 16 keys on their way: N times 16 bytes, of chunk at(i) of the row's
template <typename C> struct KeyPart {
    static constexpr int N = sizeof(C);                // (16 elements)
    uint4 x[N];
    uint32_t power;
    static __device__ __forceinline__ int at(int i, int g) { return sizeof(C) == 1 ? 16 * g : 64 * i + 16 * g; }     // bytes
    __device__ __forceinline__ auto step(int k) const {
        if constexpr (sizeof(C) == 4) {
            const uint4 &a = x[2 * k], &b = x[2 * k + 1];
            const float f[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                                __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
            return operand(f);
        } else if constexpr (sizeof(C) == 2) {
            return operand(x[k], bf16_t{});
        } else {
            return operand(k == 0 ? mx_codes(x[0].x, x[0].y, mx_power(power)) : mx_codes(x[0].z, x[0].w, mx_power(power)), bf16_t{});
        }
    }
};
// A tile of 32 values in LDS, its 16-byte chunks permuted inside a row: here a transposing read takes 32 bytes of rows 4 g .. 4 g + 3 in each group of
// 16 lanes, so that rows 2, 4 and 8 apart have to differ in the chunk's bits 2, 1 and 0 (256 bytes of banks are two rows)
__device__ __forceinline__ int chunk16_at(int row, int chunk) { return row * kTileRowBytes + ((chunk ^ ((row & 2) << 1) ^ ((row & 4) >> 1) ^ ((row & 8) >> 3)) & 7) * 16; }
__device__ __forceinline__ void put16(unsigned char* s, int row, int ch, const uint4& x, bf16_t) { *reinterpret_cast<uint4*>(s + chunk16_at(row, ch)) = x; }
__device__ __forceinline__ void put16(unsigned char* s, int row, int ch, const uint4& x, float)
{
    uint32_t p[2][3];
    split_pair(__uint_as_float(x.x), __uint_as_float(x.y), p[0]);
    split_pair(__uint_as_float(x.z), __uint_as_float(x.w), p[1]);
    unsigned char* dst = s + chunk16_at(row, ch >> 1) + (ch & 1) * 8;
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(dst + k * 32 * kTileRowBytes) = make_uint2(p[0][k], p[1][k]);
}
template <typename TC>
__device__ __forceinline__ Operand<TC> transposed16(const unsigned char* s, int m, int c, int g)
{
    const int row = 4 * g + (c >> 2), byte = 32 * m + 8 * (c & 3);
    Operand<TC> a;
#pragma unroll
    for (int i = 0; i < kParts<TC>; ++i) {
        uint2 part[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const unsigned char* p = s + i * 32 * kTileRowBytes + chunk16_at(row + 16 * t, byte >> 4) + (byte & 15);
            part[t] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((shortx4 __attribute__((address_space(3)))*)(p)));
        }
        a.v[i] = make_uint4(part[0].x, part[0].y, part[1].x, part[1].y);
    }
    return a;
}
// Weights as the second operand: bfloat16 in two parts, the small one first
__device__ __forceinline__ void weight_operand16(Operand<float> (&b)[1], const float (&w)[8]) { b[0] = operand(w); }
__device__ __forceinline__ void weight_operand16(Operand<bf16_t> (&b)[2], const float (&w)[8])
{
    uint32_t part[4][3];
#pragma unroll
    for (int i = 0; i < 4; ++i) split_pair(w[2 * i], w[2 * i + 1], part[i]);
#pragma unroll
    for (int n = 0; n < 2; ++n) b[n].v[0] = make_uint4(part[0][1 - n], part[1][1 - n], part[2][1 - n], part[3][1 - n]);
}

template <typename T, typename C, int PG>
__global__ __launch_bounds__(256, sizeof(T) == 4 || sizeof(C) == 4 ? 2 : 4)
void paged_single_kernel(Heads<const T> Q, PageHeads<const C> K, PageHeads<const C> V, PageScales ks, PageScales vs, PagedSeqs p, Heads<T> out,
                         float* __restrict__ lse, int H_kv, int causal, float scale, int n_part, float* __restrict__ part_o, float2* __restrict__ part_ml)
{
    typedef typename TileOf<C>::type TC;
    constexpr int CH = 64 * sizeof(C) / 16;
    constexpr int NL = 32 * CH / 64;                   // chunks of a tile of 32 values, to a lane
    constexpr int NU = RowChunk<C>::N;
    constexpr int NW = sizeof(T) == 4 ? 1 : 2;         // parts of a weight
    constexpr int kBytes = kTileBytes<TC, 32>;
    constexpr int kJoinBytes = 4 * 16 * kJoinRow * 4;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * kBytes > kJoinBytes ? 4 * kBytes : kJoinBytes];
    __shared__ float s_m[4][16], s_l[4][16];
    const int hk = blockIdx.x % H_kv, x = blockIdx.x / H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const Part f = find_part<false>(p, x);
    if (f.seq < 0) { outside_rows(p, out, lse, hk, x, n_part); return; }
    const int n_rows = f.nq * p.G;
    const int shift = f.nk - f.nq + 1;
    auto visible = [&](int r) { const int t = query_of(r, p.G); return causal ? min(max(t + shift, 0), f.nk) : f.nk; };
    const int row0 = f.tile * 16, rc = min(row0 + c, n_rows - 1);
    const int t = query_of(rc, p.G), head = hk * p.G + (rc - t * p.G);
    const int n_vis = visible(rc);
    const int begin = f.split * f.per * kUnit, cut = min(begin + f.per * kUnit, f.nk);
    const int end = min(cut, __builtin_amdgcn_readfirstlane(visible(min(row0 + 15, n_rows - 1))));
    const int n_every = __builtin_amdgcn_readfirstlane(visible(row0));

    Operand<T> q[2];
    load_query<T, C>(q, Q.at(head, f.q0 + t), g);
    PageWindow<C, PG> w(p, f.seq, f.nk, K, V, hk);
    unsigned char* const sV = lds + wave * kBytes;
    struct Tile {
        KeyPart<C> k[2];
        RowChunk<C> v[NL];
        uint32_t held;
    } next;
    auto fetch = [&](Tile& n, int j0) {
        w.reach(j0, 32);
        if constexpr (PG > 0) {
#pragma unroll
            for (int from = 0; from < 32; from += PG) {
                PageRows<C> pk, pv;
                pk.open(w, 0, K, ks, hk, j0 + from, f.nk);
                pv.open(w, 1, V, vs, hk, j0 + from, f.nk);
#pragma unroll
                for (int t16 = from / 16; t16 < (from + PG) / 16; ++t16) {
#pragma unroll
                    for (int i = 0; i < KeyPart<C>::N; ++i) n.k[t16].x[i] = pk.bytes(16 * t16 - from + c, KeyPart<C>::at(i, g));
                    if constexpr (sizeof(C) == 1) n.k[t16].power = pk.power(16 * t16 - from + c, g >> 1);
                }
#pragma unroll
                for (int i = from * CH / 64; i < (from + PG) * CH / 64; ++i)
                    pv.load(n.v[i], (i * 64 + lane) / CH - from, lane % CH);
            }
        } else {
#pragma unroll
            for (int t16 = 0; t16 < 2; ++t16) {
                const int j = j0 + 16 * t16 + c, page = w.lane(j), slot = w.slot(j);
                const bool valid = page >= 0 && j < f.nk;
                const unsigned char* key = reinterpret_cast<const unsigned char*>(row_at(K, hk, page, slot));
#pragma unroll
                for (int i = 0; i < KeyPart<C>::N; ++i) n.k[t16].x[i] = load_or_zero<uint4>(key + KeyPart<C>::at(i, g), valid);
                if constexpr (sizeof(C) == 1) n.k[t16].power = load_or_zero<uint8_t>(ks.at(hk, page, slot) + (g >> 1), valid);
            }
#pragma unroll
            for (int i = 0; i < NL; ++i) load_chunk(n.v[i], V, vs, hk, w, j0 + (i * 64 + lane) / CH, lane % CH, f.nk);
        }
        n.held = rows_held(w, j0, f.nk, lane & 31);
    };
    float m, l;
    floatx4 o[4];
    // Infinities and NaN of V: a weight of 0 does not keep them out of a sum, and one times a part of the other sign is NaN.  They always
    // leave an infinity or NaN in the sums, so a wave looks at those at its end and only then takes its keys once more, with such
    // values left out of the product and added afterwards to the rows that see them.
    for (int careful = 0; careful < 2; ++careful) {
        m = kMaxInit; l = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        auto take = [&](Tile& n, int j0) {
            uint4 v[NL * NU];
#pragma unroll
            for (int i = 0; i < NL; ++i) n.v[i].unpack(v + i * NU);
            bool any = false;
            if (careful) {
                any = __builtin_amdgcn_ballot_w64(nonfinite(v, TC{})) != 0;
#pragma unroll
                for (int i = 0; i < NL * NU; ++i) v[i] = finite_only(v[i], TC{});
            }
            wave_lds_sync();
#pragma unroll
            for (int i = 0; i < NL; ++i)
#pragma unroll
                for (int u = 0; u < NU; ++u) put16(sV, (i * 64 + lane) / CH, lane % CH * NU + u, v[i * NU + u], TC{});
            floatx4 s[2];
#pragma unroll
            for (int t16 = 0; t16 < 2; ++t16) {
                s[t16] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 2; ++k) s[t16] = mfma16(n.k[t16].step(k), q[k], s[t16]);
            }
            wave_lds_sync();
            const uint32_t held = n.held;
            if (j0 + 128 < end) fetch(n, j0 + 128);
            if (j0 + 32 > n_every || held != ~0u) {
                const uint32_t seen = (held & first_bits(n_vis - j0)) >> (4 * g);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] = seen >> (16 * (i >> 2) + (i & 3)) & 1 ? s[i >> 2][i & 3] : -INFINITY;
            }
            // the running maximum, as Rows32 follows it
            float top = s[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
            top = max_xor16(max_xor32(top)) * scale;
            const float m_new = top > m + kLagLog2 ? top : m;
            if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {
                const float alpha = fast_exp2(m - m_new);
                l *= alpha;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] *= alpha;
            }
            m = m_new;
            float weight[8], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) { weight[i] = fast_exp2(fmaf(s[i >> 2][i & 3], scale, -m)); sum += weight[i]; }
            l += sum;
            Operand<T> b[NW];
            weight_operand16(b, weight);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Operand<TC> a = transposed16<TC>(sV, i, c, g);
#pragma unroll
                for (int k = 0; k < NW; ++k) o[i] = mfma16(a, b[k], o[i]);
            }
            if (any) {
                for (int j = j0; j < min(j0 + 32, f.nk); ++j) {
                    const int page = w.row[j >> w.shift], slot = w.slot(j);
                    if ((unsigned)page >= (unsigned)p.n_pages) continue;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float value = value_at(row_at(V, hk, page, slot), vs.at(hk, page, slot), 16 * i + 4 * g + r);
                            if (j < n_vis && !isfinite(value)) o[i][r] += value;
                        }
                }
            }
        };
        int j0 = begin + wave * 32;
        if (j0 < end) {
            w.open(j0 >> p.shift);
            fetch(next, j0);
        }
        for (; j0 < end; j0 += 128) take(next, j0);
        float size = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) size = fmaxf(size, isfinite(o[i >> 2][i & 3]) ? 0.f : 1.f);
        if (__builtin_amdgcn_ballot_w64(size != 0.f) == 0) break;
    }
    outside_rows(p, out, lse, hk, x, n_part);
    // join: wave w's sums of row r at join[w][r]; a wave that saw no key has m = kMaxInit and sums of 0
    __syncthreads();
    float* join = reinterpret_cast<float*>(lds);
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) { s_m[wave][c] = m; s_l[wave][c] = l; }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(join + (wave * 16 + c) * kJoinRow + 16 * i + 4 * g) = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
    __syncthreads();
    // 16 threads of 4 elements to a row
    const int r = tid >> 4, e = (tid & 15) * 4;
    if (row0 + r >= n_rows) return;
    float top = s_m[0][r];
#pragma unroll
    for (int k = 1; k < 4; ++k) top = fmaxf(top, s_m[k][r]);
    float sum = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (s_m[k][r] == kMaxInit && s_l[k][r] == 0.f) continue;       // (saw no key: its accumulators may hold 0 * NaN)
        const float f1 = fast_exp2(s_m[k][r] - top);
        const float4 v = *reinterpret_cast<const float4*>(join + (k * 16 + r) * kJoinRow + e);
        sum = fmaf(s_l[k][r], f1, sum);
        a.x = fmaf(v.x, f1, a.x); a.y = fmaf(v.y, f1, a.y); a.z = fmaf(v.z, f1, a.z); a.w = fmaf(v.w, f1, a.w);
    }
    const int rt = (row0 + r) / p.G, rh = hk * p.G + (row0 + r - rt * p.G);
    if (f.splits > 1) {
        const int64_t rec = ((int64_t)(f.slot + f.split * f.tiles + f.tile) * H_kv + hk) * 16 + r;
        *reinterpret_cast<float4*>(part_o + rec * 64 + e) = a;
        if (e == 0) part_ml[rec] = make_float2(top, sum);
    } else {
        const float f1 = sum != 0.f ? 1.f / sum : 0.f;
        store4(out.at(rh, f.q0 + rt) + e, sum != 0.f ? make_float4(a.x * f1, a.y * f1, a.z * f1, a.w * f1) : make_float4(0.f, 0.f, 0.f, 0.f));
        if (lse && e == 0) lse[(int64_t)rh * p.T + f.q0 + rt] = sum == 0.f ? -INFINITY : top * kLn2 + logf(sum);
    }
}

// Joins the splits of 32 rows of a sequence that has several: 16 lanes of 4 elements to a row, with four splits on their way; where there are few
// rows, four such groups to a row, for every fourth split each.
template <typename T>
__global__ __launch_bounds__(256, 2)
void paged_join_kernel(const float* __restrict__ part_o, const float2* __restrict__ part_ml, PagedSeqs p, int H_kv, Heads<T> out, float* __restrict__ lse)
{
    const int hk = blockIdx.x % H_kv;
    const Part f = find_part<true>(p, blockIdx.x / H_kv);
    if (f.seq < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = (lane & 15) * 4, group = lane >> 4;
    const int r0 = f.tile * 32, r1 = min(r0 + 32, f.nq * p.G);
    const bool shared = r1 - r0 <= 8;                  // four groups to a row
    const int every = shared ? 4 : 1, s0 = shared ? group : 0;
    for (int r = r0 + (shared ? wave : wave * 4 + group); r < r1; r += shared ? 4 : 16) {
        const int t = query_of(r, p.G), head = hk * p.G + (r - t * p.G), tile = r >> p.row_shift, rows = 1 << p.row_shift;
        const int64_t first = ((int64_t)(f.slot + tile) * H_kv + hk) * rows + (r & (rows - 1)), step = (int64_t)f.tiles * H_kv * rows;
        float m = kMaxInit, sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int base = s0; base < f.splits; base += 4 * every) {
            float2 ml[4];
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t rec = first + min(base + every * k, f.splits - 1) * step;
                ml[k] = part_ml[rec];
                v[k] = *reinterpret_cast<const float4*>(part_o + rec * 64 + e);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)                // (a split that saw no key may hold 0 * NaN)
                if (base + every * k >= f.splits || ml[k].y == 0.f) { ml[k] = make_float2(kMaxInit, 0.f); v[k] = make_float4(0.f, 0.f, 0.f, 0.f); }
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
        if (shared) {
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
            if (group != 0) continue;
        }
        const float f1 = sum != 0.f ? 1.f / sum : 0.f;
        store4(out.at(head, f.q0 + t) + e, sum != 0.f ? make_float4(o.x * f1, o.y * f1, o.z * f1, o.w * f1) : make_float4(0.f, 0.f, 0.f, 0.f));
        if (lse && e == 0) lse[(int64_t)head * p.T + f.q0 + t] = sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
    }
}

// 16, 64 or 128 rows to a work-group?  16 for at most 32 rows to a sequence, and for calls with few work-groups.  16 | 64 or 128 rows, bfloat16: 8 sequences
// of 500 to 1500 keys and 64 rows, 4 heads, 14.8 | 16.0 us, 64 of them with 200 to 900 keys 21.6 | 19.3; 32 of 300 to 1500 keys and 32 rows, 8
// heads, 23.1 | 20.3 (float32 46.6 | 54.3); 4 of 1000 to 2000 keys and 128 rows, 8 heads, 18.5 | 17.3 (float32 40 | 28); 32 of 300 to 1000 and 100 rows 33 | 28
// (float32 75 | 48).  64 | 128 rows: 16 of 600 to 2048 keys and 64 rows 21.0 | 23.3; 64 of 200 to 900, 4 heads, 19.3 | 21.6.
//
// Shares of the work: as many as compute units hold work-groups while tiles are less than a quarter (128 rows: a third) of those, down to a quarter as
// many where they are half (two thirds) of them: their own number evens out what is left, and sums to be joined are 528 bytes of traffic a row and split.  Then, with sequences that
// can only be so long, nothing is divided, and no join launched (64 sequences of 1300 keys, 8 heads, one new row: 40 | 34 us; 64 new rows 49 | 36).  The host knows how
// long they can be, by the tables' width, not how long they are: with tables for 32768 rows the same sequences are searched for shares and joined, though nothing is divided.  Tables as
// wide as the sequences | for 32768 rows: 31.5 | 33.9 us, 64 new rows 33.5 | 36.0, 96 of 128 rows, all new, 14.7 | 18.5; where shares are searched for anyway the same (16 x 64 of 600 to 2048 20.1 | 20.1).
// A share is at least 2 units of keys; 4 where bfloat16 calls have 64 tiles of 128 rows and more, since what a row leaves for the join is as many bytes as 2 units of its
// keys and values: 32 clips of 40 to 500, 4 heads, 22.7 | 19.5 us, 16 of 2000 keys and 128 rows, 8 heads, 30.1 | 27.7, but 4 of 1000 to 2000 and 128 rows (32 tiles) 17.6 | 21.7,
// and in float32 28.5 | 41.
//
// One | two waves to the same 32 rows, float32: two where tiles are about as many as the 256 compute units, which then have two waves to a
// SIMD without a division: 24 prompts of 120 to 750, 2 heads of 2, 51.9 | 40.6 us; 16 of 512, 4 heads, 40.7 | 34.1; 32 of 500 to 1500 keys and
// 120 rows, 8 heads, 85.8 | 74.8; of 6000 to 8000 keys 430 | 400.  With fewer tiles or more four waves fill the compute units more
// evenly: 192 tiles, 8000 keys, 235 | 343; 384, 700 keys, 60.8 | 65.9; 1024 of 8 x 2048 216 | 226.
PagedPlan make_paged_plan(const psa_cache_t& cache, const psa_paged_shape_t& s)
{
    PagedPlan p{};
    const int64_t rows = (int64_t)s.T * (s.H / s.H_kv);
    const int64_t wide = (rows / 128 + s.B) * s.H_kv;
    p.few = rows <= (int64_t)32 * s.B || (rows / 16 + s.B) * s.H_kv <= 192;
    p.fine = p.few || wide < (s.causal ? 224 : 152);
    p.rows = p.few ? 16 : rows <= (int64_t)64 * s.B && s.dtype == PSA_BF16 ? 64 : 128;
    const int64_t keys = (int64_t)cache.max_pages * cache.page_rows;
    const int64_t each = (rows + s.B - 1) / s.B, tiles = s.B * ((each + p.rows - 1) / p.rows);
    p.pairs = !p.few && s.dtype == PSA_F32 && cache.format == PSA_CACHE_PLAIN && tiles * s.H_kv >= 224 && tiles * s.H_kv <= 352;
    const int64_t shares = ((p.few ? 1024 : p.pairs ? 256 : 768) + s.H_kv - 1) / s.H_kv;
    const double full = std::min(std::max((p.few ? 4.0 : 3.0) * tiles / shares - 1.0, 0.0), 1.0);
    p.least = p.rows == 128 && s.dtype == PSA_BF16 && tiles * s.H_kv >= 64 ? 4 : 2;
    p.join = keys > p.least * kUnit && !(full == 1.0 && keys <= (p.few ? 4096 : 2048));
    // (each tile's last share is half a one on average)
    p.per_head = p.join ? std::max((int64_t)1, (int64_t)((shares - 0.5 * std::min(tiles, shares)) * (1.0 - 0.75 * full))) : 0;
    // sum of ceil(tiles units / chunk) is at most per_head more than the tiles
    p.n_part = rows / p.rows + s.B + p.per_head;
    // of sequences with several splits the parts are at most twice their work over the chunk, and a row is joined in parts of 32
    const int64_t slots = p.join ? 2 * (int64_t)p.per_head : 0;
    p.n_join = std::min(slots * std::max(p.rows / 32, 1) / 2 + 1, rows / 32 + s.B);
    size_t at = 0;
    if (s.B > kPagedMany) at += ((size_t)(3 * ((s.B + 63) / 64) + 1) * sizeof(int) + 255) & ~(size_t)255;
    p.off_ml = at;
    at += ((size_t)slots * s.H_kv * p.rows * sizeof(float2) + 255) & ~(size_t)255;
    p.off_part = at;
    at += (size_t)slots * s.H_kv * p.rows * 64 * sizeof(float);
    p.total = at > 256 ? at : 256;
    return p;
}

// May a page's rows be a buffer with 32-bit offsets?
static bool rows_regular(const psa_cache_t& c, int size)
{
    auto good = [&](const psa_heads_t& t, int64_t width, int64_t bytes) {
        return t.row_stride >= width && t.row_stride * bytes <= 1 << 20 && t.row_stride * bytes * c.page_rows < INT32_MAX;
    };
    return good(c.K, 64, size) && good(c.V, 64, size) && (c.format != PSA_CACHE_MX || (good(c.K_scales, 2, 1) && good(c.V_scales, 2, 1)));
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
    auto pick = [&](auto pg) {
        constexpr int SINGLE = decltype(pg)::value, PG = SINGLE < 16 ? SINGLE : 16;
        if (p.few) return paged_single_kernel<T, C, SINGLE>;
        if constexpr (sizeof(T) == 2)
            if (p.rows == 64) return p.fine ? paged_rows_kernel<T, C, PG, 32, 2, 2, true> : paged_rows_kernel<T, C, PG, 32, 2, 2, false>;
        if constexpr (sizeof(C) == 4)
            if (p.pairs) return paged_rows_kernel<T, C, PG, KT, 4, 2, FINE>;
        return p.fine ? paged_rows_kernel<T, C, PG, KT, 4, 1, FINE> : paged_rows_kernel<T, C, PG, KT, 4, 1, false>;
    };
    using std::integral_constant;
    const int pg = rows_regular(cache, sizeof(C)) ? std::min(cache.page_rows, 32) : 0;
    (pg == 32 ? pick(integral_constant<int, 32>{}) : pg == 16 ? pick(integral_constant<int, 16>{}) : pick(integral_constant<int, 0>{}))<<<grid, p.pairs ? 512 : 256, 0, stream>>>(
        heads_of<const T>(Q), page_heads_of<const C>(cache.K), page_heads_of<const C>(cache.V), page_scales_of(cache.K_scales), page_scales_of(cache.V_scales), seqs,
        heads_of<T>(out), lse, s.H_kv, s.causal, scale, (int)p.n_part, part_o, part_ml);
    if (p.join) paged_join_kernel<T><<<(unsigned)(p.n_join * s.H_kv), 256, 0, stream>>>(part_o, part_ml, seqs, s.H_kv, heads_of<T>(out), lse);
}
hipError_t launch_paged(const PagedPlan& p, const psa_paged_shape_t& s, const psa_heads_t& Q, const int* offsets, const psa_cache_t& cache, const psa_heads_t& out,
                        float* lse, void* workspace, hipStream_t stream)
{
    const PagedSeqs seqs{offsets, cache.lengths, cache.table, s.B, s.T, s.T / s.B, s.H / s.H_kv, cache.max_pages * cache.page_rows, page_shift(cache.page_rows), cache.n_pages,
                         cache.max_pages, page_shift(p.rows), (int)p.per_head, p.least, nullptr};
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
