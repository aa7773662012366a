// A cache in pages: new rows into it, who holds its pages, compaction, and copies of pages.
//
// All of it is bound by memory, or, for the few rows and the few thousand integers of a step, by latency: the length of a chain
// of dependent loads and the number of launches.
#include <limits.h>

#include "psa_paged.h"

namespace psa {

// ---- new rows
// A wave takes as many rows as 64 chunks of 16 bytes make, of kAppendHeads heads, K and V: whole kilobytes of a head at a time, read and, on one page, written.
// What decides where a row goes is a chain of four loads (which sequence, its rows, its page); the first rows are asked for before it.
// (A row of all heads to a wave: 10213 rows of 8 heads, bfloat16, 22 us; 8-bit from float32, 4 heads, 9.8.)
__device__ __forceinline__ int sequence_of(const int* offsets, int B, int row)
{
    // the last sequence whose offset is at most `row` (offsets do not decrease); -1: none
    const int lane = threadIdx.x & 63;
    int lo = 0, n = B + 1;                             // candidates lo .. lo + n - 1
    while (true) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const uint64_t at_most = __builtin_amdgcn_ballot_w64(lane * step < n && offsets[min(i, B)] <= row);
        if (at_most == 0) return -1;
        const int k = 63 - __builtin_clzll(at_most);
        lo += k * step;
        if (step == 1) return lo;
        n = min(step, n - k * step);
    }
}

// 16 bytes of a row, chunk `ch` of head `hk`, to where the row lies in the cache.  8-bit: every lane of the 32 elements that share a
// power of two has to be here.
template <typename T>
__device__ __forceinline__ void put_chunk(const uint4& x, const PageHeads<T>& to, const PageScales&, int hk, int64_t page, int slot, int ch)
{
    *reinterpret_cast<uint4*>(to.data + hk * to.head + page * to.page + slot * to.row + ch * (16 / (int)sizeof(T))) = make_uint4(x.x, x.y, x.z, x.w);
}
// largest of the lanes of one block of 32 elements: 4 lanes of 8 elements, or 8 of 4
__device__ __forceinline__ float block_max(float a, bf16_t) { a = fmaxf(a, dpp_mov<0xB1>(a)); return fmaxf(a, dpp_mov<0x4E>(a)); }
__device__ __forceinline__ float block_max(float a, float) { a = block_max(a, bf16_t{}); return fmaxf(a, dpp_mov<0x141>(a)); }
template <typename T>
__device__ __forceinline__ void put_chunk(const uint4& x, const PageHeads<mx8_t>& to, const PageScales& scales, int hk, int64_t page, int slot, int ch)
{
    constexpr int N = kVec<T>;                         // elements of a chunk
    constexpr int LANES = 32 / N;                      // lanes of a block
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float v[N], most = 0.f;
    unpack(w, v, T{});
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, isfinite(v[i]) ? fabsf(v[i]) : 0.f);
    const uint32_t bits = __float_as_uint(block_max(most, T{}));
    // floor(log2) - 8, one more where the largest would pass 1.75 * 2^8 = 448, the largest code
    const int e = min(max((int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0), -117), 119);
    const float inverse = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t code[N / 4];
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = __builtin_amdgcn_fmed3f(v[i + k] * inverse, -448.f, 448.f);
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (!isfinite(v[i + k])) c |= 0x7F << (8 * k);
        code[i / 4] = (uint32_t)c;
    }
    mx8_t* dst = to.data + hk * to.head + page * to.page + slot * to.row + ch * N;
    if constexpr (N == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(code[0], code[1]);
    else *reinterpret_cast<uint32_t*>(dst) = code[0];
    if (ch % LANES == 0) *(scales.at(hk, (int)page, slot) + ch / LANES) = (uint8_t)(e + 127);
}

template <typename T, typename C>
__global__ __launch_bounds__(256)
void cache_append_kernel(Heads<const T> K, Heads<const T> V, PagedSeqs p, PageHeads<C> Kc, PageHeads<C> Vc, PageScales ks, PageScales vs, int H_kv)
{
    constexpr int CH = 64 * sizeof(T) / 16, ROWS = 64 / CH;
    const int lane = threadIdx.x & 63, ch = lane % CH, h0 = blockIdx.y * kAppendHeads;
    const int row0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * ROWS;
    if (row0 >= p.T) return;
    const int row1 = min(row0 + ROWS, p.T) - 1, row = min(row0 + lane / CH, row1);
    uint4 k[kAppendHeads], v[kAppendHeads];
#pragma unroll
    for (int i = 0; i < kAppendHeads; ++i) {
        const int h = min(h0 + i, H_kv - 1);
        k[i] = *reinterpret_cast<const uint4*>(K.at(h, row) + ch * kVec<T>);
        v[i] = *reinterpret_cast<const uint4*>(V.at(h, row) + ch * kVec<T>);
    }
    int s, first, n;
    bool valid = row0 + lane / CH <= row1;
    if (p.offsets) {
        // the wave's first and last row by all lanes, each row between the two by its own
        s = sequence_of(p.offsets, p.B, row0);
        const int last = sequence_of(p.offsets, p.B, row1);
        if (last < 0) return;
        for (int lo = s, hi = last; ; ) {              // the last offset of s .. last at most `row`; s may be -1
            if (__builtin_amdgcn_ballot_w64(lo < hi) == 0) { s = lo; break; }
            const int mid = (lo + hi + 1) >> 1;
            const bool right = p.offsets[max(mid, 0)] <= row;
            if (lo < hi) { if (right) lo = mid; else hi = mid - 1; }
        }
        valid = valid && s >= 0 && s < p.B;            // (else in no sequence)
        s = min(max(s, 0), p.B - 1);
        first = max(p.offsets[s], 0);
        n = min(p.offsets[s + 1], p.T) - first;
    } else {
        s = row / p.uniform;
        first = s * p.uniform;
        n = p.uniform;
    }
    const int j = min(max(p.lengths[s], 0), p.capacity) - n + (row - first);
    if (row - first < 0 || row - first >= n || j < 0) valid = false;           // (the first two only where offsets decrease)
    const int page = valid ? p.table[(int64_t)s * p.max_pages + (j >> p.shift)] : -1, slot = j & ((1 << p.shift) - 1);
    if ((unsigned)page >= (unsigned)p.n_pages) return;
#pragma unroll
    for (int i = 0; i < kAppendHeads; ++i) {
        if (h0 + i < H_kv) {
            put_chunk<T>(k[i], Kc, ks, h0 + i, page, slot, ch);
            put_chunk<T>(v[i], Vc, vs, h0 + i, page, slot, ch);
        }
    }
}

template <typename T, typename C>
static void append_go(const psa_heads_t& K, const psa_heads_t& V, const PagedSeqs& seqs, const psa_cache_t& cache, int H_kv, hipStream_t stream)
{
    constexpr int ROWS = 4 * 64 / (64 * (int)sizeof(T) / 16);                  // of a work-group
    const dim3 grid((unsigned)((seqs.T + ROWS - 1) / ROWS), (unsigned)((H_kv + kAppendHeads - 1) / kAppendHeads));
    cache_append_kernel<T, C><<<grid, 256, 0, stream>>>(heads_of<const T>(K), heads_of<const T>(V), seqs, page_heads_of<C>(cache.K), page_heads_of<C>(cache.V),
                                                        page_scales_of(cache.K_scales), page_scales_of(cache.V_scales), H_kv);
}
hipError_t launch_cache_append(const psa_heads_t& K, const psa_heads_t& V, const int* offsets, const psa_cache_t& cache, const psa_paged_shape_t& s, hipStream_t stream)
{
    const PagedSeqs seqs{offsets, cache.lengths, cache.table, s.B, s.T, s.T / s.B, 1, cache.max_pages * cache.page_rows, page_shift(cache.page_rows), cache.n_pages,
                         cache.max_pages, 0, 1, 1, nullptr};
    const bool mx = cache.format == PSA_CACHE_MX;
    if (s.dtype == PSA_F32) {
        if (mx) append_go<float, mx8_t>(K, V, seqs, cache, s.H_kv, stream);
        else append_go<float, float>(K, V, seqs, cache, s.H_kv, stream);
    } else {
        if (mx) append_go<bf16_t, mx8_t>(K, V, seqs, cache, s.H_kv, stream);
        else append_go<bf16_t, bf16_t>(K, V, seqs, cache, s.H_kv, stream);
    }
    return hipGetLastError();
}

// ---- the sequences of the next step
// Small calls (update_is_small) are one work-group's, with refs in LDS: what they cost is launches and chains of loads.  Else three
// launches: refs and the workspace; the tables' rows, with the changes of refs that they make; one work-group for what depends on all
// of them, which is little: the pages that are given away, in ascending order.  (In the last work-group that is done with its rows, by a ticket, instead of
// a launch of its own: 13.3 -> 15.7 us, everything it reads comes from memory then.)  One | three launches: 16 x 8 beams, 1161 pages, with the copies 12.5 |
// 19.9 us; 12288 pages and 256 sequences of 128 entries, updates alone, 23.8 | 10.6.  1024 sequences of 256 entries and 200000 pages, free ones among the first: 20.
// Two things take longer.  Free pages are looked for from page 0 on, 4096 at a time: 500000 pages of which 399872 are used, 512 sequences that grow by a page each, 12.6 us where the free ones
// are scattered, 94.8 where they lie behind the used ones, as after a compaction.  And the pages that one sequence grows into are given by one thread, one after the other: 24 prompts of 120 to 750 rows in
// pages of 16 8.5 | 14.5 us (small | large call), one of 32768 rows 143 | 245, 16 of them 320.
constexpr int kScanParents = 4096;         // new sequences up to which each old one looks through all of them for those that continue it
struct UpdateRoom {
    unsigned long long* over;              // pages beyond the tables' rows
    int* holes;                            // sequences that grow inside a page that they do not have
    int *growers, *first, *given;          // [n_pages]: sequences that write to a page next, the first of them; free pages in order of need
    int *last, *had, *want;                // [B_out]: the page that it writes to next (-1: a new one); pages that it has and will have
    int *at, *copied;                      // [B_out]: pages needed before it; whether its last page is copied
    int *children;                         // [B], beyond kScanParents: sequences that continue it
};
static UpdateRoom update_room(const CacheUpdate& u, void* room)
{
    UpdateRoom w{};
    w.over = static_cast<unsigned long long*>(room);
    w.holes = static_cast<int*>(room) + 2;
    int* p = static_cast<int*>(room) + 4;
    w.growers = p; p += u.n_pages;
    w.first = p; p += u.n_pages;
    w.given = p; p += u.n_pages;
    for (int** a : {&w.last, &w.had, &w.want, &w.at, &w.copied}) { *a = p; p += u.B_out; }
    if (u.B_out > kScanParents) w.children = p;
    return w;
}
size_t cache_update_bytes(int B, int B_out, int n_pages) { return ((4 + 3 * (size_t)n_pages + 5 * (size_t)B_out + (B_out > kScanParents ? B : 0)) * sizeof(int) + 255) & ~(size_t)255; }

// Sequence i of the new ones: whom it continues (-1: nobody), the rows and pages it has from there, the rows and pages it will have, and the
// pages that a row of the table cannot hold
struct Child { int parent, n, had, n_out, want; int64_t over; };
__device__ __forceinline__ Child child_of(const CacheUpdate& u, int i)
{
    Child c;
    c.parent = u.parents ? u.parents[i] : i;
    if ((unsigned)c.parent >= (unsigned)u.B) c.parent = -1;
    const int most = u.max_pages * u.page_rows, shift = __builtin_ctz((unsigned)u.page_rows);
    c.n = c.parent < 0 ? 0 : min(max(u.lengths[c.parent], 0), most);
    const int64_t grown = (int64_t)c.n + (u.grow ? max(u.grow[i], 0) : 0);
    c.had = (c.n + u.page_rows - 1) >> shift;
    c.n_out = (int)min(grown, (int64_t)most);
    c.want = (c.n_out + u.page_rows - 1) >> shift;
    c.over = ((grown + u.page_rows - 1) >> shift) - c.want;
    return c;
}
// The last page of a sequence that will write to it; -1: none.  `hole`: the sequence has rows there, but the entry names no page.  It gets none now either: its
// rows there were left out, and on a page of its own, whatever that page held would be seen in their place.
__device__ __forceinline__ int partial_page(const CacheUpdate& u, const Child& c, bool& hole)
{
    hole = false;
    if (c.n_out == c.n || (c.n & (u.page_rows - 1)) == 0) return -1;
    const int page = u.table[(int64_t)c.parent * u.max_pages + c.had - 1];
    hole = (unsigned)page >= (unsigned)u.n_pages;
    return hole ? -1 : page;
}
// What counts[1] says, of `missing` pages that were asked for and `holes`
__device__ __forceinline__ int missing_of(unsigned long long missing, int holes) { return missing != 0 ? (int)min(missing, (unsigned long long)INT_MAX) : holes; }

__global__ __launch_bounds__(256)
void update_begin_kernel(CacheUpdate u, UpdateRoom w)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < u.n_pages) {
        u.refs_out[i] = u.refs[i];
        w.growers[i] = 0;
        w.first[i] = INT_MAX;
    }
    if (w.children && i < u.B) w.children[i] = 0;
    if (i == 0) { *w.over = 0; *w.holes = 0; }
}
__global__ __launch_bounds__(256)
void update_children_kernel(CacheUpdate u, UpdateRoom w)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < u.B_out && (unsigned)u.parents[i] < (unsigned)u.B) atomicAdd(w.children + u.parents[i], 1);
}
// Work-groups 0 .. B - 1: refs follow the number of sequences that continue one; the others: a row of the new table each
__global__ __launch_bounds__(256)
void update_rows_kernel(CacheUpdate u, UpdateRoom w)
{
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < u.B) {
        if (!u.parents) return;
        const int b = blockIdx.x;
        int more = -1;
        if (w.children) {
            more += w.children[b];
        } else {
            for (int i0 = 0; i0 < u.B_out; i0 += 64) {
                const int i = i0 + (tid & 63);
                more += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < u.B_out && u.parents[min(i, u.B_out - 1)] == b));
            }
        }
        if (more == 0) return;
        const int had = (min(max(u.lengths[b], 0), u.max_pages * u.page_rows) + u.page_rows - 1) / u.page_rows;
        for (int j = tid; j < had; j += 256) {
            const int page = u.table[(int64_t)b * u.max_pages + j];
            if ((unsigned)page < (unsigned)u.n_pages) atomicAdd(u.refs_out + page, more);
        }
        return;
    }
    const int i = blockIdx.x - u.B;
    const Child c = child_of(u, i);
    for (int j = tid; j < u.max_pages; j += 256) {
        int page = -1;
        if (j < c.had) {
            page = u.table[(int64_t)c.parent * u.max_pages + j];
            if ((unsigned)page >= (unsigned)u.n_pages) page = -1;
        }
        u.table_out[(int64_t)i * u.max_pages + j] = page;
    }
    if (tid == 0) {
        u.lengths_out[i] = c.n_out;
        bool hole;
        const int page = partial_page(u, c, hole);
        w.last[i] = page;
        w.had[i] = c.had;
        w.want[i] = c.want;
        if (page >= 0) {
            atomicAdd(w.growers + page, 1);
            atomicMin(w.first + page, i);
        }
        if (c.over > 0) atomicAdd(w.over, (unsigned long long)c.over);
        if (hole) atomicAdd(w.holes, 1);
    }
}

// Exclusive prefix over a work-group of 1024 threads of one number each, and the sum of all.  `s` holds 16 ints; calls take two of them in turn.
__device__ __forceinline__ int group_scan(int x, int* s, int& all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int sum = wave_scan(x);
    if (lane == 63) s[wave] = sum;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        if (k < wave) before += s[k];
        all += s[k];
    }
    return before + sum - x;
}
constexpr int kGivenLds = 4096;
__global__ __launch_bounds__(1024)
void update_end_kernel(CacheUpdate u, UpdateRoom w)
{
    __shared__ int s[2][16];
    __shared__ int s_given[kGivenLds];
    const int tid = threadIdx.x;
    int buf = 0, all;
    // (the first pages are looked at while what is needed is counted)
    int refs[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) refs[k] = u.refs_out[min(4 * tid + k, u.n_pages - 1)];
    // pages that are needed: as many free ones are looked for
    int need = 0, last = -1, had = 0, want = 0, copied = 0, at = 0;
    for (int i0 = 0; i0 < u.B_out; i0 += 1024, buf ^= 1) {
        const int i = i0 + tid;
        int n = 0;
        if (i < u.B_out) {
            last = w.last[i]; had = w.had[i]; want = w.want[i];
            copied = last >= 0 && !(u.refs_out[last] == w.growers[last] && w.first[last] == i);
            n = want - had + copied;
        }
        at = need + group_scan(n, s[buf], all);
        if (i < u.B_out && u.B_out > 1024) { w.at[i] = at; w.copied[i] = copied; }
        need += all;                                   // (at most B_out * max_pages <= 2^30)
    }
    int* const given = need <= kGivenLds ? s_given : w.given;
    int found = 0;
    for (int p0 = 0; p0 < u.n_pages && found < need; p0 += 4096, buf ^= 1) {
        const int p = p0 + 4 * tid;
        bool is_free[4];
        int n = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            is_free[k] = p + k < u.n_pages && refs[k] == 0;
            n += is_free[k];
            refs[k] = u.refs_out[min(p + 4096 + k, u.n_pages - 1)];
        }
        int to = found + group_scan(n, s[buf], all);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (is_free[k]) { if (to < need) given[to] = p + k; ++to; }
        found += all;
    }
    __syncthreads();                                   // (all of `given` is written, and refs have been read)
    int pairs = 0;
    for (int i0 = 0; i0 < u.B_out; i0 += 1024, buf ^= 1) {
        const int i = i0 + tid;
        if (i < u.B_out && u.B_out > 1024) { last = w.last[i]; had = w.had[i]; want = w.want[i]; copied = w.copied[i]; at = w.at[i]; }
        const bool with_page = i < u.B_out && copied && at < found;
        const int pair = pairs + group_scan(with_page, s[buf], all);
        pairs += all;
        if (i < u.B_out) {
            int* row = u.table_out + (int64_t)i * u.max_pages;
            if (copied) {
                atomicAdd(u.refs_out + last, -1);
                if (with_page) { u.pairs[2 * pair] = last; u.pairs[2 * pair + 1] = given[at]; }
            }
            for (int j = had - copied; j < want; ++j, ++at) {
                const int page = at < found ? given[at] : -1;
                row[j] = page;
                if (page >= 0) u.refs_out[page] = 1;   // (it was 0: nobody else's)
            }
        }
    }
    for (int i = pairs + tid; i < u.B_out; i += 1024) u.pairs[2 * i] = u.pairs[2 * i + 1] = -1;
    if (tid == 0) {
        u.counts[0] = pairs;
        u.counts[1] = missing_of((unsigned long long)max(need - found, 0) + *w.over, *w.holes);
    }
}
// The same by one work-group.  A sequence to a thread; entries of the tables to any.
constexpr int kSmallPages = 8192, kSmallSequences = 1024, kSmallEntries = 8192;
static bool update_is_small(const CacheUpdate& u)
{
    return u.n_pages <= kSmallPages && u.B <= kSmallSequences && u.B_out <= kSmallSequences && (int64_t)u.B * u.max_pages <= kSmallEntries &&
           (int64_t)u.B_out * u.max_pages <= kSmallEntries;
}
__global__ __launch_bounds__(1024)
void update_small_kernel(CacheUpdate u)
{
    extern __shared__ int lds[];
    int *const refs = lds, *const mark = lds + u.n_pages, *const given = lds + 2 * u.n_pages;
    __shared__ int s_had_in[kSmallSequences], s_had[kSmallSequences], s_parent[kSmallSequences];
    __shared__ int s[2][16];
    __shared__ unsigned long long s_over;
    __shared__ int s_holes;
    const int tid = threadIdx.x, shift = __builtin_ctz((unsigned)u.page_rows);
    Child c{};
    int last = -1;                                     // the page that this thread's sequence writes to next, where it has rows of others
    bool hole = false;
    // (asked for before the chain of loads that each sequence is)
    constexpr int AHEAD = kSmallPages / 1024;
    int held[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) held[k] = u.refs[min(tid + 1024 * k, u.n_pages - 1)];
    if (tid == 0) { s_over = 0; s_holes = 0; }
    if (tid < u.B_out) {
        c = child_of(u, tid);
        last = partial_page(u, c, hole);
        s_had[tid] = c.had;
        s_parent[tid] = c.parent;
        u.lengths_out[tid] = c.n_out;
    }
    if (tid < u.B) s_had_in[tid] = (min(max(u.lengths[tid], 0), u.max_pages * u.page_rows) + u.page_rows - 1) >> shift;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (tid + 1024 * k < u.n_pages) { refs[tid + 1024 * k] = held[k]; mark[tid + 1024 * k] = INT_MAX; }
    __syncthreads();
    if (c.over > 0) atomicAdd(&s_over, (unsigned long long)c.over);
    if (hole) atomicAdd(&s_holes, 1);
    // who holds what: the old sequences' entries go, the new ones' come (without parents they are the same)
    const int entries = u.B * u.max_pages, entries_out = u.B_out * u.max_pages;
    if (u.parents) {
#pragma unroll 4
        for (int e = tid; e < entries; e += 1024) {
            const int b = e / u.max_pages;
            if (e - b * u.max_pages >= s_had_in[b]) continue;
            const int page = u.table[e];
            if ((unsigned)page < (unsigned)u.n_pages) atomicAdd(refs + page, -1);
        }
    }
#pragma unroll 4
    for (int e = tid; e < entries_out; e += 1024) {
        const int i = e / u.max_pages, j = e - i * u.max_pages;
        int page = -1;
        if (j < s_had[i]) {
            page = u.table[s_parent[i] * u.max_pages + j];
            if ((unsigned)page >= (unsigned)u.n_pages) page = -1;
            else if (u.parents) atomicAdd(refs + page, 1);
        }
        u.table_out[e] = page;
    }
    // of those that write to one page the first, then how many they are
    if (last >= 0) atomicMin(mark + last, tid);
    __syncthreads();
    const bool is_first = last >= 0 && mark[last] == tid;
    __syncthreads();
    if (last >= 0) mark[last] = 0;
    __syncthreads();
    if (last >= 0) atomicAdd(mark + last, 1);
    __syncthreads();
    const int copied = last >= 0 && !(is_first && refs[last] == mark[last]);
    int need, all, found = 0, buf = 0;
    int at = group_scan(tid < u.B_out ? c.want - c.had + copied : 0, s[1], need);
    for (int p0 = 0; p0 < u.n_pages && found < need; p0 += 4096, buf ^= 1) {
        const int p = p0 + 4 * tid;
        bool is_free[4];
        int n = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            is_free[k] = p + k < u.n_pages && refs[min(p + k, u.n_pages - 1)] == 0;
            n += is_free[k];
        }
        int to = found + group_scan(n, s[buf], all);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (is_free[k]) given[to++] = p + k;
        found += all;
    }
    __syncthreads();                                   // (all of `given` is written, refs have been read, and the tables' stores are done)
    int pairs;
    const bool with_page = copied && at < found;
    const int pair = group_scan(with_page, s[0], pairs);
    if (copied) atomicAdd(refs + last, -1);
    if (with_page) { u.pairs[2 * pair] = last; u.pairs[2 * pair + 1] = given[at]; }
    if (tid < u.B_out) {
        for (int j = c.had - copied; j < c.want; ++j, ++at) {
            const int page = at < found ? given[at] : -1;
            u.table_out[tid * u.max_pages + j] = page;
            if (page >= 0) refs[page] = 1;             // (it was 0: nobody else's)
        }
    }
    if (tid >= pairs && tid < u.B_out) u.pairs[2 * tid] = u.pairs[2 * tid + 1] = -1;
    if (tid == 0) {
        u.counts[0] = pairs;
        u.counts[1] = missing_of((unsigned long long)max(need - found, 0) + s_over, s_holes);
    }
    __syncthreads();
    for (int p = tid; p < u.n_pages; p += 1024) u.refs_out[p] = refs[p];
}

hipError_t launch_cache_update(const CacheUpdate& u, void* workspace, hipStream_t stream)
{
    if (update_is_small(u)) {
        if (const hipError_t e = init_cache(); e != hipSuccess) return e;
        update_small_kernel<<<1, 1024, 3 * u.n_pages * sizeof(int), stream>>>(u);
        return hipGetLastError();
    }
    const UpdateRoom w = update_room(u, workspace);
    const int n = w.children && u.B > u.n_pages ? u.B : u.n_pages;
    update_begin_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(u, w);
    if (w.children && u.parents) update_children_kernel<<<(unsigned)((u.B_out + 255) / 256), 256, 0, stream>>>(u, w);
    update_rows_kernel<<<(unsigned)(u.B + u.B_out), 256, 0, stream>>>(u, w);
    update_end_kernel<<<1, 1024, 0, stream>>>(u, w);
    return hipGetLastError();
}

// ---- compaction
// The pages in use are counted, n of them; holes before n and pages in use from n on are ranked, which pairs them; then refs and entries follow.
// Small calls are one work-group's; else blocks of kBlockPages pages are counted first, and each finds from the counts what lies before it: 1000
// pages 4.5 us, 12288 pages and 256 sequences of 128 entries 16.7 in one work-group, 11.4 in blocks, 500000 pages 14.8 (ranked by one work-group 358).
// Workspace: [n_pages], where a page at n or behind goes, and the blocks' counts.
constexpr int kBlockPages = 4096;
size_t cache_compact_bytes(int n_pages) { return (((size_t)n_pages + (n_pages + kBlockPages - 1) / kBlockPages) * sizeof(int) + 255) & ~(size_t)255; }
__device__ __forceinline__ int group_sum(int x, int* s)
{
    int all;
    group_scan(x, s, all);
    return all;
}
__global__ __launch_bounds__(1024)
void compact_count_kernel(const int* __restrict__ refs, int n_pages, int* __restrict__ count)
{
    __shared__ int s[16];
    int n = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int p = blockIdx.x * kBlockPages + k * 1024 + threadIdx.x;
        n += p < n_pages && refs[min(p, n_pages - 1)] != 0;
    }
    n = group_sum(n, s);
    if (threadIdx.x == 0) count[blockIdx.x] = n;
}
__global__ __launch_bounds__(1024)
void compact_rank_kernel(const int* __restrict__ refs, int n_pages, const int* __restrict__ count, int n_block, int* __restrict__ pairs, int* __restrict__ counts)
{
    __shared__ int s[2][16];
    const int tid = threadIdx.x, block = blockIdx.x;
    int all = 0, before = 0;                           // pages in use, in all blocks and in those before this one
    for (int i = tid; i < n_block; i += 1024) {
        all += count[i];
        before += i < block ? count[i] : 0;
    }
    const int used = group_sum(all, s[0]);
    before = group_sum(before, s[1]);
    // the block that `used` falls into: how many of its pages before there are in use, and in all blocks up to there
    const int border = min(used / kBlockPages, n_block - 1);
    int low = 0, under = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int p = border * kBlockPages + k * 1024 + tid;
        low += p < used && refs[min(p, n_pages - 1)] != 0;
    }
    for (int i = tid; i < border; i += 1024) under += count[i];
    const int front = group_sum(low + under, s[0]);    // pages in use before `used`: as many stay
    const int moved = used - front;
    const int p = block * kBlockPages + 4 * tid;
    bool is_hole[4], is_moved[4];
    int h = 0, m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const bool taken = p + k < n_pages && refs[min(p + k, n_pages - 1)] != 0;
        h += is_hole[k] = p + k < used && !taken;
        m += is_moved[k] = p + k >= used && taken;
    }
    int unused;
    h = block * kBlockPages - before + group_scan(h, s[1], unused);            // (blocks up to the border: all their pages are before `used`)
    m = max(before - front, 0) + group_scan(m, s[0], unused);                  // (blocks behind it: all their pages are behind)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (is_hole[k]) pairs[2 * (int64_t)h++ + 1] = p + k;
        if (is_moved[k]) pairs[2 * (int64_t)m++] = p + k;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (p + k >= moved && p + k < n_pages / 2) pairs[2 * (int64_t)(p + k)] = pairs[2 * (int64_t)(p + k) + 1] = -1;
    if (block == 0 && tid == 0) { counts[0] = moved; counts[1] = used; }
}
__global__ __launch_bounds__(256)
void compact_map_kernel(const int* __restrict__ refs, int n_pages, const int* __restrict__ pairs, const int* __restrict__ counts, int* __restrict__ refs_out, int* __restrict__ to)
{
    const int p = blockIdx.x * 256 + threadIdx.x, moved = counts[0], used = counts[1];
    if (p < moved) {
        const int from = pairs[2 * p], hole = pairs[2 * p + 1];
        to[from] = hole;
        refs_out[hole] = refs[from];
    }
    if (p < n_pages && (p >= used || refs[p] != 0)) refs_out[p] = p < used ? refs[p] : 0;
}
__global__ __launch_bounds__(256)
void compact_table_kernel(const int* table, int64_t entries, int n_pages, const int* __restrict__ refs, const int* __restrict__ counts, const int* __restrict__ to, int* table_out)
{
    const int used = counts[1];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += (int64_t)gridDim.x * 256) {
        const int page = table[i];
        const bool moves = page >= used && page < n_pages && refs[page] != 0;
        table_out[i] = moves ? to[page] : page;
    }
}
constexpr int kSmallCompactPages = 8192, kSmallCompactEntries = 16384;
__global__ __launch_bounds__(1024)
void compact_small_kernel(const int* table, const int* __restrict__ refs, int entries, int n_pages, int* table_out, int* __restrict__ refs_out, int* __restrict__ pairs,
                          int* __restrict__ counts)
{
    extern __shared__ int lds[];
    int *const r = lds, *const from = lds + n_pages, *const hole = from + n_pages / 2;
    __shared__ int s[2][2][16];
    const int tid = threadIdx.x;
    // (the first entries are asked for before it is known where their pages go)
    constexpr int AHEAD = 8;
    int entry[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) entry[k] = table[min(tid + 1024 * k, entries - 1)];
    int all, used = 0;
#pragma unroll 4
    for (int p = tid; p < n_pages; p += 1024) {
        const int x = refs[p];
        r[p] = x;
        used += x != 0;
    }
    group_scan(used, s[0][0], used);
    int holes = 0, moved = 0, buf = 1;
    for (int p0 = 0; p0 < n_pages; p0 += 4096, buf ^= 1) {
        const int p = p0 + 4 * tid;
        bool is_hole[4], is_moved[4];
        int h = 0, m = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool in = p + k < n_pages, taken = in && r[min(p + k, n_pages - 1)] != 0;
            h += is_hole[k] = p + k < used && !taken;
            m += is_moved[k] = p + k >= used && taken;
        }
        h = holes + group_scan(h, s[buf][0], all);
        holes += all;
        m = moved + group_scan(m, s[buf][1], all);
        moved += all;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (is_hole[k]) hole[h++] = p + k;
            if (is_moved[k]) from[m++] = p + k;
        }
    }
    __syncthreads();
    for (int p = tid; p < n_pages; p += 1024)
        if (p >= used || r[p] != 0) refs_out[p] = p < used ? r[p] : 0;
    __syncthreads();
    for (int i = tid; i < n_pages / 2; i += 1024) {
        int2 pair = make_int2(-1, -1);
        if (i < moved) {
            pair = make_int2(from[i], hole[i]);
            refs_out[pair.y] = r[pair.x];
            r[pair.x] = ~pair.y;                       // (below 0) from here on, of pages at `used` and behind: where they go
        }
        pairs[2 * i] = pair.x;
        pairs[2 * i + 1] = pair.y;
    }
    if (tid == 0) { counts[0] = moved; counts[1] = used; }
    __syncthreads();
    auto follow = [&](int page) {
        if (page < used || page >= n_pages) return page;
        const int to = r[page];
        return to < 0 ? ~to : page;
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (tid + 1024 * k < entries) table_out[tid + 1024 * k] = follow(entry[k]);
    for (int e = tid + 1024 * AHEAD; e < entries; e += 1024) table_out[e] = follow(table[e]);
}
static std::atomic<uint64_t> g_update_small{0}, g_compact_small{0};
hipError_t init_cache()
{
    hipError_t e = ensure_lds_limit(reinterpret_cast<const void*>(&update_small_kernel), 3 * kSmallPages * sizeof(int), g_update_small);
    if (e == hipSuccess) e = ensure_lds_limit(reinterpret_cast<const void*>(&compact_small_kernel), 2 * kSmallCompactPages * sizeof(int), g_compact_small);
    return e;
}
hipError_t launch_cache_compact(const int* table, const int* refs, int B, int n_pages, int max_pages, int* table_out, int* refs_out, int* pairs, int* counts, void* workspace, hipStream_t stream)
{
    const int64_t entries = (int64_t)B * max_pages, groups = (entries + 255) / 256;
    if (n_pages <= kSmallCompactPages && entries <= kSmallCompactEntries) {
        if (const hipError_t e = init_cache(); e != hipSuccess) return e;
        compact_small_kernel<<<1, 1024, 2 * n_pages * sizeof(int), stream>>>(table, refs, (int)entries, n_pages, table_out, refs_out, pairs, counts);
        return hipGetLastError();
    }
    int *const to = static_cast<int*>(workspace), *const count = to + n_pages;
    const int n_block = (n_pages + kBlockPages - 1) / kBlockPages;
    compact_count_kernel<<<n_block, 1024, 0, stream>>>(refs, n_pages, count);
    compact_rank_kernel<<<n_block, 1024, 0, stream>>>(refs, n_pages, count, n_block, pairs, counts);
    compact_map_kernel<<<(unsigned)((n_pages + 255) / 256), 256, 0, stream>>>(refs, n_pages, pairs, counts, refs_out, to);
    compact_table_kernel<<<(unsigned)(groups < 4096 ? groups : 4096), 256, 0, stream>>>(table, entries, n_pages, refs, counts, to, table_out);
    return hipGetLastError();
}

// ---- copies of pages
// 2010 pages of 128 KB in two pools to the front, 1.05 GB read and written: 197 us, 5.3 TB/s, the rate of a large copy.
constexpr int kPools = 64, kFewPools = 4;  // of a launch; those of a launch whose arguments are short
constexpr int kCopyBytes = 16384;          // of a page that a work-group takes at a time
template <int N> struct Pools { unsigned char* data[N]; int64_t stride[N], bytes[N]; int unit[N]; };
template <typename W>
__device__ __forceinline__ void copy_bytes(unsigned char* to, const unsigned char* from, int bytes)
{
    W* dst = reinterpret_cast<W*>(to);
    const W* src = reinterpret_cast<const W*>(from);
    const int n = bytes / (int)sizeof(W);
    for (int i = threadIdx.x; i < n; i += 1024) {
        const int last = n - 1;                        // (loads of four in flight: those behind the end read its last again)
        const W a = src[i], b = src[min(i + 256, last)], c = src[min(i + 512, last)], d = src[min(i + 768, last)];
        dst[i] = a;
        if (i + 256 < n) dst[i + 256] = b;
        if (i + 512 < n) dst[i + 512] = c;
        if (i + 768 < n) dst[i + 768] = d;
    }
}
template <int N>
__global__ __launch_bounds__(256)
void cache_copy_kernel(Pools<N> pools, int n_pools, int parts, int n_pages, const int* __restrict__ pairs, const int* __restrict__ counts, int n_pairs)
{
    const int n = counts ? min(max(counts[0], 0), n_pairs) : n_pairs;
    const int64_t items = (int64_t)n * n_pools * parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int part = (int)(item % parts), pool = (int)(item / parts % n_pools);
        const int64_t pair = item / parts / n_pools;
        const int from = pairs[2 * pair], to = pairs[2 * pair + 1];
        if ((unsigned)from >= (unsigned)n_pages || (unsigned)to >= (unsigned)n_pages || from == to) continue;
        const int64_t at = (int64_t)part * kCopyBytes;
        const int bytes = (int)min((int64_t)kCopyBytes, pools.bytes[pool] - at);
        if (bytes <= 0) continue;
        unsigned char* dst = pools.data[pool] + to * pools.stride[pool] + at;
        const unsigned char* src = pools.data[pool] + from * pools.stride[pool] + at;
        if (pools.unit[pool] == 16) copy_bytes<uint4>(dst, src, bytes);
        else if (pools.unit[pool] == 4) copy_bytes<uint32_t>(dst, src, bytes);
        else copy_bytes<uint8_t>(dst, src, bytes);
    }
}
template <int N>
static void copy_go(const psa_pool_t* pools, int n, int n_pages, const int* pairs, const int* counts, int n_pairs, hipStream_t stream)
{
    Pools<N> p{};
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        p.data[i] = static_cast<unsigned char*>(pools[i].data);
        p.stride[i] = pools[i].page_stride;
        p.bytes[i] = pools[i].page_bytes;
        const uintptr_t bits = reinterpret_cast<uintptr_t>(pools[i].data) | (uintptr_t)pools[i].page_stride | (uintptr_t)pools[i].page_bytes;
        p.unit[i] = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
        if (pools[i].page_bytes > most) most = pools[i].page_bytes;
    }
    const int64_t parts = (most + kCopyBytes - 1) / kCopyBytes, items = n_pairs * parts * n;
    cache_copy_kernel<N><<<(unsigned)(items < 2048 ? items : 2048), 256, 0, stream>>>(p, n, (int)parts, n_pages, pairs, counts, n_pairs);
}
hipError_t launch_cache_copy(const psa_pool_t* pools, int n_pools, int n_pages, const int* pairs, const int* counts, int n_pairs, hipStream_t stream)
{
    for (int first = 0; first < n_pools; first += kPools) {
        const int n = n_pools - first < kPools ? n_pools - first : kPools;
        (n <= kFewPools ? copy_go<kFewPools> : copy_go<kPools>)(pools + first, n, n_pages, pairs, counts, n_pairs, stream);
    }
    return hipGetLastError();
}

}  // namespace psa
