// A cache in pages: what the kernels that read it and those that write it share.
#pragma once

#include "psa_packed.h"

namespace psa {

struct mx8_t { uint8_t x; };               // an 8-bit float (e4m3); a byte for each 32 of a row holds the power of two they are multiplied by

constexpr int kUnit = 128;                 // keys: a round of the 4 waves of a work-group
constexpr int kPagedMany = 256;            // sequences beyond which the parts of a call are counted by a kernel of its own

// K or V of a pool, and the powers of two of 8-bit ones (strides in elements)
template <typename C>
struct PageHeads { C* data; int64_t page, head, row; };
template <typename C>
inline PageHeads<C> page_heads_of(const psa_heads_t& t) { return PageHeads<C>{static_cast<C*>(t.data), t.batch_stride, t.head_stride, t.row_stride}; }
struct PageScales {
    uint8_t* data; int64_t page, head, row;
    __device__ __forceinline__ uint8_t* at(int hk, int p, int slot) const { return data + hk * head + p * page + slot * row; }
};
inline PageScales page_scales_of(const psa_heads_t& t) { return PageScales{static_cast<uint8_t*>(t.data), t.batch_stride, t.head_stride, t.row_stride}; }

inline int page_shift(int page_rows) { return __builtin_ctz((unsigned)page_rows); }

// The sequences of a call: their new rows (offsets, or `uniform` each) and their rows in the cache
struct PagedSeqs {
    const int* offsets; const int* lengths; const int* table;
    int B, T, uniform, G, capacity, shift, n_pages, max_pages, row_shift, per_head, least;
    const int* before;
};

// Inclusive prefix sum over the 64 lanes: within rows of 16 by shifts, then the rows' last lanes are handed on.
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}

}  // namespace psa
