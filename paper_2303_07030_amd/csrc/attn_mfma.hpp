// The matrix-core kernels of differential attention (bfloat16, widths of at
// least eight) as the entry points call them.
#pragma once

#include "attn.hpp"

namespace nsd {
namespace attn {

// A wave's share of the heads.
struct Slab {
    int32_t hs;     // key heads
    int32_t nsub;   // shares of one key head's query heads (eight each)
    int32_t nslab;  // slabs in all
    int32_t nc, nv; // 32-column chunks of keys, 128-column groups of values
    int32_t full;   // the key columns fill their chunks
    int32_t lrh;    // log2 of the query heads that a mask row takes of the eight
};

// What the matrix cores can take, and where they are faster than the vector form.
inline bool fits_cores(const nsd_attn *s) {
    return s->dtype == NSD_BF16 && s->d >= 8 && s->dv >= 8;
}
bool cores_pay(const nsd_attn *s);

Slab make_slab(const nsd_attn *s);
Slab one_row(Slab b);      // of single rows: one mask row at a time
Slab column_slab(Slab b);  // of the pass over columns: whole key heads
int64_t mfma_blocks(int64_t items, const Slab &b);
void mfma_forward(const FwdArgs &a, const Slab &b, int64_t blocks, bool decode, hipStream_t st);
void mfma_rows(const BwdArgs &a, const Slab &b, int64_t blocks, hipStream_t st);
void mfma_columns(const BwdArgs &a, const Slab &b, int64_t blocks, hipStream_t st);

}  // namespace attn
}  // namespace nsd
