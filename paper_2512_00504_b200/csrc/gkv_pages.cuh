// Rows of a cache in pages.
#pragma once

#include "gkv_store_codes.cuh"

namespace gkv {

// Numbers that no row has (a cache has below 2^31 rows): no such row here, and a row whose place in the table holds no page.
constexpr uint32_t kNoRow = 0xffffffffu, kNoPage = 0xfffffffeu;

__device__ __forceinline__ int page_of(const PagesView& g, int row) { return (int)((uint64_t)(uint32_t)row * g.inv_page >> 40); }
// What the table of a sequence holds for a row.
__device__ __forceinline__ int32_t page_entry(const PagesView& g, const int32_t* table, int row) { return table[page_of(g, row)]; }
// Number, over all pages and heads, of a sequence's row in head `head` (its first rows' number `head0` = head * head_rows).
__device__ __forceinline__ uint32_t page_row(const PagesView& g, int32_t entry, uint32_t head0, int row) {
    if ((uint32_t)entry >= (uint32_t)g.n_pages) return kNoPage;
    return (uint32_t)entry * g.page_rows + head0 + (uint32_t)(row - page_of(g, row) * g.page_size) * g.token_rows;
}

__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
    return r;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a) : "memory");
    return r;
}
__device__ __forceinline__ uint32_t lds2(uint32_t a) {
    uint16_t r;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r) : "r"(a) : "memory");
    return r;
}

}  // namespace gkv
