// Device-side helpers of heads, cache and attention: tokens of rows, 4-bit codes.
#pragma once

#include "cache.h"
#include "rows_device.h"

namespace dcnn {

struct Token {
    int stream, pos;
    bool here;                                 // the row has a token
};
__device__ __forceinline__ Token token_of(const TokenArgs& t, int r) {
    const int i = t.idx != nullptr ? t.idx[r] : r;
    if ((uint32_t)i >= (uint32_t)t.map_rows) return {0, 0, false};
    const int q = (int)fast_div((uint32_t)i, t.period);
    return {t.stream != nullptr ? t.stream[i] : q, t.pos != nullptr ? t.pos[i] : i - q * (int)t.period.d, true};
}
// The page of block `block` (of per_stream) of a stream, -1: none.
__device__ __forceinline__ int page_of(const CacheArgs& c, int stream, int block) {
    if ((uint32_t)block >= (uint32_t)c.per_stream) return -1;
    const int64_t at = (int64_t)stream * c.per_stream + block;
    const int page = c.pages != nullptr ? c.pages[at] : (int)at;
    return (uint32_t)page < (uint32_t)c.num_pages ? page : -1;
}
// The same where stream and block are one for all lanes: through the scalar cache, so that it waits for no other load.  (No branches: what is loaded is
// waited for where it is used.  Without a table, or past its end, a word of the codes or of the table is read, and not looked at.)
__device__ __forceinline__ int page_of_all(const CacheArgs& c, int stream, int block) {
    typedef __attribute__((address_space(4))) const int32_t ConstInt;
    const bool in = (uint32_t)block < (uint32_t)c.per_stream;
    const int64_t at = (int64_t)stream * c.per_stream + (in ? block : 0);
    const int entry = *((ConstInt*)(c.pages != nullptr ? (uintptr_t)(c.pages + at) : (uintptr_t)c.codes));
    const int page = c.pages != nullptr ? entry : (int)at;
    return in && (uint32_t)page < (uint32_t)c.num_pages ? page : -1;
}
// Tokens before the first one of a page's head; `which`: 0 keys, 1 values.
__device__ __forceinline__ int64_t head_of_page(const CacheArgs& c, int page, int which, int head) {
    return (((int64_t)page * 2 + which) * c.heads + head) << c.page_shift;
}

// The scale of eight codes travels in bits 30..23 of a register: the conversions look at nothing else.
__device__ __forceinline__ float scale_of_byte(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

}  // namespace dcnn
