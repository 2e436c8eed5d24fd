// Where a row of the cache lives, and the status word: shared by the kernels that move cache rows.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace vispec {

__device__ __forceinline__ void record_status(int* status, int code) {
    if (status) atomicCAS(status, 0, code);
}

// Where logical slot `slot` of (sequence b, kv head h) lives, in 16-byte vectors from the tensor's base.
// Contiguous cache [B,Hkv,S_max,D]: table == nullptr.  Paged pool [num_blocks,Hkv,page_rows,D], or
// [num_blocks,page_rows,Hkv,D] if token_major: through the block table; -1 if the table entry is outside the pool.
struct RowMap {
    const int32_t* table; int table_stride, page_rows, num_blocks, token_major;
    __device__ __forceinline__ long long at(int b, int h, int slot, int Hkv, int S_max, int chunks) const {
        if (!table) return (((long long)b * Hkv + h) * S_max + slot) * chunks;
        const int blk = table[(size_t)b * table_stride + slot / page_rows];
        if (blk < 0 || blk >= num_blocks) return -1;
        if (token_major) return (((long long)blk * page_rows + slot % page_rows) * Hkv + h) * chunks;
        return (((long long)blk * Hkv + h) * page_rows + slot % page_rows) * chunks;
    }
};

}  // namespace vispec
