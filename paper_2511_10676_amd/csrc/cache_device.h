// Addressing of a paged key-value cache in device code.
#pragma once

#include "paep_device.h"
#include "paep_internal.h"

namespace paep {

// Page of entry i of sequence b, -1 where the entry names none (also past the table's end).
__device__ __forceinline__ int page_entry(const int32_t* table, int max_pages, int n_pages, int b, int i)
{
    if (i >= max_pages) return -1;
    const int page = table[(long long)b * max_pages + i];
    return (uint32_t)page < (uint32_t)n_pages ? page : -1;
}

// A sequence's length as every call reads it: 0 to max_len.
__device__ __forceinline__ int clamped_length(const int32_t* lengths, int b, int max_len)
{
    const int n = lengths[b];
    return n < 0 ? 0 : n > max_len ? max_len : n;
}

}  // namespace paep
