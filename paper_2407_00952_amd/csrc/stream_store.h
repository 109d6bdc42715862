// Stores of large outputs that bypass the caches.
//
// A call that moves more than half of what the last-level cache (256 MB) holds pushes out of it whatever the calls around it left
// there, with results that will mostly be gone again when their reader gets to them.  Such calls store their results with the
// non-temporal hint, smaller ones leave them in the cache for the reader.  Measured with / without, inputs changing from call to
// call: RMS norm [32768, 1024], fp32 stream, both directions, 185 / 196 us; [10001, 5120] bf16 138 / 146; embedding of 65536 tokens of
// 1024, lookup and gradient, 154 / 162.
#pragma once
#include <stddef.h>

inline bool stream_results(size_t bytes_moved) { return bytes_moved > ((size_t)128 << 20); }

// (STREAM is a template argument because two branches with the two stores become one store without the hint in the compiler)
template <bool STREAM, class V>
__device__ __forceinline__ void store_result(V *p, V v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}
