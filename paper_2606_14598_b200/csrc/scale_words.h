// MXFP4 scales of one head of a token, fetched as 4-byte words by copies that want their addresses aligned (the buffer is): from the word that the head's first
// byte is in up to its last byte, so that nothing behind the buffer is read. Host and device code.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define W8A8_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define W8A8_HOST_DEVICE inline
#endif

namespace w8a8 {

struct ScaleWords {
    int64_t from;                               // first byte fetched, a multiple of 4
    int shift;                                  // bytes of it that belong to heads before this one
    int end;                                    // bytes from `from` to the head's end
    // bytes to fetch of word i (the rest of it is filled with zeros)
    W8A8_HOST_DEVICE int bytes(int i) const {
        const int left = end - 4 * i;
        return left < 0 ? 0 : left < 4 ? left : 4;
    }
};
// entry: slot * heads + head; blocks: scales of a head
W8A8_HOST_DEVICE ScaleWords scale_words(int64_t entry, int blocks) {
    const int64_t first = entry * blocks;
    const int shift = static_cast<int>(first & 3);
    return ScaleWords{first - shift, shift, shift + blocks};
}

} // namespace w8a8
