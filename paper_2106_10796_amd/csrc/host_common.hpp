// Host-side checks that the entry points of every translation unit share.
#pragma once

namespace {

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Do [a, a + na) and [b, b + nb) share a byte?  (NULL never overlaps.)
inline bool overlap2(const void *a, size_t na, const void *b, size_t nb)
{
    if (!a || !b) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y ? y - x < na : x - y < nb;
}

// Do the byte ranges [a, a + bytes) and [b, b + bytes) share a byte?  (NULL never overlaps.)
inline bool overlap(const void *a, const void *b, size_t bytes)
{
    if (!a || !b) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y ? y - x < bytes : x - y < bytes;
}

inline int launch_status()
{
    return hipGetLastError() == hipSuccess ? CDSGD_OK : CDSGD_ERR_DEVICE;
}

}  // namespace
