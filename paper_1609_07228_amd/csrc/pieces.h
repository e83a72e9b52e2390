// Pieces of eight columns of a row that has n of them, one after the other: where a piece that begins at column `at` (a multiple of
// eight, also past the last one) is loaded from, and how it is put in its place.  No load leaves the row.  For the host too, where
// every width is checked.
#pragma once

// A row of eight columns and more: a piece that the last column is in, or past it, is loaded as the last eight ...
constexpr int piece_from(int at, int n) { return n >= 8 ? (at < n - 8 ? at : n - 8) : 0; }
// ... and moved down by so many (8 and more: nothing of it is used).
constexpr int piece_moved(int at, int n) { return n >= 8 ? at - piece_from(at, n) : 0; }
// A row of fewer columns is read one by one: column of element k.
constexpr int piece_column(int k, int n) { return k < n ? k : n - 1; }

// Eight elements from the `by`-th on (the ones after the last: anything)
template <class Y, class Eight> constexpr Eight moved_down(Eight x, int by)
{
    constexpr int kWords = 2 * sizeof(Y);
    typedef unsigned Words __attribute__((ext_vector_type(kWords)));
    Words w = __builtin_bit_cast(Words, x);
    const int words = by * (int)sizeof(Y) / 4;
#pragma unroll
    for (int bit = 1; bit < kWords; bit *= 2)
#pragma unroll
        for (int k = 0; k + bit < kWords; ++k) w[k] = words & bit ? w[k + bit] : w[k];
    if (sizeof(Y) == 2)
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = by & 1 ? w[k] >> 16 | (k + 1 < kWords ? w[k + 1] << 16 : 0) : w[k];
    return __builtin_bit_cast(Eight, w);
}
