// Where the few rows' kernels load from (gdn_few_kernel.h): plain arithmetic, the host's too.
#pragma once
#include <cstdint>

#ifdef __HIP__
#define GDN_FEW_FN __host__ __device__ __forceinline__
#else
#define GDN_FEW_FN inline
#endif

namespace gdn {
namespace few {

constexpr int STEP = 64;                          // k of a step: a row of 128 bytes

// Rows of a matrix: where they begin, the bytes up to the last one's end (what lies behind arrives as zeros), the bytes from one to the next.
struct Part {
    const char* at;
    int bytes, pitch;
};

// At most `most` rows from row `first` of a weight of N rows of K, ld elements apart; where there are none the last row stands for them (their sums go nowhere). No part
// that is loaded from at a k is empty: a load is cut off by its lane's offset against the descriptor's bytes less its scalar offset, k, and that difference must not wrap.
GDN_FEW_FN Part rows_from(const void* w, int64_t ld, int32_t N, int32_t K, int first, int most) {
    const int from = first < N ? first : N - 1, rows = N - from;
    return Part{static_cast<const char*>(w) + (int64_t)from * ld * 2, (int)((int64_t)((rows < most ? rows : most) - 1) * ld * 2 + (int64_t)K * 2), (int)(ld * 2)};
}

// Where piece `pos` (16 bytes) of row `row` of a stage comes from, at k = 0, in a part whose row `of_part` it is.  Piece p of row r lies at p ^ (r / 2) % 8: 16 rows' pieces of
// one k then spread over the banks.
GDN_FEW_FN int load_offset(int row, int of_part, int pos, int pitch) { return of_part * pitch + ((pos ^ ((row >> 1) & 7)) << 4); }

}  // namespace few
}  // namespace gdn
