// What the key-split prefill kernels (attn_split.hip, attn_split8.hip) share:
// the numbering of their column blocks.
#pragma once

#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace rc {

namespace {

constexpr int kCols = 32;  // columns (row, head) per block

// Whether a launch numbers its blocks over the column blocks that there are
// rather than n_qt for every request (and leaves a work order aside).  In a
// batch of few long and many short requests most blocks of the full grid are
// empty, and the others fall on few XCDs and CUs wherever n_qt has a factor in
// common with their number: 63 requests of one query and one of 128 over 100
// keys, 8 / 1 heads, 83 us against 14; 511 and one 431 against 31.  A full grid
// of one block per free CU slot (two 4-wave blocks or one of 8 per CU) has no
// such problem and saves the search (0.5 us: four requests of 9 to 300 queries,
// 8 / 2 heads, 28.4 us against 29.0).
bool compact_grid(const AttnArgs& a, int waves) {
    return a.n_qt > 1 && a.n_units > 1 && (long)a.n_qt * a.n_units * a.n_kv_heads > 2048 / waves;
}

// The idx-th column block in order of the requests, each one's last columns
// first: (request, column block), or request -1 past the last.  Each wave
// searches for itself, four requests per lane and step.
__device__ __forceinline__ int2 nth_col_block(const AttnArgs& a, int idx, int lane) {
    for (int u0 = 0; u0 < a.n_units; u0 += 256) {
        const int u = u0 + lane * 4;
        int c[5], n[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 5; ++i) c[i] = a.cu_q[min(u + i, a.n_units)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            n[i] = (max(0, min(c[i + 1] - c[i], a.max_rows)) * a.ratio + kCols - 1) / kCols;
            sum += n[i];
        }
        int incl = sum;
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(incl, o);
            if (lane >= o) incl += y;
        }
        int at = idx - (incl - sum);  // of the lane's column blocks
        const uint64_t hit = __builtin_amdgcn_ballot_w64(at >= 0 && at < sum);
        if (hit) {
            int2 r = make_int2(0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (at >= 0 && at < n[i]) r = make_int2(u + i, n[i] - 1 - at);
                at -= n[i];
            }
            const int l = __builtin_ctzll(hit);
            return make_int2(__builtin_amdgcn_readlane(r.x, l), __builtin_amdgcn_readlane(r.y, l));
        }
        idx -= __builtin_amdgcn_readlane(incl, 63);
    }
    return make_int2(-1, 0);
}

// The grid of a launch; fills n_qt and bounds max_rows (no unit has more rows
// than there are).
struct SplitGrid {
    bool compact;
    long blocks;
    SplitGrid(AttnArgs& b, int waves) {
        b.max_rows = (int)std::min((long)b.max_rows, b.lse_rows);
        b.n_qt = (int)(((long)b.max_rows * b.ratio + kCols - 1) / kCols);
        // compact: no more column blocks than the full ones and one begun by every request
        compact = compact_grid(b, waves);
        const long full = (long)b.n_qt * b.n_units;
        blocks = (compact ? std::min(full, (b.lse_rows * b.ratio + (kCols - 1L) * b.n_units) / kCols) : full) *
                 b.n_kv_heads;
    }
};

}  // namespace

}  // namespace rc
