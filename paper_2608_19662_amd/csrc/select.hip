// The rows of every segment that stay: its best scores, ties to the lower
// index, its first and last rows among them whatever they score, in ascending
// order.  A row's score is the sum of its weights over the planes, in 64 bits,
// rounded to 32.
//
// Scores are compared as 32-bit keys of the same order.  The k-th largest key
// of a segment is found by three histograms of 11, 11 and 10 bits, from the
// top; then every wave counts what it keeps of its part of the segment
// (consecutive rows), and after one exchange of those counts writes it in
// place.  One block per segment, the keys in its registers; segments too long
// for that have their keys formed by a grid of their own, and a block that
// reads them from memory.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace rc {

namespace {

constexpr int kItems = 16;   // keys per thread in registers
constexpr int kBins = 2048;
constexpr uint32_t kForced = 0xffffffffu;  // above every score
constexpr int kShortLen = 256 * kItems, kMidLen = 1024 * kItems;

// Keys in the order of the scores; NaN below every number, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float score) {
    if (score != score) return 0;
    const uint32_t b = __float_as_uint(score + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint32_t row_key(const SelectArgs& a, long row) {
    double sum = 0.0;
    const float* w = a.w + row;
    for (int p = 0; p < a.n_planes; ++p) sum += (double)w[(size_t)p * a.total];
    return key_of((float)sum);
}

// A segment: its rows, how many stay, which of them do in any case.
struct Segment {
    long beg;
    int len, k, first, last;
    __device__ __forceinline__ Segment(const SelectArgs& a, int s) {
        beg = a.cu[s];
        len = (int)max(0L, min((long)a.cu[s + 1], a.total) - beg);
        if (beg < 0) len = 0;
        k = max(0, min(a.cu_kept[s + 1] - a.cu_kept[s], len));
        last = min(a.keep_last, k);
        first = min(a.keep_first, k - last);
    }
    __device__ __forceinline__ bool forced(int j) const { return j < first || j >= len - last; }
};

// LONG: keys are in memory (a.keys), and kept rows go behind them for the
// gather of their weights.
template <int NW, bool LONG>
__global__ __launch_bounds__(NW * 64) void select_kernel(const SelectArgs a) {
    __shared__ int hist[kBins];
    __shared__ int scan[NW];
    __shared__ int found[2];  // the bin of the k-th key, keys above it
    __shared__ int counts[NW][2];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int s = blockIdx.x;
    const Segment seg(a, s);
    if (seg.k == 0) return;
    if (seg.len > a.max_len) {
        // a caller's size error shows: the keys in registers would not hold it
        for (long p = max(0L, (long)a.cu_kept[s]) + tid; p < min((long)a.cu_kept[s + 1], a.total_kept); p += NW * 64) {
            a.kept_idx[p] = -1;
            if (LONG && a.kept_w) a.keys[a.total + p] = kForced;
            for (int q = 0; a.kept_w && q < a.n_planes; ++q)
                a.kept_w[(size_t)q * a.total_kept + p] = __builtin_nanf("");
        }
        return;
    }
    const int ni = (seg.len + NW * 64 - 1) / (NW * 64);  // 64-row steps per wave
    const int base = wave * ni * 64 + lane;
    uint32_t keys[LONG ? 1 : kItems];
    if constexpr (!LONG) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int j = base + i * 64;
            keys[i] = 0;
            if (i < ni && j < seg.len) keys[i] = seg.forced(j) ? kForced : row_key(a, seg.beg + j);
        }
    }
    // f(step, row, key) for this lane's rows; steps past the segment's end are
    // passed too (row >= len), so that all lanes take part in each
    auto each = [&](auto&& f) {
        if constexpr (LONG) {
            for (int i = 0; i < ni; ++i) {
                const int j = base + i * 64;
                f(j, j < seg.len ? a.keys[seg.beg + j] : 0u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (i < ni) f(base + i * 64, keys[i]);
        }
    };

    // ---- the k-th largest key: its digits from the top
    uint32_t prefix = 0, fixed = 0;  // digits found, and their bits
    int need = seg.k;                // its place among the keys that share them
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
        for (int i = tid; i < bins; i += NW * 64) hist[i] = 0;
        __syncthreads();
        each([&](int j, uint32_t key) {
            if (j < seg.len && (key & fixed) == prefix) atomicAdd(&hist[(key >> shift) & (bins - 1)], 1);
        });
        __syncthreads();
        // thread t sums bins [t * per, t * per + per) counted from the top
        const int per = (bins + NW * 64 - 1) / (NW * 64);
        int sum = 0;
        for (int i = 0; i < per; ++i) {
            const int bin = bins - 1 - (tid * per + i);
            if (bin >= 0) sum += hist[bin];
        }
        int total;
        const int before = block_exclusive_scan<NW>(sum, scan, &total);
        if (need > before && need <= before + sum) {
            int above = before;
            for (int i = 0; i < per; ++i) {
                const int bin = bins - 1 - (tid * per + i);
                if (above + hist[bin] >= need) {
                    found[0] = bin;
                    found[1] = above;
                    break;
                }
                above += hist[bin];
            }
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        fixed |= (uint32_t)(bins - 1) << shift;
        need -= found[1];
        // (found and scan are written again only behind the next pass's barriers)
    }
    // `need` of the keys equal to prefix stay, the lowest rows first

    int n_above = 0, n_equal = 0;
    each([&](int j, uint32_t key) {
        const bool in = j < seg.len;
        n_above += __popcll(__builtin_amdgcn_ballot_w64(in && key > prefix));
        n_equal += __popcll(__builtin_amdgcn_ballot_w64(in && key == prefix));
    });
    if (lane == 0) {
        counts[wave][0] = n_above;
        counts[wave][1] = n_equal;
    }
    __syncthreads();
    int above = 0, equal = 0;
    for (int w = 0; w < wave; ++w) {
        above += counts[w][0];
        equal += counts[w][1];
    }
    const uint64_t below = (1ull << lane) - 1;
    const long out0 = a.cu_kept[s];
    each([&](int j, uint32_t key) {
        const bool in = j < seg.len;
        const uint64_t ma = __builtin_amdgcn_ballot_w64(in && key > prefix);
        const uint64_t me = __builtin_amdgcn_ballot_w64(in && key == prefix);
        const int eq = equal + __popcll(me & below);  // equal keys before this row
        if (in && (key > prefix || (key == prefix && eq < need))) {
            const long p = out0 + above + __popcll(ma & below) + min(eq, need);
            if (p >= 0 && p < a.total_kept) {
                a.kept_idx[p] = j;
                if constexpr (LONG) {
                    if (a.kept_w) a.keys[a.total + p] = (uint32_t)(seg.beg + j);
                } else if (a.kept_w) {
                    for (int q = 0; q < a.n_planes; ++q)
                        a.kept_w[(size_t)q * a.total_kept + p] = a.w[(size_t)q * a.total + seg.beg + j];
                }
            }
        }
        above += __popcll(ma);
        equal += __popcll(me);
    });
}

// Keys of long segments: 64 rows per wave.
__global__ __launch_bounds__(256) void score_kernel(const SelectArgs a) {
    const int lane = threadIdx.x & 63;
    const long at = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int s = find_segment(a.cu, a.n_seg, 64, 1, at, lane);
    const Segment seg(a, s);
    const long j = (at - first_item(a.cu[s], s, 64, 1)) * 64 + lane;
    if (j < 0 || j >= seg.len) return;
    a.keys[seg.beg + j] = seg.forced((int)j) ? kForced : row_key(a, seg.beg + j);
}

__global__ __launch_bounds__(256) void kept_weights_kernel(const SelectArgs a) {
    const long p = (long)blockIdx.x * 256 + threadIdx.x;
    if (p >= a.total_kept) return;
    const uint32_t at = a.keys[a.total + p];
    if (at >= a.total) return;  // (of a segment longer than max_len)
    const long row = at;
    for (int q = 0; q < a.n_planes; ++q) a.kept_w[(size_t)q * a.total_kept + p] = a.w[(size_t)q * a.total + row];
}

}  // namespace

size_t select_workspace_bytes(long total, int max_len) { return max_len > kMidLen ? (size_t)total * 8 : 0; }

hipError_t launch_select(const SelectArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)a.n_seg);
    if (a.max_len <= kShortLen) {
        hipLaunchKernelGGL((select_kernel<4, false>), grid, dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    if (a.max_len <= kMidLen) {
        hipLaunchKernelGGL((select_kernel<16, false>), grid, dim3(1024), 0, stream, a);
        return hipGetLastError();
    }
    const long waves = a.total / 64 + a.n_seg;
    hipLaunchKernelGGL(score_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, a);
    hipLaunchKernelGGL((select_kernel<16, true>), grid, dim3(1024), 0, stream, a);
    if (a.kept_w)
        hipLaunchKernelGGL(kept_weights_kernel, dim3((unsigned)((a.total_kept + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace rc
