// The rows of every segment that stay: its best scores, ties to the lower
// index, its first and last rows among them whatever they score, in ascending
// order.  A row's score is the sum of its weights over the planes, in 64 bits,
// rounded to 32.
//
// Scores are compared as 32-bit keys of the same order.  One block takes a
// segment: it finds the k-th largest key, then every wave counts what it keeps
// of its part of the segment (consecutive rows), and after one exchange of those
// counts writes it in place.
//
// Segments of up to 16 keys per thread hold them in registers.  The k-th largest
// is closed in on from the largest key by counting the keys at or above a candidate
// (ballots, no atomics): one compare per key and step, and the search ends as soon as
// k keys are, which takes about as many steps as the segment's length has bits.
// Longer segments have their keys formed by a grid of their own.  A block per
// segment then takes a histogram of the top 11 bits, searches the keys of the one
// bin that holds the k-th in LDS as above, and counts what stays of every 512 rows; a
// grid over those writes the rows.
//
// 2,048 segments of 200 to 2,000 rows, 8 planes, 30% kept: 33 us for 96 MB; 21 of
// them are left with one plane, the steps of the search with their reductions over
// lanes and waves, and all blocks are in the same phase at once.  Six segments of 12,000 to
// 100,000 rows: 40 us, 29 of them the blocks that search, each on one CU.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace rc {

namespace {

constexpr uint32_t kForced = 0xffffffffu;  // above every score
constexpr int kAll = 0x7fffffff;
constexpr int kMidLen = 16384;  // the longest segment in registers

// Keys in the order of the scores; NaN below every number, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float score) {
    if (score != score) return 0;
    const uint32_t b = __float_as_uint(score + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
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

// Keys of N rows (clamped to the segment), 16 loads in flight together.
template <int N, typename Row>
__device__ __forceinline__ void row_keys(const SelectArgs& a, const Segment& seg, uint32_t* keys, Row&& row) {
    constexpr int P = N >= 16 ? 1 : 16 / N;  // planes per step
    double sum[N] = {};
    const float* w = a.w + seg.beg;
    int at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = min(row(i), seg.len - 1);
    for (int p = 0; p < a.n_planes; p += P) {
        float x[P][N];
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const float* wp = w + (size_t)min(p + q, a.n_planes - 1) * a.total;
#pragma unroll
            for (int i = 0; i < N; ++i) x[q][i] = wp[at[i]];
        }
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (p + q < a.n_planes) sum[i] += (double)x[q][i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) keys[i] = seg.forced(row(i)) ? kForced : key_of((float)sum[i]);
}

// Sum over the lanes up to each.
__device__ __forceinline__ int wave_prefix(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);  // row_bcast:15, into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);  // row_bcast:31, into rows 2 and 3
    return x;
}

// Sum over the 64 lanes, in every lane.
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_prefix(x), 63); }

// The largest t in [lo, hi) with `need` keys or more at or above it, of the keys
// that each(f) passes to f(key) (keys that do not count are 0).  There have to be as
// many at or above lo (or lo = 0), and fewer at or above hi.  *equal: how many of the
// keys equal to t stay.  A step tries three candidates, a quarter of [lo, hi) apart; at
// first closer to hi, since scores lie closer to their largest than to zero.  Counts
// stay in the lanes (a compare and an add with carry per key and candidate) and
// are summed once a step, over the waves by LDS additions (every wave reading every
// other's was 0.4 us a step with 16 waves).  sums: 3 turns of 4 ints in LDS, zero since
// before the block's last barrier (one wave needs none).  SMALL: the block's counts
// fit 16 bits.
template <int NW, bool SMALL, typename Each>
__device__ __forceinline__ uint32_t kth_key(int need, uint32_t lo, uint32_t hi, Each&& each, int* sums, int* equal) {
    const int lane = threadIdx.x & 63;
    int turn = 0;
    auto over_block = [&](int& n1, int& n2, int& n3) {
        if (SMALL) n1 |= n2 << 16;
        n1 = wave_total(n1), n3 = wave_total(n3);
        if (!SMALL) n2 = wave_total(n2);
        if constexpr (NW > 1) {
            int* sum = sums + turn * 4;
            turn = turn == 2 ? 0 : turn + 1;
            if (lane == 0) {
                atomicAdd(sum, n1);
                atomicAdd(sum + 1, n3);
                if (!SMALL) atomicAdd(sum + 2, n2);
            }
            // the next turn's, which was read two barriers ago
            if (threadIdx.x < 4) sums[turn * 4 + threadIdx.x] = 0;
            __syncthreads();
            n1 = __builtin_amdgcn_readfirstlane(sum[0]);
            n3 = __builtin_amdgcn_readfirstlane(sum[1]);
            if (!SMALL) n2 = __builtin_amdgcn_readfirstlane(sum[2]);
        }
        if (SMALL) {
            n2 = (int)((uint32_t)n1 >> 16);
            n1 &= 0xffff;
        }
    };
    int near = 22;     // log2 of the candidates' distance from hi
    bool low = false;  // a candidate was low enough
    while (hi - lo > 1) {
        const uint32_t r = hi - lo;
        const bool by_hi = !low && near <= 28 && r >> (near + 3) != 0;
        // ascending, in [lo, hi), c2 above lo
        uint32_t c1, c2, c3;
        if (by_hi)
            c1 = hi - (4u << near), c2 = hi - (2u << near), c3 = hi - (1u << near);
        else
            c1 = lo + (r >> 2), c2 = lo + (r >> 1), c3 = hi - max(r >> 2, 1u);
        int n1 = 0, n2 = 0, n3 = 0;
        each([&](uint32_t key) {
            n1 += key >= c1;
            n2 += key >= c2;
            n3 += key >= c3;
        });
        over_block(n1, n2, n3);
        if (n3 == need || n2 == need || n1 == need) {  // exactly those stay
            *equal = kAll;
            return n3 == need ? c3 : n2 == need ? c2 : c1;
        }
        // (each way the interval gets shorter)
        low = low || n1 > need;
        if (n3 > need) lo = c3;
        else if (n2 > need) lo = c2, hi = c3;
        else if (n1 > need) lo = c1, hi = c2;
        else hi = c1 > lo ? c1 : c2;
        near += 3;
    }
    // more keys than needed are at or above t: some of those equal to it go
    int n = 0, z2 = 0, z3 = 0;
    each([&](uint32_t key) { n += key > lo; });
    over_block(n, z2, z3);
    *equal = need - n;
    return lo;
}

// Marks a segment that is longer than max_len: a caller's size error shows.
template <int NT>
__device__ __forceinline__ void mark_too_long(const SelectArgs& a, int s) {
    for (long p = max(0L, (long)a.cu_kept[s]) + threadIdx.x; p < min((long)a.cu_kept[s + 1], a.total_kept); p += NT) {
        a.kept_idx[p] = -1;
        for (int q = 0; a.kept_w && q < a.n_planes; ++q) a.kept_w[(size_t)q * a.total_kept + p] = __builtin_nanf("");
    }
}

// Writes n kept rows (local indices in LDS) of the segment at `beg` to out0 on, and
// their weights, eight planes' loads in flight together; by n_threads threads.
template <typename Index>
__device__ __forceinline__ void write_rows(const SelectArgs& a, long beg, const Index* list, int n, long out0, int tid,
                                           int n_threads) {
#pragma unroll 2
    for (int i = tid; i < n; i += n_threads) {
        const long p = out0 + i;
        if (p < 0 || p >= a.total_kept) continue;
        const int j = list[i];
        a.kept_idx[p] = j;
        if (!a.kept_w) continue;
        const float* w = a.w + beg + j;
        float* out = a.kept_w + p;
        for (int q = 0; q < a.n_planes; q += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = w[(size_t)min(q + e, a.n_planes - 1) * a.total];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (q + e < a.n_planes) out[(size_t)(q + e) * a.total_kept] = x[e];
        }
    }
}

// Segments in registers: wave w has rows [w * ni * 64, (w + 1) * ni * 64), 64 per
// step, N steps at most.
template <int NW, int N>
__device__ __forceinline__ void select_rows(const SelectArgs& a, const Segment& seg, int ni, int* sums, int2* counts,
                                           uint16_t* list) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int base = wave * ni * 64 + lane;
    constexpr int B = N < 8 ? N : 8;  // steps whose rows are loaded together
    uint32_t keys[N];
#pragma unroll
    for (int i = 0; i < N; i += B)
        if (i < ni) row_keys<B>(a, seg, keys + i, [&](int e) { return base + (i + e) * 64; });
    uint32_t most = 0;  // the largest score
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i >= ni || base + i * 64 >= seg.len) keys[i] = 0;
        if (keys[i] != kForced) most = max(most, keys[i]);
    }
    for (int o = 32; o >= 1; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
    if constexpr (NW > 1) {
        if (lane == 0) counts[wave].x = (int)most;
        if (threadIdx.x < 12) sums[threadIdx.x] = 0;
        __syncthreads();
        most = (uint32_t)counts[lane % NW].x;
        for (int o = NW / 2; o >= 1; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
    }
    most = (uint32_t)__builtin_amdgcn_readfirstlane((int)most);
    uint32_t t = kForced;
    int need = kAll;
    if (seg.first + seg.last < seg.k)
        t = kth_key<NW, true>(
            seg.k, 0, most + 1,
            [&](auto&& f) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i < ni) f(keys[i]);
            },
            sums, &need);
    // `need` of the keys equal to t stay, the lowest rows first.  Keys of no row
    // are 0, as those of a NaN score are, and come after every row: they are
    // left out where they would count, in the list.
    int above = 0, equal = 0;
    if constexpr (NW > 1) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < ni) {
                above += __popcll(__builtin_amdgcn_ballot_w64(keys[i] > t));
                equal += __popcll(__builtin_amdgcn_ballot_w64(keys[i] == t));
            }
        __syncthreads();  // (the largest scores are read, also where no search was)
        if (lane == 0) counts[wave] = make_int2(above, equal);
        __syncthreads();
        above = equal = 0;
        for (int w = 0; w < wave; ++w) {
            above += counts[w].x;
            equal += counts[w].y;
        }
    }
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < ni) {
            const uint64_t ma = __builtin_amdgcn_ballot_w64(keys[i] > t);
            const uint64_t me = __builtin_amdgcn_ballot_w64(keys[i] == t);
            const int eq = equal + __popcll(me & below);  // equal keys before this row
            const int p = above + __popcll(ma & below) + min(eq, need);
            if ((keys[i] > t || (keys[i] == t && eq < need)) && p < seg.k) list[p] = (uint16_t)(base + i * 64);
            above += __popcll(ma);
            equal += __popcll(me);
        }
    if constexpr (NW > 1) __syncthreads();
}

constexpr int steps_of(int nw) { return nw == 1 ? 8 : 16; }

// One block of NW waves per segment; 8 or 16 steps of 64 rows per wave.
template <int NW>
__global__ __launch_bounds__(NW * 64, 8) void select_kernel(const SelectArgs a) {
    constexpr int N = steps_of(NW);
    __shared__ int sums[12];
    __shared__ int2 counts[NW];
    __shared__ uint16_t list[NW * 64 * N];  // the kept rows
    const int s = blockIdx.x;
    const Segment seg(a, s);
    if (seg.k == 0) return;
    if (seg.len > min(a.max_len, NW * 64 * N)) return mark_too_long<NW * 64>(a, s);
    const int ni = (seg.len + NW * 64 - 1) / (NW * 64);
    if (ni <= N / 4)
        select_rows<NW, N / 4>(a, seg, ni, sums, counts, list);
    else if (ni <= N / 2)
        select_rows<NW, N / 2>(a, seg, ni, sums, counts, list);
    else
        select_rows<NW, N>(a, seg, ni, sums, counts, list);
    write_rows(a, seg.beg, list, seg.k, a.cu_kept[s], threadIdx.x, NW * 64);
}

// ---- long segments

constexpr int kLongWaves = 16, kBins = 2048, kTopShift = 21;
constexpr int kCopies = 8;  // of the histogram, by lane: most scores share a few
                            // bins, and additions to one address take turns
constexpr int kCandidates = 16384;  // keys of one bin that LDS takes
constexpr int kGroup = 2048;        // rows of a wave's step
constexpr int kChunk = 512;         // rows that one wave writes

// Four consecutive keys from any 4-byte boundary.
struct __attribute__((packed, aligned(4))) Keys4 {
    uint32_t k[4];
};

// The workspace: keys [total], per chunk the rows that stay above the k-th key and
// at it, of the chunks before it, per segment that key and how many equal ones stay.
struct LongSpace {
    uint32_t* keys;
    int2* before;
    int2* kth;
    __device__ __forceinline__ LongSpace(const SelectArgs& a) {
        keys = a.keys;
        before = reinterpret_cast<int2*>(keys + (a.total + 1) / 2 * 2);
        kth = before + first_item(a.total, a.n_seg, kChunk, 1);
    }
};

// A wave's keys of rows [r0, r0 + ROWS) of a segment, all loads in flight together:
// f(row, rows left, keys, u) for four consecutive rows at a time, lane l's at
// r0 + 256 u + 4 l.
template <int ROWS, typename F>
__device__ __forceinline__ void chunk_keys(const uint32_t* keys, int r0, int len, int lane, F&& f) {
    constexpr int U = ROWS / 256;
    Keys4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = r0 + u * 256 + lane * 4;
        if (r0 + (u + 1) * 256 <= len) {
            x[u] = *reinterpret_cast<const Keys4*>(keys + j);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[u].k[e] = j + e < len ? keys[j + e] : 0u;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = r0 + u * 256 + lane * 4;
        f(j, len - j, x[u].k, u);
    }
}

__global__ __launch_bounds__(kLongWaves * 64) void kth_long_kernel(const SelectArgs a) {
    constexpr int NW = kLongWaves, NT = NW * 64;
    __shared__ __attribute__((aligned(16))) int hist[kBins * kCopies];
    __shared__ uint32_t cand[kCandidates];
    __shared__ int scan[2 * NW], found[3], n_cand, sums[12];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int s = blockIdx.x;
    const Segment seg(a, s);
    if (seg.k == 0 || seg.len > a.max_len) return;
    const LongSpace ws(a);
    const uint32_t* keys = ws.keys + seg.beg;
    auto each = [&](auto&& f) {
        for (int r0 = wave * kGroup; r0 < seg.len; r0 += NW * kGroup) chunk_keys<kGroup>(keys, r0, seg.len, lane, f);
    };

    // ---- the bin of the k-th largest key
    for (int i = tid; i < kBins * kCopies; i += NT) hist[i] = 0;
    if (tid == 0) n_cand = 0;
    if (tid < 12) sums[tid] = 0;
    __syncthreads();
    each([&](int, int left, const uint32_t* k, int) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) atomicAdd(&hist[(k[e] >> kTopShift) * kCopies + lane % kCopies], 1);
    });
    __syncthreads();
    {
        constexpr int P = kBins / NT;  // bins per thread, from the top
        int n[P], sum = 0;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int* h = hist + (kBins - 1 - (tid * P + i)) * kCopies;
            n[i] = 0;
#pragma unroll
            for (int c = 0; c < kCopies; ++c) n[i] += h[c];
            sum += n[i];
        }
        int total, before = block_exclusive_scan<NW>(sum, scan, &total);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (seg.k > before && seg.k <= before + n[i]) {
                found[0] = kBins - 1 - (tid * P + i);
                found[1] = before;
                found[2] = n[i];
            }
            before += n[i];
        }
    }
    __syncthreads();
    const uint32_t bin = (uint32_t)found[0];
    const int in_bin = found[2], need_bin = seg.k - found[1];

    // ---- the key itself
    const uint32_t lo = bin << kTopShift, hi = bin == kBins - 1 ? kForced : lo + (1u << kTopShift);
    uint32_t t = lo;
    int need = kAll;  // (the whole bin stays)
    if (seg.first + seg.last == seg.k) {
        t = kForced;
    } else if (in_bin > need_bin && in_bin <= kCandidates) {
        // one LDS addition per wave and step: every lane's share lies together
        for (int r0 = wave * kGroup; r0 < seg.len; r0 += NW * kGroup) {
            uint32_t mine[kGroup / 64];
            int n = 0;
            chunk_keys<kGroup>(keys, r0, seg.len, lane, [&](int, int left, const uint32_t* k, int u) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    mine[u * 4 + e] = e < left ? k[e] : ~0u;  // (in the bin of forced rows, which is not searched)
                    n += mine[u * 4 + e] >> kTopShift == bin;
                }
            });
            int at = wave_prefix(n);
            const int all = __builtin_amdgcn_readlane(at, 63);
            int base = 0;
            if (lane == 0) base = atomicAdd(&n_cand, all);
            at += __builtin_amdgcn_readfirstlane(base) - n;
#pragma unroll
            for (int i = 0; i < kGroup / 64; ++i)
                if (mine[i] >> kTopShift == bin) cand[at++] = mine[i];
        }
        __syncthreads();
        t = kth_key<NW, true>(
            need_bin, lo, hi,
            [&](auto&& f) {
                for (int i = wave * 64; i < in_bin; i += NT) f(i + lane < in_bin ? cand[i + lane] : 0u);
            },
            sums, &need);
    } else if (in_bin > need_bin) {
        // more of them than LDS takes (equal scores, most often): from memory
        t = kth_key<NW, false>(
            seg.k, lo, hi,
            [&](auto&& f) {
                each([&](int, int left, const uint32_t* k, int) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) f(e < left ? k[e] : 0u);
                });
            },
            sums, &need);
    }
    if (tid == 0) ws.kth[s] = make_int2((int)t, need);

    // ---- what stays of every chunk, then of the chunks before it
    int2* before = ws.before + first_item(seg.beg, s, kChunk, 1);
    const int n_chunks = (seg.len + kChunk - 1) / kChunk;
    constexpr int C = kGroup / kChunk;
    for (int r0 = wave * kGroup; r0 < seg.len; r0 += NW * kGroup) {
        int n[C] = {};  // above the k-th, and at it from bit 16 on
        chunk_keys<kGroup>(keys, r0, seg.len, lane, [&](int, int left, const uint32_t* k, int u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) n[u * C / (kGroup / 256)] += e < left ? (k[e] > t) + ((k[e] == t) << 16) : 0;
        });
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int sum = wave_total(n[i]);
            if (lane == 0 && r0 + i * kChunk < seg.len) before[r0 / kChunk + i] = make_int2(sum & 0xffff, sum >> 16);
        }
    }
    __syncthreads();
    int above = 0, equal = 0;
    for (int c0 = 0; c0 < n_chunks; c0 += NT) {
        const int c = c0 + tid;
        const int2 n = c < n_chunks ? before[c] : make_int2(0, 0);
        int na, ne;
        const int pa = block_exclusive_scan<NW>(n.x, scan, &na);
        const int pe = block_exclusive_scan<NW>(n.y, scan + NW, &ne);
        if (c < n_chunks) before[c] = make_int2(above + pa, equal + pe);
        above += na;
        equal += ne;
        __syncthreads();  // (the totals are read)
    }
}

// One wave per chunk.
__global__ __launch_bounds__(256) void write_long_kernel(const SelectArgs a) {
    __shared__ int lists[4][kChunk];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long at = (long)blockIdx.x * 4 + wave;
    const int s = find_segment(a.cu, a.n_seg, kChunk, 1, at, lane);
    const Segment seg(a, s);
    const long c = at - first_item(a.cu[s], s, kChunk, 1);
    if (seg.k == 0 || c < 0 || c * kChunk >= seg.len) return;
    const long out0 = a.cu_kept[s];
    if (seg.len > a.max_len) {
        for (long p = max(0L, out0) + c * 64 + lane; p < min(out0 + seg.k, a.total_kept);
             p += (seg.len + kChunk - 1L) / kChunk * 64) {
            a.kept_idx[p] = -1;
            for (int q = 0; a.kept_w && q < a.n_planes; ++q) a.kept_w[(size_t)q * a.total_kept + p] = __builtin_nanf("");
        }
        return;
    }
    const LongSpace ws(a);
    const int2 before = ws.before[at], kth = ws.kth[s];
    const uint32_t t = (uint32_t)kth.x;
    const int need = kth.y;
    const uint64_t below = (1ull << lane) - 1;
    int* list = lists[wave];
    int above = 0, equal = before.y;
    const int eq0 = min(equal, need);
    chunk_keys<kChunk>(ws.keys + seg.beg, (int)c * kChunk, seg.len, lane, [&](int j, int left, const uint32_t* k, int) {
        int ab = above, eq = equal;  // before this lane's rows
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t ma = __builtin_amdgcn_ballot_w64(e < left && k[e] > t);
            const uint64_t me = __builtin_amdgcn_ballot_w64(e < left && k[e] == t);
            above += __popcll(ma);
            equal += __popcll(me);
            ab += __popcll(ma & below);
            eq += __popcll(me & below);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool more = e < left && k[e] > t, same = e < left && k[e] == t;
            if (more || (same && eq < need)) list[ab + min(eq, need) - eq0] = j + e;
            ab += more;
            eq += same;
        }
    });
    // (only this wave reads its list)
    write_rows(a, seg.beg, list, above + min(equal, need) - eq0, out0 + before.x + eq0, lane, 64);
}

// Keys of long segments: 64 rows per wave.
__global__ __launch_bounds__(256) void score_kernel(const SelectArgs a) {
    const int lane = threadIdx.x & 63;
    const long at = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int s = find_segment(a.cu, a.n_seg, 64, 1, at, lane);
    const Segment seg(a, s);
    const long j = (at - first_item(a.cu[s], s, 64, 1)) * 64 + lane;
    if (j < 0 || j >= seg.len) return;
    uint32_t key;
    row_keys<1>(a, seg, &key, [&](int) { return (int)j; });
    a.keys[seg.beg + j] = key;
}

}  // namespace

size_t select_workspace_bytes(int n_seg, long total, int max_len) {
    return max_len > kMidLen ? (size_t)((total + 1) / 2 + total / kChunk + 2L * n_seg) * 8 : 0;
}

constexpr int kManySegments = 512;

hipError_t launch_select(const SelectArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)a.n_seg);
    // One wave per segment where there are enough of them and they are short: most
    // of a step of the search is the same for any number of keys, and paid by every
    // wave (2,048 segments of 31 to 60 rows, 8 planes: 7.6 us instead of 13.2 with
    // four waves, of 151 to 300 11.2 instead of 16.2; of 550 to 1,100 27.6 against 24.8).
    if (a.max_len <= 64 * steps_of(1) && a.n_seg >= kManySegments) {
        hipLaunchKernelGGL(select_kernel<1>, grid, dim3(64), 0, stream, a);
        return hipGetLastError();
    }
    if (a.max_len <= 4096) {
        hipLaunchKernelGGL(select_kernel<4>, grid, dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    if (a.max_len <= kMidLen) {
        hipLaunchKernelGGL(select_kernel<16>, grid, dim3(1024), 0, stream, a);
        return hipGetLastError();
    }
    const long waves = a.total / 64 + a.n_seg, chunks = a.total / kChunk + a.n_seg;
    hipLaunchKernelGGL(score_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, a);
    hipLaunchKernelGGL(kth_long_kernel, grid, dim3(kLongWaves * 64), 0, stream, a);
    hipLaunchKernelGGL(write_long_kernel, dim3((unsigned)((chunks + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace rc
