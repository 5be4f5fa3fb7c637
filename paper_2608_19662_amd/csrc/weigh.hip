// The attention weight that every cached row receives, and the inverse of the
// request lists that it is summed over.
//
//     w[g][key] = w0[g][key] + sum over the queries (request, head of g, row) that see the key of
//                 exp(scale * q . k - lse)
// with the visibility of the attention call that left lse.  No softmax is
// taken: each probability is formed again from the row's log-sum-exp.
//
// Work is split by keys, so that no two blocks add to one sum and its order is
// fixed: a block owns 64 rows of one segment and plane (32 in fp32), holds them
// as the A operand of its MFMAs for its whole life, and walks the queries that
// see them in order of the requests, 32 (row, head) columns at a time:
//     S = K Q^T (32x32 MFMA)      column c of every lane is one query, so that
//     w += exp2(S - lse)          the log-sum-exp is one register and the sum over
//                                 queries stays in the lanes until the end
// Its waves take the column tiles in turn.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace rc {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// MFMA operands of one 32-row tile: HD / 2 elements of a row per lane (row
// lane % 32; bf16: chunks of 8, chunk 2t + half in step t; fp32: the half row
// of `half`, an element per step; K and Q alike).
template <typename T, int HD>
struct Frag;
template <int HD>
struct Frag<uint16_t, HD> {
    static constexpr int kBlocks = 2;  // 32-key blocks per wave
    u32x4 w[HD / 16];
    __device__ __forceinline__ void load(const uint16_t* row, int half) {
#pragma unroll
        for (int t = 0; t < HD / 16; ++t) w[t] = *reinterpret_cast<const u32x4*>(row + t * 16 + half * 8);
    }
    static __device__ __forceinline__ f32x16 product(const Frag& a, const Frag& b) {
        f32x16 c = {};
#pragma unroll
        for (int t = 0; t < HD / 16; ++t)
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.w[t]),
                                                        __builtin_bit_cast(bf16x8, b.w[t]), c, 0, 0, 0);
        return c;
    }
};
template <int HD>
struct Frag<float, HD> {
    static constexpr int kBlocks = 1;
    f32x4 w[HD / 8];
    __device__ __forceinline__ void load(const float* row, int half) {
#pragma unroll
        for (int t = 0; t < HD / 8; ++t) w[t] = *reinterpret_cast<const f32x4*>(row + half * (HD / 2) + t * 4);
    }
    static __device__ __forceinline__ f32x16 product(const Frag& a, const Frag& b) {
        f32x16 c = {};
#pragma unroll
        for (int t = 0; t < HD / 8; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w[t][i], b.w[t][i], c, 0, 0, 0);
        return c;
    }
};

// Sums of N values over the 32 lanes of a half wave, halving the values with the
// lanes (step O: between lanes O apart): with N = 32 lane l ends with the total of
// value l, with 16 of value l / 2.
template <int N, int O = 16>
__device__ __forceinline__ float lane_totals(const float* v, int lane) {
    if constexpr (O == 0) {
        return v[0];
    } else if constexpr (N == 1) {
        const float sum = v[0] + __shfl_xor(v[0], O);
        return lane_totals<1, O / 2>(&sum, lane);
    } else {
        float half[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float keep = lane & O ? v[i + N / 2] : v[i], send = lane & O ? v[i] : v[i + N / 2];
            half[i] = keep + __shfl_xor(send, O);
        }
        return lane_totals<N / 2, O / 2>(half, lane);
    }
}

template <typename T, int HD, int NW>
__global__ __launch_bounds__(NW * 64, 2) void weigh_kernel(const WeighArgs a) {
    constexpr int NKB = Frag<T, HD>::kBlocks, KT = 32 * NKB;
    __shared__ float part[NW][KT];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int R = a.ratio, G = a.n_kv_heads;

    // ---- this block's keys: tile j of a resource's rows or of a context
    long bid = blockIdx.x;
    const long n_r = a.r_w ? (a.res_off ? a.r_items : a.r_items * G) : 0;
    const bool ctx = bid >= n_r;
    int g, u0, u1;   // plane, and the users of the segment: user_req[u0 .. u1), or request u0 itself
    long row0;       // first key row
    int n;           // keys
    int off = 0;     // context: query i sees keys up to off + i of the tile
    if (!ctx) {
        int r;
        long j, beg;
        if (a.res_off) {
            const int s = find_segment(a.res_off, a.n_res * G, KT, 1, bid, lane);
            r = s / G;
            g = s % G;
            beg = a.res_off[s];
            j = bid - first_item(beg, s, KT, 1);
        } else {
            g = (int)(bid % G);
            bid /= G;
            r = find_segment(a.cu_kept, a.n_res, KT, 1, bid, lane);
            beg = a.cu_kept[r];
            j = bid - first_item(beg, r, KT, 1);
        }
        long len = (long)a.cu_kept[r + 1] - a.cu_kept[r];
        const bool seen = a.mask[((size_t)r * a.n_layers + a.layer) * G + g] != 0;
        if (a.res_off && !seen) len = 0;  // (a route that the store does not hold)
        row0 = beg + j * KT;
        n = j < 0 ? 0 : (int)max(0L, min((long)KT, len - j * KT));
        u0 = seen ? max(a.user_off[r], 0) : 0;
        u1 = seen ? min(a.user_off[r + 1], a.n_users) : 0;
    } else {
        bid -= n_r;
        g = (int)(bid % G);
        bid /= G;
        const int b = find_segment(a.cu_ctx, a.n_req, KT, 1, bid, lane);
        const long beg = a.cu_ctx[b], len = a.cu_ctx[b + 1] - beg;
        const long j = bid - first_item(beg, b, KT, 1);
        row0 = beg + j * KT;
        n = j < 0 ? 0 : (int)max(0L, min((long)KT, len - j * KT));
        off = (int)(len - (a.cu_q[b + 1] - a.cu_q[b]) - j * KT);
        u0 = b;
        u1 = b + 1;
    }
    const long rows = ctx ? a.c_rows : a.r_rows;
    if (row0 < 0) n = 0;
    n = (int)min((long)n, max(rows - row0, 0L));  // in bounds whatever the offsets hold
    if (n <= 0) return;
    const size_t plane = (ctx || !a.res_off) ? (size_t)g * rows : 0;

    Frag<T, HD> kf[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
        kf[kb].load(static_cast<const T*>(ctx ? a.ck : a.rk) + (plane + row0 + min(kb * 32 + l32, n - 1)) * HD, half);

    float acc[NKB * 16] = {};
    // One tile of columns: this lane's query row and head, and from which key
    // offset on it sees none (KT or more: sees all); used: the column counts.
    auto columns = [&](long row, int head, bool used, int last, bool wrong) {
        row = max(0L, min(row, a.total_q - 1));
        Frag<T, HD> qf;
        qf.load(static_cast<const T*>(a.q) + ((size_t)row * a.n_q_heads + head) * HD, half);
        float lse2 = used ? a.lse[(size_t)head * a.total_q + row] * kLog2e : INFINITY;
        if (wrong) lse2 = __builtin_nanf("");  // (a caller's size error shows)
        const bool diag = __builtin_amdgcn_ballot_w64(last < KT - 1) != 0;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            f32x16 s = Frag<T, HD>::product(kf[kb], qf);
            if (diag) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (kb * 32 + (r >> 2) * 8 + half * 4 + (r & 3) > last) s[r] = -INFINITY;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[kb * 16 + r] += __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2, -lse2));
        }
    };
    if (a.one_query && !ctx) {
        // one query per request: columns run over the users
        const int n_cols = (u1 - u0) * R;
        for (int j0 = wave * 32; j0 < n_cols; j0 += NW * 32) {
            const int j = min(j0 + l32, n_cols - 1);
            const int b = max(0, min(a.user_req[u0 + j / R], a.n_req - 1));
            const int q0 = a.cu_q[b];
            columns(q0, g * R + j % R, j0 + l32 < n_cols, KT, a.cu_q[b + 1] - q0 != 1);
        }
    } else {
        int turn = 0;  // column tiles so far, modulo the waves
        for (int u = u0; u < u1; ++u) {
            const int b = ctx ? u : max(0, min(a.user_req[u], a.n_req - 1));
            const int q0 = a.cu_q[b], n_cols = (a.cu_q[b + 1] - q0) * R;
            // context: rows before -off see none of these keys
            const int first = ctx ? max(0, -off) * R / 32 * 32 : 0;
            for (int j0 = first; j0 < n_cols; j0 += 32) {
                if (turn == wave) {
                    const int j = min(j0 + l32, n_cols - 1);
                    columns((long)q0 + j / R, g * R + j % R, j0 + l32 < n_cols, ctx ? off + j / R : KT, false);
                }
                turn = turn + 1 == NW ? 0 : turn + 1;
            }
        }
    }

    // ---- the sums of the lanes, then of the waves
    const float total = lane_totals<NKB * 16>(acc, lane);
    const int v = NKB == 2 ? l32 : l32 >> 1;  // value of this lane: block v / 16, register v % 16
    const int key = (v >> 4) * 32 + ((v & 15) >> 2) * 8 + half * 4 + (v & 3);
    if (NKB == 2 || !(l32 & 1)) part[wave][key] = total;
    __syncthreads();
    if (tid < n) {
        float* w = ctx ? a.c_w : a.r_w;
        const float* prior = ctx ? a.c_prior : a.r_prior;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) sum += part[i][tid];
        w[plane + row0 + tid] = (prior ? prior[plane + row0 + tid] : 0.f) + sum;
    }
}

// One wave per resource: its users are the list entries that name it, in
// order, and its offset the number of entries that name a resource before it.
__global__ __launch_bounds__(256) void users_kernel(int n_req, const int32_t* req_res_off, const int32_t* req_res,
                                                    int total, int n_res, int32_t* user_off, int32_t* user_req) {
    const int lane = threadIdx.x & 63;
    const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (r > n_res) return;  // (wave n_res writes the last offset)
    int before = 0;
    for (int i = lane; i < total; i += 64) before += req_res[i] < r;
    for (int o = 32; o >= 1; o >>= 1) before += __shfl_xor(before, o);
    if (lane == 0) user_off[r] = before;
    if (r == n_res) return;
    int at = before;
    for (int i0 = 0; i0 < total; i0 += 64) {
        const int i = i0 + lane;
        const bool mine = i < total && req_res[i] == r;
        const uint64_t m = __builtin_amdgcn_ballot_w64(mine);
        if (mine) {
            // the request of entry i: the last whose list starts at i or before
            int lo = 0, hi = n_req - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (req_res_off[mid] <= i) lo = mid; else hi = mid - 1;
            }
            const int p = at + __popcll(m & ((1ull << lane) - 1));
            if (p < total) user_req[p] = lo;
        }
        at += __popcll(m);
    }
}

template <typename T, int HD>
hipError_t launch(const WeighArgs& b, hipStream_t stream) {
    WeighArgs a = b;
    constexpr int KT = 32 * Frag<T, HD>::kBlocks;
    a.r_items = a.res_off ? a.r_rows / KT + (long)a.n_res * a.n_kv_heads : a.r_rows / KT + a.n_res;
    a.c_items = a.c_rows / KT + a.n_req;
    const long blocks = (a.r_w ? (a.res_off ? a.r_items : a.r_items * a.n_kv_heads) : 0) +
                        (a.c_w ? a.c_items * a.n_kv_heads : 0);
    if (blocks <= 0) return hipSuccess;
    if (blocks > 0x7fffffffL) return hipErrorInvalidValue;
    if (a.one_query)
        hipLaunchKernelGGL((weigh_kernel<T, HD, 1>), dim3((unsigned)blocks), dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL((weigh_kernel<T, HD, 4>), dim3((unsigned)blocks), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_weigh(const WeighArgs& a, int elem_bytes, int head_dim, hipStream_t stream) {
    if (elem_bytes == 4) return head_dim == 128 ? launch<float, 128>(a, stream) : launch<float, 64>(a, stream);
    return head_dim == 128 ? launch<uint16_t, 128>(a, stream) : launch<uint16_t, 64>(a, stream);
}

hipError_t launch_resource_users(int n_req, const int32_t* req_res_off, const int32_t* req_res, int total,
                                 int n_res, int32_t* user_off, int32_t* user_req, hipStream_t stream) {
    hipLaunchKernelGGL(users_kernel, dim3((unsigned)((n_res + 4L) / 4)), dim3(256), 0, stream, n_req, req_res_off,
                       req_res, total, n_res, user_off, user_req);
    return hipGetLastError();
}

}  // namespace rc
