// Split-KV decode over caches in 8 bits (quant8.hpp): what decode.hip computes,
// on e4m3 rows with a power of two per 64 tokens.
//
// Memory-bound like decode.hip, on half of its bytes.  The products run on the
// same bf16 MFMAs: a code times its block's scale is exact in bf16, so the
// conversion (one instruction for two codes, scale included) adds no rounding.
//     S^T = K Q^T      (A = 16 keys x 32 dims of K, from HBM into VGPRs)
//     O^T += V^T P^T   (A = V^T by 8-bit transpose reads from LDS)
// A tile is one scale block: up to 64 consecutive rows of one segment (a
// resource's kept rows, or the context).  Its rows are one run of memory and
// its two scales are uniform, so that a tile costs no per-key lookups: a
// buffer resource whose extent is the tile (rows past its end read as zeros and
// are masked; all of an offset is per lane, where it takes part in the check),
// constant offsets per lane, and the two scales as operands of the conversions.
// Segments end inside a tile now and then; what a partial tile loses is matrix
// and vector work, which this kernel has to spare, no bytes.
//
// 64 requests of 4,096 context rows over 32 resources each, 32 / 8 heads (887 MB):
// 160 us with the merge, 5.5 TB/s; 12 requests of 60 to 9,000 context rows 20 us;
// one request over 3,400 keys 8 us and 4 for the merge, each a chain of dependent
// round trips.
//
// K dims are taken in the order in which 16-byte loads bring them: lane group
// g holds dims 64 c + 16 g + [0, 16) in the two MFMA steps of chunk c, for K
// and Q alike.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"
#include "quant8.hpp"

namespace rc {

namespace {

constexpr int kThreads = 256;
constexpr int kTk = kBlk8;  // keys per wave tile
constexpr int kMaxSeg = 1024;
// Third dword of a gfx9 buffer resource for raw (unformatted) loads.
constexpr int kBufferFlags = 0x00020000;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef int v2i __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v2i lds_v2i;

template <int C>
struct Tag {
    static constexpr int value = C;
};

template <int HD>
struct DT8 {
    static constexpr int CPR = HD / 16;       // 16-byte chunks per row
    static constexpr int TILEB = kTk * HD;    // bytes of one V tile
    static constexpr int NC = HD / 64;        // 16-byte K loads per key block and lane
    static constexpr int NKB = kTk / 16;      // 16-key blocks per tile
    static constexpr int NDB = HD / 16;       // 16-dim blocks of O^T
    static constexpr int RPI = 64 / CPR;      // rows per 1 KB wave copy
    static constexpr int NJ = kTk / RPI;      // copies per V tile
    static constexpr int NLOAD = NKB * NC + NJ + 1;  // vector memory operations per tile
    // s_waitcnt immediate for vmcnt(NLOAD), other counters unconstrained
    static constexpr int WAIT_PREV = (NLOAD & 15) | ((NLOAD >> 4) << 14) | 0x0F70;
};

// Segments of a stream in tiles: segment i has tiles [end[i - 1], end[i]).  The
// merge's (max, sum) take the same memory after the loop.
union Dec8Smem {
    struct {
        int end[kMaxSeg];
        int row[kMaxSeg];  // first row
        int len[kMaxSeg];  // rows
        int id[kMaxSeg];   // number in its cache, of the scale slots
    } seg;
    float ml[4][16][2];  // per wave and head: max, sum
};

// Chunk swizzle of a V tile row: the 16 rows x 16 bytes that half a wave's
// transpose read touches fall on distinct banks.
template <int HD>
__device__ __forceinline__ int v_mask8(int row) {
    return HD == 128 ? (((row >> 1) & 3) | (((row >> 4) & 1) << 2)) : (((row >> 2) & 1) | (((row >> 4) & 1) << 1));
}

__device__ __forceinline__ float xor16_max(float x) { return fmaxf(x, __shfl_xor(x, 16)); }
__device__ __forceinline__ float xor16_sum(float x) { return x + __shfl_xor(x, 16); }

__device__ __forceinline__ uint64_t uniform64(uint64_t x) {
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// NT: context rows are loaded with the non-temporal hint, as in decode.hip.
template <int HD, bool NT>
__global__ __launch_bounds__(kThreads, 2) void decode8_kernel(const Decode8Args a) {
    using T = DT8<HD>;
    __shared__ Dec8Smem sm;
    // Per wave two V tile buffers, in two arrays, so that the compiler sees
    // that copies into one do not touch the other.  Before the loop the first
    // holds the scan of the segment lengths, after it the two hold the wave's
    // O, fp32 [16 heads][HD] each half.
    __shared__ __attribute__((aligned(16))) char v_all0[4][T::TILEB], v_all1[4][T::TILEB];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, grp = lane >> 4;  // MFMA column and row group of this lane

    int bid = blockIdx.x;
    const int split = bid % a.d.n_splits;
    bid /= a.d.n_splits;
    int g = bid % a.d.n_kv_heads;
    int b = bid / a.d.n_kv_heads;
    if (a.d.plan) {
        const int n_pairs = a.d.n_req * a.d.n_kv_heads;
        int p = a.d.plan[(size_t)a.d.layer * n_pairs + bid];
        p = min(max(p, 0), n_pairs - 1);  // in bounds whatever the plan holds
        b = p / a.d.n_kv_heads;
        g = p % a.d.n_kv_heads;
    }
    const int R = a.d.ratio;

    // ---- Q^T (B operand): head l16 of the group (zero beyond R), in K's order of dims
    const int qrow = max(0, min(a.d.cu_q[b], (int)a.d.lse_rows - 1));
    bf16x8_t qf[T::NC * 2];
#pragma unroll
    for (int i = 0; i < T::NC * 2; ++i) {
        u32x4 w = {0u, 0u, 0u, 0u};
        if (l16 < R)
            w = *reinterpret_cast<const u32x4*>(a.d.q + ((size_t)qrow * a.d.n_q_heads + g * R + l16) * HD +
                                                (i >> 1) * 64 + grp * 16 + (i & 1) * 8);
        qf[i] = __builtin_bit_cast(bf16x8_t, w);
    }

    const size_t e = ((size_t)b * a.d.n_layers + a.d.layer) * a.d.n_kv_heads + g;
    const int r0 = a.d.route_off[e];
    const int n_seg = a.d.route_off[e + 1] - r0;
    if (n_seg > kMaxSeg || a.d.cu_q[b + 1] - a.d.cu_q[b] != 1) {
        // as in decode.hip: a caller's size error shows as NaN outputs
        for (int idx = tid; idx < R * HD; idx += kThreads) {
            const size_t slot = ((size_t)b * a.d.n_q_heads + g * R + idx / HD) * a.d.n_splits + split;
            a.d.ws_o[slot * HD + idx % HD] = __builtin_nanf("");
            if (idx % HD == 0) {
                a.d.ws_ml[slot * 2 + 0] = INFINITY;
                a.d.ws_ml[slot * 2 + 1] = __builtin_nanf("");
            }
        }
        return;
    }
    // ---- the segments' tiles
    int n_segt = 0;
    {
        int* scan = reinterpret_cast<int*>(v_all0[0]);
        for (int s0 = 0, k = 0; s0 < n_seg; s0 += kThreads, k ^= 1) {
            const int s = s0 + tid;
            int tiles = 0;
            if (s < n_seg) {
                const int r = a.d.route_res[r0 + s];
                const int k0 = a.d.cu_kept[r];
                const int id = a.d.res_off ? r * a.d.n_kv_heads + g : r;
                const int len = max(a.d.cu_kept[r + 1] - k0, 0);
                sm.seg.row[s] = a.d.res_off ? a.d.res_off[id] : k0;
                sm.seg.len[s] = len;
                sm.seg.id[s] = id;
                tiles = (len + kTk - 1) / kTk;
            }
            int total;
            const int at = n_segt + block_exclusive_scan<4>(tiles, scan + k * 4, &total);
            if (s < n_seg) sm.seg.end[s] = at + tiles;
            n_segt += total;
        }
        __syncthreads();
        n_segt = __builtin_amdgcn_readfirstlane(n_segt);
    }
    const int c0 = __builtin_amdgcn_readfirstlane(a.d.cu_ctx[b]);
    const int tc = __builtin_amdgcn_readfirstlane(a.ctx_len ? a.ctx_len[b] : a.d.cu_ctx[b + 1] - c0);
    const int n_tiles = n_segt + (max(tc, 0) + kTk - 1) / kTk;
    // this split's tiles [t0, t1)
    const int chunk = (n_tiles + a.d.n_splits - 1) / a.d.n_splits;
    const int t0 = min(split * chunk, n_tiles), t1 = min(t0 + chunk, n_tiles);

    // ---- loads of one tile
    char* const v_st0 = v_all0[wave];
    char* const v_st1 = v_all1[wave];
    const int k_lane = l16 * HD + grp * 16;
    int v_lane[2];  // byte offset of this lane in V copy j, from the copy's first row, for (j * RPI / 16) & 1
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = lane / T::CPR + h * 16;  // (copies of a lane differ in row bit 4 only, as far as the mask goes)
        v_lane[h] = lane / T::CPR * HD + (((lane % T::CPR) ^ v_mask8<HD>(row)) << 4);
    }
    u32x4 kreg[2][T::NKB][T::NC];
    int exps[2];  // lanes 0 .. 31: the tile's K exponent, others: V's
    int n_in[2];  // its keys
    int u_i = 0, u_lo = 0;  // wave-uniform walk over the segments: the current one, its first tile
    auto load_tile = [&](auto buf_tag, auto aux_tag, int i) {
        constexpr int buf = decltype(buf_tag)::value, AUX = decltype(aux_tag)::value;
        const int t = t0 + wave + 4 * i;
        const bool seg = t < n_segt;
        long row, slot, rows;
        int n;
        if (seg) {
            int hi = __builtin_amdgcn_readfirstlane(sm.seg.end[u_i]);
            while (t >= hi && u_i + 1 < n_seg) {
                ++u_i;
                u_lo = hi;
                hi = __builtin_amdgcn_readfirstlane(sm.seg.end[u_i]);
            }
            const int j = t - u_lo, beg = __builtin_amdgcn_readfirstlane(sm.seg.row[u_i]);
            row = (long)beg + (long)j * kTk;
            slot = block_slot(beg, __builtin_amdgcn_readfirstlane(sm.seg.id[u_i])) + j;
            n = __builtin_amdgcn_readfirstlane(sm.seg.len[u_i]) - j * kTk;
            rows = a.d.r_rows;
            slot = max(0L, min(slot, a.r_slots - 1));
        } else {
            const int j = t - n_segt;
            row = (long)c0 + (long)j * kTk;
            slot = block_slot(c0, b) + j;
            n = tc - j * kTk;
            rows = a.d.c_rows;
            slot = max(0L, min(slot, a.c_slots - 1));
        }
        // in bounds whatever the tables hold: the tile's extent ends at the plane's
        row = max(0L, min(row, rows - 1));
        n = (int)max(0L, min((long)min(n, kTk), rows - row));
        n_in[buf] = n;
        const size_t base = ((size_t)g * (seg ? a.d.r_gstride : a.d.c_rows) + row) * HD;
        const uint64_t kp = uniform64((uint64_t)((seg ? a.rk : a.ck) + base));
        const uint64_t vp = uniform64((uint64_t)((seg ? a.rv : a.cv) + base));
        const int bytes = __builtin_amdgcn_readfirstlane(n * HD);
        const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc((void*)kp, (short)0, bytes, kBufferFlags);
        const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc((void*)vp, (short)0, bytes, kBufferFlags);
        const size_t at = (size_t)g * (seg ? a.r_sstride : a.c_slots) + slot;
        exps[buf] = lane < 32 ? (seg ? a.rk_exp : a.ck_exp)[at] : (seg ? a.rv_exp : a.cv_exp)[at];
#pragma unroll
        for (int kb = 0; kb < T::NKB; ++kb)
#pragma unroll
            for (int c = 0; c < T::NC; ++c)
                kreg[buf][kb][c] = __builtin_amdgcn_raw_buffer_load_b128(kr, k_lane + kb * 16 * HD + c * 64, 0, AUX);
        char* dst = buf ? v_st1 : v_st0;
#pragma unroll
        for (int j = 0; j < T::NJ; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void*)(dst + j * 1024), 16,
                                                     (int)(v_lane[(j * T::RPI >> 4) & 1] + j * 1024), 0, 0, AUX);
    };

    // ---- transpose reads: in a 16-lane group, lanes 2k and 2k + 1 point at the
    // two halves of row k's chunk, and lane i receives column i of the 8 rows.
    // Rows: the keys whose weights this lane group holds in the S^T
    // accumulators of two 16-key blocks, grp*4 + [0, 4) and 16 + grp*4 + [0, 4).
    uint32_t v_rd0;
    {
        const int k = l16 >> 1, row = (k >> 2) * 16 + grp * 4 + (k & 3);
        v_rd0 = (uint32_t)(row * HD + (v_mask8<HD>(row) << 4) + (l16 & 1) * 8);
    }

    const float sl2 = a.d.scale_log2;
    const bf16x2 ones2 = __builtin_bit_cast(bf16x2, 0x3F803F80u);  // (1.0, 1.0) in bf16
    float m = -INFINITY;  // running max (log2 units) for head l16
    float lsum = 0.f;     // this lane's part of the row sum
    f32x4 oacc[T::NDB];   // O^T: dims db*16 + grp*4 + [0, 4) of head l16
#pragma unroll
    for (int db = 0; db < T::NDB; ++db) oacc[db] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto compute = [&](auto buf_tag) {
        constexpr int buf = decltype(buf_tag)::value;
        const float ksc = block_scale((uint32_t)__builtin_amdgcn_readlane(exps[buf], 0));
        const float vsc = block_scale((uint32_t)__builtin_amdgcn_readlane(exps[buf], 32));
        const int n = n_in[buf];
        f32x4 sacc[T::NKB];
#pragma unroll
        for (int kb = 0; kb < T::NKB; ++kb) {
            sacc[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < T::NC; ++c) {
                const u32x4 w = kreg[buf][kb][c];
                sacc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8_t, codes_to_bf16x8(w[0], w[1], ksc)), qf[c * 2], sacc[kb], 0, 0, 0);
                sacc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8_t, codes_to_bf16x8(w[2], w[3], ksc)), qf[c * 2 + 1], sacc[kb], 0, 0, 0);
            }
        }
        if (n < kTk) {  // keys past the tile's end
#pragma unroll
            for (int kb = 0; kb < T::NKB; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (kb * 16 + grp * 4 + r >= n) sacc[kb][r] = -INFINITY;
        }
        float mt = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < T::NKB; ++kb)
            mt = fmaxf(mt, fmaxf(fmaxf(sacc[kb][0], sacc[kb][1]), fmaxf(sacc[kb][2], sacc[kb][3])));
        mt = pair_max(xor16_max(mt)) * sl2;  // over the tile's keys, log2 units
        // lazy rescale, as in decode.hip: weights stay <= 2^8
        if (__builtin_amdgcn_ballot_w64(mt > m + 8.f)) {
            const float m_new = fmaxf(m, mt);
            const float alpha = __builtin_amdgcn_exp2f(m - m_new);  // 0 when m == -inf
            lsum *= alpha;
#pragma unroll
            for (int db = 0; db < T::NDB; ++db) oacc[db] *= alpha;
            m = m_new;
        }
        uint32_t w[T::NKB * 2];
#pragma unroll
        for (int kb = 0; kb < T::NKB; ++kb)
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[kb][r], sl2, -m));
                const float p1 = __builtin_amdgcn_exp2f(fmaf(sacc[kb][r + 1], sl2, -m));
                const uint32_t pk = pack_bf16x2(p0, p1);
                w[kb * 2 + r / 2] = pk;
                // row sum of the weights as rounded for the P V product
                lsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones2, lsum, false);
            }
        const char* st = buf ? v_st1 : v_st0;
#pragma unroll
        for (int s = 0; s < T::NKB / 2; ++s) {
            const bf16x8_t pf =
                __builtin_bit_cast(bf16x8_t, u32x4{w[s * 4], w[s * 4 + 1], w[s * 4 + 2], w[s * 4 + 3]});
#pragma unroll
            for (int db = 0; db < T::NDB; ++db) {
                const v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (lds_v2i*)(st + (v_rd0 ^ (uint32_t)(db << 4)) + s * 32 * HD));
                const bf16x8_t av =
                    __builtin_bit_cast(bf16x8_t, codes_to_bf16x8((uint32_t)x[0], (uint32_t)x[1], vsc));
                oacc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, pf, oacc[db], 0, 0, 0);
            }
        }
    };

    // This wave's tiles are wave, wave + 4, ... of the range; the loads of the
    // next one are in flight while one is computed.
#define RC_TILES(AUX, FIRST, LAST)                            \
    if (const int i0 = FIRST, i1 = LAST; i0 < i1) {           \
        load_tile(Tag<0>{}, Tag<AUX>{}, i0);                  \
        for (int i = i0;; i += 2) {                           \
            if (i + 1 >= i1) {                                \
                __builtin_amdgcn_s_waitcnt(0x0F70);           \
                compute(Tag<0>{});                            \
                break;                                        \
            }                                                 \
            load_tile(Tag<1>{}, Tag<AUX>{}, i + 1);           \
            __builtin_amdgcn_s_waitcnt(T::WAIT_PREV);         \
            compute(Tag<0>{});                                \
            if (i + 2 >= i1) {                                \
                __builtin_amdgcn_s_waitcnt(0x0F70);           \
                compute(Tag<1>{});                            \
                break;                                        \
            }                                                 \
            load_tile(Tag<0>{}, Tag<AUX>{}, i + 2);           \
            __builtin_amdgcn_s_waitcnt(T::WAIT_PREV);         \
            compute(Tag<1>{});                                \
        }                                                     \
    }
    auto tiles_of = [&](int n) { return n > wave ? (n - wave + 3) / 4 : 0; };
    if constexpr (NT) {
        // the resource tiles, then the context tiles with their own loads
        const int n_res = max(0, min(t1, n_segt) - t0);
        RC_TILES(0, 0, tiles_of(n_res))
        RC_TILES(2, tiles_of(n_res), tiles_of(t1 - t0))
    } else {
        RC_TILES(0, 0, tiles_of(t1 - t0))
    }
#undef RC_TILES

    // ---- merge, as in decode.hip: the row groups of a head hold disjoint dims
    // of O^T and parts of its row sum; then the four waves, through LDS
    lsum = pair_sum(xor16_sum(lsum));
    static_assert(16 * HD * 4 == T::TILEB, "a wave's O fills a V buffer");
    __syncthreads();  // (ml shares the segment table's memory)
#pragma unroll
    for (int db = 0; db < T::NDB; ++db)
        *reinterpret_cast<f32x4*>(v_st0 + (l16 * (HD / 4) + ((db * 4 + grp) ^ l16)) * 16) = oacc[db];
    if (grp == 0) {
        sm.ml[wave][l16][0] = m;
        sm.ml[wave][l16][1] = lsum;
    }
    __syncthreads();
    for (int idx = tid; idx < R * HD; idx += kThreads) {
        const int h = idx / HD, d = idx % HD;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm.ml[w][h][0]);
        float num = 0.f, den = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = sm.ml[w][h][0];
            const float sc = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mx);
            const char* o = v_all0[w] + (h * (HD / 4) + ((d >> 2) ^ h)) * 16 + (d & 3) * 4;
            num += sc * *reinterpret_cast<const float*>(o);
            den += sc * sm.ml[w][h][1];
        }
        const size_t slot = ((size_t)b * a.d.n_q_heads + g * R + h) * a.d.n_splits + split;
        a.d.ws_o[slot * HD + d] = num;
        if (d == 0) {
            a.d.ws_ml[slot * 2 + 0] = mx;
            a.d.ws_ml[slot * 2 + 1] = den;
        }
    }
}

}  // namespace

// As many splits as decode.hip makes of half the keys, whose rows have twice the
// bytes (12 requests of 60 to 9,000 context rows, 16 / 8 heads: 20.4 us instead of
// 25.1 with all of its splits; one request over 3,400 keys 10.2 instead of 11.2, with
// a third of them 11.4; the merge included).
int decode8_splits(int n_req, int n_kv_heads, int max_kv) {
    return decode_splits(n_req, n_kv_heads, max_kv / 2 + max_kv % 2);
}

hipError_t launch_decode8(const Decode8Args& a, hipStream_t s) {
    const long blocks = (long)a.d.n_req * a.d.n_kv_heads * a.d.n_splits;
    if (blocks > 0x7fffffffL || a.d.ratio < 1 || a.d.ratio > 16) return hipErrorInvalidValue;
    // context rows past the caches by the rule of decode.hip, on their bytes here
    const bool nt = (unsigned long)std::min(a.d.c_rows, a.d.max_ctx_rows) * a.d.n_kv_heads * a.d.head_dim * 2 >=
                    (512UL << 20);
    const dim3 grid((unsigned)blocks), block(kThreads);
    if (a.d.head_dim == 128) {
        if (nt)
            hipLaunchKernelGGL((decode8_kernel<128, true>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((decode8_kernel<128, false>), grid, block, 0, s, a);
    } else {
        if (nt)
            hipLaunchKernelGGL((decode8_kernel<64, true>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((decode8_kernel<64, false>), grid, block, 0, s, a);
    }
    const hipError_t err = hipGetLastError();
    return err != hipSuccess ? err : launch_decode_merge(a.d, s);
}

}  // namespace rc
