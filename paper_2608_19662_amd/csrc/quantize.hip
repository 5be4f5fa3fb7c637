// 16- or 32-bit K and V rows into the 8-bit cache format (quant8.hpp).
//
// For each block of 64 tokens of a segment and plane:
//     e = the smallest e >= 1 with max |x| <= 448 * 2^(e - 127)   (448: the largest e4m3 value)
//     code = rne_e4m3(x * 2^(127 - e))
// New rows are a segment's last ones.  Where rows were there before them in
// their first block, e is at least what it was, and where it grows the old
// codes are rounded again to the new scale.
//
// HBM-bound: a row is read and written once.  A wave takes one block of K or of V
// at a time: all of its loads (16 KB of bf16 at head_dim 128) are in flight together,
// the maximum is a reduction over its lanes, and the codes are formed from the
// same registers.  A store of 2,048 resources, 0.70 GB of bf16 rows read and
// 0.35 GB of codes written: 175 us, 6.0 TB/s; 64 appended tokens 5 us.
#include "common.hpp"
#include "kernels.hpp"
#include "quant8.hpp"

namespace rc {

namespace {

constexpr int kWaves = 4;  // per block

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Eight elements of a row, as loaded.  take_max: the largest magnitudes into acc, read
// back by max_bits; codes: all of them over scale, each NaN or at most 448 scale.
template <typename T>
struct Raw8;
template <>
struct Raw8<uint16_t> {
    u32x4 w;
    template <int AUX>
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        w = __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, AUX);
    }
    __device__ __forceinline__ void take_max(uint32_t& acc) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, acc),
                                                                         __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu)));
    }
    static __device__ __forceinline__ uint32_t max_bits(uint32_t acc) { return max(acc & 0xffff0000u, acc << 16); }
    // What is not finite becomes NaN (e4m3 has no infinities) and takes no part in acc.
    __device__ __forceinline__ void drop_infinities(uint32_t& acc) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool lo = (w[i] & 0x7f80u) == 0x7f80u, hi = (w[i] & 0x7f800000u) == 0x7f800000u;
            const uint32_t x = w[i] & 0x7fff7fffu & (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
            acc = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, acc),
                                                                         __builtin_bit_cast(u16x2, x)));
            w[i] |= (lo ? 0x7fffu : 0u) | (hi ? 0x7fff0000u : 0u);
        }
    }
    __device__ __forceinline__ u32x2 codes(float scale) const {
        u32x2 y;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // (a bit cast of a vector's element itself would take its first one)
            const uint32_t lo = w[2 * h], hi = w[2 * h + 1];
            s16x2 c = {0, 0};
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, lo), scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, hi), scale, true);
            y[h] = __builtin_bit_cast(uint32_t, c);
        }
        return y;
    }
};
template <>
struct Raw8<float> {
    u32x4 w[2];
    template <int AUX>
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        w[0] = __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, AUX);
        w[1] = __builtin_amdgcn_raw_buffer_load_b128(r, (int)(at + 16u), 0, AUX);
    }
    __device__ __forceinline__ uint32_t bits(int e) const { return w[e >> 2][e & 3]; }
    __device__ __forceinline__ void take_max(uint32_t& acc) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc = max(acc, bits(e) & 0x7fffffffu);
    }
    static __device__ __forceinline__ uint32_t max_bits(uint32_t acc) { return acc; }
    __device__ __forceinline__ void drop_infinities(uint32_t& acc) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t x = bits(e) & 0x7fffffffu;
            if (x < 0x7f800000u)
                acc = max(acc, x);
            else
                w[e >> 2][e & 3] |= 0x7fffffffu;
        }
    }
    __device__ __forceinline__ u32x2 codes(float scale) const {
        u32x2 y;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            auto f = [&](int e) { return __uint_as_float(w[h][e]); };
            s16x2 c = {0, 0};
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, f(0), f(1), scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, f(2), f(3), scale, true);
            y[h] = __builtin_bit_cast(uint32_t, c);
        }
        return y;
    }
};

// Maximum over the 64 lanes, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#define RC_STEP(ctrl, rows) \
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, true));
    RC_STEP(0x111, 0xf)  // row_shr:1, 2, 4, 8
    RC_STEP(0x112, 0xf)
    RC_STEP(0x114, 0xf)
    RC_STEP(0x118, 0xf)
    RC_STEP(0x142, 0xa)  // row_bcast:15, into rows 1 and 3
    RC_STEP(0x143, 0xc)  // row_bcast:31, into rows 2 and 3
#undef RC_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

constexpr uint32_t kInf = 0x7f800000u;

// e of a block whose largest finite |x| has these bits (448 = 1.75 * 2^8).
__device__ __forceinline__ int exponent_for(uint32_t amax) {
    return max(1, (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0));
}

__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// `bytes` bytes from p on: loads past them return zeros, stores past them do
// nothing.  (Offsets before p, too: they are taken as unsigned.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t extent(const void* p, long bytes) {
    const uint64_t u = (uint64_t)p;
    const uint64_t base = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32) |
                          (uint32_t)__builtin_amdgcn_readfirstlane((int)u);
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, __builtin_amdgcn_readfirstlane((int)bytes),
                                             0x00020000);
}

// NT: rows go past the caches, both ways.
template <typename T, int HD, bool NT>
__global__ __launch_bounds__(kWaves * 64, 2) void quantize_kernel(const QuantizeArgs a) {
    constexpr int AUX = NT ? 2 : 0;
    constexpr int CPR = HD / 8;           // 8-element chunks per row
    constexpr int RPI = 64 / CPR;         // rows per load of the wave
    constexpr int NL = kBlk8 / RPI;       // loads per block
    const int lane = threadIdx.x & 63;
    const long wid = (long)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_v = wid & 1;
    const int plane = (int)((wid >> 1) % a.n_planes);
    const long at = (wid >> 1) / a.n_planes;  // of the blocks that new rows may touch
    if (at >= a.n_blocks) return;
    // with counts of new rows a segment's can touch one block more than they fill
    const int32_t* cu_src = a.cu_new ? a.cu_new : a.cu;
    const int per = a.cu_new ? 2 : 1;
    const int s = find_segment(cu_src, a.n_seg, kBlk8, per, at, lane);
    const long src0 = cu_src[s], beg = a.cu[s];
    const long len = a.len ? a.len[s] : a.cu[s + 1] - beg;
    const long n_new = min(a.cu_new ? (long)a.cu_new[s + 1] - src0 : len, len);
    const long first = len - n_new;  // first new token of the segment
    const long j = first / kBlk8 + (at - first_item(src0, s, kBlk8, per));
    const long t0 = j * kBlk8;  // first token of the block
    const long row = beg + t0, slot = block_slot(beg, s) + j;
    const int n_old = (int)min(max(first - t0, 0L), (long)kBlk8);  // its tokens that were there
    const long src = src0 + t0 + n_old - first;                    // source row of its first new one
    // its tokens, in bounds whatever the offsets hold
    const int n = (int)min(min(len - t0, (long)kBlk8), min(a.rows - row, n_old + a.src_rows - src));
    if (n_new <= 0 || j < 0 || n <= n_old || beg < 0 || src < 0 || slot < 0 || slot >= a.n_slots) return;

    // ---- its rows.  Rows that were there lie before the extent of the new ones:
    // their loads return zeros and their stores do nothing.
    const int r0 = lane / CPR, col = (lane % CPR) * 8;
    const uint32_t row_bytes = (uint32_t)a.row_stride * sizeof(T);
    Raw8<T> raw[NL];
    {
        const auto from = extent(static_cast<const T*>(is_v ? a.v : a.k) + plane * a.plane_stride + src * a.row_stride,
                                 (n - n_old - 1) * (long)row_bytes + HD * sizeof(T));
        const uint32_t o = (uint32_t)(r0 - n_old) * row_bytes + (uint32_t)(col * sizeof(T));
#pragma unroll
        for (int i = 0; i < NL; ++i) raw[i].template load<AUX>(from, o + (uint32_t)(i * RPI) * row_bytes);
    }
    uint8_t* codes = (is_v ? a.v8 : a.k8) + ((size_t)plane * a.rows + row) * HD;
    uint8_t* exps = (is_v ? a.v_exp : a.k_exp) + (size_t)plane * a.n_slots;
    int e_old = 1;
    if (n_old > 0) e_old = max((int)exps[slot], 1);
    uint32_t acc = 0;
#pragma unroll
    for (int i = 0; i < NL; ++i) raw[i].take_max(acc);
    uint32_t amax = wave_max(Raw8<T>::max_bits(acc));
    if (amax >= kInf) {  // the maximum of those that are finite
        acc = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) raw[i].drop_infinities(acc);
        amax = wave_max(Raw8<T>::max_bits(acc));
    }
    const int e_new = max(e_old, exponent_for(amax));
    const float scale = block_scale((uint32_t)e_new);
    const auto dst = extent(codes + n_old * HD, (n - n_old) * HD);
    const uint32_t o = (uint32_t)((r0 - n_old) * HD + col);
#pragma unroll
    for (int i = 0; i < NL; ++i)
        __builtin_amdgcn_raw_buffer_store_b64(raw[i].codes(scale), dst, (int)(o + i * RPI * HD), 0, AUX);
    if (n_old > 0 && e_new > e_old) {
        // the old codes at the new scale (exact, but for those that become subnormal)
        const float down = __uint_as_float((uint32_t)max(127 + e_old - e_new, 0) << 23);
        for (int r = r0; r < n_old; r += RPI) {
            u32x2* p = reinterpret_cast<u32x2*>(codes + r * HD + col);
            const u32x2 w = *p;
            u32x2 y;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false);
                const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
                y[h] = pack_codes(lo[0] * down, lo[1] * down, hi[0] * down, hi[1] * down);
            }
            *p = y;
        }
    }
    if (lane == 0) exps[slot] = (uint8_t)e_new;
}

template <typename T, int HD>
hipError_t launch(const QuantizeArgs& a, hipStream_t stream) {
    const long waves = a.n_blocks * a.n_planes * 2, blocks = (waves + kWaves - 1) / kWaves;
    if (blocks > 0x7fffffffL) return hipErrorInvalidValue;
    // Past the caches where the rows are twice the 256 MB last-level cache or more
    // (1.05 GB: 175 us instead of 190); smaller ones are wanted there by whoever
    // reads them next, and found there (16,000 rows of 8 heads, 49 MB: 15.8 us
    // instead of 18.4).
    const bool nt = waves * (kBlk8 * HD) * (long)(sizeof(T) + 1) >= (512L << 20);
    const dim3 grid((unsigned)blocks), block(kWaves * 64);
    if (nt)
        hipLaunchKernelGGL((quantize_kernel<T, HD, true>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((quantize_kernel<T, HD, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs& a, int elem_bytes, int head_dim, hipStream_t stream) {
    if (a.n_blocks <= 0) return hipSuccess;
    if (elem_bytes == 4) return head_dim == 128 ? launch<float, 128>(a, stream) : launch<float, 64>(a, stream);
    return head_dim == 128 ? launch<uint16_t, 128>(a, stream) : launch<uint16_t, 64>(a, stream);
}

}  // namespace rc
