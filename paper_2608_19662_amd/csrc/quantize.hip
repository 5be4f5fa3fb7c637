// 16- or 32-bit K and V rows into the 8-bit cache format (quant8.hpp).
//
// For each block of 64 tokens of a segment and plane:
//     e = the smallest e >= 1 with max |x| <= 448 * 2^(e - 127)   (448: the largest e4m3 value)
//     code = rne_e4m3(x * 2^(127 - e))
// New rows are a segment's last ones.  Where rows were there before them in
// their first block, e is at least what it was, and where it grows the old
// codes are rounded again to the new scale.
//
// HBM-bound: a row is read and written once.  One wave takes one block of K or
// of V: all of its loads (16 KB of bf16 at head_dim 128) are in flight
// together, the maximum is a reduction over its lanes, and the codes are formed
// from the same registers.
#include "common.hpp"
#include "kernels.hpp"
#include "quant8.hpp"

namespace rc {

namespace {

constexpr int kWaves = 4;  // per block

// Eight elements of a row, as loaded; as floats.
template <typename T>
struct Raw8;
template <>
struct Raw8<uint16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void zero() { w = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ uint32_t bits(int e) const { return e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16; }
};
template <>
struct Raw8<float> {
    u32x4 w[2];
    __device__ __forceinline__ void load(const float* p) {
        w[0] = reinterpret_cast<const u32x4*>(p)[0];
        w[1] = reinterpret_cast<const u32x4*>(p)[1];
    }
    __device__ __forceinline__ void zero() { w[0] = w[1] = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ uint32_t bits(int e) const { return w[e >> 2][e & 3]; }
};

constexpr uint32_t kInf = 0x7f800000u;

// e of a block whose largest finite |x| has these bits (448 = 1.75 * 2^8).
__device__ __forceinline__ int exponent_for(uint32_t amax) {
    return max(1, (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0));
}

// A float that is not finite becomes NaN: e4m3 has no infinities.
__device__ __forceinline__ float finite_or_nan(uint32_t bits) {
    return __uint_as_float((bits & kInf) == kInf ? 0x7fc00000u : bits);
}

__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

template <typename T, int HD>
__global__ __launch_bounds__(kWaves * 64) void quantize_kernel(const QuantizeArgs a) {
    constexpr int CPR = HD / 8;           // 8-element chunks per row
    constexpr int RPI = 64 / CPR;         // rows per load of the wave
    constexpr int NL = kBlk8 / RPI;       // loads per block
    const int lane = threadIdx.x & 63;
    const long item = (long)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int is_v = (int)(item & 1);
    const int plane = (int)((item >> 1) % a.n_planes);
    const long at = (item >> 1) / a.n_planes;  // of the blocks that new rows may touch
    if (at >= a.n_blocks) return;
    // ---- the segment and its block.  With counts of new rows a segment's can
    // touch one block more than they fill.
    const int32_t* cu_src = a.cu_new ? a.cu_new : a.cu;
    const int per = a.cu_new ? 2 : 1;
    const int s = find_segment(cu_src, a.n_seg, kBlk8, per, at, lane);
    const long src0 = cu_src[s], beg = a.cu[s];
    const long len = a.len ? a.len[s] : a.cu[s + 1] - beg;
    const long n_new = min(a.cu_new ? (long)a.cu_new[s + 1] - src0 : len, len);
    const long first = len - n_new;  // first new token of the segment
    const long j = first / kBlk8 + (at - first_item(src0, s, kBlk8, per));
    if (n_new <= 0 || j < 0 || j * kBlk8 >= len) return;
    const long t0 = j * kBlk8;                                    // first token of the block
    const int n = (int)min(len - t0, (long)kBlk8);                // its tokens
    const int n_old = (int)min(max(first - t0, 0L), (long)n);     // those that were there
    const long slot = block_slot(beg, s) + j;
    if (beg < 0 || slot < 0 || slot >= a.n_slots) return;  // (offsets that do not fit the cache)

    const T* x = static_cast<const T*>(is_v ? a.v : a.k) + plane * a.plane_stride;
    uint8_t* codes = (is_v ? a.v8 : a.k8) + (size_t)plane * a.rows * HD;
    uint8_t* exps = (is_v ? a.v_exp : a.k_exp) + (size_t)plane * a.n_slots;

    const int r0 = lane / CPR, col = (lane % CPR) * 8;
    Raw8<T> raw[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int r = i * RPI + r0;
        const long src = src0 + (t0 + r - first);
        if (r >= n_old && r < n && src >= 0 && src < a.src_rows)
            raw[i].load(x + src * a.row_stride + col);
        else
            raw[i].zero();
    }
    int e_old = 1;
    if (n_old > 0) e_old = max((int)exps[slot], 1);
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = raw[i].bits(e) & 0x7fffffffu;
            amax = max(amax, b < kInf ? b : 0u);
        }
    for (int o = 32; o >= 1; o >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o));
    const int e_new = max(e_old, exponent_for(amax));
    const float inv = __uint_as_float((uint32_t)(254 - e_new) << 23);  // 2^(127 - e)
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int r = i * RPI + r0;
        const long row = beg + t0 + r;
        if (r >= n_old && r < n && row < a.rows) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = finite_or_nan(raw[i].bits(e)) * inv;
            *reinterpret_cast<u32x2*>(codes + row * HD + col) =
                u32x2{pack_codes(f[0], f[1], f[2], f[3]), pack_codes(f[4], f[5], f[6], f[7])};
        }
    }
    if (n_old > 0 && e_new > e_old) {
        // the old codes at the new scale (exact, but for those that become subnormal)
        const float down = __uint_as_float((uint32_t)max(127 + e_old - e_new, 0) << 23);
        for (int r = r0; r < n_old; r += RPI) {
            const long row = beg + t0 + r;
            if (row >= a.rows) break;
            u32x2* p = reinterpret_cast<u32x2*>(codes + row * HD + col);
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

}  // namespace

hipError_t launch_quantize(const QuantizeArgs& a, int elem_bytes, int head_dim, hipStream_t stream) {
    if (a.n_blocks <= 0) return hipSuccess;
    const long waves = a.n_blocks * a.n_planes * 2, blocks = (waves + kWaves - 1) / kWaves;
    if (blocks > 0x7fffffffL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(kWaves * 64);
    if (elem_bytes == 4) {
        if (head_dim == 128)
            hipLaunchKernelGGL((quantize_kernel<float, 128>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((quantize_kernel<float, 64>), grid, block, 0, stream, a);
    } else {
        if (head_dim == 128)
            hipLaunchKernelGGL((quantize_kernel<uint16_t, 128>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((quantize_kernel<uint16_t, 64>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace rc
