// MXFP4 quantization and its inverse (OCP Microscaling Formats v1.0): blocks
// of 32 elements share a scale 2^e, e = floor(log2 amax) - 2 from the
// exponent field of the block's largest magnitude; elements are E2M1.
//
// Both kernels read every input byte and write every output byte once, so
// they are bound by HBM at large sizes (235 M fp32 values 214 us, 5.0 TB/s;
// back to bf16 101 to 113 us, 5.9 to 5.3, the codes partly or not in the
// last-level cache, back to fp32 199 us, 5.3; a copy reaches 5.1) and by the launch at small ones
// (257 x 14336 bf16 3.2 and 3.6 us, from the last-level cache).  A thread owns
// eight consecutive elements (16 or 32 bytes in, 4 bytes of codes out), four
// consecutive lanes a block, whose largest magnitude they find with two quad
// permutations: no LDS, no barrier.
#include "kernels.h"
#include "mx4_common.h"

namespace catk {

constexpr int kMxThreads = 256;
constexpr int64_t kMxMaxBlocks = 1 << 20;  // beyond it threads take several vectors

template <typename T>
__global__ __launch_bounds__(kMxThreads) void mx4_quant_kernel(const T* __restrict__ x,
                                                               int64_t vecs,
                                                               uint32_t* __restrict__ codes,
                                                               uint8_t* __restrict__ scales) {
    // vecs is a multiple of 4 and so is the stride: a block's four lanes
    // leave the loop together
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kMxThreads;
    for (int64_t v = static_cast<int64_t>(blockIdx.x) * kMxThreads + threadIdx.x; v < vecs;
         v += stride) {
        float f[8];
        load8(x + 8 * v, f);
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = abs_bits(f[i]);
            amax = b > amax ? b : amax;
        }
        const uint32_t byte = mx4_scale_byte(quad_max(amax));
        codes[v] = byte == kMxByteNan ? 0u : mx4_encode8(f, mx4_inverse_scale(byte));
        if ((v & 3) == 0) scales[v >> 2] = static_cast<uint8_t>(byte);
    }
}

template <typename T>
__global__ __launch_bounds__(kMxThreads) void mx4_dequant_kernel(
    const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t vecs,
    T* __restrict__ out) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kMxThreads;
    for (int64_t v = static_cast<int64_t>(blockIdx.x) * kMxThreads + threadIdx.x; v < vecs;
         v += stride) {
        const uint32_t w = codes[v];
        const float s = mx4_scale(scales[v >> 2]);
        const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
        const f32x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
        const f32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
        const f32x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
        const float f[8] = {p0[0] * s, p0[1] * s, p1[0] * s, p1[1] * s,
                            p2[0] * s, p2[1] * s, p3[0] * s, p3[1] * s};
        store8(out + 8 * v, f);
    }
}

static unsigned mx4_blocks(int64_t vecs) {
    const int64_t b = (vecs + kMxThreads - 1) / kMxThreads;
    return static_cast<unsigned>(b < kMxMaxBlocks ? b : kMxMaxBlocks);
}

hipError_t launch_mx4_quant(const void* x, int x_bf16, int64_t n, int64_t d, uint8_t* codes,
                            uint8_t* scales, hipStream_t stream) {
    const int64_t vecs = n * (d / 8);
    uint32_t* c = reinterpret_cast<uint32_t*>(codes);
    if (x_bf16)
        mx4_quant_kernel<uint16_t><<<mx4_blocks(vecs), kMxThreads, 0, stream>>>(
            static_cast<const uint16_t*>(x), vecs, c, scales);
    else
        mx4_quant_kernel<float><<<mx4_blocks(vecs), kMxThreads, 0, stream>>>(
            static_cast<const float*>(x), vecs, c, scales);
    return hipGetLastError();
}

hipError_t launch_mx4_dequant(const uint8_t* codes, const uint8_t* scales, int64_t n, int64_t d,
                              void* out, int out_bf16, hipStream_t stream) {
    const int64_t vecs = n * (d / 8);
    const uint32_t* c = reinterpret_cast<const uint32_t*>(codes);
    if (out_bf16)
        mx4_dequant_kernel<uint16_t><<<mx4_blocks(vecs), kMxThreads, 0, stream>>>(
            c, scales, vecs, static_cast<uint16_t*>(out));
    else
        mx4_dequant_kernel<float><<<mx4_blocks(vecs), kMxThreads, 0, stream>>>(
            c, scales, vecs, static_cast<float*>(out));
    return hipGetLastError();
}

}  // namespace catk
