// MXFP4 product, dense and grouped by expert:
//   y[i, o] = sum_b 2^(ex[i, b] + ew[o, b] - 254) sum_{j in b} cx[i, j] cw[o, j]
// on the block-scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4:
// lane L holds row L % 16, elements [32 (L / 16), 32 (L / 16) + 32) of a
// step of 128 (16 bytes of codes) and that block's scale byte.
#include "kernels.h"
#include "mx4_common.h"

namespace catk {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// acc += A B for one step; a and b are a lane's 16 bytes of codes, sa and sb
// their scale bytes (bits 0-7).
__device__ __forceinline__ f32x4 mx4_mfma(u32x4 a, u32x4 b, f32x4 acc, int sa, int sb) {
    const i32x8 av = {static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]),
                      static_cast<int>(a[3]), 0, 0, 0, 0};
    const i32x8 bv = {static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]),
                      static_cast<int>(b[3]), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc, 4, 4, 0, sa, 0, sb);
}

// Operands of a call; the dense product is one group of n rows.
struct Mx4Args {
    const uint8_t* cx;          // [n x d_in/2]
    const uint8_t* ex;          // [n x d_in/32]
    const uint8_t* cw;          // [groups x d_out x d_in/2]
    const uint8_t* ew;          // [groups x d_out x d_in/32]
    const int32_t* row_ids;     // [m] or NULL
    const int32_t* offsets;     // [groups + 1] or NULL (dense)
    void* y;                    // [m x d_out]
    int n, m, groups, d_in, d_out;
};

// The rows of row tile `tile` (BM rows of one expert): the expert's index,
// the first row and the end of the rows.  Experts' tiles are numbered one
// expert after the other; every wave finds its own by scanning the experts'
// tile counts, 64 at a time.  Offsets are clamped to [0, m], so no value in
// them leads outside the buffers.
struct Mx4Rows {
    int group, first, end;
};

template <int BM>
__device__ __forceinline__ bool mx4_rows(const Mx4Args& a, int tile, Mx4Rows& r) {
    if (!a.offsets) {
        r = Mx4Rows{0, tile * BM, a.m};
        return r.first < a.m;
    }
    const int lane = threadIdx.x & (kWave - 1);
    int before = 0;
    for (int g0 = 0; g0 < a.groups; g0 += kWave) {
        const int g = g0 + lane;
        int lo = 0, hi = 0;
        if (g < a.groups) {
            lo = a.offsets[g];
            hi = a.offsets[g + 1];
            lo = lo < 0 ? 0 : (lo > a.m ? a.m : lo);
            hi = hi < lo ? lo : (hi > a.m ? a.m : hi);
        }
        const int tiles = (hi - lo) / BM + ((hi - lo) % BM != 0 ? 1 : 0);
        int incl = tiles;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        const int start = before + incl - tiles;
        const uint64_t hit = __ballot(tile >= start && tile < start + tiles);
        if (hit) {
            const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
            r.group = g0 + src;
            r.first = __shfl(lo, src) + (tile - __shfl(start, src)) * BM;
            r.end = __shfl(hi, src);
            return true;
        }
        before += __shfl(incl, kWave - 1);
    }
    return false;
}

__device__ __forceinline__ int mx4_source_row(const Mx4Args& a, int i) {
    int s = a.row_ids ? a.row_ids[i] : i;
    return s < 0 ? 0 : (s < a.n ? s : a.n - 1);
}

__device__ __forceinline__ void mx4_store(float* y, float v) { *y = v; }
__device__ __forceinline__ void mx4_store(uint16_t* y, float v) {
    *y = static_cast<uint16_t>(pack_bf16(v, 0.0f));
}

// One wave per 16 outputs x 16 rows, operands straight from global memory.
template <typename Y>
__global__ __launch_bounds__(kWave) void mx4_gemm_kernel(Mx4Args a) {
    Mx4Rows r;
    if (!mx4_rows<16>(a, static_cast<int>(blockIdx.x), r)) return;
    const int lane = threadIdx.x, l16 = lane & 15, q = lane >> 4;
    const int blocks = a.d_in / kMxBlock;
    const int o = static_cast<int>(blockIdx.y) * 16 + l16;
    const int oc = o < a.d_out ? o : a.d_out - 1;
    const int64_t wrow = static_cast<int64_t>(r.group) * a.d_out + oc;
    const int i = r.first + l16 < r.end ? r.first + l16 : r.end - 1;
    const int64_t xrow = mx4_source_row(a, i);
    const u32x4* pw = reinterpret_cast<const u32x4*>(a.cw) + wrow * blocks;
    const u32x4* px = reinterpret_cast<const u32x4*>(a.cx) + xrow * blocks;
    const uint8_t* sw = a.ew + wrow * blocks;
    const uint8_t* sx = a.ex + xrow * blocks;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int b0 = 0; b0 < blocks; b0 += 4) {
        const int b = b0 + q;
        u32x4 cw = {0, 0, 0, 0}, cx = {0, 0, 0, 0};
        int ew = kMxByteOne, ex = kMxByteOne;
        if (b < blocks) {
            cw = pw[b];
            cx = px[b];
            ew = sw[b];
            ex = sx[b];
        }
        acc = mx4_mfma(cw, cx, acc, ew, ex);
    }
    // lane: row l16 of the tile, outputs 4 q .. 4 q + 3
    const int row = r.first + l16;
    if (row >= r.end) return;
    Y* y = static_cast<Y*>(a.y) + static_cast<int64_t>(row) * a.d_out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int col = static_cast<int>(blockIdx.y) * 16 + 4 * q + e;
        if (col < a.d_out) mx4_store(y + col, acc[e]);
    }
}

static hipError_t launch(const Mx4Args& a, int y_bf16, hipStream_t stream) {
    const int64_t row_tiles = (a.m + 15) / 16 + (a.offsets ? a.groups : 0);
    const dim3 grid(static_cast<unsigned>(row_tiles), static_cast<unsigned>((a.d_out + 15) / 16));
    if (y_bf16) mx4_gemm_kernel<uint16_t><<<grid, kWave, 0, stream>>>(a);
    else mx4_gemm_kernel<float><<<grid, kWave, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_mx4_linear(const uint8_t* cx, const uint8_t* ex, const uint8_t* cw,
                             const uint8_t* ew, int64_t n, int64_t d_in, int64_t d_out, void* y,
                             int y_bf16, hipStream_t stream) {
    const Mx4Args a{cx, ex, cw, ew, nullptr, nullptr, y, static_cast<int>(n), static_cast<int>(n), 1,
                    static_cast<int>(d_in), static_cast<int>(d_out)};
    return launch(a, y_bf16, stream);
}

hipError_t launch_mx4_linear_grouped(const uint8_t* cx, const uint8_t* ex, int64_t n,
                                     const int32_t* row_ids, int64_t m, const int32_t* offsets,
                                     int64_t groups, const uint8_t* cw, const uint8_t* ew,
                                     int64_t d_in, int64_t d_out, void* y, int y_bf16,
                                     hipStream_t stream) {
    const Mx4Args a{cx, ex, cw, ew, row_ids, offsets, y, static_cast<int>(n), static_cast<int>(m),
                    static_cast<int>(groups), static_cast<int>(d_in), static_cast<int>(d_out)};
    return launch(a, y_bf16, stream);
}

}  // namespace catk
