// RMS norm with the residual's addition and quantized output:
//   h = fl(x + residual), r = fl32(1 / sqrt(mean h^2 + eps)),
//   y = fl(fl(h w) r), written as per-token int8 codes or MXFP4.
//
// One pass over HBM: a row's h stays in the registers of its threads between
// the statistics and the codes (rows of up to 32768 elements).  r is one
// number a row and positive, and rounding is monotonic, so max |y| =
// fl(max |fl(h w)| * r): the sum of squares and the int8 scale come out of one
// reduction.  The sum is held in fp64 (an fp64 multiply-add costs what an fp32
// one does here): it neither overflows nor depends noticeably on the order,
// so codes next to a rounding border are those of the exact sum.
//
// Bound by HBM: bf16 with a residual reads 4 and writes 2 bytes an element
// and 1 (int8) or 0.53 (MXFP4) of codes.  Measured over 130 M elements, where
// a copy reaches 5.1 TB/s: 5.2 to 5.9 TB/s for rows of 32 to 16384, 4.8 at
// 32768, 4.0 beyond (read twice); int8 from bf16 without a residual, 3 bytes
// an element, 4.5 (its conversions).  Threads per row are the fewest that hold
// it with up to four vectors: 256 threads for every row up to 2048 left lanes
// idle (1024 elements 3.8 TB/s, now 5.6; 32 elements 0.5, now 5.7).  Rows
// whose length is no multiple of 8 start at any address and are loaded with
// 16-byte loads all the same: 3.4 TB/s where single elements gave 1.7.
#include "kernels.h"
#include "mx4_common.h"

namespace catk {

enum : int { kOutInt8 = 0, kOutMx4 = 1 };

struct RowStats {
    double ss;          // sum of h^2
    uint32_t amax;      // bits of max |fl(h w)|
};

// Statistics of a row over the TPR threads that share it (a power of two up
// to a wave, or several waves).  Every wave adds the partial sums in the same
// order, so all threads get the same bits.
template <int TPR>
__device__ __forceinline__ RowStats row_stats(RowStats s) {
#pragma unroll
    for (int o = 1; o < (TPR < kWave ? TPR : kWave); o <<= 1) {
        s.ss += __shfl_xor(s.ss, o);
        const uint32_t b = static_cast<uint32_t>(__shfl_xor(static_cast<int>(s.amax), o));
        s.amax = b > s.amax ? b : s.amax;
    }
    if constexpr (TPR > kWave) {
        constexpr int W = TPR / kWave;
        __shared__ double ss[W];
        __shared__ uint32_t mx[W];
        const int wave = threadIdx.x / kWave;
        if (threadIdx.x % kWave == 0) {
            ss[wave] = s.ss;
            mx[wave] = s.amax;
        }
        __syncthreads();
        s = RowStats{0.0, 0u};
#pragma unroll
        for (int i = 0; i < W; ++i) {
            s.ss += ss[i];
            s.amax = mx[i] > s.amax ? mx[i] : s.amax;
        }
    }
    return s;
}

// NaN for a row that is not finite, so that all of it becomes NaN.
__device__ __forceinline__ float inverse_rms(double ss, int64_t d, double eps) {
    const double v = ss / static_cast<double>(d) + eps;
    if (v == 0.0) return 0.0f;
    return v < __builtin_huge_val() ? static_cast<float>(1.0 / sqrt(v)) : __uint_as_float(0x7FC00000u);
}

// The int8 quantizer of a row: its scale, the factor of the codes, and a mask
// of them (0 where the codes are to be 0: a row of zeros, one so small that
// the factor is infinite, or one that is not finite).
struct Int8Scale {
    float s, inv;
    uint32_t keep;
};
__device__ __forceinline__ Int8Scale int8_scale(uint32_t amax_hw, float r) {
    const float amax = __uint_as_float(amax_hw) * r;
    if (!(abs_bits(amax) < 0x7F800000u)) return {__uint_as_float(0x7FC00000u), 0.0f, 0u};
    const float inv = 127.0f / amax;
    if (abs_bits(inv) == 0x7F800000u) return {0.0f, 0.0f, 0u};
    return {amax / 127.0f, inv, 0xFFFFFFFFu};
}
// Code of y, in the low byte: adding 1.5 * 2^23 rounds the product to the
// nearest integer, ties to even, and leaves its two's complement in the low
// bits.  |y * inv| <= 127 (1 + 2^-23), so no code exceeds 127.
__device__ __forceinline__ uint32_t int8_bits(float y, float inv) {
    return __float_as_uint(y * inv + 12582912.0f);
}
__device__ __forceinline__ uint32_t int8_pack4(const float* y, float inv) {
    const uint32_t lo = __builtin_amdgcn_perm(int8_bits(y[1], inv), int8_bits(y[0], inv), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(int8_bits(y[3], inv), int8_bits(y[2], inv), 0x0C0C0400u);
    return lo | (hi << 16);
}

// Eight elements of a row that starts at any address, one by one at its end
// (left of them exist).  Global loads and stores of 16 bytes may start at any
// byte here.
template <typename T>
__device__ __forceinline__ void load8_any(const T* p, int left, float* v) {
    if (left >= 8) {
        T raw[8];
        __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = load_as_f32(raw, i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? load_as_f32(p, i) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store8_any(T* p, int left, const float* v) {
    T raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) raw[i] = v[i];
        else raw[i] = static_cast<T>(pack_bf16(v[i], 0.0f));
    }
    if (left >= 8) {
        __builtin_memcpy(p, raw, sizeof(raw));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = raw[i];
    }
}

// One vector of eight elements: loads of x and the residual, and of the
// weight; stores of the residual and of the codes.  ANY: rows may start at any
// address (d % 8 != 0).
template <typename T, bool ANY>
__device__ __forceinline__ void load_h(const T* x, const T* res, int64_t at, int left, float* h) {
    if constexpr (ANY) load8_any(x + at, left, h);
    else load8(x + at, h);
    if (res) {
        float e[8];
        if constexpr (ANY) load8_any(res + at, left, e);
        else load8(res + at, e);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += e[i];
    }
}
template <typename W, bool ANY>
__device__ __forceinline__ void load_w(const W* w, int64_t c, int left, float* g) {
    if constexpr (ANY) load8_any(w + c, left, g);
    else load8(w + c, g);
}
template <typename T, bool ANY>
__device__ __forceinline__ void store_h(T* out, int64_t at, int left, const float* h) {
    if constexpr (ANY) store8_any(out + at, left, h);
    else store8(out + at, h);
}
// y of a vector from h w and r, and its codes at element `at` of the matrix
template <int OUT, bool ANY>
__device__ __forceinline__ void store_codes(uint8_t* codes, void* scales, int64_t at, int left, int t,
                                            float* h, float r, const Int8Scale& q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] *= r;
    if constexpr (OUT == kOutInt8) {
        const u32x2 c = {int8_pack4(h, q.inv) & q.keep, int8_pack4(h + 4, q.inv) & q.keep};
        if constexpr (!ANY) {
            *reinterpret_cast<u32x2*>(codes + at) = c;
        } else if (left >= 8) {
            __builtin_memcpy(codes + at, &c, 8);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) codes[at + i] = static_cast<uint8_t>(c[i / 4] >> (8 * (i % 4)));
        }
    } else {                               // d % 32 == 0: the four lanes of a block together
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = abs_bits(h[i]);
            amax = b > amax ? b : amax;
        }
        const uint32_t byte = mx4_scale_byte(quad_max(amax));
        reinterpret_cast<uint32_t*>(codes)[at / 8] =
            byte == kMxByteNan ? 0u : mx4_encode8(h, mx4_inverse_scale(byte));
        if (t % 4 == 0) static_cast<uint8_t*>(scales)[at / kMxBlock] = static_cast<uint8_t>(byte);
    }
}

// NV vectors a thread, TPR threads a row; rows of at most 8 TPR NV elements.
// res_out may be res or x: every load of a row comes before its first store.
template <typename T, typename W, int OUT, int TPR, int NV, bool ANY>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rmsnorm_kernel(
    const T* x, const T* res, T* res_out, const W* __restrict__ w, int64_t n, int64_t d,
    double eps, uint8_t* __restrict__ codes, void* __restrict__ scales) {
    static_assert(!ANY || OUT == kOutInt8, "MXFP4 rows are whole blocks");
    constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;     // rows per workgroup
    const int t = threadIdx.x % TPR;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    if (ROWS > 1 && row >= n) return;                   // all threads of a row together
    const int64_t at = row * d;
    const int dd = static_cast<int>(d);

    float h[NV][8];
    RowStats st{0.0, 0u};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TPR + t) * 8;
        if (c < dd) load_h<T, ANY>(x, res, at + c, dd - c, h[v]);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TPR + t) * 8;
        if (c >= dd) continue;
        if (res) store_h<T, ANY>(res_out, at + c, dd - c, h[v]);
        float g[8];
        load_w<W, ANY>(w, c, dd - c, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            st.ss += static_cast<double>(h[v][i]) * h[v][i];
            h[v][i] *= g[i];
            if constexpr (OUT == kOutInt8) {
                const uint32_t b = abs_bits(h[v][i]);
                st.amax = b > st.amax ? b : st.amax;
            }
        }
    }
    st = row_stats<TPR>(st);
    const float r = inverse_rms(st.ss, d, eps);
    const Int8Scale q = OUT == kOutInt8 ? int8_scale(st.amax, r) : Int8Scale{};
    if (OUT == kOutInt8 && t == 0) static_cast<float*>(scales)[row] = q.s;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * TPR + t) * 8;
        if (c < dd) store_codes<OUT, ANY>(codes, scales, at + c, dd - c, t, h[v], r, q);
    }
}

// Rows too long for registers: the row is read a second time for the codes
// (from L2), and the updated residual is written only then, each element by
// the thread that reads it, so that it may replace the residual or x.
template <typename T, typename W, int OUT, bool ANY>
__global__ __launch_bounds__(1024) void rmsnorm_long_kernel(
    const T* x, const T* res, T* res_out, const W* __restrict__ w, int64_t n, int64_t d,
    double eps, uint8_t* __restrict__ codes, void* __restrict__ scales) {
    static_assert(!ANY || OUT == kOutInt8, "MXFP4 rows are whole blocks");
    constexpr int TPR = 1024;
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x, at = row * d;
    auto left = [&](int64_t c) { return static_cast<int>(d - c < 8 ? d - c : 8); };
    RowStats st{0.0, 0u};
    for (int64_t c = static_cast<int64_t>(t) * 8; c < d; c += TPR * 8) {
        float h[8], g[8];
        load_h<T, ANY>(x, res, at + c, left(c), h);
        load_w<W, ANY>(w, c, left(c), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            st.ss += static_cast<double>(h[i]) * h[i];
            const uint32_t b = abs_bits(h[i] * g[i]);
            st.amax = b > st.amax ? b : st.amax;
        }
    }
    st = row_stats<TPR>(st);
    const float r = inverse_rms(st.ss, d, eps);
    const Int8Scale q = int8_scale(st.amax, r);
    if (OUT == kOutInt8 && t == 0) static_cast<float*>(scales)[row] = q.s;
    for (int64_t c = static_cast<int64_t>(t) * 8; c < d; c += TPR * 8) {
        float h[8], g[8];
        load_h<T, ANY>(x, res, at + c, left(c), h);
        load_w<W, ANY>(w, c, left(c), g);
        if (res) store_h<T, ANY>(res_out, at + c, left(c), h);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] *= g[i];
        store_codes<OUT, ANY>(codes, scales, at + c, left(c), t, h, r, q);
    }
}

// Calls fn(first row, rows) so that no launch exceeds 2^31 threads.
template <typename F>
static hipError_t row_launches(int64_t n, int threads, int rows_per_block, F fn) {
    const int64_t most = (int64_t{1} << 31) / threads * rows_per_block;
    for (int64_t r = 0; r < n; r += most) {
        fn(r, n - r < most ? n - r : most);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

// Threads per row and vectors per thread: the smallest that hold the row.
template <typename T, typename W, int OUT, bool ANY>
static hipError_t launch_rows(const T* x, const T* res, T* res_out, const W* w, int64_t n,
                              int64_t d, double eps, uint8_t* codes, void* scales,
                              hipStream_t stream) {
    auto scales_at = [&](int64_t r) -> void* {
        return OUT == kOutInt8 ? static_cast<void*>(static_cast<float*>(scales) + r)
                               : static_cast<void*>(static_cast<uint8_t*>(scales) + r * (d / kMxBlock));
    };
    auto codes_at = [&](int64_t r) { return codes + (OUT == kOutInt8 ? r * d : r * (d / 2)); };
#define CAT_NORM(TPR, NV)                                                                        \
    if (d <= TPR * NV * 8) {                                                                     \
        constexpr int rows = TPR < 256 ? 256 / TPR : 1, threads = TPR < 256 ? 256 : TPR;         \
        return row_launches(n, threads, rows, [&](int64_t r, int64_t c) {                        \
            rmsnorm_kernel<T, W, OUT, TPR, NV, ANY>                                              \
                <<<static_cast<unsigned>((c + rows - 1) / rows), threads, 0, stream>>>(          \
                    x + r * d, res ? res + r * d : nullptr, res ? res_out + r * d : nullptr, w,  \
                    c, d, eps, codes_at(r), scales_at(r));                                       \
        });                                                                                      \
    }
    CAT_NORM(4, 1)
    CAT_NORM(8, 1)
    CAT_NORM(16, 1)
    CAT_NORM(32, 1)
    CAT_NORM(64, 1)
    CAT_NORM(64, 2)
    CAT_NORM(64, 4)
    CAT_NORM(256, 2)
    CAT_NORM(256, 4)
    CAT_NORM(1024, 2)
    CAT_NORM(1024, 4)
#undef CAT_NORM
    return row_launches(n, 1024, 1, [&](int64_t r, int64_t c) {
        rmsnorm_long_kernel<T, W, OUT, ANY><<<static_cast<unsigned>(c), 1024, 0, stream>>>(
            x + r * d, res ? res + r * d : nullptr, res ? res_out + r * d : nullptr, w, c, d, eps,
            codes_at(r), scales_at(r));
    });
}

template <typename T, typename W>
static hipError_t launch_typed(const void* x, const void* res, void* res_out, const void* w,
                               int64_t n, int64_t d, double eps, int mx4, uint8_t* codes,
                               void* scales, hipStream_t stream) {
    const T* xt = static_cast<const T*>(x);
    const T* rt = static_cast<const T*>(res);
    T* ro = static_cast<T*>(res_out);
    const W* wt = static_cast<const W*>(w);
    if (mx4) return launch_rows<T, W, kOutMx4, false>(xt, rt, ro, wt, n, d, eps, codes, scales, stream);
    if (d % 8 == 0)
        return launch_rows<T, W, kOutInt8, false>(xt, rt, ro, wt, n, d, eps, codes, scales, stream);
    return launch_rows<T, W, kOutInt8, true>(xt, rt, ro, wt, n, d, eps, codes, scales, stream);
}

hipError_t launch_rmsnorm(const void* x, int x_bf16, int64_t n, int64_t d, const void* res,
                          void* res_out, const void* w, int w_bf16, double eps, int mx4,
                          uint8_t* codes, void* scales, hipStream_t stream) {
    if (x_bf16)
        return w_bf16 ? launch_typed<uint16_t, uint16_t>(x, res, res_out, w, n, d, eps, mx4, codes, scales, stream)
                      : launch_typed<uint16_t, float>(x, res, res_out, w, n, d, eps, mx4, codes, scales, stream);
    return w_bf16 ? launch_typed<float, uint16_t>(x, res, res_out, w, n, d, eps, mx4, codes, scales, stream)
                  : launch_typed<float, float>(x, res, res_out, w, n, d, eps, mx4, codes, scales, stream);
}

}  // namespace catk
