// RMS norm with the residual's addition and quantized output:
//   h = fl(x + residual), r = fl32(1 / sqrt(mean h^2 + eps)),
//   y = fl(fl(h w) r), written as per-token int8 codes or MXFP4.
//
// One pass over HBM: a row's h stays in the registers of its threads between
// the statistics and the codes.  r is one number a row and positive, and
// rounding is monotonic, so max |y| = fl(max |fl(h w)| * r): the sum of
// squares and the int8 scale come out of one reduction.  The sum is held in
// fp64 (an fp64 multiply-add costs what an fp32 one does here, and the
// kernel waits for memory): it neither overflows nor depends noticeably on
// the order, so codes next to a rounding border are those of the exact sum.
// Bound by HBM: bf16 with a residual reads 4 and writes 2 bytes an element
// and 1 (int8) or 0.53 (MXFP4) of codes.
#include "kernels.h"
#include "mx4_common.h"

namespace catk {

enum : int { kOutInt8 = 0, kOutMx4 = 1 };

struct RowStats {
    double ss;          // sum of h^2
    uint32_t amax;      // bits of max |fl(h w)|
};

__device__ __forceinline__ RowStats wave_stats(RowStats s) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        s.ss += __shfl_xor(s.ss, o);
        const uint32_t b = static_cast<uint32_t>(__shfl_xor(static_cast<int>(s.amax), o));
        s.amax = b > s.amax ? b : s.amax;
    }
    return s;
}

// Statistics of a row over the TPR threads that share it.  Every wave adds
// the partial sums in the same order, so all threads get the same bits.
template <int TPR>
__device__ __forceinline__ RowStats row_stats(RowStats s) {
    s = wave_stats(s);
    if constexpr (TPR > kWave) {
        constexpr int W = TPR / kWave;
        __shared__ double ss[W];
        __shared__ uint32_t mx[W];
        const int wave = threadIdx.x / kWave;
        __syncthreads();    // an earlier row's readers
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

__device__ __forceinline__ float inverse_rms(double ss, int64_t d, double eps) {
    const double v = ss / static_cast<double>(d) + eps;
    return v > 0.0 ? static_cast<float>(1.0 / sqrt(v)) : (v == 0.0 ? 0.0f : __uint_as_float(0x7FC00000u));
}

// The int8 quantizer of a row: its scale, and the factor of the codes (0
// where the codes are to be 0: an all-zero row, or one that is not finite).
struct Int8Scale {
    float s, inv;
};
__device__ __forceinline__ Int8Scale int8_scale(uint32_t amax_hw, float r) {
    const float amax = __uint_as_float(amax_hw) * r;
    if (amax == 0.0f) return {0.0f, 0.0f};
    if (!(abs_bits(amax) < 0x7F800000u)) return {__uint_as_float(0x7FC00000u), 0.0f};
    return {amax / 127.0f, 127.0f / amax};
}
__device__ __forceinline__ int int8_code(float y, float inv) {
    if (inv == 0.0f) return 0;
    const float q = fminf(fmaxf(rintf(y * inv), -127.0f), 127.0f);
    return static_cast<int>(q);
}

// NV vectors of eight elements a thread, TPR threads a row.  VEC: a vector
// is eight consecutive elements (d % 8 == 0); otherwise eight elements TPR
// apart, loaded one by one (rows of any length start at any address, and
// consecutive lanes still read consecutive elements).  res_out may be res or
// x: every load of a row comes before its first store.
template <typename T, typename W, int OUT, int TPR, int NV, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rmsnorm_kernel(
    const T* x, const T* res, T* res_out, const W* __restrict__ w, int64_t n, int64_t d,
    double eps, uint8_t* __restrict__ codes, void* __restrict__ scales) {
    static_assert(VEC || OUT == kOutInt8, "MXFP4 rows are whole blocks");
    constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;     // rows per workgroup
    const int t = threadIdx.x % TPR;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    if (ROWS > 1 && row >= n) return;                   // whole waves
    const int64_t at = row * d;
    const int dd = static_cast<int>(d);

    float h[NV][8];
    RowStats st{0.0, 0u};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if constexpr (VEC) {
            const int c = (v * TPR + t) * 8;
            if (c < dd) {
                load8(x + at + c, h[v]);
                if (res) {
                    float e[8];
                    load8(res + at + c, e);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[v][i] += e[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] = 0.0f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = (v * 8 + i) * TPR + t;
                h[v][i] = 0.0f;
                if (c < dd) {
                    h[v][i] = load_as_f32(x + at, c);
                    if (res) h[v][i] += load_as_f32(res + at, c);
                }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if constexpr (VEC) {
            const int c = (v * TPR + t) * 8;
            if (c < dd) {
                if (res) store8(res_out + at + c, h[v]);
                float g[8];
                load8(w + c, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    st.ss += static_cast<double>(h[v][i]) * h[v][i];
                    h[v][i] *= g[i];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = (v * 8 + i) * TPR + t;
                if (c < dd) {
                    if (res) {
                        if constexpr (sizeof(T) == 4) res_out[at + c] = h[v][i];
                        else res_out[at + c] = static_cast<T>(pack_bf16(h[v][i], 0.0f));
                    }
                    st.ss += static_cast<double>(h[v][i]) * h[v][i];
                    h[v][i] *= load_as_f32(w, c);
                }
            }
        }
        if constexpr (OUT == kOutInt8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = abs_bits(h[v][i]);
                st.amax = b > st.amax ? b : st.amax;
            }
        }
    }
    st = row_stats<TPR>(st);
    const float r = inverse_rms(st.ss, d, eps);

    if constexpr (OUT == kOutInt8) {
        const Int8Scale q = int8_scale(st.amax, r);
        int8_t* row_codes = reinterpret_cast<int8_t*>(codes) + at;
        if (t == 0) static_cast<float*>(scales)[row] = q.s;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (VEC) {
                const int c = (v * TPR + t) * 8;
                if (c < dd) {
                    uint32_t lo = 0, hi = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        lo |= (static_cast<uint32_t>(int8_code(h[v][i] * r, q.inv)) & 0xFFu) << (8 * i);
                        hi |= (static_cast<uint32_t>(int8_code(h[v][4 + i] * r, q.inv)) & 0xFFu) << (8 * i);
                    }
                    *reinterpret_cast<u32x2*>(row_codes + c) = u32x2{lo, hi};
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = (v * 8 + i) * TPR + t;
                    if (c < dd) row_codes[c] = static_cast<int8_t>(int8_code(h[v][i] * r, q.inv));
                }
            }
        }
    } else {
        uint32_t* row_codes = reinterpret_cast<uint32_t*>(codes + at / 2);
        uint8_t* row_scales = static_cast<uint8_t*>(scales) + at / kMxBlock;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * TPR + t) * 8;
            if (c < dd) {       // d % 32 == 0: the four lanes of a block together
                uint32_t amax = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    h[v][i] *= r;
                    const uint32_t b = abs_bits(h[v][i]);
                    amax = b > amax ? b : amax;
                }
                const uint32_t byte = mx4_scale_byte(quad_max(amax));
                row_codes[c / 8] = byte == kMxByteNan ? 0u : mx4_encode8(h[v], mx4_inverse_scale(byte));
                if (t % 4 == 0) row_scales[c / kMxBlock] = static_cast<uint8_t>(byte);
            }
        }
    }
}

// Rows too long for registers: the row is read a second time for the codes
// (from L2), and the updated residual is written only then, each element by
// the thread that reads it, so that it may replace the residual.
template <typename T, typename W, int OUT, bool VEC>
__global__ __launch_bounds__(1024) void rmsnorm_long_kernel(
    const T* x, const T* res, T* res_out, const W* __restrict__ w, int64_t n, int64_t d,
    double eps, uint8_t* __restrict__ codes, void* __restrict__ scales) {
    static_assert(VEC || OUT == kOutInt8, "MXFP4 rows are whole blocks");
    constexpr int TPR = 1024;
    constexpr int E = VEC ? 8 : 1;
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x, at = row * d;
    auto load = [&](int64_t c, float* h) {
        if constexpr (VEC) {
            load8(x + at + c, h);
            if (res) {
                float e[8];
                load8(res + at + c, e);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] += e[i];
            }
        } else {
            h[0] = load_as_f32(x + at, c);
            if (res) h[0] += load_as_f32(res + at, c);
        }
    };
    auto load_w = [&](int64_t c, float* g) {
        if constexpr (VEC) load8(w + c, g);
        else g[0] = load_as_f32(w, c);
    };
    RowStats st{0.0, 0u};
    for (int64_t c = static_cast<int64_t>(t) * E; c < d; c += TPR * E) {
        float h[E], g[E];
        load(c, h);
        load_w(c, g);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            st.ss += static_cast<double>(h[i]) * h[i];
            const uint32_t b = abs_bits(h[i] * g[i]);
            st.amax = b > st.amax ? b : st.amax;
        }
    }
    st = row_stats<TPR>(st);
    const float r = inverse_rms(st.ss, d, eps);
    const Int8Scale q = int8_scale(st.amax, r);
    if (OUT == kOutInt8 && t == 0) static_cast<float*>(scales)[row] = q.s;
    for (int64_t c = static_cast<int64_t>(t) * E; c < d; c += TPR * E) {
        float h[E], g[E];
        load(c, h);
        load_w(c, g);
        if (res) {
            if constexpr (VEC) store8(res_out + at + c, h);
            else if constexpr (sizeof(T) == 4) res_out[at + c] = h[0];
            else res_out[at + c] = static_cast<T>(pack_bf16(h[0], 0.0f));
        }
#pragma unroll
        for (int i = 0; i < E; ++i) h[i] = (h[i] * g[i]) * r;
        if constexpr (OUT == kOutInt8) {
            int8_t* row_codes = reinterpret_cast<int8_t*>(codes) + at;
            if constexpr (VEC) {
                uint32_t lo = 0, hi = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lo |= (static_cast<uint32_t>(int8_code(h[i], q.inv)) & 0xFFu) << (8 * i);
                    hi |= (static_cast<uint32_t>(int8_code(h[4 + i], q.inv)) & 0xFFu) << (8 * i);
                }
                *reinterpret_cast<u32x2*>(row_codes + c) = u32x2{lo, hi};
            } else {
                row_codes[c] = static_cast<int8_t>(int8_code(h[0], q.inv));
            }
        } else {
            uint32_t amax = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = abs_bits(h[i]);
                amax = b > amax ? b : amax;
            }
            const uint32_t byte = mx4_scale_byte(quad_max(amax));
            reinterpret_cast<uint32_t*>(codes + at / 2)[c / 8] =
                byte == kMxByteNan ? 0u : mx4_encode8(h, mx4_inverse_scale(byte));
            if (t % 4 == 0)
                static_cast<uint8_t*>(scales)[at / kMxBlock + c / kMxBlock] = static_cast<uint8_t>(byte);
        }
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
template <typename T, typename W, int OUT, bool VEC>
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
            rmsnorm_kernel<T, W, OUT, TPR, NV, VEC>                                              \
                <<<static_cast<unsigned>((c + rows - 1) / rows), threads, 0, stream>>>(          \
                    x + r * d, res ? res + r * d : nullptr, res ? res_out + r * d : nullptr, w,  \
                    c, d, eps, codes_at(r), scales_at(r));                                       \
        });                                                                                      \
    }
    CAT_NORM(64, 1)
    CAT_NORM(256, 1)
    CAT_NORM(256, 2)
    CAT_NORM(256, 4)
    CAT_NORM(1024, 2)
    CAT_NORM(1024, 4)
#undef CAT_NORM
    return row_launches(n, 1024, 1, [&](int64_t r, int64_t c) {
        rmsnorm_long_kernel<T, W, OUT, VEC><<<static_cast<unsigned>(c), 1024, 0, stream>>>(
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
    if (mx4) return launch_rows<T, W, kOutMx4, true>(xt, rt, ro, wt, n, d, eps, codes, scales, stream);
    if (d % 8 == 0)
        return launch_rows<T, W, kOutInt8, true>(xt, rt, ro, wt, n, d, eps, codes, scales, stream);
    return launch_rows<T, W, kOutInt8, false>(xt, rt, ro, wt, n, d, eps, codes, scales, stream);
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
