// MXFP4 product, dense and grouped by expert:
//   y[i, o] = sum_b 2^(ex[i, b] + ew[o, b] - 254) sum_{j in b} cx[i, j] cw[o, j]
// on the block-scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4:
// lane L holds row L % 16, elements [32 (L / 16), 32 (L / 16) + 32) of a
// step of 128 (16 bytes of codes) and that block's scale byte.  Weights are
// the first operand, so that a lane's four sums are consecutive outputs.
//
// The order of the reduction is free as long as both operands take the same,
// which every kernel here uses to load whole pieces of rows.
//
// Three forms, picked by an estimate of their times (mx4_pick.h):
//   line   few rows: small tiles, their reduction shared out among the waves of
//          a workgroup; bound by the weights' bytes
//   tile   many rows: 128 x 128, 128 x 256 or 256 x 256 outputs a workgroup;
//          bound by the copies and the matrix rate, which the power of random
//          data holds at 6.9 to 7.05 PFLOP/s of the nominal 10 (a loop of the
//          instruction alone; 6.0 is the prompt's loop without its copies)
//   split  rows of less than 512 elements, a wave for each 128 of them; bound
//          by the outputs' bytes
// Kernel times, weights in the last-level cache (rows x inputs -> outputs):
//   1 x 4096 -> 4096 3.5 us, 48 x 4096 -> 14336 7.1 to 7.5, 100 x 4096 -> 4096
//   5.9, 257 x 14336 -> 4096 22, 1000 x 4096 -> 4096 15 to 16.5, 8192 x 4096
//   -> 14336 220 to 250 (3.8 to 4.4 PFLOP/s), 8192 x 256 -> 4096 27; 128 rows of
//   64 experts 2048 -> 1024 9.5, 16384 rows of 8 uneven experts 14336 -> 4096
//   506 to 530 (3.6 to 3.8).
#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "mx4_common.h"
#include "mx4_pick.h"

namespace catk {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kMxXcd = 8;

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

// Most row tiles of bm rows that a call can have: every expert with rows may
// end inside one.
__host__ __device__ inline int64_t mx4_row_tiles_most(const Mx4Args& a, int bm) {
    return (a.m + bm - 1) / bm + (a.offsets ? (a.groups < a.m ? a.groups : a.m) : 0);
}

__device__ __forceinline__ int mx4_source_row(const Mx4Args& a, int i) {
    int s = a.row_ids ? a.row_ids[i] : i;
    return s < 0 ? 0 : (s < a.n ? s : a.n - 1);
}

__device__ __forceinline__ void mx4_store(float* y, float v) { *y = v; }
__device__ __forceinline__ void mx4_store(uint16_t* y, float v) {
    *y = static_cast<uint16_t>(pack_bf16(v, 0.0f));
}

// Four outputs of row `row` and column `col` of the tile at (first, n0), of
// which rows x cols exist.
template <typename Y>
__device__ __forceinline__ void mx4_store4(Y* y, int d_out, int first, int n0, int rows, int cols,
                                           int row, int col, f32x4 v) {
    if (row >= rows || col >= cols) return;
    y += static_cast<int64_t>(first + row) * d_out + n0 + col;
    if (col + 4 <= cols) {                 // stores of 8 and 16 bytes may start at any byte here
        if constexpr (sizeof(Y) == 4) {
            __builtin_memcpy(y, &v, 16);
        } else {
            const u32x2 p = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            __builtin_memcpy(y, &p, 8);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < cols) mx4_store(y + e, v[e]);
    }
}

// global -> LDS copies as dma16 and dma4 of the common header (16 or 4 bytes a
// lane, the lane's bytes at lds + 16 or 4 lane), with M0 as an operand that the
// compiler writes instead of saved and restored around each: a copy is then
// three instructions.  From a wave-uniform base and a 32-bit offset a lane, or
// from an address a lane.
__device__ __forceinline__ void mx4_copy16(const uint8_t* base, uint32_t off, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void mx4_copy4(const uint8_t* base, uint32_t off, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void mx4_copy16(const uint8_t* p, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void mx4_copy4(const uint8_t* p, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(p), "{m0}"(lds) : "memory");
}

// -------------------------------------------------------- tiles for short rows
// Rows of less than 512 elements, up to four chunks of 128: a workgroup owns 16
// A rows x 16 B outputs and has a wave for each chunk, which copies its A + B
// KiB of codes and their scale bytes to LDS (global -> LDS copies, all in
// flight at once) and multiplies them; the waves' partial sums are then added
// in LDS in the chunks' order.
//
// A chunk's copies: 16 rows x 64 bytes of codes per fragment (four lanes on
// 64 contiguous bytes; unit u of row r at slot 4 r + (u ^ ((r >> 2) & 3))),
// and one dword of scale bytes per row, 64 rows a copy.  Rows whose scale
// bytes are not dword-aligned (d_in % 128 != 0; ALN = false) copy the two
// aligned dwords that hold them (bytes of the buffers' last dword past its
// end are read with it, never used) and a lane picks its byte, at a place
// that depends on its row only.  Units past a row's end count as zero with
// scale 1.
//
// 8192 x 256 -> 4096 27 us and 1000 x 480 -> 4096 8.5; with eight waves of
// which half or more had no chunk, and a ring for each, 92 and 16.

// Adds the partial sums of the workgroup's waves (W at most) in the waves'
// order through LDS and stores them.
template <typename Y, int A, int B, int W, int BYTES>
__device__ __forceinline__ void mx4_join(const Mx4Args& a, const Mx4Rows& r, int n0, int waves,
                                         uint8_t (*lds)[BYTES], const f32x4 (&acc)[A][B]) {
    constexpr int RT = mx4_round(A, B, W), ROUNDS = (A * B + RT - 1) / RT;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int rows_x = r.end - r.first, rows_w = a.d_out - n0;
#pragma unroll
    for (int rd = 0; rd < ROUNDS; ++rd) {
        __syncthreads();                   // the ring (or the last round) is read
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int tl = rd * RT + t;
            if (tl < A * B) reinterpret_cast<f32x4*>(&lds[wave][0])[t * kWave + lane] = acc[tl / B][tl % B];
        }
        __syncthreads();
        for (int t = wave; t < RT; t += waves) {
            const int tl = rd * RT + t;
            if (tl >= A * B) break;
            f32x4 v = reinterpret_cast<const f32x4*>(&lds[0][0])[t * kWave + lane];
#pragma unroll
            for (int w = 1; w < W; ++w) {
                if (w >= waves) break;
                const f32x4 p = reinterpret_cast<const f32x4*>(&lds[w][0])[t * kWave + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += p[e];
            }
            // a lane holds row lane % 16, outputs 4 (lane / 16) .. + 3
            mx4_store4(static_cast<Y*>(a.y), a.d_out, r.first, n0, rows_x, rows_w,
                       (tl / B) * 16 + (lane & 15), (tl % B) * 16 + 4 * (lane >> 4), v);
        }
    }
}

template <typename Y, int A, int B, bool ALN>
__device__ __forceinline__ void mx4_split_tile(const Mx4Args& a, const Mx4Rows& r, int n0,
                                               uint8_t (*lds)[sp_wave_bytes(A, B, ALN)]) {
    constexpr int BM = 16 * A, BN = 16 * B;
    constexpr int L = A + B;               // code copies per chunk
    constexpr int SC = (L + 3) / 4;        // scale copies per chunk and dword
    constexpr int kScaleAt = L * 1024;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l16 = lane & 15, q = lane >> 4;
    const uint32_t rb = static_cast<uint32_t>(a.d_in) / 2;
    const uint32_t sb = static_cast<uint32_t>(a.d_in) / 32;
    const int chunk = wave;
    const int rows_x = r.end - r.first < BM ? r.end - r.first : BM;
    const int rows_w = a.d_out - n0 < BN ? a.d_out - n0 : BN;
    const int64_t w0 = static_cast<int64_t>(r.group) * a.d_out + n0;
    // row i of the tile's tokens (i < BM) or weights (BM + o); rows past the
    // end read the last one (their results are not stored)
    auto x_row = [&](int i) {
        return static_cast<int64_t>(mx4_source_row(a, r.first + (i < rows_x ? i : rows_x - 1)));
    };
    auto w_row = [&](int o) { return w0 + (o < rows_w ? o : rows_w - 1); };

    const uint8_t* src[L];
    const int cr = lane >> 2;
    const uint32_t cu = 16u * static_cast<uint32_t>((lane & 3) ^ ((lane >> 4) & 3));
#pragma unroll
    for (int g = 0; g < L; ++g)
        src[g] = g < A ? a.cx + x_row(16 * g + cr) * rb : a.cw + w_row(16 * (g - A) + cr) * rb;
    const uint8_t* ssrc[SC];               // scale row of lane's row 64 g + lane
    const uint8_t* send[SC];               // last aligned dword of its buffer
#pragma unroll
    for (int g = 0; g < SC; ++g) {
        const int i = 64 * g + lane < 16 * L ? 64 * g + lane : 16 * L - 1;
        const bool x = i < BM;
        ssrc[g] = x ? a.ex + x_row(i) * sb : a.ew + w_row(i - BM) * sb;
        if constexpr (!ALN) {
            const int64_t bytes = x ? static_cast<int64_t>(a.n) * sb
                                    : static_cast<int64_t>(a.groups) * a.d_out * sb;
            send[g] = (x ? a.ex : a.ew) + ((bytes - 1) & ~int64_t{3});
        }
    }
    const uint32_t at0 = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(lds_addr(&lds[wave][0])));
    uint32_t col = static_cast<uint32_t>(chunk) * 64u + cu;
    if (!ALN) col = col < rb ? col : 0;            // past the row's end: any unit of it
#pragma unroll
    for (int g = 0; g < L; ++g) mx4_copy16(src[g] + col, at0 + g * 1024u);
#pragma unroll
    for (int g = 0; g < SC; ++g) {
        const uint8_t* p = ssrc[g] + 4 * chunk;
        if constexpr (ALN) {
            mx4_copy4(p, at0 + kScaleAt + g * 256u);
        } else {
            const uint64_t lo = reinterpret_cast<uint64_t>(p) & ~uint64_t{3};
            const uint64_t end = reinterpret_cast<uint64_t>(send[g]);
            mx4_copy4(reinterpret_cast<const uint8_t*>(lo < end ? lo : end), at0 + kScaleAt + g * 256u);
            mx4_copy4(reinterpret_cast<const uint8_t*>(lo + 4 < end ? lo + 4 : end),
                      at0 + kScaleAt + (SC + g) * 256u);
        }
    }
    // byte of the lane's scale, by fragment
    int sat[L];
#pragma unroll
    for (int g = 0; g < L; ++g) {
        const int i = 16 * g + l16;
        int byte = q, dword = 0;
        if constexpr (!ALN) {
            const uint64_t row = g < A ? reinterpret_cast<uint64_t>(a.ex) + x_row(i) * sb
                                       : reinterpret_cast<uint64_t>(a.ew) + w_row(i - BM) * sb;
            const int at = static_cast<int>(row & 3) + q;
            byte = at & 3;
            dword = at >> 2;
        }
        sat[g] = kScaleAt + dword * (SC * 256) + 4 * i + byte;
    }
    wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    const int slot = 16 * (4 * l16 + (q ^ (l16 >> 2)));
    u32x4 f[L];
    int s[L];
#pragma unroll
    for (int g = 0; g < L; ++g) {
        f[g] = *reinterpret_cast<const u32x4*>(&lds[wave][g * 1024 + slot]);
        s[g] = lds[wave][sat[g]];
    }
    if (!ALN && 4 * chunk + q >= static_cast<int>(sb)) {
#pragma unroll
        for (int g = 0; g < L; ++g) {
            s[g] = kMxByteOne;
            f[g] = u32x4{0u, 0u, 0u, 0u};
        }
    }
    f32x4 acc[A][B];
#pragma unroll
    for (int i = 0; i < A; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j)
            acc[i][j] = mx4_mfma(f[A + j], f[i], f32x4{0.0f, 0.0f, 0.0f, 0.0f}, s[A + j], s[i]);

    mx4_join<Y, A, B, kSpWaves>(a, r, n0, static_cast<int>(blockDim.x) / kWave, lds, acc);
}

// The same with whole cache lines, for rows of at least 512 elements: a chunk
// is 256 elements, 128 bytes of every row (8 rows a copy).  Copies of whole
// lines reach almost twice the rate of 64-byte pieces, and what a copy costs
// grows with the rows it touches: scale bytes therefore come 32 of a row at a
// time (32 rows a copy), which serve four chunks.  Sixteen for every chunk, 64
// rows a copy, took up to a third of the time (257 x 14336 -> 4096 29 us).
// Wave w of W takes the w-th part of the chunks, in order.
//
// EX: d_in % 256 == 0, so that chunks are whole and scale bytes begin at dwords;
// windows begin where none of their 16-byte pieces passes a row's end with its
// first half in it.  Otherwise the 32 bytes serve three chunks and begin at the
// dword that holds the first one's first byte; each half of them is moved back
// where it would pass the buffer's last dword, and a lane finds its bytes in
// it; units past a row's end count as zero with scale 1.
template <typename Y, int A, int B, int D, int W, bool EX>
__device__ __forceinline__ void mx4_line_tile(const Mx4Args& a, const Mx4Rows& r, int n0,
                                              uint8_t (*lds)[ln_wave_bytes(A, B, D, W)]) {
    constexpr int BM = 16 * A, BN = 16 * B;
    constexpr int L = A + B;
    constexpr int SC = (L + 1) / 2;        // scale copies per window
    constexpr int P = EX ? 4 : 3;          // chunks per window of scale bytes
    constexpr int COPIES = 2 * L;          // per chunk, and SC before a window's first
    static_assert((COPIES + SC) * D < 64, "copies in flight must fit the vmcnt range");
    constexpr int kStageBytes = ln_stage_bytes(A, B), kScaleBytes = ln_scale_bytes(A, B);
    constexpr int kScaleAt = D * kStageBytes;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l16 = lane & 15, q = lane >> 4;
    const uint32_t rb = static_cast<uint32_t>(a.d_in) / 2;
    const uint32_t sb = static_cast<uint32_t>(a.d_in) / 32;
    const int nk = (a.d_in + 255) / 256;
    const int c0 = nk * wave / W, cnt = nk * (wave + 1) / W - c0;
    const int rows_x = r.end - r.first < BM ? r.end - r.first : BM;
    const int rows_w = a.d_out - n0 < BN ? a.d_out - n0 : BN;
    const int64_t w0 = static_cast<int64_t>(r.group) * a.d_out + n0;
    // rows past the end read the last one (their results are not stored)
    auto x_row = [&](int i) {
        return static_cast<int64_t>(mx4_source_row(a, r.first + (i < rows_x ? i : rows_x - 1)));
    };
    auto w_row = [&](int o) { return o < rows_w ? o : rows_w - 1; };

    // copy 2 f + h of a chunk: rows 8 h .. 8 h + 7 of fragment f, unit u of row
    // r at slot 8 r + (u ^ (r >> 1))
    const int cr = lane >> 3;
    const uint32_t cu = 16u * static_cast<uint32_t>((lane & 7) ^ (lane >> 4));
    const uint8_t* src_x[2 * A];
    uint32_t src_w[2 * B];
#pragma unroll
    for (int g = 0; g < 2 * A; ++g) src_x[g] = a.cx + x_row(8 * g + cr) * rb;
#pragma unroll
    for (int g = 0; g < 2 * B; ++g) src_w[g] = static_cast<uint32_t>(w_row(8 * g + cr)) * rb;
    const uint8_t* const base_w = a.cw + w0 * rb;
    // A scale row by its byte address; the last place where 16 bytes may be
    // read from its buffer.
    auto scale_row = [&](int i) {          // tokens, then weights
        return reinterpret_cast<uint64_t>(i < BM ? a.ex + x_row(i) * sb : a.ew + (w0 + w_row(i - BM)) * sb);
    };
    auto scale_most = [&](int i) {
        const uint64_t first = reinterpret_cast<uint64_t>(i < BM ? a.ex : a.ew);
        const int64_t bytes = (i < BM ? static_cast<int64_t>(a.n) : static_cast<int64_t>(a.groups) * a.d_out) * sb;
        return first + static_cast<uint64_t>((bytes - 1) & ~int64_t{3}) - 12;
    };
    // Copy g of a window: 32 bytes of rows 32 g .. 32 g + 31, half u of row r
    // at slot 2 r + (u ^ ((r >> 3) & 1)).
    const uint32_t su = 16u * static_cast<uint32_t>((lane & 1) ^ ((lane >> 4) & 1));
    uint64_t ssrc[SC], smost[SC];
#pragma unroll
    for (int g = 0; g < SC; ++g) {
        const int i = 32 * g + (lane >> 1) < 16 * L ? 32 * g + (lane >> 1) : 16 * L - 1;
        ssrc[g] = scale_row(i);
        if (!EX) {
            ssrc[g] &= ~uint64_t{3};
            smost[g] = scale_most(i);
        }
    }
    const uint32_t ring = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(lds_addr(&lds[wave][0])));
    // Whole chunks: windows begin at chunks as even or odd as the row's end.
    // The first one begins a chunk early for that, or, at the row's start, holds
    // one chunk alone.
    const int odd = EX ? (c0 ^ nk) & 1 : 0;
    const bool lone = odd && c0 == 0;
    const int w0_chunk = lone ? 0 : c0 - odd;
    // next chunk's window, its place there, the window's end and buffer
    int iw = w0_chunk, ik = c0 - w0_chunk, ie = lone ? 1 : P, ib = 0;
    // Of the wave's i-th chunk the weights and scales, the tokens, or both.
    constexpr int kWeights = 1, kTokens = 2, kBoth = 3;
    auto issue = [&](int i, int st, int part) {
        const uint32_t at = ring + static_cast<uint32_t>(st * kStageBytes);
        const int c = c0 + i;
        if ((part & kWeights) && (i == 0 || ik == 0)) {
            const uint32_t to = static_cast<uint32_t>(
                __builtin_amdgcn_readfirstlane(static_cast<int>(ring) + kScaleAt + ib * kScaleBytes));
#pragma unroll
            for (int g = 0; g < SC; ++g) {
                uint32_t off = static_cast<uint32_t>(iw) * 8u + su;
                if (EX) off = off + 16u <= sb ? off : sb - 16u;    // past the row's end: any piece of it
                uint64_t p = ssrc[g] + off;
                if (!EX) p = p < smost[g] ? p : smost[g];
                mx4_copy16(reinterpret_cast<const uint8_t*>(p), to + g * 1024u);
            }
        }
        if ((part & kWeights) && ++ik == ie) {
            iw += ie;
            ik = 0;
            ie = P;
            ib = D > 1 ? ib ^ 1 : 0;
        }
        uint32_t col[2];                   // of even and odd copies
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            col[h] = static_cast<uint32_t>(c) * 128u + (cu ^ (64u * h));
            if (!EX) col[h] = col[h] < rb ? col[h] : 0;        // past the row's end: any unit of it
        }
#pragma unroll
        for (int g = 0; g < 2 * B; ++g)
            if (part & kWeights) mx4_copy16(base_w, src_w[g] + col[g & 1], at + (2 * A + g) * 1024u);
#pragma unroll
        for (int g = 0; g < 2 * A; ++g)
            if (part & kTokens) mx4_copy16(src_x[g] + col[g & 1], at + g * 1024u);
    };
    const int at0 = 16 * (8 * l16 + (q ^ (l16 >> 1))), at1 = at0 ^ 64;
    // General rows: a lane's byte of the window at chunk w, place k, is byte
    // near + 8 k of the 32, in a half that begins 8 w + 16 u bytes behind the
    // row's dword, or at `far` where that is less.
    int near[EX ? 1 : L], far[EX ? 1 : L];
    if (!EX) {
#pragma unroll
        for (int g = 0; g < L; ++g) {
            const uint64_t row = scale_row(16 * g + l16);
            const int64_t left = static_cast<int64_t>(scale_most(16 * g + l16) - (row & ~uint64_t{3}));
            near[g] = static_cast<int>(row & 3) + q;
            far[g] = static_cast<int>(left < (1 << 30) ? left : (1 << 30));
        }
    }
    const int swap = 16 * (l16 >> 3);
    int rw = iw, rk = ik, re = ie, rs = 0;                 // the same of the next chunk read
    u32x4 f[2][L];
    int s[2][L];
    auto read = [&](int i, int st, int part) {
        const uint8_t* at = &lds[wave][st * kStageBytes];
        const uint8_t* sc = &lds[wave][kScaleAt + rs * kScaleBytes + 32 * l16];
        const int c = c0 + i;
#pragma unroll
        for (int g = 0; g < L; ++g) {
            if (part & kWeights) {
                const uint8_t* p = sc + 512 * g;
                int i0 = 8 * rk + q, i1 = i0 + 4;
                if (!EX) {                 // bytes past the row's end: any of the 32
                    i0 = near[g] + 8 * rk;
                    i1 = i0 + 4;
                    const int over0 = 8 * rw + (i0 & 16) - far[g], over1 = 8 * rw + (i1 & 16) - far[g];
                    i0 = (i0 + (over0 > 0 ? over0 : 0)) & 31;
                    i1 = (i1 + (over1 > 0 ? over1 : 0)) & 31;
                }
                s[0][g] = p[i0 ^ swap];
                s[1][g] = p[i1 ^ swap];
            }
            if (part & (g < A ? kTokens : kWeights)) {
                f[0][g] = *reinterpret_cast<const u32x4*>(at + g * 2048 + at0);
                f[1][g] = *reinterpret_cast<const u32x4*>(at + g * 2048 + at1);
            }
        }
        if ((part & kWeights) && ++rk == re) {
            rw += re;
            rk = 0;
            re = P;
            rs = D > 1 ? rs ^ 1 : 0;
        }
        if ((part & kTokens) && !EX && c == nk - 1) {      // units past the row's end
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool past = 8 * c + 4 * h + q >= static_cast<int>(sb);
#pragma unroll
                for (int g = 0; g < L; ++g) {
                    s[h][g] = past ? kMxByteOne : s[h][g];
                    f[h][g] = past ? u32x4{0u, 0u, 0u, 0u} : f[h][g];
                }
            }
        }
    };
    f32x4 acc[A][B];
#pragma unroll
    for (int i = 0; i < A; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto compute = [&]() {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < A; ++i)
#pragma unroll
                for (int j = 0; j < B; ++j)
                    acc[i][j] = mx4_mfma(f[h][A + j], f[h][i], acc[i][j], s[h][A + j], s[h][i]);
    };
#pragma unroll
    for (int st = 0; st < D; ++st)
        if (st < cnt) issue(st, st, kBoth);
    int i = 0, st = 0;
    for (; i + D < cnt; ++i) {
        wait_vmcnt<(D - 1) * COPIES>();
        asm volatile("" ::: "memory");
        if constexpr (A > 2) {
            // the weights' copies leave before the tokens are read: 48 x 4096
            // -> 14336 7.1 us, 7.6 with all of them behind all reads; with
            // fewer fragments the second wait costs as much (64 rows on 32 x
            // 64 outputs 8.4, 8.0)
            read(i, st, kWeights);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            issue(i + D, st, kWeights);
            read(i, st, kTokens);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            issue(i + D, st, kTokens);
        } else {
            read(i, st, kBoth);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            issue(i + D, st, kBoth);
        }
        compute();
        st = st + 1 == D ? 0 : st + 1;
    }
    wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    for (; i < cnt; ++i) {
        read(i, st, kBoth);
        compute();
        st = st + 1 == D ? 0 : st + 1;
    }

    mx4_join<Y, A, B, W>(a, r, n0, W, lds, acc);
}

// Tiles of the call, walked so that XCD x (workgroups are dealt to the 8 of
// them in turn) takes one contiguous range, the row tiles of a column panel
// next to each other: its weights then enter that XCD's L2 once.
template <int BM, int BN, typename F>
__device__ __forceinline__ void mx4_walk(const Mx4Args& a, F tile) {
    const int tiles_n = (a.d_out + BN - 1) / BN;
    const int64_t row_tiles = mx4_row_tiles_most(a, BM);
    const int64_t T = row_tiles * tiles_n;
    const int64_t per_xcd = (T + kMxXcd - 1) / kMxXcd;
    for (int64_t j = blockIdx.x / kMxXcd; j < per_xcd; j += gridDim.x / kMxXcd) {
        const int64_t tau = (blockIdx.x % kMxXcd) * per_xcd + j;
        if (tau >= T) return;
        const int tn = static_cast<int>(tau / row_tiles);
        Mx4Rows r;
        if (!mx4_rows<BM>(a, static_cast<int>(tau - tn * row_tiles), r)) continue;
        r.group = __builtin_amdgcn_readfirstlane(r.group);
        r.first = __builtin_amdgcn_readfirstlane(r.first);
        r.end = __builtin_amdgcn_readfirstlane(r.end);
        tile(r, tn * BN);
        __syncthreads();                   // the sums are read before the next ring
    }
}

template <typename Y, int A, int B, bool ALN>
__global__ __launch_bounds__(kSpWaves * kWave) void mx4_split_kernel(Mx4Args a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t dynamic_lds[];
    uint8_t (*const lds)[sp_wave_bytes(A, B, ALN)] = reinterpret_cast<uint8_t (*)[sp_wave_bytes(A, B, ALN)]>(dynamic_lds);
    mx4_walk<16 * A, 16 * B>(a, [&](const Mx4Rows& r, int n0) { mx4_split_tile<Y, A, B, ALN>(a, r, n0, lds); });
}

template <typename Y, int A, int B, int D, int W, bool EX>
__global__ __launch_bounds__(W * kWave) void mx4_line_kernel(Mx4Args a) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[W][ln_wave_bytes(A, B, D, W)];
    mx4_walk<16 * A, 16 * B>(a, [&](const Mx4Rows& r, int n0) { mx4_line_tile<Y, A, B, D, W, EX>(a, r, n0, lds); });
}

// ------------------------------------------------------------- large tiles
// BM rows x BN outputs per workgroup of four waves (2 x 2): a wave holds BN/2
// outputs x BM/2 rows of fp32 sums (256 registers with 256 x 256, the
// accumulation half of the register file), so that a fragment read from LDS
// serves 8 matrix instructions.  One workgroup per CU, or two with 128 x 128:
// half the copies of 64 x 64 outputs an operation where larger tiles leave CUs
// idle (1000 x 4096 -> 4096 16.5 us; 20.3 on 64 x 64, 20.9 on 128 x 256).
//
// The reduction goes in pairs of stages. A stage is 128 elements, one matrix
// step; a pair is 128 bytes of every row, a whole cache line: global -> LDS
// copies (global_load_lds_dwordx4) of rows of 64 bytes reach 27 to 34 bytes
// per clock and CU with all CUs reading, of 128 bytes 53.  Two pairs fit the
// LDS.  In a stage a wave multiplies its BN/32 weight fragments, read during the
// stage before, with token fragments that it reads three ahead of their use.
// After the last token fragment of a pair's second stage has been read there
// is a barrier: behind it the pair's buffer is free, the next pair but one is
// requested into it, and (vmcnt) the next pair has arrived.
//
// Scale bytes come in 16 a row, two pairs, likewise straight into LDS; a lane
// keeps the four of its block column in one register, whose byte s the matrix
// instruction of stage s selects.
//
// Workgroups are persistent and their tiles form one stream of pairs, so the
// requests run ahead across tiles; past the last one they repeat the last
// tile's first ones, which keeps the stages free of branches.
//
// LDS: unit u (16 bytes) of row r sits at slot 8 r + (u ^ ((r >> 1) & 7)): a
// fragment's 16 rows at one unit fall on 16 different 16-byte bank groups.
constexpr int kTlThreads = 256;
constexpr int kTlUnits = 8;                // 16-byte units of a row per pair of stages
constexpr int kTlPair = 256;               // elements of the reduction per pair
constexpr int kTlGroupM = 4;               // row panels that are walked together

// Row tiles of the call.
template <int BM>
__device__ __forceinline__ int mx4_row_tiles(const Mx4Args& a) {
    if (!a.offsets) return (a.m + BM - 1) / BM;
    const int lane = threadIdx.x & (kWave - 1);
    int tiles = 0;
    for (int g = lane; g < a.groups; g += kWave) {
        int lo = a.offsets[g], hi = a.offsets[g + 1];
        lo = lo < 0 ? 0 : (lo > a.m ? a.m : lo);
        hi = hi < lo ? lo : (hi > a.m ? a.m : hi);
        tiles += (hi - lo + BM - 1) / BM;
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) tiles += __shfl_xor(tiles, o);
    // offsets that decrease could give more: never more work than that
    const int64_t most = mx4_row_tiles_most(a, BM);
    return tiles < 0 || tiles > most ? static_cast<int>(most) : tiles;
}

// One matrix step with scale byte S of sw and sx, the sum in place in the
// accumulation registers.  Written as an instruction because a wave's sums
// fill that half of the register file: left to the builtin, they are moved
// back and forth between the halves.  A sum is used again no sooner than 16
// steps later, so the steps need no waits among each other.
template <int S>
__device__ __forceinline__ void mx4_mfma_acc(u32x4 a, u32x4 b, f32x4& acc, int sw, int sx) {
    static_assert(S >= 0 && S < 4, "scale byte");
#define CAT_MFMA(SEL)                                                                         \
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 " SEL " cbsz:4 blgp:4" \
                 : "+a"(acc)                                                                  \
                 : "v"(a), "v"(b), "v"(sw), "v"(sx))
    if constexpr (S == 0) CAT_MFMA("op_sel:[0,0,0] op_sel_hi:[0,0,0]");
    if constexpr (S == 1) CAT_MFMA("op_sel:[1,1,0] op_sel_hi:[0,0,0]");
    if constexpr (S == 2) CAT_MFMA("op_sel:[0,0,0] op_sel_hi:[1,1,0]");
    if constexpr (S == 3) CAT_MFMA("op_sel:[1,1,0] op_sel_hi:[1,1,0]");
#undef CAT_MFMA
}

template <typename Y, int BM, int BN, bool EX>
__global__ __launch_bounds__(kTlThreads, BN == 128 ? 2 : 1) void mx4_tile_kernel(Mx4Args a) {
    constexpr int IO = BN / 32;            // 16-output fragments of a wave
    constexpr int IT = BM / 32;            // 16-row fragments of a wave
    constexpr int ROWS = BN + BM;          // LDS rows: weights, then tokens
    constexpr int LW = BN / 32, LX = BM / 32;     // copies a wave and pair
    constexpr int NL = LW + LX, NM = IO * IT;
    constexpr int XB = 4;                  // token fragments in registers
    constexpr int WN = BN / 2, LPR = BN / 16;       // outputs of a wave, lanes that store a row of them
    __shared__ __attribute__((aligned(16))) u32x4 codes[2][ROWS * kTlUnits];
    __shared__ __attribute__((aligned(16))) u32x4 scales[2][ROWS];
    __shared__ __attribute__((aligned(16))) u32x4 outs[kTlThreads / kWave][BN];

    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wo = wave & 1, wt = wave >> 1;
    const int l16 = lane & 15, q = lane >> 4;
    const uint32_t rb = static_cast<uint32_t>(a.d_in) / 2;       // bytes of a code row
    const uint32_t sb = static_cast<uint32_t>(a.d_in) / 32;      // bytes of a scale row
    const int np = (a.d_in + 2 * kTlPair - 1) / (2 * kTlPair) * 2;      // even

    // Tiles are numbered so that each XCD (workgroups are dealt to the 8 of
    // them in turn) walks one contiguous range, kTlGroupM row panels at a
    // time: the workgroups of an XCD share panels in its L2.
    const int tiles_m = __builtin_amdgcn_readfirstlane(mx4_row_tiles<BM>(a));
    const int tiles_n = (a.d_out + BN - 1) / BN;
    const int64_t T = static_cast<int64_t>(tiles_m) * tiles_n;
    const int64_t per_xcd = (T + kMxXcd - 1) / kMxXcd;
    const int64_t wg_per_xcd = gridDim.x / kMxXcd;
    struct Tile {
        int group, first, end, n0;
    };
    auto tile_at = [&](int64_t k, Tile& t) {
        const int64_t local = blockIdx.x / kMxXcd + k * wg_per_xcd;
        const int64_t tau = (blockIdx.x % kMxXcd) * per_xcd + local;
        if (local >= per_xcd || tau >= T) return false;
        const int64_t panel = tau / (static_cast<int64_t>(kTlGroupM) * tiles_n);
        const int m1 = static_cast<int>(panel) * kTlGroupM;
        const int gm = tiles_m - m1 < kTlGroupM ? tiles_m - m1 : kTlGroupM;
        const int in = static_cast<int>(tau - panel * kTlGroupM * tiles_n);
        Mx4Rows r;
        if (!mx4_rows<BM>(a, m1 + in % gm, r)) return false;
        t.group = __builtin_amdgcn_readfirstlane(r.group);
        t.first = __builtin_amdgcn_readfirstlane(r.first);
        t.end = __builtin_amdgcn_readfirstlane(r.end);
        t.n0 = in / gm * BN;
        return true;
    };

    // ---- the load cursor: the tile and pair requested next
    Tile lt{};
    int64_t lk = 0;                        // its number in this workgroup's list
    int ls = 0;                            // its next pair
    if (!tile_at(0, lt)) return;
    Tile tile = lt;
    // Copy j of this wave fills the 64 slots of 8 rows: weights' rows
    // 8 (4 j + wave) .. + 7, then the tokens' likewise.
    const uint32_t unit = 16u * static_cast<uint32_t>((lane & 7) ^ ((lane >> 4) | ((wave & 1) << 2)));
    const uint8_t *base_w, *base_x, *base_sw, *base_sx;
    uint32_t off_w[LW], off_x[LX], off_sw, off_sx;
    // general rows: base_sw and base_sx are dword-aligned, and these the last
    // offsets from them where 16 bytes may be read
    uint32_t most_sw = 0, most_sx = 0;
    auto set_rows = [&]() {
        const int64_t w0 = static_cast<int64_t>(lt.group) * a.d_out + lt.n0;
        base_w = a.cw + w0 * rb;
        base_sw = a.ew + w0 * sb;
        const int left_w = a.d_out - lt.n0 < BN ? a.d_out - lt.n0 : BN;
        const int left_x = lt.end - lt.first < BM ? lt.end - lt.first : BM;
        const uint32_t in_row = EX ? unit : 0u;
        // rows past the end read the last one (their results are not stored)
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const int r = 8 * (4 * j + wave) + (lane >> 3);
            off_w[j] = static_cast<uint32_t>(r < left_w ? r : left_w - 1) * rb + in_row;
        }
        const int rw = 64 * wave + lane;
        off_sw = static_cast<uint32_t>(rw < left_w ? rw : left_w - 1) * sb;
        const bool by_id = a.row_ids != nullptr;
        base_x = a.cx + (by_id ? 0 : static_cast<int64_t>(lt.first) * rb);
        base_sx = a.ex + (by_id ? 0 : static_cast<int64_t>(lt.first) * sb);
        auto src = [&](int r) {
            const int c = r < left_x ? r : left_x - 1;
            return static_cast<uint32_t>(by_id ? mx4_source_row(a, lt.first + c) : c);
        };
#pragma unroll
        for (int j = 0; j < LX; ++j) off_x[j] = src(8 * (4 * j + wave) + (lane >> 3)) * rb + in_row;
        off_sx = src(64 * wave + lane) * sb;
        if (!EX) {
            auto align = [&](const uint8_t*& base, uint32_t& off, const uint8_t* first, int64_t rows) {
                const uint32_t low = static_cast<uint32_t>(reinterpret_cast<uint64_t>(base)) & 3u;
                base -= low;
                off += low;
                const int64_t at = ((rows * sb - 1) & ~int64_t{3}) - 12 - (base - first);
                return static_cast<uint32_t>(at < (int64_t{1} << 31) ? at : (int64_t{1} << 31));
            };
            most_sw = align(base_sw, off_sw, a.ew, static_cast<int64_t>(a.groups) * a.d_out);
            most_sx = align(base_sx, off_sx, a.ex, a.n);
        }
    };
    set_rows();
    const uint32_t lds_codes =
        static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(lds_addr(&codes[0][0]))) +
        static_cast<uint32_t>(wave) * 1024u;
    const uint32_t lds_scales =
        static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(lds_addr(&scales[0][0]))) +
        static_cast<uint32_t>(wave) * 1024u;
    auto load_codes = [&](int j, int buf) {            // j < NL
        const uint32_t dst = lds_codes + static_cast<uint32_t>(buf) * (ROWS * kTlUnits * 16u);
        const uint32_t col = static_cast<uint32_t>(ls) * 128u;
        // general rows: past the end any unit of the row
        const uint32_t at = EX ? 0u : (col + unit < rb ? col + unit : 0u);
        if (j < LW) mx4_copy16(base_w + (EX ? col : 0u), off_w[j] + at, dst + static_cast<uint32_t>(j) * 4096u);
        else mx4_copy16(base_x + (EX ? col : 0u), off_x[j - LW] + at, dst + BN * 128u + static_cast<uint32_t>(j - LW) * 4096u);
    };
    uint32_t load_super = 0;               // byte offset of the cursor's scale buffer
    // General rows: the 16 bytes lie in the five dwords from the one that holds
    // the first of them, the fifth copied to the wave's output space (which is
    // not in use then; without it where rows begin at dwords).  At the buffer's
    // end the 16 bytes begin earlier.
    const bool fifths = sb % 4 != 0;
    const uint32_t lds_fifth = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(lds_addr(&outs[wave][0])));
    auto load_scales = [&]() {             // before the codes of an even pair
        const uint32_t dst = lds_scales + load_super, col = static_cast<uint32_t>(ls) * 8u;
        if (EX) {
            if (BN == 256 || wave < BN / 64) mx4_copy16(base_sw + col, off_sw, dst);
            if (BM == 256 || wave < BM / 64) mx4_copy16(base_sx + col, off_sx, dst + BN * 16u);
        } else {
            const uint32_t w = (off_sw & ~3u) + col, x = (off_sx & ~3u) + col;
            if (BN == 256 || wave < BN / 64) {
                mx4_copy16(base_sw, w < most_sw ? w : most_sw, dst);
                if (fifths) mx4_copy4(base_sw, w + 4 < most_sw ? w + 16 : most_sw + 12, lds_fifth);
            }
            if (BM == 256 || wave < BM / 64) {
                mx4_copy16(base_sx, x < most_sx ? x : most_sx, dst + BN * 16u);
                if (fifths) mx4_copy4(base_sx, x + 4 < most_sx ? x + 16 : most_sx + 12, lds_fifth + 256u);
            }
        }
        load_super ^= ROWS * 16u;
    };
    // general rows: the token units past the end of pair `pair` in buffer `buf`
    // count as zero
    auto clear_tail = [&](int pair, int buf) {
        if (EX || static_cast<uint32_t>(pair) * 128u + 128u <= rb) return;
        if (static_cast<uint32_t>(pair) * 128u + unit < rb) return;
#pragma unroll
        for (int j = 0; j < LX; ++j)
            codes[buf][BN * kTlUnits + (4 * j + wave) * kWave + lane] = u32x4{0u, 0u, 0u, 0u};
    };

    // ---- fragments
    u32x4 fw[2][IO], fx[XB];
    int sw[IO], sx[IT];
    // lane (l16, q) reads row l16, unit 4 (stage % 2) + q
    const int at0 = l16 * kTlUnits + (q ^ (l16 >> 1)), at1 = at0 ^ 4;
    const u32x4* const rd_w = &codes[0][wo * WN * kTlUnits];
    const u32x4* const rd_x = &codes[0][(BN + wt * (BM / 2)) * kTlUnits];
    auto frag_at = [&](int st, int i) {    // stage 0 .. 3: pair st / 2, half st % 2
        return (st / 2) * (ROWS * kTlUnits) + i * 16 * kTlUnits + (st % 2 ? at1 : at0);
    };
    auto read_w = [&](int i, int st) { fw[st % 2][i] = rd_w[frag_at(st, i)]; };
    auto read_x = [&](int j, int st) { fx[j % XB] = rd_x[frag_at(st, j)]; };
    // Scale bytes: the lane that copied a row's 16 bytes (byte 4 s + q for
    // stage s, block column q) turns them in place into four dwords by q, byte
    // s for stage s, once they have arrived.  A fragment's dword then needs no
    // arithmetic: a vector instruction's result may be read by a matrix
    // instruction only two wait states later, and the compiler does not see
    // the ones written as text.
    uint32_t turn_super = 0;
    auto turn = [&](u32x4* p, const uint32_t* fifth, uint32_t off, uint32_t most, int pair) {
        u32x4 v = *p;
        if (!EX) {
            uint32_t w[5] = {v[0], v[1], v[2], v[3], *fifth};
            const uint32_t at = (off & ~3u) + static_cast<uint32_t>(pair) * 8u;
            const uint32_t early = at > most ? (at - most) / 4u : 0u;      // dwords
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = early > t ? w[i + 1] : w[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = __builtin_amdgcn_alignbyte(w[i + 1], w[i], off & 3u);
                // blocks past the row's end: scale 1
                const int left = static_cast<int>(sb) - pair * 8 - 4 * i;
                const uint32_t keep = left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
                v[i] = (v[i] & keep) | (0x7F7F7F7Fu & ~keep);
            }
        }
        const uint32_t a0 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u);    // 00 10 01 11
        const uint32_t a1 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u);    // 02 12 03 13
        const uint32_t b0 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u);
        const uint32_t b1 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
        *p = u32x4{__builtin_amdgcn_perm(b0, a0, 0x05040100u), __builtin_amdgcn_perm(b0, a0, 0x07060302u),
                   __builtin_amdgcn_perm(b1, a1, 0x05040100u), __builtin_amdgcn_perm(b1, a1, 0x07060302u)};
    };
    auto turn_scales = [&](int pair) {     // of this pair and the next
        u32x4* const p = &scales[0][turn_super + 64 * wave + lane];
        const uint32_t* const fifth = reinterpret_cast<const uint32_t*>(&outs[wave][0]) + lane;
        if (BN == 256 || wave < BN / 64) turn(p, fifth, off_sw, most_sw, pair);
        if (BM == 256 || wave < BM / 64) turn(p + BN, fifth + kWave, off_sx, most_sx, pair);
        turn_super ^= ROWS;
    };
    const int* const rd_sw = reinterpret_cast<const int*>(&scales[0][wo * WN + l16]) + q;
    const int* const rd_sx = reinterpret_cast<const int*>(&scales[0][BN + wt * (BM / 2) + l16]) + q;
    uint32_t read_super = 0;
    auto read_sw = [&](int i) { sw[i] = rd_sw[read_super + 64 * i]; };
    auto read_sx = [&](int j) { sx[j] = rd_sx[read_super + 64 * j]; };

    f32x4 acc[IO][IT];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < IO; ++i)
#pragma unroll
            for (int j = 0; j < IT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    };

    // Accumulator (i, j) holds outputs WN wo + 16 i + 4 q + e of row (BM/2) wt
    // + 16 j + l16.  Sixteen rows at a time pass through LDS of the wave's own
    // (16-byte unit u of row r at u ^ (r % LPR)), so that LPR lanes store 256
    // (128 with BN = 128) contiguous bytes of a row: stored from the
    // accumulators, pieces of 32 bytes, a prefill's y took 68 us of 289.
    u32x4* const out_lds = &outs[wave][0];
    // FULL: all of the wave's outputs exist, and rows are addressed by 32-bit
    // offsets from its first one.
    auto store_as = [&](const Tile& t, auto full_) {
        constexpr bool FULL = decltype(full_)::value;
        // what depends on the lane is computed here again: kept through the
        // stages it would take their registers
        int el = lane;
        asm volatile("" : "+v"(el));
        const int l16 = el & 15, q = el >> 4;
        // The last matrix step's result takes up to 18 wait states; the reads
        // below come behind them because they take `ready`.  They read in
        // place: as ordinary values all 256 sums would change registers.
        int ready;
        asm volatile("s_nop 15\n\ts_nop 15\n\ts_mov_b32 %0, 0" : "=s"(ready)::"memory");
        auto sum = [&](int i, int j, int e) {
            float v;
            asm("v_accvgpr_read_b32 %0, %1 ; %2" : "=v"(v) : "a"(acc[i][j][e]), "s"(ready));
            return v;
        };
        constexpr int PER = 16 / sizeof(Y);            // outputs of a unit
        constexpr int PARTS = sizeof(Y) == 4 ? 2 : 1;  // pieces of a wave's row, LPR units each
        constexpr int RPL = kWave / LPR;               // rows a store
        const int lr = el / LPR, lu = el % LPR;
        const int rows = t.end - t.first - wt * (BM / 2), cols = a.d_out - t.n0 - wo * WN;
        Y* const yw = static_cast<Y*>(a.y) + static_cast<int64_t>(t.first + wt * (BM / 2)) * a.d_out + t.n0 + wo * WN;
        const uint32_t pitch = static_cast<uint32_t>(a.d_out) * sizeof(Y);
        const uint32_t at = static_cast<uint32_t>(lr) * pitch + static_cast<uint32_t>(lu) * 16u;
#pragma unroll
        for (int j = 0; j < IT; ++j) {
#pragma unroll
            for (int h = 0; h < PARTS; ++h) {
#pragma unroll
                for (int ii = 0; ii < IO / PARTS; ++ii) {
                    const int i = h * (IO / PARTS) + ii;
                    const float v0 = sum(i, j, 0), v1 = sum(i, j, 1), v2 = sum(i, j, 2), v3 = sum(i, j, 3);
                    if constexpr (sizeof(Y) == 4) {
                        out_lds[l16 * LPR + ((4 * ii + q) ^ (l16 % LPR))] =
                            u32x4{__float_as_uint(v0), __float_as_uint(v1), __float_as_uint(v2), __float_as_uint(v3)};
                    } else {
                        reinterpret_cast<u32x2*>(&out_lds[l16 * LPR + ((2 * ii + (q >> 1)) ^ (l16 % LPR))])[q & 1] =
                            u32x2{pack_bf16(v0, v1), pack_bf16(v2, v3)};
                    }
                }
                u32x4 v[16 / RPL];
#pragma unroll
                for (int r = 0; r < 16 / RPL; ++r) {
                    const int row = RPL * r + lr;
                    v[r] = out_lds[row * LPR + (lu ^ (row % LPR))];
                }
                const int c = h * (WN / PARTS) + lu * PER;
#pragma unroll
                for (int r = 0; r < 16 / RPL; ++r) {
                    const int row = 16 * j + RPL * r + lr;
                    // 16-byte stores may start at any byte here
                    if constexpr (FULL) {
                        char* const base = reinterpret_cast<char*>(yw + h * (WN / PARTS)) + static_cast<uint64_t>(16 * j + RPL * r) * pitch;
                        __builtin_memcpy(base + at, &v[r], 16);
                    } else if (row < rows && c < cols) {
                        Y* const y = yw + static_cast<int64_t>(row) * a.d_out + c;
                        if (c + PER <= cols) {
                            __builtin_memcpy(y, &v[r], 16);
                        } else {
#pragma unroll
                            for (int e = 0; e < PER; ++e) {
                                if (c + e >= cols) continue;
                                if constexpr (sizeof(Y) == 4) y[e] = __uint_as_float(v[r][e]);
                                else y[e] = static_cast<uint16_t>(v[r][e / 2] >> (16 * (e % 2)));
                            }
                        }
                    }
                }
            }
        }
    };
    auto store = [&](const Tile& t) {
        const bool full = t.end - t.first - wt * (BM / 2) >= BM / 2 && a.d_out - t.n0 - wo * WN >= WN;
        if (full && a.d_out < (1 << 22)) store_as(t, std::true_type{});
        else store_as(t, std::false_type{});
    };

    // The barrier of a stage comes behind row IT - 4 of its matrix steps; the
    // AFTER steps that follow it are where the next stage's first fragments
    // are read.  Copy c of a pair is issued SP c steps behind the barrier of a
    // second stage, the last ones in the stage after it.
    constexpr int BAR = (IT - 3) * IO - 1, AFTER = NM - 1 - BAR, SP = IT / 2;
    constexpr int BEGUN = AFTER / SP + 1 < NL ? AFTER / SP + 1 : NL;   // copies issued before that stage ends
    static_assert((NL - 1) * SP < AFTER + BAR, "copies are issued before the scales are waited for");

    // ---- prologue: pair 0 and the begun part of pair 1 (np >= 2)
    load_scales();
#pragma unroll
    for (int j = 0; j < NL; ++j) load_codes(j, 0);
    ls = 1;
#pragma unroll
    for (int j = 0; j < BEGUN; ++j) load_codes(j, 1);
    wait_vmcnt<BEGUN>();
    asm volatile("" ::: "memory");
    turn_scales(0);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < IO; ++i) {
        read_w(i, 0);
        read_sw(i);
    }
#pragma unroll
    for (int j = 0; j < IT; ++j) read_sx(j);
#pragma unroll
    for (int j = 0; j < XB - 1; ++j) read_x(j, 0);
    clear();

    auto copy_at = [&](int steps, int buf) {   // copies due `steps` behind the barrier
        if (steps % SP == 0 && steps / SP < NL) load_codes(steps / SP, buf);
    };
    auto stage = [&](auto st_) {
        constexpr int B = decltype(st_)::value, N = (B + 1) % 4;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            const int j = m / IO, i = m % IO;
            mx4_mfma_acc<B>(fw[B % 2][i], fx[j % XB], acc[i][j], sw[i], sx[j]);
            if (i == 0 && j + XB - 1 < IT) read_x(j + XB - 1, B);
            if (m == BAR) {
                if (B % 2 == 1) {
                    wait_vmcnt<0>();
                    if (!EX) clear_tail(ls > 0 ? ls - 1 : np - 1, B == 1 ? 1 : 0);
                    lds_barrier();
                    if (B == 1) load_scales();
                } else if (B == 2) {
                    wait_vmcnt<NL>();
                    asm volatile("" ::: "memory");
                    turn_scales(ls);
                }
                if (B == 3) {
                    read_super ^= 4 * ROWS;
#pragma unroll
                    for (int e = 0; e <= j; ++e) read_sx(e);
                }
            }
            // copies: into buffer 0 behind stage 1's barrier, 1 behind stage 3's
            if (B % 2 == 1 && m >= BAR) copy_at(m - BAR, B / 2);
            if (B % 2 == 0) copy_at(m + 1 + AFTER, N == 3 ? 0 : 1);
            // next stage's fragments: of another pair only behind the barrier
            if (i == 0 && j + XB - 1 >= IT) read_x(j + XB - 1 - IT, N);
            if (B % 2 == 1) {
                if (m > BAR && (m - BAR) % 3 == 2 && (m - BAR) / 3 < IO) read_w((m - BAR) / 3, N);
            } else if (m % (NM / IO) == NM / IO / 2) {
                read_w(m / (NM / IO), N);
            }
            // the next two pairs' scales, each behind its last use
            if (B == 3 && i == IO - 1 && m > BAR) read_sx(j);
            if (B == 3 && j == IT - 1) read_sw(i);
        }
        if (B % 2 == 0) {
            ++ls;
            if (B == 0 && ls == np) {      // after an odd pair only
                ls = 0;
                if (tile_at(++lk, lt)) set_rows();
            }
        }
    };
    for (int64_t k = 0;;) {
        for (int p = 0; p < np; p += 2) {
            stage(std::integral_constant<int, 0>{});
            stage(std::integral_constant<int, 1>{});
            stage(std::integral_constant<int, 2>{});
            stage(std::integral_constant<int, 3>{});
        }
        store(tile);
        if (!tile_at(++k, tile)) break;
        clear();
    }
    wait_vmcnt<0>();                       // the requests past the last pair
}

// ---------------------------------------------------------------- dispatch
// A launch covers fewer than 2^32 threads; workgroups then take several tiles.
constexpr int64_t kSpMaxGrid = int64_t{1} << 22;
static unsigned small_grid(const Mx4Args& a, int bm, int bn) {
    const int64_t T = mx4_row_tiles_most(a, bm) * ((a.d_out + bn - 1) / bn);
    const int64_t wgs = (T + kMxXcd - 1) / kMxXcd * kMxXcd;
    return static_cast<unsigned>(wgs < kSpMaxGrid ? wgs : kSpMaxGrid);
}

template <typename Y, bool ALN>
static hipError_t launch_split(const Mx4Args& a, int tile, hipStream_t stream) {
    const int waves = (a.d_in + 127) / 128;
    switch (tile) {
#define CAT_CASE(id, A, B)                                                                \
    case id:                                                                              \
        mx4_split_kernel<Y, A, B, ALN><<<small_grid(a, 16 * A, 16 * B), waves * kWave,    \
                                         waves * sp_wave_bytes(A, B, ALN), stream>>>(a);  \
        break;
        CAT_SPLIT_TILES(CAT_CASE)
#undef CAT_CASE
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <typename Y, bool EX>
static hipError_t launch_line(const Mx4Args& a, int tile, hipStream_t stream) {
    switch (tile) {
#define CAT_CASE(id, A, B, D, W)                                                          \
    case id:                                                                              \
        mx4_line_kernel<Y, A, B, D, W, EX>                                                \
            <<<small_grid(a, 16 * A, 16 * B), W * kWave, 0, stream>>>(a);                 \
        break;
        CAT_LINE_TILES(CAT_CASE)
#undef CAT_CASE
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <typename Y, int BM, int BN, bool EX>
static hipError_t launch_tiles(const Mx4Args& a, int cus, hipStream_t stream) {
    const unsigned grid = static_cast<unsigned>(cus >= kMxXcd ? cus / kMxXcd * kMxXcd : kMxXcd) * (BN == 128 ? 2 : 1);
    mx4_tile_kernel<Y, BM, BN, EX><<<grid, kTlThreads, 0, stream>>>(a);
    return hipGetLastError();
}

// CUs of the current device, asked once a device: the question takes 0.3 us of
// a call's 4.
static hipError_t device_cus(int& cus) {
    constexpr int kKept = 64;
    static std::atomic<int> kept[kKept];
    int dev = 0;
    hipError_t err = hipGetDevice(&dev);
    if (err != hipSuccess) return err;
    cus = dev < kKept ? kept[dev].load(std::memory_order_relaxed) : 0;
    if (cus > 0) return hipSuccess;
    err = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
    if (err == hipSuccess && dev < kKept) kept[dev].store(cus, std::memory_order_relaxed);
    return err;
}

template <typename Y, bool EX>
static hipError_t launch_tile(const Mx4Args& a, int shape, int cus, hipStream_t stream) {
    if (shape == 0) return launch_tiles<Y, 128, 128, EX>(a, cus, stream);
    if (shape == 1) return launch_tiles<Y, 128, 256, EX>(a, cus, stream);
    return launch_tiles<Y, 256, 256, EX>(a, cus, stream);
}

template <typename Y>
static hipError_t launch(const Mx4Args& a, hipStream_t stream) {
    int cus = 0;
    const hipError_t err = device_cus(cus);
    if (err != hipSuccess) return err;
    const Mx4Sizes z{a.n, a.m, a.groups, a.d_in, a.d_out, a.offsets != nullptr, a.row_ids != nullptr};
    const Mx4Pick p = mx4_pick(z, cus);
    switch (p.form) {
        case Mx4Form::split:
            return p.whole ? launch_split<Y, true>(a, p.shape, stream) : launch_split<Y, false>(a, p.shape, stream);
        case Mx4Form::line:
            return p.whole ? launch_line<Y, true>(a, p.shape, stream) : launch_line<Y, false>(a, p.shape, stream);
        case Mx4Form::tile: break;
    }
    return p.whole ? launch_tile<Y, true>(a, p.shape, cus, stream) : launch_tile<Y, false>(a, p.shape, cus, stream);
}

hipError_t launch_mx4_linear(const uint8_t* cx, const uint8_t* ex, const uint8_t* cw,
                             const uint8_t* ew, int64_t n, int64_t d_in, int64_t d_out, void* y,
                             int y_bf16, hipStream_t stream) {
    const Mx4Args a{cx, ex, cw, ew, nullptr, nullptr, y, static_cast<int>(n), static_cast<int>(n), 1,
                    static_cast<int>(d_in), static_cast<int>(d_out)};
    return y_bf16 ? launch<uint16_t>(a, stream) : launch<float>(a, stream);
}

hipError_t launch_mx4_linear_grouped(const uint8_t* cx, const uint8_t* ex, int64_t n,
                                     const int32_t* row_ids, int64_t m, const int32_t* offsets,
                                     int64_t groups, const uint8_t* cw, const uint8_t* ew,
                                     int64_t d_in, int64_t d_out, void* y, int y_bf16,
                                     hipStream_t stream) {
    const Mx4Args a{cx, ex, cw, ew, row_ids, offsets, y, static_cast<int>(n), static_cast<int>(m),
                    static_cast<int>(groups), static_cast<int>(d_in), static_cast<int>(d_out)};
    return y_bf16 ? launch<uint16_t>(a, stream) : launch<float>(a, stream);
}

}  // namespace catk
