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

// ------------------------------------------------------------- large tiles
// BM rows x 256 outputs per workgroup of four waves (2 x 2), one workgroup
// per CU: a wave holds 128 outputs x BM/2 rows of fp32 sums (256 registers
// with BM = 256, the accumulation half of the register file), so a fragment
// read from LDS serves 8 matrix instructions.
//
// A stage is 128 elements of the reduction, 64 bytes of every row: one matrix
// step.  Stages go from global memory into a ring of four LDS buffers with
// global_load_lds_dwordx4, requested three ahead.  During stage h a wave
// multiplies its weight fragments (read during h - 1) with the token
// fragments of h (read three fragments ahead of their use), reads the weight
// fragments of h + 1 and requests stage h + 3 into the buffer of h - 1.  One
// barrier a stage: behind it all waves are done with h - 1, and (vmcnt) h + 1
// has arrived.
//
// Scale bytes come in 16 a row, four stages, likewise straight into LDS; a
// lane reads a row's 16 bytes and keeps the four of its block column q (byte
// 4 s + q for stage s) in one register, whose byte s the matrix instruction
// of stage s selects.
//
// Workgroups are persistent and their tiles form one stream of stages, so
// the requests run ahead across tiles; past the last stage they repeat the
// last tile's first ones, which keeps the stages free of branches.
//
// LDS: unit u (16 bytes) of row r sits at slot 4 r + (u ^ ((r >> 2) & 3)): a
// fragment's 16 rows at one unit fall on 16 different 16-byte bank groups.
constexpr int kTlThreads = 256;
constexpr int kTlN = 256;                  // outputs per tile
constexpr int kTlUnits = 4;                // 16-byte units of a row per stage
constexpr int kTlStage = 128;              // elements of the reduction per stage
constexpr int kTlRing = 4;
constexpr int kTlGroupM = 4;               // row panels that are walked together
constexpr int kMxXcd = 8;

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
    return tiles;
}

// One matrix step with scale byte S of sw and sx, the sum in place in the
// accumulation registers.  Written as an instruction because a wave's sums
// fill that half of the register file: left to the builtin, they are moved
// back and forth between the halves.  The steps' sums are used again no
// sooner than NM / 2 steps later, so they need no waits among each other.
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

template <typename Y, int BM>
__global__ __launch_bounds__(kTlThreads, 1) void mx4_tile_kernel(Mx4Args a) {
    constexpr int IO = 8;                  // 16-output fragments of a wave
    constexpr int IT = BM / 32;            // 16-row fragments of a wave
    constexpr int ROWS = kTlN + BM;        // LDS rows: weights, then tokens
    constexpr int LW = kTlN / 64, LX = BM / 64;     // direct loads a wave and stage
    constexpr int NL = LW + LX, NM = IO * IT;
    constexpr int XB = 4;                  // token fragments in registers
    __shared__ __attribute__((aligned(16))) u32x4 codes[kTlRing][ROWS * kTlUnits];
    __shared__ __attribute__((aligned(16))) u32x4 scales[2][ROWS];

    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wo = wave & 1, wt = wave >> 1;
    const int l16 = lane & 15, q = lane >> 4;
    const uint32_t rb = static_cast<uint32_t>(a.d_in) / 2;       // bytes of a code row
    const uint32_t sb = static_cast<uint32_t>(a.d_in) / 32;      // bytes of a scale row
    const int nk = a.d_in / kTlStage;      // a multiple of 4

    // Tiles are numbered so that each XCD (workgroups are dealt to the 8 of
    // them in turn) walks one contiguous range, kTlGroupM row panels at a
    // time: the workgroups of an XCD share panels in its L2.
    const int tiles_m = __builtin_amdgcn_readfirstlane(mx4_row_tiles<BM>(a));
    const int tiles_n = (a.d_out + kTlN - 1) / kTlN;
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
        t.n0 = in / gm * kTlN;
        return true;
    };

    // ---- the load cursor: the tile and stage requested next
    Tile lt{};
    int64_t lk = 0;                        // its number in this workgroup's list
    int ls = 0;                            // its next stage
    if (!tile_at(0, lt)) return;
    Tile tile = lt;
    // Direct load j of this wave fills the 64 slots of 16 rows: weights' rows
    // 16 (4 j + wave) .. + 15, then the tokens' likewise.
    const uint32_t unit = 16u * static_cast<uint32_t>((lane & 3) ^ ((lane >> 4) & 3));
    const uint8_t *base_w, *base_x, *base_sw, *base_sx;
    uint32_t off_w[LW], off_x[LX], off_sw, off_sx;
    auto set_rows = [&]() {
        const int64_t w0 = static_cast<int64_t>(lt.group) * a.d_out + lt.n0;
        base_w = a.cw + w0 * rb;
        base_sw = a.ew + w0 * sb;
        const int left_w = a.d_out - lt.n0 < kTlN ? a.d_out - lt.n0 : kTlN;
        const int left_x = lt.end - lt.first < BM ? lt.end - lt.first : BM;
        // rows past the end read the last one (their results are not stored)
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const int r = 16 * (4 * j + wave) + (lane >> 2);
            off_w[j] = static_cast<uint32_t>(r < left_w ? r : left_w - 1) * rb + unit;
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
        for (int j = 0; j < LX; ++j) off_x[j] = src(16 * (4 * j + wave) + (lane >> 2)) * rb + unit;
        off_sx = src(64 * wave + lane) * sb;
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
        if (j < LW) dma16(base_w + ls * 64, off_w[j], dst + static_cast<uint32_t>(j) * 4096u);
        else dma16(base_x + ls * 64, off_x[j - LW], dst + kTlN * 64u + static_cast<uint32_t>(j - LW) * 4096u);
    };
    uint32_t load_super = 0;               // byte offset of the cursor's scale buffer
    auto load_scales = [&]() {             // before the loads of a stage that is 0 modulo 4
        const uint32_t dst = lds_scales + load_super;
        dma16(base_sw + ls * 4, off_sw, dst);
        if (BM == 256 || wave < BM / 64) dma16(base_sx + ls * 4, off_sx, dst + kTlN * 16u);
        load_super ^= ROWS * 16u;
    };

    // ---- fragments
    u32x4 fw[2][IO], fx[XB];
    int sw[IO], sx[IT], nsw[IO], nsx[IT];
    const int frag0 = l16 * kTlUnits + (q ^ (l16 >> 2));
    const u32x4* const rd_w = &codes[0][wo * 128 * kTlUnits + frag0];
    const u32x4* const rd_x = &codes[0][(kTlN + wt * (BM / 2)) * kTlUnits + frag0];
    auto read_w = [&](int i, int buf, int to) { fw[to][i] = rd_w[buf * (ROWS * kTlUnits) + i * 16 * kTlUnits]; };
    auto read_x = [&](int j, int buf) { fx[j % XB] = rd_x[buf * (ROWS * kTlUnits) + j * 16 * kTlUnits]; };
    // bytes q of a scale row's four dwords
    const uint32_t pick = static_cast<uint32_t>(q) | (static_cast<uint32_t>(4 + q) << 8) | 0x0C0C0000u;
    int read_super = 0;
    auto gather = [&](u32x4 v) {
        const uint32_t lo = __builtin_amdgcn_perm(v[1], v[0], pick);
        const uint32_t hi = __builtin_amdgcn_perm(v[3], v[2], pick);
        return static_cast<int>(lo | (hi << 16));
    };
    const u32x4* const rd_sw = &scales[0][wo * 128 + l16];
    const u32x4* const rd_sx = &scales[0][kTlN + wt * (BM / 2) + l16];
    auto read_sw = [&](int i) { nsw[i] = gather(rd_sw[read_super + 16 * i]); };
    auto read_sx = [&](int j) { nsx[j] = gather(rd_sx[read_super + 16 * j]); };
    auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < IO; ++i) sw[i] = nsw[i];
#pragma unroll
        for (int j = 0; j < IT; ++j) sx[j] = nsx[j];
        read_super ^= ROWS;
    };

    f32x4 acc[IO][IT];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < IO; ++i)
#pragma unroll
            for (int j = 0; j < IT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    };

    // accumulator (i, j): outputs 128 wo + 16 i + 4 q + e, row (BM/2) wt + 16 j + l16
    auto store = [&](const Tile& t) {
        const int rows = t.end - t.first, cols = a.d_out - t.n0;
        const bool vec = (a.d_out & 3) == 0;
#pragma unroll
        for (int j = 0; j < IT; ++j) {
            const int row = wt * (BM / 2) + 16 * j + l16;
            if (row >= rows) continue;
            Y* y = static_cast<Y*>(a.y) + static_cast<int64_t>(t.first + row) * a.d_out + t.n0;
#pragma unroll
            for (int i = 0; i < IO; ++i) {
                const int c = wo * 128 + 16 * i + 4 * q;
                const f32x4 v = acc[i][j];
                if (vec) {
                    if (c >= cols) continue;
                    if constexpr (sizeof(Y) == 4) *reinterpret_cast<f32x4*>(y + c) = v;
                    else *reinterpret_cast<u32x2*>(y + c) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < cols) mx4_store(y + c + e, v[e]);
                }
            }
        }
    };

    // The sums are read by other instructions only behind this: the last
    // matrix step's result takes up to 18 wait states.
    auto settle = [&]() {
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int i = 0; i < IO; ++i)
#pragma unroll
            for (int j = 0; j < IT; ++j) asm volatile("" : "+a"(acc[i][j]));
    };

    // ---- prologue: stages 0, 1 and 2 (nk >= 4)
    load_scales();
#pragma unroll
    for (int b = 0; b < 3; ++b) {
#pragma unroll
        for (int j = 0; j < NL; ++j) load_codes(j, b);
        ++ls;
    }
    wait_vmcnt<2 * NL>();
    lds_barrier();
#pragma unroll
    for (int i = 0; i < IO; ++i) {
        read_w(i, 0, 0);
        read_sw(i);
    }
#pragma unroll
    for (int j = 0; j < IT; ++j) read_sx(j);
#pragma unroll
    for (int j = 0; j < XB - 1; ++j) read_x(j, 0);
    clear();

    for (int64_t k = 0;;) {
        for (int kt = 0; kt < nk; kt += 4) {
            take_scales();
#define CAT_STAGE(B)                                                                             \
    {                                                                                            \
        constexpr int L = (B + 3) % 4;                                                           \
        wait_vmcnt<NL + (B == 2 ? (BM == 256 ? 2 : 1) : 0)>();                                   \
        lds_barrier();                                                                           \
        if (L == 0) load_scales();                                                               \
        _Pragma("unroll") for (int m = 0; m < NM; ++m) {                                         \
            const int j = m / IO, i = m % IO;                                                    \
            mx4_mfma_acc<B>(fw[B & 1][i], fx[j % XB], acc[i][j], sw[i], sx[j]);                  \
            if (m % 4 == 1 && m / 4 < NL) load_codes(m / 4, L);                           \
            if (i == 0) {                                                                        \
                if (j + XB - 1 < IT) read_x(j + XB - 1, B);                                      \
                else read_x(j + XB - 1 - IT, (B + 1) % 4);                                       \
            }                                                                                    \
            if (m % (NM / IO) == NM / IO / 2) read_w(m / (NM / IO), (B + 1) % 4, (B + 1) & 1);   \
            if (B == 3 && i == 2) {                                                              \
                read_sx(j);                                                                      \
                if (IT == 8) read_sw(j);                                                         \
                else read_sw(2 * j), read_sw(2 * j + 1);                                         \
            }                                                                                    \
        }                                                                                        \
        ++ls;                                                                                    \
        if (L == 3 && ls == nk) {                                                                \
            ls = 0;                                                                              \
            if (tile_at(++lk, lt)) set_rows();                                                   \
        }                                                                                        \
    }
            CAT_STAGE(0)
            CAT_STAGE(1)
            CAT_STAGE(2)
            CAT_STAGE(3)
#undef CAT_STAGE
        }
        settle();
        store(tile);
        if (!tile_at(++k, tile)) break;
        clear();
    }
    wait_vmcnt<0>();                       // the requests past the last stage
}

// Large tiles need whole pairs of stages (scale rows of whole 16 bytes) and
// 32-bit offsets into gathered rows.
static bool tile_fits(const Mx4Args& a) {
    return a.d_in % 512 == 0 &&
           (!a.row_ids || static_cast<int64_t>(a.n) * (a.d_in / 2) < (int64_t{1} << 32));
}

template <int BM>
static hipError_t launch_tiles(const Mx4Args& a, int y_bf16, hipStream_t stream) {
    int dev = 0, cus = 0;
    hipError_t err = hipGetDevice(&dev);
    if (err == hipSuccess) err = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
    if (err != hipSuccess) return err;
    const unsigned grid = static_cast<unsigned>(cus >= kMxXcd ? cus / kMxXcd * kMxXcd : kMxXcd);
    if (y_bf16) mx4_tile_kernel<uint16_t, BM><<<grid, kTlThreads, 0, stream>>>(a);
    else mx4_tile_kernel<float, BM><<<grid, kTlThreads, 0, stream>>>(a);
    return hipGetLastError();
}

static hipError_t launch(const Mx4Args& a, int y_bf16, hipStream_t stream) {
    if (tile_fits(a) && a.m >= 256) return launch_tiles<256>(a, y_bf16, stream);
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
