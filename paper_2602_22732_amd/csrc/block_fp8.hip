// FP8 (OCP E4M3) operands with a scale for every block of 128 values along the contraction, and their product:
//     C[m, n] = sum_kb sa[kb, m] sw[kb, n / 128] sum_{k in block kb} Aq[m, k] Wq[n, k]  (+ bias[n]).
//
//  * quantize_blocks<..>     1 x 128 or 128 x 128 blocks, one pass over the values.
//  * gemm_block_few<..>      up to 64 rows: the weights stream from memory to the matrix cores' operands, wavefronts split K.
//  * gemm_block_ring<..>     256 x 256 tiles of C, for products that have enough of them to fill the chip.
//  * gemm_block_stream<..>   128 x 128 and 64 x 64 tiles for the shapes between.
//  * gemm_block_tile<..>     the same tiles for rows that do not start on 16 bytes.
//
// v_mfma_f32_16x16x128_f8f6f4 contracts exactly one block, so a block's product leaves it as 16 x 16 sums that one multiply-add each scales into the
// float32 accumulators.  The weights are the first operand: a lane then owns one row of A, whose scale is one register, and four consecutive columns of C.
#include <type_traits>

#include "common.h"

namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint2 e4m3x8(const float (&v)[8], float f) {
    int w0 = 0, w1 = 0;
    w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * f, v[1] * f, w0, false);
    w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * f, v[3] * f, w0, true);
    w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * f, v[5] * f, w1, false);
    w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * f, v[7] * f, w1, true);
    return make_uint2((unsigned)w0, (unsigned)w1);
}

__device__ __forceinline__ float row16_max(float v) {  // over the 16 lanes of a row
    v = fmaxf(v, dpp_move<0x128, 0xF>(v, v));
    v = fmaxf(v, dpp_move<0x124, 0xF>(v, v));
    v = fmaxf(v, dpp_move<0x122, 0xF>(v, v));
    return fmaxf(v, dpp_move<0x121, 0xF>(v, v));
}

struct BlockScale {
    float scale, inv;
    __device__ __forceinline__ explicit BlockScale(float amax) {
        const bool zero = amax < 0x1p-100f;
        scale = zero ? 1.0f : amax / 448.0f;
        inv = zero ? 1.0f : 448.0f / amax;
    }
};

// Sixteen lanes hold a row's block, eight values each.  TALL: a workgroup owns one block of 128 x 128 (16 rows at a time, 8 times); otherwise 16 rows by STEPS
// blocks.  All of a thread's values are requested at once and kept, so they are read once.  wide: workgroups along a row, which are successive ones (bf16,
// 16384 x 4096: 50 us; with the rows in turn 55).  keep: the bytes stay in the caches; outputs that would fill them and lie on 8 bytes pass by (41 us).
// Bound by the bytes: bf16, 4096 x 4096 in rows 12 us, 4.2 TB/s; float32, 16384 x 1040 in squares 18 us, 4.7 TB/s, 16384 x 4096 50 us, 6.7 TB/s (with
// outputs that stay in the caches 59).
template <typename T, bool TALL> __global__ __launch_bounds__(256) void quantize_blocks(const T *__restrict__ x, int64_t ldx, uint8_t *__restrict__ q, float *__restrict__ scale, int rows,
                                                                                        int n, int wide, int bands, int keep) {
    constexpr int STEPS = TALL ? 8 : 2;
    const int band = blockIdx.x / wide, kb0 = blockIdx.x % wide * (TALL ? 1 : STEPS), lane16 = threadIdx.x % 16, r16 = threadIdx.x / 16;
    float v[STEPS][8], amax[STEPS];
    auto row_of = [&](int i) { return TALL ? band * 128 + i * 16 + r16 : band * 16 + r16; };
    auto col_of = [&](int i) { return (TALL ? kb0 : kb0 + i) * 128 + lane16 * 8; };
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
        const int r = row_of(i), c = col_of(i);
#pragma unroll
        for (int e = 0; e < 8; e++) v[i][e] = 0.0f;
        if (r < rows && c < n) {
            const T *src = x + (int64_t)r * ldx + c;
            if (c + 8 <= n) {  // (rows may start anywhere)
                T t[8];
                __builtin_memcpy(t, src, 8 * sizeof(T));
#pragma unroll
                for (int e = 0; e < 8; e++) v[i][e] = to_f(t[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (c + e < n) v[i][e] = to_f(src[e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
        amax[i] = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e++) amax[i] = fmaxf(amax[i], fabsf(v[i][e]));
    }
    if (TALL) {
        __shared__ float part[4];
        float m = amax[0];
#pragma unroll
        for (int i = 1; i < STEPS; i++) m = fmaxf(m, amax[i]);
        m = wave_max(m);
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = m;
        __syncthreads();
        m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
#pragma unroll
        for (int i = 0; i < STEPS; i++) amax[i] = m;
        if (threadIdx.x == 0) scale[(int64_t)kb0 * bands + band] = BlockScale(m).scale;
    }
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
        const BlockScale s(TALL ? amax[i] : row16_max(amax[i]));
        const int r = row_of(i), c = col_of(i);
        if (r >= rows || c >= n) continue;
        if (!TALL && lane16 == 0) scale[(int64_t)(kb0 + i) * rows + r] = s.scale;
        const uint2 w = e4m3x8(v[i], s.inv);
        uint8_t *dst = q + (int64_t)r * n + c;
        if (c + 8 <= n) {
            if (keep) __builtin_memcpy(dst, &w, 8);
            else __builtin_nontemporal_store((uint64_t)w.y << 32 | w.x, (uint64_t *)dst);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (c + e < n) dst[e] = (uint8_t)((e < 4 ? w.x : w.y) >> (8 * (e % 4)));
        }
    }
}

// 16 bytes at column k of a row of K bytes, zeros past its end; rows may start anywhere
__device__ __forceinline__ intx4 bytes16(const uint8_t *row, int k, int K) {
    intx4 r = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&r, row + k, 16);
    } else {
        for (int i = 0; i < 16 && k + i < K; i++) r[i / 4] |= (int)row[k + i] << (8 * (i % 4));
    }
    return r;
}
__device__ __forceinline__ intx8 join8(intx4 lo, intx4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ floatx4 mfma_block(intx8 w, intx8 a) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, floatx4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}

struct BlockGemm {
    const uint8_t *A, *W;
    const float *sa, *sw, *bias;
    void *C;
    int M, N, K, nb, wb;  // blocks along K, and along N
    int out_f16;
};

__device__ __forceinline__ uint16_t half_of(const BlockGemm &g, float x) {
    uint16_t h;
    if (g.out_f16) {
        const _Float16 y = (_Float16)x;
        __builtin_memcpy(&h, &y, 2);
    } else {
        const bf16 y = (bf16)x;
        __builtin_memcpy(&h, &y, 2);
    }
    return h;
}
// four consecutive columns of one row of C
__device__ __forceinline__ void store4(const BlockGemm &g, int m, int n, floatx4 v) {
    if (m >= g.M) return;
    uint16_t h[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        h[e] = half_of(g, v[e] + (g.bias && n + e < g.N ? g.bias[n + e] : 0.0f));
    }
    uint16_t *dst = (uint16_t *)g.C + (int64_t)m * g.N + n;
    if (n + 4 <= g.N) {
        __builtin_memcpy(dst, h, 8);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (n + e < g.N) dst[e] = h[e];
    }
}

// 16 GM x 16 GN results of a wavefront, through LDS of its own (store_bytes of it) so that they leave as whole rows of 16-byte pieces: pieces of 8 bytes, 32
// of a row at a time, took a 256 x 256 tile of 16384 x 4096 x 1024 about as long as its products.
template <int GM, int GN> constexpr int store_bytes() { return 16 * GM * (32 * GN + 16); }
template <int GM, int GN> __device__ __forceinline__ void store_rows(const BlockGemm &g, char *lds, int m0, int n0, const floatx4 (&acc)[GM][GN]) {
    const int lane = threadIdx.x % 64, r = lane % 16, c = lane / 16;
    if (g.N % 8 || (uintptr_t)g.C % 16) {
#pragma unroll
        for (int i = 0; i < GM; i++)
#pragma unroll
            for (int j = 0; j < GN; j++) store4(g, m0 + 16 * i + r, n0 + 16 * j + 4 * c, acc[i][j]);
        return;
    }
    constexpr int STRIDE = 32 * GN + 16, PER = 2 * GN, ROWS = 64 / PER;  // bytes of a staged row; pieces of a row, rows of one store
#pragma unroll
    for (int j = 0; j < GN; j++) {
        floatx4 b = {0.0f, 0.0f, 0.0f, 0.0f};
        if (g.bias)
#pragma unroll
            for (int e = 0; e < 4; e++) b[e] = g.bias[min(n0 + 16 * j + 4 * c + e, g.N - 1)];
#pragma unroll
        for (int i = 0; i < GM; i++) {
            uint16_t h[4];
#pragma unroll
            for (int e = 0; e < 4; e++) h[e] = half_of(g, acc[i][j][e] + b[e]);
            __builtin_memcpy(lds + (16 * i + r) * STRIDE + (16 * j + 4 * c) * 2, h, 8);
        }
    }
    const int p = lane % PER;
#pragma unroll 4
    for (int row = lane / PER; row < 16 * GM; row += ROWS) {
        const intx4 x = *(const intx4 *)(lds + row * STRIDE + p * 16);
        if (m0 + row < g.M && n0 + p * 8 < g.N) *(intx4 *)((uint16_t *)g.C + (int64_t)(m0 + row) * g.N + n0 + p * 8) = x;
    }
}

// Up to 16 MG rows: 16 NG columns of C per workgroup, whose 8 wavefronts take blocks of K in turn and are joined in LDS in their order.  (A wavefront reads
// the rows' fragments anew for every NG column groups: 64 rows x 16384 x 8192 79 us with one group, 38 with four, 3.5 TB/s; NG is chosen so that workgroups
// still fill the chip.)  Few and small ones are latency: 5 x 4096 x 1024 3.4 us, where the weights' bytes are worth 0.8.
template <int MG, int NG> __global__ __launch_bounds__(512) void gemm_block_few(BlockGemm g) {
    constexpr int NW = 8;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, c = lane / 16, n0 = blockIdx.x * 16 * NG;
    const uint8_t *w[NG], *a[MG];
    int m[MG];
#pragma unroll
    for (int j = 0; j < NG; j++) w[j] = g.W + (int64_t)min(n0 + 16 * j + r, g.N - 1) * g.K;
#pragma unroll
    for (int i = 0; i < MG; i++) {
        m[i] = min(16 * i + r, g.M - 1);
        a[i] = g.A + (int64_t)m[i] * g.K;
    }
    floatx4 acc[MG][NG];
#pragma unroll
    for (int i = 0; i < MG; i++)
#pragma unroll
        for (int j = 0; j < NG; j++) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    auto block = [&](int kb, auto whole) {
        const int k = kb * 128 + 32 * c;
        auto frag = [&](const uint8_t *row) {
            if constexpr (decltype(whole)::value) {
                intx8 f;
                __builtin_memcpy(&f, row + k, 32);
                return f;
            } else {
                return join8(bytes16(row, k, g.K), bytes16(row, k + 16, g.K));
            }
        };
        intx8 wf[NG], af[MG];
        float s[MG], sw[NG];
#pragma unroll
        for (int j = 0; j < NG; j++) {
            wf[j] = frag(w[j]);
            sw[j] = g.sw[(int64_t)kb * g.wb + min((n0 + 16 * j) / 128, g.wb - 1)];
        }
#pragma unroll
        for (int i = 0; i < MG; i++) {
            af[i] = frag(a[i]);
            s[i] = g.sa[(int64_t)kb * g.M + m[i]];
        }
#pragma unroll
        for (int i = 0; i < MG; i++)
#pragma unroll
            for (int j = 0; j < NG; j++) {
                const floatx4 p = mfma_block(wf[j], af[i]);
#pragma unroll
                for (int v = 0; v < 4; v++) acc[i][j][v] = fmaf(p[v], s[i] * sw[j], acc[i][j][v]);
            }
    };
    const int whole = g.K / 128;
    int kb = wave;
#pragma unroll 2
    for (; kb < whole; kb += NW) block(kb, std::true_type());
    if (kb < g.nb) block(kb, std::false_type());  // (the last block, if it is a part of one)
    constexpr int AT_ONCE = MG * NG < 4 ? MG * NG : 4;  // 16 x 16 tiles that are joined at a time
    __shared__ floatx4 part[NW][AT_ONCE][64];
#pragma unroll
    for (int first = 0; first < MG * NG; first += AT_ONCE) {
        if (first) __syncthreads();
#pragma unroll
        for (int x = 0; x < AT_ONCE; x++) part[wave][x][lane] = acc[(first + x) / NG][(first + x) % NG];
        __syncthreads();
        if (wave < AT_ONCE) {
            const int x = first + wave;
            floatx4 s = part[0][wave][lane];
#pragma unroll
            for (int y = 1; y < NW; y++) s += part[y][wave][lane];
            store4(g, 16 * (x / NG) + r, n0 + 16 * (x % NG) + 4 * c, s);
        }
    }
}

// Rows that do not start on 16 bytes, or are too long for 32-bit places: TM x TN tiles of C on four wavefronts (2 x 2).  The next block's operands travel to
// registers while this one's multiply.  A tile row is one block, 128 bytes; its 16-byte chunk p lies at p ^ (row / 2 % 8).  3000 x 5000 x 1111: 57 us,
// 0.58 PFLOP/s; 200 x 300 x 1999 17 us, the walk of one tile along K.
template <int TM, int TN> __global__ __launch_bounds__(256) void gemm_block_tile(BlockGemm g) {
    constexpr int WM = TM / 2, WN = TN / 2, GM = WM / 16, GN = WN / 16, LA = TM * 8 / 256, LW = TN * 8 / 256;
    __shared__ intx4 sA[TM * 8], sW[TN * 8];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, c = lane / 16;
    const int wm = wave / 2, wn = wave % 2, tiles_m = (g.M + TM - 1) / TM;
    const int m0 = (int)(blockIdx.x % tiles_m) * TM, n0 = (int)(blockIdx.x / tiles_m) * TN;
    intx4 ra[LA], rw[LW];
    auto load = [&](int kb) {
        const bool whole = kb * 128 + 128 <= g.K;  // (uniform: only the last block looks at every byte)
        auto piece = [&](const uint8_t *row, int k) {
            if (!whole) return bytes16(row, k, g.K);
            intx4 f;
            __builtin_memcpy(&f, row + k, 16);
            return f;
        };
#pragma unroll
        for (int i = 0; i < LA; i++) {
            const int id = i * 256 + threadIdx.x;
            ra[i] = piece(g.A + (int64_t)min(m0 + id / 8, g.M - 1) * g.K, kb * 128 + id % 8 * 16);
        }
#pragma unroll
        for (int i = 0; i < LW; i++) {
            const int id = i * 256 + threadIdx.x;
            rw[i] = piece(g.W + (int64_t)min(n0 + id / 8, g.N - 1) * g.K, kb * 128 + id % 8 * 16);
        }
    };
    auto slot = [](int row, int p) { return row * 8 + (p ^ ((row >> 1) & 7)); };
    floatx4 acc[GM][GN];
#pragma unroll
    for (int i = 0; i < GM; i++)
#pragma unroll
        for (int j = 0; j < GN; j++) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    load(0);
    for (int kb = 0; kb < g.nb; kb++) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < LA; i++) {
            const int id = i * 256 + threadIdx.x;
            sA[slot(id / 8, id % 8)] = ra[i];
        }
#pragma unroll
        for (int i = 0; i < LW; i++) {
            const int id = i * 256 + threadIdx.x;
            sW[slot(id / 8, id % 8)] = rw[i];
        }
        __syncthreads();
        if (kb + 1 < g.nb) load(kb + 1);
        const float sw = g.sw[(int64_t)kb * g.wb + (n0 + wn * WN) / 128];
        intx8 wf[GN];
#pragma unroll
        for (int j = 0; j < GN; j++) {
            const int row = wn * WN + 16 * j + r;
            wf[j] = join8(sW[slot(row, c)], sW[slot(row, c + 4)]);
        }
#pragma unroll
        for (int i = 0; i < GM; i++) {
            const int row = wm * WM + 16 * i + r;
            const intx8 af = join8(sA[slot(row, c)], sA[slot(row, c + 4)]);
            const float s = g.sa[(int64_t)kb * g.M + min(m0 + row, g.M - 1)] * sw;
#pragma unroll
            for (int j = 0; j < GN; j++) {
                const floatx4 p = mfma_block(wf[j], af);
#pragma unroll
                for (int v = 0; v < 4; v++) acc[i][j][v] = fmaf(p[v], s, acc[i][j][v]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < GM; i++)
#pragma unroll
        for (int j = 0; j < GN; j++) store4(g, m0 + wm * WM + 16 * i + r, n0 + wn * WN + 16 * j + 4 * c, acc[i][j]);
}

// ---------------------------------------------------------------------------------------------------------------------
// Large products: 256 x 256 tiles of C on 8 wavefronts (2 x 4, 128 x 64 each), one workgroup per compute unit.  A block of K is a half-tile of A and one of
// W (256 rows x 128 bytes), which travel from memory to LDS without passing registers: three slots for A, two for W (160 KB), so that a block's A has two
// blocks' time to land and its W one.  Chunk p of row r lies at p ^ (r / 2 % 8), applied where it is read from memory.
// Per block and wavefront 24 KB of fragments feed 32 MFMAs; each one's sums are scaled into the accumulators while the next ones run.
// 16384 x 4096 x 4096: 258 us, 2.13 PFLOP/s (an FP8 product with one scale in all reaches 2.68 as a library's): the matrix cores are busy for 54 % of the cycles
// at the 1.86 GHz that the chip holds under them; the scaling takes four vector instructions per MFMA.
// ---------------------------------------------------------------------------------------------------------------------
__device__ __attribute__((aligned(16))) uint8_t zero_chunk[16];  // stands for the chunks past the end of a row

constexpr int kRing = 256;  // rows of a half-tile
// RAGGED: K is no multiple of 128; EDGE: M is no multiple of 256
template <bool RAGGED, bool EDGE> __global__ __launch_bounds__(512, 2) void gemm_block_ring(BlockGemm g, int tiles_m, int tiles_n) {
    extern __shared__ intx4 smem[];  // 3 + 2 half-tiles of 2048 chunks
    constexpr int HALF = kRing * 8;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, c = lane / 16, wm = wave / 4, wn = wave % 4;
    // Every XCD (workgroup id % 8) owns a contiguous range of tiles, 8 row blocks deep and then along the columns, so that its workgroups share operands in its L2
    const int total = tiles_m * tiles_n, per = (total + 7) / 8, l = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || l >= total) return;
    const int deep = 8 * tiles_n, grp = l / deep, in = l - grp * deep, rows_here = min(8, tiles_m - grp * 8), col = in / rows_here;
    const int m0 = (grp * 8 + in - col * rows_here) * kRing, n0 = col * kRing;

    // loads: load j of a wavefront fills rows (4 wave + j) 8 .. + 7 of a half-tile, lane -> row lane / 8, place lane % 8; which chunk that is changes with j's parity
    const int row0 = wave * 32 + lane / 8, ch0 = (lane % 8) ^ ((lane / 8) >> 1);
    const uint8_t *base_a = g.A + (int64_t)m0 * g.K, *base_w = g.W + (int64_t)n0 * g.K;
    const int last_a = g.M - 1 - m0, last_w = g.N - 1 - n0;
    unsigned a_off[4], w_off[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {  // (rows past the edge re-read the last one)
        const unsigned k = (unsigned)(ch0 ^ ((j & 1) * 4)) * 16;
        a_off[j] = (unsigned)min(row0 + 8 * j, last_a) * (unsigned)g.K + k;
        w_off[j] = (unsigned)min(row0 + 8 * j, last_w) * (unsigned)g.K + k;
    }
    auto dma = [&](const uint8_t *src, int slot, int j) {
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1))) *)src, (void __attribute__((address_space(3))) *)(smem + slot * HALF + (wave * 4 + j) * 64), 16, 0, 0);
    };
    auto piece = [&](const uint8_t *base, unsigned off, int kb, int slot, int j) {
        const uint8_t *at = base + kb * 128;  // (uniform: a whole block's load adds nothing per lane)
        if constexpr (!RAGGED) dma(at + off, slot, j);
        else dma(kb * 128 + (ch0 ^ ((j & 1) * 4)) * 16 < g.K ? at + off : zero_chunk, slot, j);
    };
    typedef const __attribute__((address_space(3))) intx4 *LdsChunk;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const unsigned swz = (unsigned)(c ^ ((r >> 1) & 7)) * 16;  // chunk c of row r of 16; chunk c + 4 lies 64 bytes off (their bit 2 differs)
    const unsigned a_lane = lds0 + (unsigned)(wm * 128 + r) * 128 + swz, w_lane = lds0 + 3 * HALF * 16 + (unsigned)(wn * 64 + r) * 128 + swz;
    auto frag = [&](unsigned at, int i) { return join8(*((LdsChunk)at + i * 128), *((LdsChunk)(at ^ 64u) + i * 128)); };

    // scales of a block: a row's in its lane (8 row groups), the weights' for 64 successive blocks one per lane
    const float *sa = g.sa + m0;
    const unsigned m_lane = (unsigned)(wm * 128 + r);
    auto row_scales = [&](float (&s)[8], const float *of) {
        if constexpr (!EDGE) {
#pragma unroll
            for (int i = 0; i < 8; i++) s[i] = (of + 16 * i)[m_lane];
        } else {
            int at = (int)m_lane;
            asm volatile("" : "+v"(at));  // (the places are formed here and not kept in registers over the loop)
#pragma unroll
            for (int i = 0; i < 8; i++) s[i] = of[min(at + 16 * i, last_a)];
        }
    };
    const int nblk = min((n0 + wn * 64) / 128, g.wb - 1);
    float sw64 = 0.0f;
    auto weight_scale = [&](int kb) {
        if (kb % 64 == 0) {
            const float *src = g.sw + (int64_t)min(kb + lane, g.nb - 1) * g.wb + nblk;
            asm volatile("global_load_dword %0, %1, off\n\ts_waitcnt vmcnt(0)" : "=&v"(sw64) : "v"(src) : "memory");
        }
        return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sw64), kb % 64));
    };
    floatx4 acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    float s_now[8], s_next[8];
    const int nb = g.nb;
    row_scales(s_next, sa);
#pragma unroll
    for (int j = 0; j < 4; j++) piece(base_a, a_off[j], 0, 0, j);
#pragma unroll
    for (int j = 0; j < 4; j++) piece(base_w, w_off[j], 0, 3, j);
#pragma unroll
    for (int j = 0; j < 4; j++) piece(base_a, a_off[j], min(1, nb - 1), 1, j);
    // All but A of the block after next has landed (the compiler sees this wait and knows that the scales have), and everybody has read the block before.
    auto meet = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(4 | 7 << 4);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    intx8 wf[4], af[3];  // fragments: the block's columns, and row groups i % 3
    int a_slot = 0, a_next = 1;
    meet();
    {
        const unsigned at_a = a_lane, at_w = w_lane;
        af[0] = frag(at_a, 0);
#pragma unroll
        for (int j = 0; j < 4; j++) wf[j] = frag(at_w, j);
        af[1] = frag(at_a, 1);
    }
#pragma unroll
    for (int i = 0; i < 8; i++) s_now[i] = s_next[i];
    constexpr int SKEW = 3;  // MFMAs between one and the use of its sums
    for (int kb = 0; kb < nb; kb++) {
        const float sw = weight_scale(kb);
        const int next = min(kb + 1, nb - 1), after = min(kb + 2, nb - 1), a_free = 3 - a_slot - a_next, w_next = (kb & 1) ^ 1;
        sa += next > kb ? g.M : 0;
        row_scales(s_next, sa);
        const unsigned at_a = a_lane + (unsigned)a_slot * HALF * 16;
        const unsigned next_a = a_lane + (unsigned)a_next * HALF * 16, next_w = w_lane + (unsigned)w_next * HALF * 16;
        floatx4 p[SKEW + 1];
        float s = 0.0f;
#pragma unroll
        for (int t = 0; t < 32 + SKEW; t++) {
            const int i = t / 4, j = t % 4, u = t - SKEW;
            if (t == 28) {  // the last row group is in registers: on to the next block, whose fragments are read under this one's last MFMAs
                meet();
                af[(8 + 0) % 3] = frag(next_a, 0);
            }
            if (t < 32) {
                if (j == 0 && i < 6) af[(i + 2) % 3] = frag(at_a, i + 2);
                p[t % (SKEW + 1)] = mfma_block(wf[j], af[i % 3]);
                if (i == 7) wf[j] = frag(next_w, j);
                // (the slots that block kb - 1 left take W of the next block and A of the one after, a load at a time)
                if (t % 3 == 2 && t / 3 < 8) {
                    const int q = t / 3;
                    if (q < 4) piece(base_w, w_off[q], next, 3 + w_next, q);
                    else piece(base_a, a_off[q - 4], after, a_free, q - 4);
                }
            }
            if (u >= 0) {
                if (u % 4 == 0) s = s_now[u / 4] * sw;
#pragma unroll
                for (int v = 0; v < 4; v++) acc[u / 4][u % 4][v] = fmaf(p[u % (SKEW + 1)][v], s, acc[u / 4][u % 4][v]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // row groups 0 and 1 of the next block belong into places 0 and 1 (group 7 was in place 1, 8 is in place 2)
        af[0] = af[2];
        af[1] = frag(next_a, 1);
#pragma unroll
        for (int i = 0; i < 8; i++) s_now[i] = s_next[i];
        a_slot = a_next;
        a_next = a_free;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads in flight own their slots)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_assert(8 * store_bytes<8, 4>() <= 5 * HALF * 16, "staged results fit the slots");
    store_rows<8, 4>(g, (char *)smem + wave * store_bytes<8, 4>(), m0 + wm * 128, n0 + wn * 64, acc);
}

int too_many_tiles(const BlockGemm &g) { return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "linear_fp8_block: sizes %d x %d x %d", g.M, g.N, g.K); }

// More than 64 KB of LDS has to be asked for, on each device: every launch asks for its own.
int allow_lds(const void *kernel, int bytes) {
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e == hipSuccess ? GR4AD_OK : thread_hip_error("linear_fp8_block", e);
}

int launch_ring(const BlockGemm &g, hipStream_t st) {
    constexpr int LDS = 5 * kRing * 128;
    const bool ragged = g.K % 128, edge = g.M % kRing;
    const auto kernel = ragged ? (edge ? gemm_block_ring<true, true> : gemm_block_ring<true, false>) : (edge ? gemm_block_ring<false, true> : gemm_block_ring<false, false>);
    const int64_t tiles_m = ceil_div64(g.M, kRing), tiles_n = ceil_div64(g.N, kRing), grid = (tiles_m * tiles_n + 7) / 8 * 8;
    if (!launchable(grid, 512)) return too_many_tiles(g);
    const int s = allow_lds((const void *)kernel, LDS);
    if (s) return s;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(512), LDS, st, g, (int)tiles_m, (int)tiles_n);
    GR4AD_LAUNCH_CHECK_AS("linear_fp8_block");
    return GR4AD_OK;
}

// ---------------------------------------------------------------------------------------------------------------------
// Products of a round or two of tiles: TM x TN tiles of C on four wavefronts (2 x 2), operands and row scales straight to LDS, SLOTS blocks of K on their
// way or in use.  With few tiles the time is one tile's walk along K, so what counts is that a block costs its MFMAs and a barrier and no memory latency.
// 517 x 1000 x 1104 7.7 us (144 tiles, 9 blocks), 1024 x 4096 x 4096 34 us, 2048 x 4096 x 4096 46 us, 1.5 PFLOP/s.
// ---------------------------------------------------------------------------------------------------------------------
template <int TM, int TN, int SLOTS, bool RAGGED> __global__ __launch_bounds__(256) void gemm_block_stream(BlockGemm g) {
    constexpr int WM = TM / 2, WN = TN / 2, GM = WM / 16, GN = WN / 16, LA = TM / 32, LW = TN / 32, LEAD = SLOTS - 1, LOADS = LA + LW + 1;
    static_assert(TM >= 64, "a wavefront's load of 64 scales stays in the tile's rows");
    constexpr int SLOT = (TM + TN) * 128 + 4 * TM;  // bytes: rows of A, rows of W, A's scales
    extern __shared__ intx4 smem[];
    char *lds = (char *)smem;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, c = lane / 16;
    const int wm = wave / 2, wn = wave % 2, tiles_m = (g.M + TM - 1) / TM;
    const int m0 = (int)(blockIdx.x % tiles_m) * TM, n0 = (int)(blockIdx.x / tiles_m) * TN;
    const int last_a = g.M - 1 - m0, last_w = g.N - 1 - n0, ch0 = (lane % 8) ^ ((lane / 8) >> 1);
    const uint8_t *base_a = g.A + (int64_t)m0 * g.K, *base_w = g.W + (int64_t)n0 * g.K;
    unsigned a_off[LA], w_off[LW];
#pragma unroll
    for (int j = 0; j < LA; j++) a_off[j] = (unsigned)min((wave * LA + j) * 8 + lane / 8, last_a) * (unsigned)g.K + (unsigned)(ch0 ^ (((wave * LA + j) & 1) * 4)) * 16;
#pragma unroll
    for (int j = 0; j < LW; j++) w_off[j] = (unsigned)min((wave * LW + j) * 8 + lane / 8, last_w) * (unsigned)g.K + (unsigned)(ch0 ^ (((wave * LW + j) & 1) * 4)) * 16;
    const int s_row = min((wave * 64) % TM + lane, last_a);  // (what several wavefronts load twice is the same)
    auto dma16 = [&](const void *src, int at) {
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1))) *)src, (void __attribute__((address_space(3))) *)(lds + at), 16, 0, 0);
    };
    auto dma4 = [&](const void *src, int at) {
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1))) *)src, (void __attribute__((address_space(3))) *)(lds + at), 4, 0, 0);
    };
    auto issue = [&](int kb, int slot) {
        const int at = slot * SLOT;
        auto from = [&](const uint8_t *base, unsigned off, int l) {
            const uint8_t *src = base + kb * 128 + off;
            if constexpr (RAGGED)
                if (kb * 128 + (ch0 ^ ((l & 1) * 4)) * 16 >= g.K) src = zero_chunk;
            return src;
        };
#pragma unroll
        for (int j = 0; j < LA; j++) dma16(from(base_a, a_off[j], wave * LA + j), at + (wave * LA + j) * 1024);
#pragma unroll
        for (int j = 0; j < LW; j++) dma16(from(base_w, w_off[j], wave * LW + j), at + TM * 128 + (wave * LW + j) * 1024);
        dma4(g.sa + (int64_t)kb * g.M + m0 + s_row, at + (TM + TN) * 128 + (wave * 256) % (4 * TM));
    };
    typedef const __attribute__((address_space(3))) intx4 *LdsChunk;
    typedef const __attribute__((address_space(3))) float *LdsFloat;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)smem, swz = (unsigned)(c ^ ((r >> 1) & 7)) * 16;
    const unsigned a_lane = lds0 + (unsigned)(wm * WM + r) * 128 + swz, w_lane = lds0 + (unsigned)(TM + wn * WN + r) * 128 + swz, s_lane = lds0 + (unsigned)((TM + TN) * 128 + (wm * WM + r) * 4);
    auto frag = [&](unsigned at, int i) { return join8(*((LdsChunk)at + i * 128), *((LdsChunk)(at ^ 64u) + i * 128)); };
    const int nblk = min((n0 + wn * WN) / 128, g.wb - 1);
    float sw64 = 0.0f;
    auto weight_scale = [&](int kb) {
        if (kb % 64 == 0) {
            const float *src = g.sw + (int64_t)min(kb + lane, g.nb - 1) * g.wb + nblk;
            asm volatile("global_load_dword %0, %1, off\n\ts_waitcnt vmcnt(0)" : "=&v"(sw64) : "v"(src) : "memory");
        }
        return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sw64), kb % 64));
    };
    floatx4 acc[GM][GN];
#pragma unroll
    for (int i = 0; i < GM; i++)
#pragma unroll
        for (int j = 0; j < GN; j++) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    const int nb = g.nb;
#pragma unroll
    for (int x = 0; x < LEAD; x++) issue(min(x, nb - 1), x);
    int slot = 0;
    for (int kb = 0; kb < nb; kb++) {
        const float sw = weight_scale(kb);
        // this block has landed, everybody's part of it; the block before is read out, and its slot takes the block LEAD ahead (past the end the last one again,
        // into slots that nobody reads)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((LEAD - 1) * LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        issue(min(kb + LEAD, nb - 1), slot == 0 ? LEAD : slot - 1);
        const unsigned at = (unsigned)slot * SLOT;
        intx8 wf[GN];
#pragma unroll
        for (int j = 0; j < GN; j++) wf[j] = frag(w_lane + at, j);
#pragma unroll
        for (int i = 0; i < GM; i++) {
            const intx8 af = frag(a_lane + at, i);
            const float s = *((LdsFloat)(s_lane + at) + 16 * i) * sw;
#pragma unroll
            for (int j = 0; j < GN; j++) {
                const floatx4 p = mfma_block(wf[j], af);
#pragma unroll
                for (int v = 0; v < 4; v++) acc[i][j][v] = fmaf(p[v], s, acc[i][j][v]);
            }
        }
        slot = slot + 1 == SLOTS ? 0 : slot + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads in flight own their slots)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    static_assert(4 * store_bytes<GM, GN>() <= SLOTS * SLOT, "staged results fit the slots");
    store_rows<GM, GN>(g, lds + wave * store_bytes<GM, GN>(), m0 + wm * WM, n0 + wn * WN, acc);
}

template <int TM, int TN, int SLOTS> int launch_stream(const BlockGemm &g, hipStream_t st) {
    constexpr int LDS = SLOTS * ((TM + TN) * 128 + 4 * TM);
    const int64_t grid = ceil_div64(g.M, TM) * ceil_div64(g.N, TN);
    if (!launchable(grid, 256)) return too_many_tiles(g);
    const auto kernel = g.K % 128 ? gemm_block_stream<TM, TN, SLOTS, true> : gemm_block_stream<TM, TN, SLOTS, false>;
    if (LDS > 65536) {
        const int s = allow_lds((const void *)kernel, LDS);
        if (s) return s;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), LDS, st, g);
    GR4AD_LAUNCH_CHECK_AS("linear_fp8_block");
    return GR4AD_OK;
}

template <int TM, int TN> int launch_tile(const BlockGemm &g, hipStream_t st) {
    const int64_t grid = ceil_div64(g.M, TM) * ceil_div64(g.N, TN);
    if (!launchable(grid, 256)) return too_many_tiles(g);
    hipLaunchKernelGGL((gemm_block_tile<TM, TN>), dim3((unsigned)grid), dim3(256), 0, st, g);
    GR4AD_LAUNCH_CHECK_AS("linear_fp8_block");
    return GR4AD_OK;
}

template <int MG> int launch_few(const BlockGemm &g, hipStream_t st) {
    // as many column groups per workgroup as leave 256 workgroups (64 rows x 16384 x 8192: one 79 us, four 38)
    const int groups = (g.N + 15) / 16, each = MG == 1 || groups < 512 ? 1 : groups < 1024 ? 2 : 4;
    const dim3 grid((groups + each - 1) / each);
    if (!launchable(grid.x, 512)) return too_many_tiles(g);
    if constexpr (MG > 1) {
        if (each == 4) hipLaunchKernelGGL((gemm_block_few<MG, 4>), grid, dim3(512), 0, st, g);
        if (each == 2) hipLaunchKernelGGL((gemm_block_few<MG, 2>), grid, dim3(512), 0, st, g);
    }
    if (each == 1) hipLaunchKernelGGL((gemm_block_few<MG, 1>), grid, dim3(512), 0, st, g);
    GR4AD_LAUNCH_CHECK_AS("linear_fp8_block");
    return GR4AD_OK;
}

// The variants by size.  Up to 64 rows every weight is read once by whoever needs it (64 rows, captured, in tiles of 64 instead: x 4096 x 4096 11.8 us against 14.1, x 8192 x 8192 25.2
// against 25.3; only where a tile for every compute unit comes together are tiles faster, x 16384 x 8192 40.9 against 32.5, 16 rows 34.3 against 31.7).  Then the time is the rounds of tiles: a compute unit holds two workgroups of
// 64 x 64 or 128 x 128 tiles and one of 256 x 256, so each size is left when it needs more rounds than the next (x 4096 x 4096, tiles of 64, 128, 256: 128 rows 15,
// 35, 46 us; 1024 rows, two rounds of the smallest, 34, 36, 45; 2048 rows, one round of the middle ones, 65, 46, 47; 2816 rows 90, 74, 49; 4096 rows 125, 86, 60).  Rows
// that do not start on 16 bytes take tiles of 128 from a tile per compute unit on (tiles of 64 | 128, x 5000 x 1111: 500 rows 21 | 26 us, 800 rows 32.7 | 32.4, 3000 rows 78 | 56; x 4096 x 4001:
// 800 rows 60 | 63, 1200 rows 82 | 74).
int launch_block_gemm(const BlockGemm &g, hipStream_t st) {
    // rows in pieces of 16 bytes (and a tile's rows within 32 bits of its first): direct loads to LDS
    const bool aligned = g.K % 16 == 0 && g.K < (1 << 23) && (uintptr_t)g.A % 16 == 0 && (uintptr_t)g.W % 16 == 0;
    const int64_t tiles64 = ceil_div64(g.M, 64) * ceil_div64(g.N, 64), tiles128 = ceil_div64(g.M, 128) * ceil_div64(g.N, 128);
    const int cls = g.M <= 64 ? KC_GEMM_F8_FEW : !aligned ? KC_GEMM_F8_ANY : tiles64 <= 1024 ? KC_GEMM_F8_64 : tiles128 <= 512 ? KC_GEMM_F8_128 : KC_GEMM_F8_256;
    ProfScope ps(cls, st, 2.0 * (double)g.M * g.N * g.K, ((double)g.M + g.N) * g.K + 2.0 * (double)g.M * g.N);
    switch (cls) {
        case KC_GEMM_F8_FEW: return g.M <= 16 ? launch_few<1>(g, st) : g.M <= 32 ? launch_few<2>(g, st) : launch_few<4>(g, st);
        case KC_GEMM_F8_64: return launch_stream<64, 64, 4>(g, st);
        case KC_GEMM_F8_128: return launch_stream<128, 128, 2>(g, st);
        case KC_GEMM_F8_256: return launch_ring(g, st);
        default: return tiles128 < 256 ? launch_tile<64, 64>(g, st) : launch_tile<128, 128>(g, st);
    }
}

}  // namespace

extern "C" {

int gr4ad_op_quantize_blocks(gr4ad_dtype dtype, const void *x, int64_t x_stride, void *q, float *scale, int32_t rows, int32_t n, int32_t block_rows, void *hip_stream) {
    if (!x || !q || !scale) return gr4ad_set_thread_error(GR4AD_EINVAL, "quantize_blocks: NULL pointer");
    if (dtype != GR4AD_F32 && dtype != GR4AD_BF16) return gr4ad_set_thread_error(GR4AD_EINVAL, "quantize_blocks: dtype %d", (int)dtype);
    if (rows < 1 || n < 1 || x_stride < n) return gr4ad_set_thread_error(GR4AD_EINVAL, "quantize_blocks: %d rows of %d values, %lld apart", rows, n, (long long)x_stride);
    if (block_rows != 1 && block_rows != 128) return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "quantize_blocks: block_rows %d (1 or 128)", block_rows);
    const size_t e = dtype == GR4AD_BF16 ? 2 : 4;
    if ((uintptr_t)x % e || (uintptr_t)scale % 4) return gr4ad_set_thread_error(GR4AD_EINVAL, "quantize_blocks: misaligned pointer");
    const bool tall = block_rows == 128;
    const int64_t nb = ceil_div64(n, 128), bands = ceil_div64(rows, tall ? 128 : 16), steps = tall ? 1 : 2, wide = ceil_div64(nb, steps), grid = bands * wide;
    const int keep = (int64_t)rows * n < (8 << 20) || n % 8 || (uintptr_t)q % 8;
    if (!launchable(grid, 256) || n > 0x7fffff00) return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "quantize_blocks: %d rows of %d values", rows, n);
    hipStream_t st = (hipStream_t)hip_stream;
    ProfScope ps(KC_QUANTIZE_BLOCKS, st, 0.0, (double)rows * n * (e + 1));
#define QUANTIZE_(T, TALL) hipLaunchKernelGGL((quantize_blocks<T, TALL>), dim3((unsigned)grid), dim3(256), 0, st, (const T *)x, x_stride, (uint8_t *)q, scale, rows, n, (int)wide, (int)bands, keep)
    if (dtype == GR4AD_BF16) { if (tall) QUANTIZE_(bf16, true); else QUANTIZE_(bf16, false); }
    else if (tall) QUANTIZE_(float, true);
    else QUANTIZE_(float, false);
#undef QUANTIZE_
    GR4AD_LAUNCH_CHECK_AS("quantize_blocks");
    return GR4AD_OK;
}

int gr4ad_op_linear_fp8_block(const void *Aq, const float *a_scale, const void *Wq, const float *w_scale, const float *bias, void *C, int32_t M, int32_t N, int32_t K, int32_t out_f16,
                              void *hip_stream) {
    if (!Aq || !a_scale || !Wq || !w_scale || !C) return gr4ad_set_thread_error(GR4AD_EINVAL, "linear_fp8_block: NULL pointer");
    if (M < 1 || N < 1 || K < 1) return gr4ad_set_thread_error(GR4AD_EINVAL, "linear_fp8_block: sizes %d x %d x %d must be positive", M, N, K);
    if (M > 0x7fffff00 || N > 0x7fffff00 || K > 0x7fffff00) return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "linear_fp8_block: sizes %d x %d x %d", M, N, K);
    if ((uintptr_t)C % 2 || (uintptr_t)a_scale % 4 || (uintptr_t)w_scale % 4 || (uintptr_t)bias % 4) return gr4ad_set_thread_error(GR4AD_EINVAL, "linear_fp8_block: misaligned pointer");
    BlockGemm g = {(const uint8_t *)Aq, (const uint8_t *)Wq, a_scale, w_scale, bias, C, M, N, K, (K + 127) / 128, (N + 127) / 128, out_f16 ? 1 : 0};
    return launch_block_gemm(g, (hipStream_t)hip_stream);
}

}  // extern "C"
