// Attention of new tokens over a paged cache of keys and values, with the cache's update.
//
// Sequence b has m_b new tokens, rows q_start[b] .. q_start[b+1]-1 of q, and len_b tokens with them; its row i stands at position
// p = len_b - m_b + i and sees key j if 0 <= j <= p and (no window, or p - j < window, or j < sinks):
//     out[row, h, :] = sum_j softmax_j(scale * q[row, h, :] . k_j) v_j,        keys and values of head h / (H / H_kv).
//
// The cache: keys [page][H_kv][slot][dh], values transposed [page][H_kv][dh][slot], so that a page of one head is one stretch of memory
// and both operands of the two products, S^T = K Q^T and O^T = V^T P^T, are read along their contraction in 16-byte pieces.
//
//  * paged_append<DH>       new keys and values into their pages (ahead of paged_flash; the others take them where they are).
//  * paged_rows<T, DH, MR>  16 or 32 rows (token, head of the group) of one (sequence, key head) per workgroup, whose wavefronts walk
//                           stretches of the keys of their own; operands go from memory to registers.
//  * paged_flash<DH, ..>    128 or 256 rows per workgroup, keys and values staged in LDS (bf16).
//  * paged_join<T, DH>      joins the stretches of several workgroups.
#include <type_traits>

#include "common.h"

namespace {

constexpr int kRows = 16;       // rows of a tile of the join
constexpr int kAppendKeys = 64; // positions of a tile of the update

struct PagedArgs {
    const void *q;
    int64_t q_stride;
    const void *k_new, *v_new;
    int64_t kv_stride;
    const int32_t *q_start, *seq_len, *table;
    void *k, *v;
    int n_pages, page_shift, max_pages;
    int B, N, H, Hkv, group;
    float scale_log2e;
    int window, sinks;  // window 0: none
    void *out;
    float *part;        // [N][H][nsplit][DH + 2]: sums, maximum, normaliser (nsplit > 1)
    int nsplit;
};

struct Sequence { int b, tile, start, m, len; };  // tile: number inside the sequence

// The sequence that tile t lies in, sequences having tiles(m, len) tiles each: every wavefront adds them up, 64 sequences at a time.  What lies on the
// device is clamped to what exists, so a bad table reads and writes nothing out of range.
template <typename F> __device__ __forceinline__ bool find_sequence(const PagedArgs &a, int64_t t, F tiles, Sequence &s) {
    const int lane = threadIdx.x % 64, most = a.max_pages << a.page_shift;
    int64_t before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int b = b0 + lane;
        int start = 0, m = 0, len = 0, count = 0;
        if (b < a.B) {
            start = min(max(a.q_start[b], 0), a.N);
            m = min(max(a.q_start[b + 1], start), a.N) - start;
            len = min(max(a.seq_len[b], 0), most);
            count = tiles(m, len);
        }
        const int upto = wave_scan(count), all = __builtin_amdgcn_readlane(upto, 63);
        if (t < before + all) {
            const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + upto > t));
            s.b = b0 + src;
            s.start = __builtin_amdgcn_readlane(start, src);
            s.m = __builtin_amdgcn_readlane(m, src);
            s.len = __builtin_amdgcn_readlane(len, src);
            s.tile = (int)(t - before) - (__builtin_amdgcn_readlane(upto, src) - __builtin_amdgcn_readlane(count, src));
            return true;
        }
        before += all;
    }
    return false;
}

// The same with the longest sequences first (B <= 64), so that their tiles do not start last; otherwise in their order.
template <typename F> __device__ __forceinline__ bool find_longest_first(const PagedArgs &a, int64_t t, F tiles, Sequence &s) {
    if (a.B > 64) return find_sequence(a, t, tiles, s);
    const int lane = threadIdx.x % 64;
    int start = 0, m = 0, len = -1, count = 0, rank = 0;
    if (lane < a.B) {
        start = min(max(a.q_start[lane], 0), a.N);
        m = min(max(a.q_start[lane + 1], start), a.N) - start;
        len = min(max(a.seq_len[lane], 0), a.max_pages << a.page_shift);
        count = tiles(m, len);
    }
    for (int i = 0; i < a.B; i++) {
        const int other = __builtin_amdgcn_readlane(len, i);
        rank += other > len || (other == len && i < lane) ? 1 : 0;
    }
    if (lane >= a.B) rank = lane;
    auto sorted = [&](int v) { return __builtin_amdgcn_ds_permute(rank * 4, v); };
    const int b = sorted(lane);
    start = sorted(start);
    m = sorted(m);
    len = sorted(len);
    count = sorted(count);
    const int upto = wave_scan(count);
    if (t >= __builtin_amdgcn_readlane(upto, 63)) return false;
    const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > t));
    s.b = __builtin_amdgcn_readlane(b, src);
    s.start = __builtin_amdgcn_readlane(start, src);
    s.m = __builtin_amdgcn_readlane(m, src);
    s.len = __builtin_amdgcn_readlane(len, src);
    s.tile = (int)t - (__builtin_amdgcn_readlane(upto, src) - __builtin_amdgcn_readlane(count, src));
    return true;
}

__device__ __forceinline__ int page_of(const PagedArgs &a, int b, int key) { return a.table[(int64_t)b * a.max_pages + (key >> a.page_shift)]; }

// New keys and values of 64 positions (counted from the sequence's first) and one key head.  Positions on a page number that does not exist are left out.
// Both are read in 16-byte pieces; the values turn in LDS and leave in pieces of 8 positions (one by one where not all of them are new): written one by one
// from their rows they took most of 51 us for 4048 tokens of 8 heads of 128 columns.
template <int DH> __global__ __launch_bounds__(256) void paged_append(PagedArgs a) {
    constexpr int P = 8, CH = DH / P;  // values of a piece, pieces of a row
    __shared__ bf16 turn[kAppendKeys][DH + 2];
    Sequence s;
    const int64_t t = blockIdx.x / a.Hkv;
    const int h = blockIdx.x % a.Hkv;
    auto tiles = [&](int m, int len) {
        const int first = max(len - m, 0);
        return m > 0 && len > first ? (len - 1) / kAppendKeys - first / kAppendKeys + 1 : 0;
    };
    if (!find_sequence(a, t, tiles, s)) return;
    const int base = s.len - s.m, tile0 = (max(base, 0) / kAppendKeys + s.tile) * kAppendKeys, k0 = max(tile0, max(base, 0)), k1 = min(tile0 + kAppendKeys, s.len);
    const int page = 1 << a.page_shift;
    for (int i = threadIdx.x; i < (k1 - k0) * CH; i += 256) {
        const int key = k0 + i / CH, c = i % CH * P, id = page_of(a, s.b, key);
        const int64_t src = (int64_t)(s.start + key - base) * a.kv_stride + h * DH + c;
        const bf16x8 k = *(const bf16x8 *)((const bf16 *)a.k_new + src), v = *(const bf16x8 *)((const bf16 *)a.v_new + src);
        if (id >= 0 && id < a.n_pages) *(bf16x8 *)((bf16 *)a.k + (((int64_t)id * a.Hkv + h) * page + (key & (page - 1))) * DH + c) = k;
#pragma unroll
        for (int e = 0; e < P; e++) turn[key - tile0][c + e] = v[e];
    }
    __syncthreads();
    constexpr int G = kAppendKeys / P;  // groups of P positions (P divides the page: on one of them)
    for (int i = threadIdx.x; i < G * DH; i += 256) {
        const int g = i % G * P, c = i / G, key = tile0 + g;
        if (key + P <= k0 || key >= k1) continue;
        const int id = page_of(a, s.b, key);
        if (id < 0 || id >= a.n_pages) continue;
        bf16 *dst = (bf16 *)a.v + (((int64_t)id * a.Hkv + h) * DH + c) * page + (key & (page - 1));
        if (key >= k0 && key + P <= k1) {
            bf16x8 v;
#pragma unroll
            for (int e = 0; e < P; e++) v[e] = turn[g + e][c];
            *(bf16x8 *)dst = v;
        } else {
#pragma unroll
            for (int e = 0; e < P; e++)
                if (key + e >= k0 && key + e < k1) dst[e] = turn[g + e][c];
        }
    }
}

// The keys a tile of rows sees, in blocks of KB keys: blocks [0, first) hold the tokens that stay visible, blocks [from, from + count - first) the rest.
struct Blocks {
    int first, from, count;
    __device__ __forceinline__ int at(int x) const { return x < first ? x : from + x - first; }
};
template <int KB> __device__ __forceinline__ Blocks visible_blocks(const PagedArgs &a, int p_lo, int p_hi) {
    Blocks r = {0, 0, 0};
    if (p_hi < 0) return r;
    const int end = p_hi / KB + 1;
    if (a.window) {
        r.first = (min(a.sinks, p_hi + 1) + KB - 1) / KB;
        r.from = max(max(p_lo - a.window + 1, 0) / KB, r.first);
    }
    r.count = r.first + max(end - r.from, 0);
    return r;
}
__device__ __forceinline__ bool sees(const PagedArgs &a, int p, int key) { return key <= p && (!a.window || p - key < a.window || key < a.sinks); }

// What a tile leaves of one row: the result, or this workgroup's share of it for the join.
template <typename T, int DH> __device__ __forceinline__ T *out_row(const PagedArgs &a, int row, int head) { return (T *)a.out + ((int64_t)row * a.H + head) * DH; }
template <int DH> __device__ __forceinline__ float *part_row(const PagedArgs &a, int row, int head, int split) {
    return a.part + (((int64_t)row * a.H + head) * a.nsplit + split) * (DH + 2);
}

// One row over blocks [x0, x1), key by key: only visible keys and values are read.  The form for tiles whose sums are no numbers: where a key that
// some rows do not see holds an infinity or a NaN, the tile's product with p = 0 would carry it into those rows.  Rows of a wavefront go one by one, 0.35 us a key, so it
// is the form of broken data alone: with one infinity among a sequence's first values, which every row sees, 64 sequences of 512 to 8192 keys and a token each take
// 349 us for 224, and 1000 tokens over 8192 keys (32 heads of 128 over 8) 91 ms for 0.2.
template <typename T, int DH, int KB>
__device__ void plain_row(const PagedArgs &a, const Sequence &s, const Blocks &bl, int x0, int x1, int kvh, int row, int head, int p, int split) {
    const int lane = threadIdx.x % 64, page = 1 << a.page_shift;
    constexpr int E = (DH + 63) / 64;
    const T *q = (const T *)a.q + (int64_t)row * a.q_stride + head * DH;
    float qv[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; e++) {
        qv[e] = lane + 64 * e < DH ? to_f(q[lane + 64 * e]) : 0.0f;
        o[e] = 0.0f;
    }
    for (int x = x0; x < x1; x++)
        for (int key = bl.at(x) * KB; key < bl.at(x) * KB + KB; key++) {
            if (!sees(a, p, key) || key >= s.len) continue;
            const int id = page_of(a, s.b, key), slot = key & (page - 1);
            if (id < 0 || id >= a.n_pages) continue;
            // (a new token where it is: another workgroup may be writing it into its page)
            const int64_t hd = (int64_t)id * a.Hkv + kvh, at = (int64_t)(s.start + key - (s.len - s.m)) * a.kv_stride + kvh * DH;
            const bool fresh = a.k_new && key >= s.len - s.m;
            const T *kr = fresh ? (const T *)a.k_new + at : (const T *)a.k + (hd * page + slot) * DH, *vr = fresh ? (const T *)a.v_new + at : (const T *)a.v + hd * DH * page + slot;
            const int vs = fresh ? 1 : page;
            float dot = 0.0f, v[E];
#pragma unroll
            for (int e = 0; e < E; e++) {
                const int c = lane + 64 * e;
                v[e] = 0.0f;
                if (c < DH) {
                    dot = fmaf(qv[e], to_f(kr[c]), dot);
                    v[e] = to_f(vr[c * vs]);
                }
            }
            dot = wave_sum(dot) * a.scale_log2e;
            const float mn = dot > m ? dot : m;  // (a NaN stays out of the maximum and enters the sums through its term)
            const float keep = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn), w = dot == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(dot - mn);
            m = mn;
            l = fmaf(l, keep, w);
#pragma unroll
            for (int e = 0; e < E; e++) o[e] = o[e] * keep + w * v[e];
        }
    float *part = a.nsplit > 1 ? part_row<DH>(a, row, head, split) : nullptr;
#pragma unroll
    for (int e = 0; e < E; e++) {
        const int c = lane + 64 * e;
        if (c >= DH) continue;
        if (part) part[c] = o[e];
        else out_row<T, DH>(a, row, head)[c] = from_f<T>(l == 0.0f ? 0.0f : o[e] / l);
    }
    if (part && lane == 0) {
        part[DH] = m;
        part[DH + 1] = l;
    }
}

// The kernel's arguments, read again where this stands: what only the rare path needs does not occupy scalar registers before it.
__device__ __forceinline__ PagedArgs late_args() {
    const __attribute__((address_space(4))) char *at = (const __attribute__((address_space(4))) char *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    PagedArgs a;
    __builtin_memcpy(&a, (const char *)at, sizeof(a));
    return a;
}

// Numbers of 64 successive pages of sequence b from `first` on, one per lane; -1 past the table.  Load and wait in one: a load that the compiler tracks
// would have every later use of the numbers wait for all keys and values on their way.
__device__ __forceinline__ int page_numbers(const PagedArgs &a, int b, int first) {
    const int at = first + threadIdx.x % 64;
    const int32_t *src = a.table + (int64_t)b * a.max_pages + min(at, a.max_pages - 1);
    int id;
    asm volatile("global_load_dword %0, %1, off\n\ts_waitcnt vmcnt(0)" : "=&v"(id) : "v"(src) : "memory");
    return at < a.max_pages ? id : -1;
}

// Fragments of one block of keys as the two products take them.  bf16: v_mfma_f32_16x16x32_bf16, 32 keys; float32: v_mfma_f32_16x16x4_f32, 16 keys.
// A lane holds row lane % 16 of the first operand and c = lane / 16 says which part of the contraction; of S^T it gets query lane % 16 and four rows.
// bf16: key rows enter in an order that makes the eight keys a lane then holds of P consecutive, as its piece of V^T has them.
// New tokens among a block's keys, [first, end) of it: k, v are where its key 0 would lie among their rows
template <typename T> struct NewRows {
    const T *k, *v;
    int64_t stride;
    int first, end, keep_from, keep_to;  // [keep_from, keep_to]: keys this workgroup writes
    __device__ __forceinline__ bool has(int key) const { return key >= first && key < end; }
    __device__ __forceinline__ bool keeps(int key) const { return key >= keep_from && key <= keep_to; }
    __device__ __forceinline__ int near(int key) const { return min(max(key, first), end - 1); }  // itself if it is new, otherwise one that is
};
template <typename T, int DH> struct Frags;
template <int DH> struct Frags<bf16, DH> {
    static constexpr int KB = 32, KF = (DH + 31) / 32, VF = DH / 16;
    bf16x8 k[2][KF], v[VF];
    __device__ __forceinline__ static bf16x8 zero() { return bf16x8{}; }
    __device__ __forceinline__ static void load_q(bf16x8 (&q)[KF], const bf16 *row) {
        const int c = threadIdx.x % 64 / 16;
#pragma unroll
        for (int f = 0; f < KF; f++) {
            q[f] = zero();
            if (32 * f + 8 * c < DH) q[f] = *(const bf16x8 *)(row + 32 * f + 8 * c);
        }
    }
    // key of the block behind row r of S^T's tile u
    __device__ __forceinline__ static int key_of(int u, int r) { return 8 * (r / 4) + 4 * u + r % 4; }
    // k0: this head's keys from the block's first on, k1: from its key 16 on (v0, v1: their values)
    __device__ __forceinline__ void load_k(const bf16 *k0, const bf16 *k1) {
        const int r = threadIdx.x % 16, c = threadIdx.x % 64 / 16;
        const bf16 *base = r < 8 ? k0 : k1;  // (key_of(u, r) < 16)
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const bf16 *src = base + (key_of(u, r) % 16) * DH + 8 * c;
#pragma unroll
            for (int f = 0; f < KF; f++) {
                if (DH % 32 == 0 || 8 * c < DH) k[u][f] = *(const bf16x8 *)(src + 32 * f);
                else k[u][f] = zero();
            }
        }
    }
    __device__ __forceinline__ void load_v(const bf16 *v0, const bf16 *v1, int page) {
        const int r = threadIdx.x % 16, c = threadIdx.x % 64 / 16;
        const bf16 *src = (c < 2 ? v0 : v1) + (8 * c) % 16 + r * page;
        asm volatile("" : "+s"(page));  // (its multiples are formed here: kept over the loop they cost scalar registers that spill)
#pragma unroll
        for (int t = 0; t < VF; t++) v[t] = *(const bf16x8 *)(src + 16 * t * page);
    }
    __device__ __forceinline__ void scores(floatx4 (&s)[2], const bf16x8 (&q)[KF]) const {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            s[u] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int f = 0; f < KF; f++) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[u][f], q[f], s[u], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void add_values(floatx4 (&o)[VF], const floatx4 (&p)[2]) const {
        // A weight as the sum of two bf16 numbers, 16 bits of it: the second product costs nothing where memory is what bounds, and the result then carries
        // one rounding, its own (with one product of rounded weights it is off by 0.0022 to 0.0023 of its norm, with two by 0.0017, as a float32 form is).
        bf16x8 w, rest;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            w[e] = (bf16)p[e / 4][e % 4];
            rest[e] = (bf16)(p[e / 4][e % 4] - (float)w[e]);
        }
#pragma unroll
        for (int t = 0; t < VF; t++) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[t], w, o[t], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < VF; t++) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[t], rest, o[t], 0, 0, 0);
    }
    __device__ __forceinline__ void take_new(const NewRows<bf16> &n, bf16 *k0, bf16 *k1, bf16 *v0, bf16 *v1, int valid, int page) {
        const int r = threadIdx.x % 16, c = threadIdx.x % 64 / 16;
#pragma unroll
        for (int u = 0; u < 2; u++) {  // (all of a row from one place or the other, without a branch)
            const int key = key_of(u, r);
            const bf16 *src = (n.has(key) ? n.k + (int64_t)key * n.stride : (r < 8 ? k0 : k1) + (key % 16) * DH) + 8 * c;
#pragma unroll
            for (int f = 0; f < KF; f++)
                if (DH % 32 == 0 || 8 * c < DH) k[u][f] = *(const bf16x8 *)(src + 32 * f);
        }
        bf16 *dst = (c < 2 ? v0 : v1) + (8 * c) % 16 + r * page;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {  // two keys' values are requested together
            const int key = 8 * c + e;
            if (!n.has(key) && !n.has(key + 1)) continue;
            bf16 x[2][VF];
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int t = 0; t < VF; t++) x[i][t] = n.v[(int64_t)n.near(key + i) * n.stride + 16 * t + r];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const bool has = n.has(key + i), keep = has && n.keeps(key + i) && (valid >> (key / 16) & 1);
#pragma unroll
                for (int t = 0; t < VF; t++) {
                    v[t][e + i] = has ? x[i][t] : v[t][e + i];
                    if (keep) dst[16 * t * page + e + i] = x[i][t];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const int key = key_of(u, r);
            bf16 *dk = (r < 8 ? k0 : k1) + (key % 16) * DH + 8 * c;
            if (n.has(key) && n.keeps(key) && (valid >> (key / 16) & 1) && 8 * c < DH)
#pragma unroll
                for (int f = 0; f < KF; f++) *(bf16x8 *)(dk + 32 * f) = k[u][f];
        }
    }
    // values of keys nobody in the tile may use (slots behind the last token, pages that do not exist): out of the product
    __device__ __forceinline__ void drop_values(int from, int valid) {
        const int c = threadIdx.x % 64 / 16;
#pragma unroll
        for (int t = 0; t < VF; t++)
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (8 * c + e >= from || !(valid >> (c / 2) & 1)) v[t][e] = (bf16)0.0f;
    }
    static constexpr int TILES = 2;
    using Q = bf16x8[KF];
};
template <int DH> struct Frags<float, DH> {
    static constexpr int KB = 16, KF = DH / 16, VF = DH / 16;
    floatx4 k[KF], v[VF];
    __device__ __forceinline__ static void load_q(floatx4 (&q)[KF], const float *row) {
        const int c = threadIdx.x % 64 / 16;
#pragma unroll
        for (int f = 0; f < KF; f++) q[f] = *(const floatx4 *)(row + 16 * f + 4 * c);
    }
    __device__ __forceinline__ static int key_of(int, int r) { return r; }
    __device__ __forceinline__ void load_k(const float *k0, const float *) {
        const int r = threadIdx.x % 16, c = threadIdx.x % 64 / 16;
#pragma unroll
        for (int f = 0; f < KF; f++) k[f] = *(const floatx4 *)(k0 + r * DH + 16 * f + 4 * c);
    }
    __device__ __forceinline__ void load_v(const float *v0, const float *, int page) {
        const int r = threadIdx.x % 16, c = threadIdx.x % 64 / 16;
        const float *src = v0 + r * page + 4 * c;
        asm volatile("" : "+s"(page));
#pragma unroll
        for (int t = 0; t < VF; t++) v[t] = *(const floatx4 *)(src + 16 * t * page);
    }
    __device__ __forceinline__ void scores(floatx4 (&s)[1], const floatx4 (&q)[KF]) const {
        s[0] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int f = 0; f < KF; f++)
#pragma unroll
            for (int e = 0; e < 4; e++) s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[f][e], q[f][e], s[0], 0, 0, 0);
    }
    __device__ __forceinline__ void add_values(floatx4 (&o)[VF], const floatx4 (&p)[1]) const {
#pragma unroll
        for (int e = 0; e < 4; e++)
#pragma unroll
            for (int t = 0; t < VF; t++) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][e], p[0][e], o[t], 0, 0, 0);
    }
    __device__ __forceinline__ void take_new(const NewRows<float> &n, float *k0, float *, float *v0, float *, int valid, int page) {
        const int r = threadIdx.x % 16, c = threadIdx.x % 64 / 16;
        const float *src = (n.has(r) ? n.k + (int64_t)r * n.stride : k0 + r * DH) + 4 * c;
#pragma unroll
        for (int f = 0; f < KF; f++) k[f] = *(const floatx4 *)(src + 16 * f);
        constexpr int AT_ONCE = DH > 64 ? 1 : 4;  // keys whose values are requested before any is used, without a branch (as many as the registers take)
#pragma unroll
        for (int e0 = 0; e0 < 4; e0 += AT_ONCE) {
            float x[AT_ONCE][VF];
#pragma unroll
            for (int i = 0; i < AT_ONCE; i++)
#pragma unroll
                for (int t = 0; t < VF; t++) x[i][t] = n.v[(int64_t)n.near(4 * c + e0 + i) * n.stride + 16 * t + r];
#pragma unroll
            for (int i = 0; i < AT_ONCE; i++) {
                const int key = 4 * c + e0 + i;
                const bool has = n.has(key), keep = has && n.keeps(key) && valid;
#pragma unroll
                for (int t = 0; t < VF; t++) {
                    v[t][e0 + i] = has ? x[i][t] : v[t][e0 + i];
                    if (keep) v0[(16 * t + r) * page + key] = x[i][t];
                }
            }
        }
        if (n.has(r) && n.keeps(r) && valid)
#pragma unroll
            for (int f = 0; f < KF; f++) *(floatx4 *)(k0 + r * DH + 16 * f + 4 * c) = k[f];
    }
    __device__ __forceinline__ void drop_values(int from, int valid) {
        const int c = threadIdx.x % 64 / 16;
#pragma unroll
        for (int t = 0; t < VF; t++)
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (4 * c + e >= from || !valid) v[t][e] = 0.0f;
    }
    static constexpr int TILES = 1;
    using Q = floatx4[KF];
};

// maximum and sum over the four lanes that hold one query's scores
__device__ __forceinline__ float query_max(float v) {
    v = halves_max(v);
    const uintx2 p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float query_sum(float v) {
    v = halves_sum(v);
    const uintx2 p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Few rows: MR groups of 16 rows per workgroup (each key read serves them all), whose four wavefronts walk blocks of the keys in turn, joined in LDS.
// The softmax runs with the walk: maximum and sum so far, the sums rescaled when the maximum grows.  New tokens are taken from k_new and v_new where the walk
// meets them, and the tile that they belong to leaves them on their page: a call of single tokens has no launch of its own for them.
// With one token per sequence the time is the reading: bf16, 64 sequences of 512 to 8192 keys, 8 key heads of 128 columns, 217 us, 5.2 TB/s; two of 100001 to
// 131072 keys in 32 parts 164 us, 5.7 TB/s (a copy reaches 5.25).  Many float32 rows are bound by their products: 16 sequences of 300 tokens over 4000, 16 heads of
// 64 columns, 741 us, 0.1 PFLOP/s, three quarters of a large product's rate; 32 heads of 128 columns 2960 (16 rows per workgroup 4170: every key is read twice as
// often).  Where 832 tiles meet 768 places, as with 32 sequences, 1 to 96 tokens of 16 heads of 64 columns and a window of 1024 (101 us), half of that.
template <typename T, int DH, int MR> __global__ __launch_bounds__(256, MR * DH <= 64 ? 4 : MR == 2 && DH <= 64 ? 3 : 2) void paged_rows(PagedArgs a) {
    using F = Frags<T, DH>;
    constexpr int KB = F::KB, VF = F::VF, NW = 4, ROWS = 16 * MR;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, c = lane / 16;
    const int split = blockIdx.x % a.nsplit, kvh = blockIdx.x / a.nsplit % a.Hkv, page = 1 << a.page_shift;
    Sequence s;
    if (!find_longest_first(a, blockIdx.x / (a.nsplit * a.Hkv), [&](int m, int) { return (m * a.group + ROWS - 1) / ROWS; }, s)) return;
    const int R0 = s.tile * ROWS, R1 = min(R0 + ROWS, s.m * a.group), base = s.len - s.m;
    const int p_lo = base + R0 / a.group, p_hi = base + (R1 - 1) / a.group;
    const Blocks bl = visible_blocks<KB>(a, p_lo, p_hi);
    const int each = (bl.count + a.nsplit * NW - 1) / (a.nsplit * NW);
    // The wavefronts take the workgroup's blocks [y0, y1) in turn, so that each has its share of the new tokens, which cost more (16 sequences of 300 float32 tokens
    // over 4000: 3150 us with stretches of their own, 2960 in turn; two tokens over 100001 to 131072 172 and 164).  Of a few blocks they take stretches: the last
    // wavefront, which meets the new token, then has the fewest (one token over 777: 10 us, 11.2 in turn; the widest kind has no register left for the choice).
    const int y0 = min(split * NW * each, bl.count), y1 = min(y0 + NW * each, bl.count);
    const int step = MR * DH <= 128 && each <= 16 ? 1 : NW, x0 = step == 1 ? min(y0 + wave * each, y1) : y0 + wave, x1 = step == 1 ? min(x0 + each, y1) : y1;

    int p[MR];
    typename F::Q q[MR];
#pragma unroll
    for (int i = 0; i < MR; i++) {
        const int R = R0 + 16 * i + n, tok = R / a.group, head = kvh * a.group + R - tok * a.group;
        p[i] = R < R1 ? base + tok : -1;
        // (rows past the last repeat a token's: they are computed and dropped)
        F::load_q(q[i], (const T *)a.q + (int64_t)(s.start + min(tok, s.m - 1)) * a.q_stride + head * DH);
    }

    // page numbers: one of 64 successive pages per lane
    int ids = 0, ids_from = -64;
    auto page_id = [&](int key) {
        const int pg = key >> a.page_shift;
        if (pg >= ids_from + 64) {
            ids_from = pg;
            ids = page_numbers(a, s.b, pg);
        }
        return __builtin_amdgcn_readlane(ids, pg - ids_from);
    };
    struct Source { const T *k0, *k1, *v0, *v1; int valid; };  // valid: bit i: keys 16 i .. 16 i + 15 of the block lie on a page that exists
    auto source = [&](int x) {
        Source r;
        const int key = bl.at(x) * KB, id = page_id(key), slot = key & (page - 1);
        const bool there = id >= 0 && id < a.n_pages;
        const int64_t hd = (int64_t)(there ? id : 0) * a.Hkv + kvh;
        r.valid = there ? 3 : 0;
        r.k0 = (const T *)a.k + (hd * page + slot) * DH;
        r.v0 = (const T *)a.v + hd * DH * page + slot;
        r.k1 = r.k0 + 16 * DH;
        r.v1 = r.v0 + 16;
        if (KB == 32 && page == 16) {  // the block's second half lies on the next page
            const int id1 = page_id(key + 16);
            const bool there1 = id1 >= 0 && id1 < a.n_pages;
            const int64_t hd1 = (int64_t)(there1 ? id1 : 0) * a.Hkv + kvh;
            r.valid = (there ? 1 : 0) | (there1 ? 2 : 0);
            r.k1 = (const T *)a.k + hd1 * page * DH;
            r.v1 = (const T *)a.v + hd1 * DH * page;
        }
        return r;
    };

    F f;
    floatx4 o[MR][VF];
    float m_run[MR], l_run[MR];
#pragma unroll
    for (int i = 0; i < MR; i++) {
        m_run[i] = -INFINITY;
        l_run[i] = 0.0f;
#pragma unroll
        for (int t = 0; t < VF; t++) o[i][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // One block; NEXT: the keys and values of the next are requested when this one's have been used; NEW: there may be new tokens in it.  (No branch stands
    // between a request and its use: the compiler would wait for everything behind it.)
    Source src;
    auto block = [&](auto next, auto fresh, int x) {
        constexpr bool NEXT = decltype(next)::value, NEW = decltype(fresh)::value;
        const int key0 = bl.at(x) * KB, valid = src.valid;
        if constexpr (NEW) {
            const int64_t row = (int64_t)(s.start + key0 - base) * a.kv_stride + kvh * DH;
            const NewRows<T> nr = {(const T *)a.k_new + row, (const T *)a.v_new + row, a.kv_stride, base - key0, s.len - key0, p_lo - key0, p_hi - key0};
            f.take_new(nr, (T *)src.k0, (T *)src.k1, (T *)src.v0, (T *)src.v1, valid, page);
        }
        floatx4 sc[MR][F::TILES];
#pragma unroll
        for (int i = 0; i < MR; i++) f.scores(sc[i], q[i]);
        if constexpr (NEXT) {
            src = source(x + step);
            f.load_k(src.k0, src.k1);
        }
        const bool whole = valid == 3 && key0 + KB - 1 <= p_lo && (!a.window || p_hi - key0 < a.window || key0 + KB <= a.sinks);
        if (!whole) {
#pragma unroll
            for (int i = 0; i < MR; i++)
#pragma unroll
                for (int u = 0; u < F::TILES; u++)
#pragma unroll
                    for (int v = 0; v < 4; v++) {
                        const int kk = F::key_of(u, 4 * c + v);
                        if (!sees(a, p[i], key0 + kk) || !(valid >> (kk / 16) & 1)) sc[i][u][v] = -INFINITY;
                    }
            if (key0 + KB - 1 > p_hi || valid != 3) f.drop_values(p_hi + 1 - key0, valid);
        }
        float mx[MR];
        bool outgrown = false;
#pragma unroll
        for (int i = 0; i < MR; i++) {
            mx[i] = -INFINITY;
#pragma unroll
            for (int u = 0; u < F::TILES; u++)
#pragma unroll
                for (int v = 0; v < 4; v++) mx[i] = fmaxf(mx[i], sc[i][u][v]);
            mx[i] = query_max(mx[i]) * a.scale_log2e;
            outgrown |= mx[i] > m_run[i] + 8.0f;
        }
        // the maximum in use follows when it is outgrown by 2^8: terms up to 256 harm nothing
        if (__builtin_amdgcn_ballot_w64(outgrown) != 0) {
            asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");  // (in place by hand, as in paged_flash; the matrix instructions' results may be read after the pause)
#pragma unroll
            for (int i = 0; i < MR; i++) {
                const float mn = mx[i] > m_run[i] + 8.0f ? mx[i] : m_run[i];
                const float alpha = m_run[i] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[i] - mn);
                m_run[i] = mn;
                l_run[i] *= alpha;
#pragma unroll
                for (int t = 0; t < VF; t++)
#pragma unroll
                    for (int v = 0; v < 4; v++) {
                        float y = o[i][t][v];
                        asm volatile("v_mul_f32 %0, %0, %1" : "+v"(y) : "v"(alpha));
                        o[i][t][v] = y;
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < MR; i++) {
            const float neg = m_run[i] == -INFINITY ? 0.0f : -m_run[i];
#pragma unroll
            for (int u = 0; u < F::TILES; u++)
#pragma unroll
                for (int v = 0; v < 4; v++) {
                    sc[i][u][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][u][v], a.scale_log2e, neg));
                    l_run[i] += sc[i][u][v];
                }
            f.add_values(o[i], sc[i]);
        }
        if constexpr (NEXT) f.load_v(src.v0, src.v1, page);
    };
    if (x0 < x1) {
        src = source(x0);
        f.load_k(src.k0, src.k1);
        f.load_v(src.v0, src.v1, page);
        constexpr std::true_type yes;
        constexpr std::false_type no;
        // From block xn on there are new tokens: they are read where they are, and written into their pages by the tile of the token's own rows, which always
        // walks its block (where two tiles share a token they write the same).
        int xn = x1;
        if (a.k_new) {
            const int first = max(base, 0) / KB;
            xn = min(max(first < bl.first ? first : max(bl.first, first - bl.from + bl.first), x0), x1);
        }
        int x = x0;
        for (; x < xn && x + step < x1; x += step) block(yes, no, x);
        for (; x + step < x1; x += step) block(yes, yes, x);
        if (x < xn) block(no, no, x);
        else block(no, yes, x);
    }

    // the wavefronts' shares, joined in their order, 16 rows at a time
    const PagedArgs z = late_args();
    __shared__ float sm[NW][16], sl[NW][16];
    __shared__ __attribute__((aligned(16))) float so[NW][16][DH + 4];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < MR; i++) {
        const float l = query_sum(l_run[i]);
        if (i) __syncthreads();
        if (c == 0) {
            sm[wave][n] = m_run[i];
            sl[wave][n] = l;
        }
#pragma unroll
        for (int t = 0; t < VF; t++) *(floatx4 *)&so[wave][n][16 * t + 4 * c] = o[i][t];
        __syncthreads();
        for (int j = threadIdx.x; j < 16 * DH; j += 256) {
            const int r = j / DH, d = j % DH, RR = R0 + 16 * i + r;
            if (RR >= R1) continue;
            float m = sm[0][r];
#pragma unroll
            for (int w = 1; w < NW; w++) m = fmaxf(m, sm[w][r]);
            float sum = 0.0f, v = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; w++) {
                const float f_ = sm[w][r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm[w][r] - m);
                sum = fmaf(sl[w][r], f_, sum);
                v = fmaf(so[w][r][d], f_, v);
                bad |= !(fabsf(so[w][r][d]) < INFINITY) || !(sl[w][r] < INFINITY);
            }
            const int tk = RR / z.group, row = s.start + tk, hd = kvh * z.group + RR - tk * z.group;
            if (z.nsplit > 1) {
                float *part = part_row<DH>(z, row, hd, split);
                part[d] = v;
                if (d == 0) {
                    part[DH] = m;
                    part[DH + 1] = sum;
                }
            } else {
                out_row<T, DH>(z, row, hd)[d] = from_f<T>(sum == 0.0f ? 0.0f : v / sum);
            }
        }
    }
    if (__syncthreads_or(bad)) {
        for (int r = wave; r < R1 - R0; r += NW) {
            const int RR = R0 + r, tk = RR / z.group;
            plain_row<T, DH, KB>(z, s, bl, y0, y1, kvh, s.start + tk, kvh * z.group + RR - tk * z.group, base + tk, split);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Many rows: 32 NW rows (token, head of the group) of one (sequence, key head) per workgroup, 32 to a wavefront.  The keys stream through LDS in
// tiles of 64 [64 x DH] with their values [DH x 64], SLOTS of each, filled by direct global->LDS loads.  Both products are transposed, so a lane owns
// a row: its maximum and sum are its own, and P^T leaves the first product as the second's operand (key rows enter with bits 2 and 3 of their index
// swapped, which makes the eight keys a lane holds for one MFMA step consecutive; the weights are rounded to bf16 there, while their sum keeps 32 bits).
// The matrix cores and the vector instructions of the softmax need about the same time, so a wavefront runs them side by side: the scores of tile x + 1 are
// formed while those of tile x become weights.  (64 rows per wavefront halve the reads of LDS and do not fit the registers: 1075 us for what takes 314.)
// bf16, 4 sequences of 1000 to 1024 new tokens among up to 8192, 32 heads of 128 columns over 8: 314 us under the tracer, and 292 to 302 for a call among others, the
// pages' update with it, 0.9 PFLOP/s of the products that the mask leaves; the matrix cores are busy for 40 % of the cycles, the rest is the softmax's and the reads of LDS.
// ---------------------------------------------------------------------------------------------------------------------
template <int DH, int NW, int SLOTS> __global__ __launch_bounds__(NW * 64, 2) void paged_flash(PagedArgs a) {
    constexpr int ROWS = NW * 32, KT = 64, KCH = DH / 8, HALF = KT * KCH, KSTEPS = DH / 16, MT = DH / 32, KI = HALF / 64 / NW, LEAD = SLOTS - 1;
    static_assert(KI * 64 * NW == HALF, "every wavefront loads as much of a tile");
    extern __shared__ bf16x8 smem[];  // keys of SLOTS tiles, values of SLOTS tiles: HALF chunks each
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), frow = lane % 32, hf = lane / 32;
    const int split = blockIdx.x / a.Hkv % a.nsplit, kvh = blockIdx.x % a.Hkv, page = 1 << a.page_shift;
    Sequence s;
    if (!find_longest_first(a, blockIdx.x / (a.nsplit * a.Hkv), [&](int m, int) { return (m * a.group + ROWS - 1) / ROWS; }, s)) return;
    // (the last rows of a sequence see the most keys: first)
    const int R0 = ((s.m * a.group + ROWS - 1) / ROWS - 1 - s.tile) * ROWS, R1 = min(R0 + ROWS, s.m * a.group), base = s.len - s.m;
    const int p_lo = base + R0 / a.group, p_hi = base + (R1 - 1) / a.group;
    const Blocks bl = visible_blocks<KT>(a, p_lo, p_hi);
    const int each = (bl.count + a.nsplit - 1) / a.nsplit, x0 = min(split * each, bl.count), x1 = min(x0 + each, bl.count);

    const int W0 = R0 + wave * 32;  // the wavefront's first row
    int p;
    bf16x8 qf[KSTEPS];
    {
        const int R = W0 + frow, tok = R / a.group, head = kvh * a.group + R - tok * a.group;
        p = R < R1 ? base + tok : -1;
        // (rows past the last repeat a token's: they are computed and dropped)
        const bf16 *q = (const bf16 *)a.q + (int64_t)(s.start + min(tok, s.m - 1)) * a.q_stride + head * DH + 8 * hf;
#pragma unroll
        for (int st = 0; st < KSTEPS; st++) qf[st] = *(const bf16x8 *)(q + 16 * st);
    }

    // Page numbers: one of 64 successive pages per lane.  Every wavefront loads its share of a tile, so all keep them.
    int ids = 0, ids_from = 0;
    auto want_pages = [&](int x) {  // uniform
        const int first = bl.at(x) * KT >> a.page_shift, last = (bl.at(x) * KT + KT - 1) >> a.page_shift;
        if (x == x0 || last >= ids_from + 64) {
            ids_from = first;
            ids = page_numbers(a, s.b, first);
        }
    };
    auto exists = [&](int id) { return id >= 0 && id < a.n_pages; };
    // A lane's place in a load of 64 chunks does not depend on which of its loads it is: chunk c of row r lies at c ^ swizzle(r)
    constexpr int KR = 64 / KCH;  // rows of K per load
    auto swizzle = [](int r) { return KCH == 16 ? r & 15 : KCH == 8 ? (r >> 1) & 7 : (r >> 2) & 3; };  // 16 successive rows' same chunk: 256 bytes of LDS, all banks once
    const int k_row = lane / KCH, k_swz = swizzle(wave * KR + k_row);
    const unsigned k_off = (unsigned)(k_row * DH + (((lane % KCH) ^ k_swz) * 8));
    const int v_row = wave * 8 + lane / 8, v_chunk = (lane % 8) ^ ((v_row >> 1) & 7);
    const unsigned v_off = (unsigned)(v_row * page + 8 * v_chunk);
    auto dma = [&](const bf16 *src, bf16x8 *dst) {
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1))) *)src, (void __attribute__((address_space(3))) *)dst, 16, 0, 0);
    };
    // A tile on one page (page_size >= 64): where this head's part of the page begins, and whether the page exists (otherwise page 0 is loaded and masked)
    auto page_start = [&](int x, bool &there) {
        const int id = __builtin_amdgcn_readlane(ids, (bl.at(x) * KT >> a.page_shift) - ids_from);
        there = exists(id);
        return ((int64_t)(there ? id : 0) * a.Hkv + kvh) * (DH << a.page_shift);
    };
    auto issue_k_at = [&](int64_t start, int slot0, int buf) {
        const bf16 *src = (const bf16 *)a.k + start + (slot0 + wave * KR) * DH;
        bf16x8 *dst = smem + buf * HALF + wave * 64;
#pragma unroll
        for (int i = 0; i < KI; i++) dma(src + i * NW * KR * DH + k_off, dst + i * NW * 64);
    };
    auto issue_v_at = [&](int64_t start, int slot0, int buf) {
        const bf16 *src = (const bf16 *)a.v + start + slot0;
        bf16x8 *dst = smem + (SLOTS + buf) * HALF + wave * 64;
#pragma unroll
        for (int i = 0; i < KI; i++) dma(src + i * NW * 8 * page + v_off, dst + i * NW * 64);
    };
    // Tiles on several small pages: a page per load of keys (at most 16 rows each), a page per lane for the values
    auto issue_k_small = [&](int x, int buf) {
        const int key0 = bl.at(x) * KT, slot0 = key0 & (page - 1), pg0 = (key0 >> a.page_shift) - ids_from;
        bf16x8 *dst = smem + buf * HALF + wave * 64;
#pragma unroll
        for (int i = 0; i < KI; i++) {
            const int slot = slot0 + (i * NW + wave) * KR, id = __builtin_amdgcn_readlane(ids, pg0 + (slot >> a.page_shift));
            dma((const bf16 *)a.k + (((int64_t)(exists(id) ? id : 0) * a.Hkv + kvh) * page + (slot & (page - 1))) * DH + k_off, dst + i * NW * 64);
        }
    };
    auto issue_v_small = [&](int x, int buf) {
        const int key0 = bl.at(x) * KT, slot = (key0 & (page - 1)) + 8 * v_chunk, pg = (key0 >> a.page_shift) - ids_from;
        const int id = __builtin_amdgcn_ds_bpermute((pg + (slot >> a.page_shift)) * 4, ids);
        const bf16 *src = (const bf16 *)a.v + (((int64_t)(exists(id) ? id : 0) * a.Hkv + kvh) * DH + v_row) * page + (slot & (page - 1));
        bf16x8 *dst = smem + (SLOTS + buf) * HALF + wave * 64;
#pragma unroll
        for (int i = 0; i < KI; i++) dma(src + i * NW * 8 * page, dst + i * NW * 64);
    };
    // bit i: chunk i of a tile's keys lies on a page that exists
    auto valid_small = [&](int x) -> unsigned {
        const int key0 = bl.at(x) * KT, slot = (key0 & (page - 1)) + 8 * (lane % 8);
        const int id = __builtin_amdgcn_ds_bpermute(((key0 >> a.page_shift) - ids_from + (slot >> a.page_shift)) * 4, ids);
        return (unsigned)__builtin_amdgcn_ballot_w64(exists(id)) & 0xFFu;
    };

    float m_run = -INFINITY, l_run = 0.0f;
    floatx16 o[MT];
#pragma unroll
    for (int mt = 0; mt < MT; mt++)
#pragma unroll
        for (int v = 0; v < 16; v++) o[mt][v] = 0.0f;
    // Fragments by their LDS address: chunk c of row r lies at c ^ swizzle(r), and c = 2 step + hf, so a step flips bits above the lane's own address; the
    // address is made anew for every tile (kept for every step it costs registers that spill).
    typedef const __attribute__((address_space(3))) bf16x8 *LdsChunk;
    const int krow = (frow & 0x13) | ((frow & 4) << 1) | ((frow & 8) >> 1);
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const unsigned k_lane = lds0 + (unsigned)(krow * KCH + (hf ^ swizzle(krow))) * 16, v_lane = lds0 + SLOTS * HALF * 16 + (unsigned)(frow * 8 + (hf ^ ((frow >> 1) & 7))) * 16;
    auto at_tile = [&](unsigned lane_address, int buf) {
        unsigned r = lane_address + (unsigned)buf * (HALF * 16);
        asm volatile("" : "+v"(r));
        return r;
    };
    auto key_frag = [&](unsigned k, int sub, int st) { return *((LdsChunk)(k ^ (unsigned)(st << 5)) + sub * 32 * KCH); };
    auto value_frag = [&](unsigned v, int ks, int mt) { return *((LdsChunk)(v ^ (unsigned)(ks << 5)) + mt * 256); };
    struct Scores { floatx16 s[2]; };  // a lane holds, of its row, keys 32 sub + 16 (v / 8) + 8 hf + v % 8
    bf16x8 pf[4];  // weights, rounded once as the operand of the matrix instruction (the normaliser adds them unrounded)
    float neg;     // minus the maximum in use
    // two weights of the lane's row, keys 2 u and 2 u + 1 of its 32, in two parts: the exponentials, and (a step later, when they are there) their sum and rounding
    auto weigh = [&](Scores &c, int u) {
#pragma unroll
        for (int e = 2 * u; e < 2 * u + 2; e++) {
            float w = __builtin_amdgcn_exp2f(__builtin_fmaf(c.s[e / 16][e % 16], a.scale_log2e, neg));
            asm volatile("" : "+v"(w));  // (formed here, beside the matrix instructions, and not in the later block that uses it)
            c.s[e / 16][e % 16] = w;
        }
    };
    auto settle = [&](const Scores &c, int u) {
#pragma unroll
        for (int e = 2 * u; e < 2 * u + 2; e++) {
            const float w = c.s[e / 16][e % 16];
            l_run += w;
            pf[e / 8][e % 8] = (bf16)w;
        }
        asm volatile("" : "+v"(l_run));
        if (u % 4 == 3) asm volatile("" : "+v"(pf[u / 4]));
    };
    auto weights_upto = [&](Scores &c, int u0, int u1) {
#pragma unroll
        for (int u = u0; u < u1; u++) {
            weigh(c, u);
            if (u > 0) settle(c, u - 1);
        }
    };
#define SB __builtin_amdgcn_sched_barrier(0)
    constexpr int AHEAD = 4;
    constexpr int PAIRS = 16, UNDER_SCORES = 12;  // pairs of weights of a tile; those formed under the next tile's first product
    // scores of a tile into n, beside the weights of the tile in c (WEIGH; without NEXT the weights alone).  The two halves of the keys in turn, so that the
    // weights have left half of c's registers before the second half of n needs its own.
    auto scores = [&](auto next, auto weights, unsigned sk, Scores &n, Scores &c) {
        constexpr bool NEXT = decltype(next)::value, WEIGH = decltype(weights)::value;
        constexpr int MM = 2 * KSTEPS;
        bf16x8 kf[AHEAD];  // fragments are read AHEAD - 1 steps before their MFMAs: the LDS answers in the time of several
        if constexpr (NEXT) {
#pragma unroll
            for (int f = 0; f < AHEAD - 1; f++) kf[f] = key_frag(sk, f / KSTEPS, f % KSTEPS);
        }
#pragma unroll
        for (int sub = 0; sub < 2; sub++) {
            if constexpr (NEXT) {
#pragma unroll
                for (int v = 0; v < 16; v++) n.s[sub][v] = 0.0f;
            }
#pragma unroll
            for (int st = 0; st < KSTEPS; st++) {
                const int f = sub * KSTEPS + st, ahead = f + AHEAD - 1;
                if constexpr (NEXT)
                    if (ahead < 2 * KSTEPS) kf[ahead % AHEAD] = key_frag(sk, ahead / KSTEPS, ahead % KSTEPS);
                if constexpr (NEXT) n.s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[f % AHEAD], qf[st], n.s[sub], 0, 0, 0);
                if constexpr (WEIGH) weights_upto(c, f * UNDER_SCORES / MM, (f + 1) * UNDER_SCORES / MM);
                SB;
            }
        }
    };
    float mx;
    // values of a tile, beside its last weights and the maxima of the scores in n
    auto values = [&](auto next, unsigned sv, Scores &c, Scores &n) {
        constexpr bool NEXT = decltype(next)::value;
        constexpr int MM = 4 * MT, LATE = PAIRS - UNDER_SCORES, half = MM / 2;
        mx = -INFINITY;
        bf16x8 vf[AHEAD];
#pragma unroll
        for (int g = 0; g < AHEAD - 1; g++) vf[g] = value_frag(sv, g / MT, g % MT);
#pragma unroll
        for (int ks = 0; ks < 4; ks++)
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                const int g = ks * MT + mt;
                if (g + AHEAD - 1 < 4 * MT) vf[(g + AHEAD - 1) % AHEAD] = value_frag(sv, (g + AHEAD - 1) / MT, (g + AHEAD - 1) % MT);
                o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[g % AHEAD], pf[ks], o[mt], 0, 0, 0);
                if (g < half) {
                    weights_upto(c, UNDER_SCORES + g * LATE / half, UNDER_SCORES + (g + 1) * LATE / half);
                    if (g == half - 1) settle(c, PAIRS - 1);
                } else if constexpr (NEXT) {
#pragma unroll
                    for (int u = (g - half) * PAIRS / half; u < (g - half + 1) * PAIRS / half; u++) mx = fmaxf(fmaxf(mx, n.s[u / 8][2 * u % 16]), n.s[u / 8][2 * u % 16 + 1]);
                }
                SB;
            }
    };
    auto mask = [&](int key0, unsigned valid, Scores &n) {
        if (valid != 0xFF || key0 + KT - 1 > p_lo || (a.window && p_hi - key0 >= a.window && key0 + KT > a.sinks)) {
            int hf_ = hf;
            asm volatile("" : "+v"(hf_));  // (nothing of this is kept in registers over the tiles that need none of it)
            const unsigned ok = valid >> hf_;
            const int k0 = key0 + 8 * hf_, sinks = a.window ? a.sinks - k0 : KT;
            const int last = p - k0, from = a.window ? last - a.window + 1 : 0;  // of the lane's keys, counted from k0
#pragma unroll
            for (int sub = 0; sub < 2; sub++)
#pragma unroll
                for (int v = 0; v < 16; v++) {
                    const int kk = 32 * sub + 16 * (v / 8) + v % 8;
                    const bool seen = (kk <= last) & ((kk >= from) | (kk < sinks)) & ((ok >> (kk / 8) & 1) != 0);
                    n.s[sub][v] = seen ? n.s[sub][v] : -INFINITY;
                }
        }
    };
    auto follow = [&]() {  // the maximum in use follows when some row outgrew it by 2^8: terms up to 256 harm nothing
        mx = halves_max(mx) * a.scale_log2e;
        const bool outgrown = mx > m_run + 8.0f;
        if (__builtin_amdgcn_ballot_w64(outgrown) != 0) {
            // In place by hand: as plain products the sums get second registers and a copy on the common path, 64 of them at DH = 128.  The matrix
            // instructions' results may be read after the pause (at most 19 wait states).
            asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
            const float mn = outgrown ? mx : m_run, alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run - mn);
            m_run = mn;
            l_run *= alpha;
#pragma unroll
            for (int mt = 0; mt < MT; mt++)
#pragma unroll
                for (int v = 0; v < 16; v++) {
                    float x = o[mt][v];
                    asm volatile("v_mul_f32 %0, %0, %1" : "+v"(x) : "v"(alpha));
                    o[mt][v] = x;
                }
        }
        neg = m_run == -INFINITY ? 0.0f : -m_run;
    };
    // Group x of the loads: the values of tile x and the keys of tile x + 1, into slots x and x + 1 (modulo SLOTS).  Past the end the last tile is loaded again,
    // into slots that nobody reads any more, so that the waits need no cases.
    uint64_t valid = 0;  // byte i: valid chunks of tile x + i
    const bool paged_tiles = a.page_shift >= 6;
    int64_t start = 0;   // page_start of the tile whose keys were requested last
    auto issue_k = [&](int x, int slot, int byte) {
        want_pages(x);
        if (paged_tiles) {
            bool there;
            start = page_start(x, there);
            issue_k_at(start, (bl.at(x) * KT) & (page - 1), slot);
            valid |= (uint64_t)(there ? 0xFF : 0) << (8 * byte);
        } else {
            issue_k_small(x, slot);
            valid |= (uint64_t)valid_small(x) << (8 * byte);
        }
    };
    auto issue = [&](int x, int slot, int byte) {
        const int here = min(x, x1 - 1);
        if (paged_tiles) issue_v_at(start, (bl.at(here) * KT) & (page - 1), slot);
        else issue_v_small(here, slot);
        issue_k(min(x + 1, x1 - 1), slot + 1 == SLOTS ? 0 : slot + 1, byte + 1);
    };
    auto meet = [&](auto left) {  // all but the newest `left` groups have landed, everybody's
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(left)::value * 2 * KI) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::true_type yes;
    constexpr std::false_type no;
    if (x0 < x1) {
        Scores s0, s1;
        issue_k(x0, 0, 0);
#pragma unroll
        for (int g = 0; g < LEAD; g++) issue(x0 + g, g, g);
        meet(std::integral_constant<int, LEAD>());
        scores(yes, no, at_tile(k_lane, 0), s0, s1);
        mask(bl.at(x0) * KT, (unsigned)valid & 0xFF, s0);
        mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < 32; k++) mx = fmaxf(mx, s0.s[k / 16][k % 16]);
        follow();
        int slot = 0;  // of tile x
        auto after = [&](int n) { return slot + n >= SLOTS ? slot + n - SLOTS : slot + n; };
        auto arrive = [&](int x) {  // tile x's values and tile x + 1's keys have landed
            meet(std::integral_constant<int, LEAD - 1>());
            issue(x + LEAD, after(LEAD), LEAD);
            const int key0 = bl.at(x) * KT;
            const unsigned here = (unsigned)valid & 0xFF;
            if (here != 0xFF || key0 + KT - 1 > p_hi) {
                // values no row of the workgroup may use: out of the product, where p = 0 would not keep an infinity or a NaN out
                bf16x8 *sv = smem + (SLOTS + slot) * HALF;
                int id = threadIdx.x;
                asm volatile("" : "+v"(id));
                for (; id < HALF; id += NW * 64) {
                    const int r = id / 8, ch = (id % 8) ^ ((r >> 1) & 7);
                    bf16x8 v = sv[id];
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (!(here >> ch & 1) || key0 + 8 * ch + e > p_hi) v[e] = (bf16)0.0f;
                    sv[id] = v;
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
        };
        // tile x, whose scores are in c; the next tile's go to n
        const bool idle = W0 >= R1;  // a wavefront without rows loads for the others
        auto step = [&](int x, Scores &c, Scores &n) {
            arrive(x);
            if (!idle) {
            scores(yes, yes, at_tile(k_lane, after(1)), n, c);
            mask(bl.at(x + 1) * KT, (unsigned)(valid >> 8) & 0xFF, n);
            values(yes, at_tile(v_lane, slot), c, n);
            follow();
            }
            valid >>= 8;
            slot = after(1);
        };
        auto last = [&](int x, Scores &c) {
            arrive(x);
            if (idle) return;
            scores(no, yes, 0u, c, c);
            values(no, at_tile(v_lane, slot), c, c);
        };
        int x = x0;
        for (; x + 1 < x1; x++) {
            step(x, s0, s1);
            s0 = s1;
        }
        last(x, s0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads in flight own their slots)
    }
#undef SB
    const PagedArgs z = late_args();
    bool bad = false;
    const float l = halves_sum(l_run);
    const int R = W0 + frow, tok = R / z.group, head = kvh * z.group + R - tok * z.group, row = s.start + tok;
    if (R < R1) {
        bad |= !(l < INFINITY);
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
            for (int v = 0; v < 16; v++) bad |= !(fabsf(o[mt][v]) < INFINITY);
        if (z.nsplit > 1) {
            float *part = part_row<DH>(z, row, head, split);
#pragma unroll
            for (int mt = 0; mt < MT; mt++)
#pragma unroll
                for (int v = 0; v < 16; v++) part[mt * 32 + 8 * (v / 4) + 4 * hf + v % 4] = o[mt][v];
            if (hf == 0) {
                part[DH] = m_run;
                part[DH + 1] = l;
            }
        } else {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            bf16 *dst = out_row<bf16, DH>(z, row, head);
#pragma unroll
            for (int mt = 0; mt < MT; mt++)
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    bf16x4 pk;
#pragma unroll
                    for (int j = 0; j < 4; j++) pk[j] = (bf16)(o[mt][4 * g + j] * inv);
                    *(bf16x4 *)(dst + mt * 32 + 8 * g + 4 * hf) = pk;
                }
        }
    }
    if (__builtin_amdgcn_ballot_w64(bad) != 0)
        for (int r = W0; r < W0 + 32 && r < R1; r++) {
            const int tk = r / z.group;
            plain_row<bf16, DH, KT>(z, s, bl, x0, x1, kvh, s.start + tk, kvh * z.group + r - tk * z.group, base + tk, split);
        }
}

// Joins the workgroups' shares of a row, out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s: WAVES wavefronts per row, each with shares of its own, four
// from 16 shares on.  Latency: 2048 rows of 128 columns in two shares 6.4 us, 64 rows in 32 shares 7.0.
template <typename T, int DH, int WAVES> __global__ __launch_bounds__(256) void paged_join(PagedArgs a) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, part_of = wave % WAVES;
    const int64_t w = (int64_t)blockIdx.x * (4 / WAVES) + wave / WAVES;  // (tile, key head, row)
    const int r = (int)(w % kRows), kvh = (int)(w / kRows % a.Hkv);
    Sequence s;
    const bool found = find_sequence(a, w / (kRows * a.Hkv), [&](int m, int) { return (m * a.group + kRows - 1) / kRows; }, s);
    const int R = found ? s.tile * kRows + r : 0;
    if (!found || R >= s.m * a.group) return;  // (all wavefronts of a row alike)
    const int tok = R / a.group, row = s.start + tok, head = kvh * a.group + R - tok * a.group;
    constexpr int E = (DH + 63) / 64;
    const float *part = part_row<DH>(a, row, head, 0);
    float m = -INFINITY, l = 0.0f;  // of share `lane` (at most 64)
    if (lane < a.nsplit) {
        m = part[(int64_t)lane * (DH + 2) + DH];
        l = part[(int64_t)lane * (DH + 2) + DH + 1];
    }
    const float most = wave_max(m), f = m == most ? (lane < a.nsplit ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f(m - most);
    l = wave_sum(l * f);
    float o[E] = {};
    const int each = (a.nsplit + WAVES - 1) / WAVES, i1 = min((part_of + 1) * each, a.nsplit);
#pragma unroll 8
    for (int i = part_of * each; i < i1; i++) {
        const float fi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i));
#pragma unroll
        for (int e = 0; e < E; e++)
            if (lane + 64 * e < DH) o[e] = fmaf(part[(int64_t)i * (DH + 2) + lane + 64 * e], fi, o[e]);
    }
    if (WAVES > 1) {
        __shared__ float sums[4][64 * E];
#pragma unroll
        for (int e = 0; e < E; e++) sums[wave][lane + 64 * e] = o[e];
        __syncthreads();
        if (part_of) return;
#pragma unroll
        for (int x = 1; x < WAVES; x++)
#pragma unroll
            for (int e = 0; e < E; e++) o[e] += sums[x][lane + 64 * e];
    }
#pragma unroll
    for (int e = 0; e < E; e++)
        if (lane + 64 * e < DH) out_row<T, DH>(a, row, head)[lane + 64 * e] = from_f<T>(l == 0.0f ? 0.0f : o[e] / l);
}

int shift_of(int page) {
    int s = 0;
    while ((1 << s) < page) s++;
    return s;
}

constexpr int kFlashRows = 256, kHalfFlashRows = 128;

// bound of the tiles of `rows` rows, of one key head
int64_t tiles_of(int N, int B, int group, int rows) {
    const int64_t all = (int64_t)N * group, n = all / rows + B;
    return n < all ? n : all;
}

// rows: of a tile: 16 or 32 (paged_rows), or 128 or 256 that share staged keys (paged_flash).  nsplit: workgroups that share a tile's keys.
struct Plan {
    int rows;
    int64_t tiles, join_tiles;
    int nsplit;
    size_t bytes;
    bool flash() const { return rows >= kHalfFlashRows; }
};
Plan plan_of(gr4ad_dtype dtype, int B, int N, int H, int Hkv, int dh, int page, int max_pages, int window, int sinks) {
    Plan p;
    const int group = H / Hkv;
    const int64_t rows = ceil_div64((int64_t)N * group, B);  // of a sequence and key head, on average
    // Rows share staged keys where there are more than two tiles of 32, or one of 16 with 128 columns (bf16; 8 key heads of 4 heads each; captured, us, not staged | staged.  64 columns,
    // 64 rows of a sequence: 4 sequences of 8000 keys 30.0 | 32.0, 32 of 2000 42.2 | 44.6; 96 rows: 44.6 | 33.3, 59.1 | 50.1.  128 columns, 32 rows: 42.1 | 37.8, 89.6 | 58.8, but 4 of 2000, which
    // are latency, 24.1 | 35.5).  Tiles of 256 rows halve the reads of the keys and tiles of 128 end earlier (128 columns, 128 rows | 256: 4 sequences of 8000 keys, 2048 rows 275 | 267; 32 of 2000
    // 581 | 600; 4 of 2000, 144 rows 42 | 50).
    if (dtype == GR4AD_BF16 && dh >= 32 && rows > (dh == 128 ? 16 : 64)) p.rows = rows > 128 && dh > 32 ? kFlashRows : kHalfFlashRows;  // (a tile of 32 columns is one load for each of four wavefronts)
    else p.rows = rows <= 16 ? 16 : 32;
    p.tiles = tiles_of(N, B, group, p.rows);
    p.join_tiles = tiles_of(N, B, group, kRows);
    const bool flash = p.flash();
    // Workgroups enough to fill the chip (counted as if all sequences had the same number of rows): one per compute unit for tiles of 256 rows, two for the
    // others (tiles of 32 rows, 832 of them: 102 us alone, 113 in halves with their join); with tiles of 16 rows, which stand for many sequences of their own
    // lengths, four where that many are near (512 of up to 8192 keys: alone 256 us, in halves 224, in quarters 236; 16 of 131072 keys in 16 parts 176 us, in 32 parts
    // 172, in 64 parts 190).  A part has 256 keys at least (1024 of the staged kinds), and a tile of 16 rows with 256 KB of keys and values at most stays whole: a call
    // from a program is bound by its launches, of which parts have one more and a workspace (one row of 777 keys, calls in a row, whole | in parts: bf16 of 64 columns 9.8 | 14.7 us; fp32 of
    // 128, twice beyond, 23.4 | 15.2.  Captured, bf16 of 64 columns: 512 keys 8.7 | 9.6, 777 10.2 | 9.4, 1024 12.1 | 10.0, 2048 19.1 | 11.3).
    const int64_t blocks = (int64_t)B * ceil_div64(rows, p.rows) * Hkv, enough = p.rows == kFlashRows ? 256 : p.rows == 16 && blocks >= 256 ? 1024 : 512, least = flash ? 1024 : 256;
    int64_t keys = (int64_t)max_pages * page;
    if (window && (int64_t)window + sinks + 64 < keys) keys = (int64_t)window + sinks + 64;
    const int64_t want = (enough + blocks - 1) / blocks, most = (keys + least - 1) / least, n = want < most ? want : most;
    const bool whole = p.rows == 16 && keys * 2 * dh * (dtype == GR4AD_BF16 ? 2 : 4) <= 256 << 10;
    p.nsplit = (int)(whole || n < 1 ? 1 : n > 64 ? 64 : n);
    p.bytes = p.nsplit > 1 ? (size_t)N * H * p.nsplit * (dh + 2) * sizeof(float) : 0;
    return p;
}

// More than 64 KB of LDS has to be asked for, on each device: every launch asks for its own.
int allow_lds(const void *kernel, int bytes) {
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e == hipSuccess ? GR4AD_OK : thread_hip_error("paged attention", e);
}

template <int DH, int NW, int SLOTS> int launch_flash(const PagedArgs &a, unsigned grid, hipStream_t st) {
    constexpr int LDS = 2 * SLOTS * 64 * DH * 2;
    if (LDS > 65536) {
        const int s = allow_lds((const void *)paged_flash<DH, NW, SLOTS>, LDS);
        if (s) return s;
    }
    hipLaunchKernelGGL((paged_flash<DH, NW, SLOTS>), dim3(grid), dim3(NW * 64), LDS, st, a);
    return GR4AD_OK;
}

template <typename T, int DH> int launch_rows(const PagedArgs &a, const Plan &p, hipStream_t st) {
    const int64_t grid = p.tiles * a.Hkv * a.nsplit, joined = p.join_tiles * a.Hkv * kRows;
    if (!launchable(grid, p.rows == kFlashRows ? 512 : 256) || (a.nsplit > 1 && !launchable(joined, 256))) return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "paged attention: %d rows of %d heads", a.N, a.H);
    if (p.rows == 16) {
        hipLaunchKernelGGL((paged_rows<T, DH, 1>), dim3((unsigned)grid), dim3(256), 0, st, a);
    } else if (p.rows == 32) {
        // (more than 16 bf16 rows of 128 columns are always staged)
        if constexpr (DH <= 64 || sizeof(T) == 4) hipLaunchKernelGGL((paged_rows<T, DH, 2>), dim3((unsigned)grid), dim3(256), 0, st, a);
    } else if constexpr (sizeof(T) == 2 && DH >= 32) {
        // (half the rows: two workgroups share a compute unit and its LDS)
        int s = GR4AD_OK;
        if (p.rows == kHalfFlashRows) s = launch_flash<DH, kHalfFlashRows / 32, DH == 128 ? 2 : 4>(a, (unsigned)grid, st);
        else if constexpr (DH > 32) s = launch_flash<DH, kFlashRows / 32, 4>(a, (unsigned)grid, st);
        if (s) return s;
    }
    GR4AD_LAUNCH_CHECK_AS("paged attention");
    if (a.nsplit > 1) {
        if (a.nsplit >= 16) hipLaunchKernelGGL((paged_join<T, DH, 4>), dim3((unsigned)joined), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((paged_join<T, DH, 1>), dim3((unsigned)(joined / 4)), dim3(256), 0, st, a);
        GR4AD_LAUNCH_CHECK_AS("paged attention");
    }
    return GR4AD_OK;
}
template <typename T> int launch_width(const PagedArgs &a, int dh, const Plan &p, hipStream_t st) {
    switch (dh) {
        case 16: return launch_rows<T, 16>(a, p, st);
        case 32: return launch_rows<T, 32>(a, p, st);
        case 64: return launch_rows<T, 64>(a, p, st);
        default: return launch_rows<T, 128>(a, p, st);
    }
}

const int kMostKeys = 1 << 30;  // positions and their differences stay in 32 bits

// what both entry points check; a message and a status for the caller
int check_shape(gr4ad_dtype dtype, const gr4ad_paged_cache *c, int32_t B, int32_t N, int32_t H, int32_t window, int32_t sinks) {
    if (!c) return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: cache is NULL");
    if (dtype != GR4AD_F32 && dtype != GR4AD_BF16) return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: dtype %d", (int)dtype);
    if (B < 1 || N < 1 || H < 1 || c->H_kv < 1 || c->n_pages < 1 || c->max_pages < 1 || window < 0 || sinks < 0)
        return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: sizes must be positive (B %d, N %d, H %d, H_kv %d, n_pages %d, max_pages %d), window %d and sinks %d not negative", B, N, H,
                                      c->H_kv, c->n_pages, c->max_pages, window, sinks);
    if (H % c->H_kv) return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: H = %d is not divisible by H_kv = %d", H, c->H_kv);
    if (c->dh != 16 && c->dh != 32 && c->dh != 64 && c->dh != 128) return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "paged attention: head width %d (16, 32, 64, 128)", c->dh);
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
        return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "paged attention: page_size %d is not a power of two from 16 to 1024", c->page_size);
    if ((int64_t)c->max_pages * c->page_size > kMostKeys || (int64_t)N * H > kMostKeys || (int64_t)B * c->H_kv > kMostKeys)
        return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "paged attention: more than 2^30 positions of a sequence, rows times heads or sequences times heads");
    if ((int64_t)H * c->dh > 0x7fffffffLL)  // (a column's place in its row is a number of 32 bits)
        return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "paged attention: rows of 2^31 values or more (%d heads of %d)", H, c->dh);
    return GR4AD_OK;
}

}  // namespace

extern "C" {

size_t gr4ad_op_paged_attention_workspace_bytes(gr4ad_dtype dtype, const gr4ad_paged_cache *cache, int32_t B, int32_t N, int32_t H, int32_t window, int32_t sinks) {
    if (check_shape(dtype, cache, B, N, H, window, sinks)) return 0;
    return plan_of(dtype, B, N, H, cache->H_kv, cache->dh, cache->page_size, cache->max_pages, window, sinks).bytes;
}

int gr4ad_op_paged_attention(gr4ad_dtype dtype, const gr4ad_paged_cache *cache, const void *q, int64_t q_stride, const void *k_new, const void *v_new, int64_t kv_stride,
                             const int32_t *q_start, const int32_t *seq_len, void *out, int32_t B, int32_t N, int32_t H, float scale, int32_t window, int32_t sinks,
                             void *workspace, size_t workspace_bytes, void *hip_stream) {
    int s = check_shape(dtype, cache, B, N, H, window, sinks);
    if (s) return s;
    const gr4ad_paged_cache &c = *cache;
    if (!q || !q_start || !seq_len || !out || !c.k_pages || !c.v_pages || !c.page_table || !k_new != !v_new)
        return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: NULL pointer (k_new and v_new: both or neither)");
    if (!(scale > 0.0f) || !(scale < INFINITY)) return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: scale must be positive and finite");
    const int piece = dtype == GR4AD_BF16 ? 8 : 4;
    if (q_stride < (int64_t)H * c.dh || (k_new && kv_stride < (int64_t)c.H_kv * c.dh)) return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: rows overlap (strides in elements)");
    if (q_stride % piece || kv_stride % piece || (uintptr_t)k_new % 16 || (uintptr_t)v_new % 16 || (uintptr_t)q % 16 || (uintptr_t)c.k_pages % 16 || (uintptr_t)c.v_pages % 16 || (uintptr_t)out % 16)
        return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: q, k_new, v_new, their rows, the pages and out must be 16-byte aligned");
    const Plan p = plan_of(dtype, B, N, H, c.H_kv, c.dh, c.page_size, c.max_pages, window, sinks);
    if (p.bytes && (!workspace || workspace_bytes < p.bytes || (uintptr_t)workspace % 16))
        return gr4ad_set_thread_error(GR4AD_EWORKSPACE, "paged attention: workspace of %zu bytes needed, 16-byte aligned", p.bytes);
    const int e = dtype == GR4AD_BF16 ? 2 : 4;
    // What is written shares no byte with anything else of the call (without new tokens the pages are only read).
    const int64_t page_bytes = (int64_t)c.H_kv * c.page_size * c.dh * e, pages = page_bytes > INT64_MAX / 4 / c.n_pages ? INT64_MAX / 4 : page_bytes * c.n_pages, new_width = k_new ? (int64_t)c.H_kv * c.dh * e : 0;
    const Span all[] = {{out, (int64_t)N * H * c.dh * e}, {workspace, (int64_t)p.bytes}, {c.k_pages, pages}, {c.v_pages, pages}, {q, (int64_t)H * c.dh * e, N, q_stride * e},
                        {k_new, new_width, N, kv_stride * e}, {v_new, new_width, N, kv_stride * e}, {c.page_table, (int64_t)B * c.max_pages * 4}, {q_start, (B + 1LL) * 4}, {seq_len, B * 4LL}};
    for (int i = 0; i < (k_new ? 4 : 2); i++)
        for (size_t j = i + 1; j < sizeof(all) / sizeof(all[0]); j++)
            if (overlap(all[i], all[j])) return gr4ad_set_thread_error(GR4AD_EINVAL, "paged attention: %s overlaps another buffer of the call", i == 0 ? "out" : i == 1 ? "the workspace" : "a page array");
    hipStream_t st = (hipStream_t)hip_stream;
    PagedArgs a = {q, q_stride, k_new, v_new, kv_stride, q_start, seq_len, c.page_table, c.k_pages, c.v_pages, c.n_pages, shift_of(c.page_size), c.max_pages, B, N, H, c.H_kv,
                   H / c.H_kv, scale * 1.4426950408889634f, window > kMostKeys ? kMostKeys : window, sinks > kMostKeys ? kMostKeys : sinks, out, (float *)workspace, p.nsplit};
    if (k_new && p.flash()) {  // (the smaller tiles take the new tokens where they are)
        int64_t tiles = (int64_t)N / kAppendKeys + 2 * (int64_t)B;
        if (tiles > N) tiles = N;
        const int64_t grid = tiles * c.H_kv;
        if (!launchable(grid, 256)) return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "paged attention: %d new tokens in %d sequences of %d key heads", N, B, c.H_kv);
        ProfScope ps(KC_PAGED_APPEND, st, 0.0, 4.0 * N * c.H_kv * c.dh * e);
        // (tiles of many rows: bf16, widths from 32 on)
        if (c.dh == 32) hipLaunchKernelGGL((paged_append<32>), dim3((unsigned)grid), dim3(256), 0, st, a);
        else if (c.dh == 64) hipLaunchKernelGGL((paged_append<64>), dim3((unsigned)grid), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((paged_append<128>), dim3((unsigned)grid), dim3(256), 0, st, a);
        GR4AD_LAUNCH_CHECK_AS("paged attention");
    }
    // Lengths lie on the device and a table may be far longer: counted are the keys that a window leaves, for the sequences' average of new tokens; without one nothing.
    const double table = (double)c.max_pages * c.page_size, per_row = fmin(table, (double)window + sinks), per_sequence = fmin(table, per_row + ceil((double)N / B) - 1.0);
    ProfScope ps(p.flash() ? KC_PAGED_FLASH : KC_PAGED_ATTN, st, window ? 4.0 * N * per_row * H * c.dh : 0.0, window ? e * (2.0 * B * per_sequence * c.H_kv * c.dh + 2.0 * N * H * c.dh) : 0.0);
    return dtype == GR4AD_BF16 ? launch_width<bf16>(a, c.dh, p, st) : launch_width<float>(a, c.dh, p, st);
}

}  // extern "C"
