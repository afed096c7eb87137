// Penalties for repeated tokens, biases and grammar masks on rows of logits, in front of the selection.
//
//     l = c > 0 ? (l > 0 ? l / repetition : l * repetition) : l;  l -= frequency c + (c > 0 ? presence : 0);  l += bias;  forbidden: -inf
//
// c: how often the token occurs in the row's history.  One pass over the logits: a workgroup owns a stretch of one row, whose tokens it counts in LDS
// (integer additions, so their order changes nothing) while the stretch's logits are on their way.  Bound by the bytes: 16384 rows of 8192 half-precision
// logits with all rules 124 us, 4.3 TB/s (the biases, twice as wide as the logits, come out of L2: without them 102).  keep = 0: outputs that would fill the caches
// and lie on 16 bytes pass them by (the same 161 us where they do not).
#include "common.h"

namespace {

struct LogitArgs {
    const void *in;
    void *out;
    int rows, V;
    gr4ad_logit_rules r;
};

// 16 bytes of a row that may start anywhere (rows of V elements: a row's start is as aligned as V is)
template <typename T> struct Piece {
    static constexpr int N = 16 / sizeof(T);
    T v[N];
    __device__ __forceinline__ void load(const T *p) { __builtin_memcpy(v, p, 16); }
    __device__ __forceinline__ void store(T *p, bool keep) const {
        if (keep) {
            __builtin_memcpy(p, v, 16);
        } else {
            intx4 w;
            __builtin_memcpy(&w, v, 16);
            __builtin_nontemporal_store(w, (intx4 *)p);
        }
    }
};

// PIECES 16-byte pieces per thread
template <typename T, int PIECES> __global__ __launch_bounds__(256) void adjust_logits(LogitArgs a, int stretches, int keep) {
    constexpr int E = Piece<T>::N;
    extern __shared__ unsigned count[];
    const int span = blockDim.x * E * PIECES, row = blockIdx.x / stretches, v0 = (blockIdx.x - row * stretches) * span, V = a.V;
    const gr4ad_logit_rules &r = a.r;
    const int64_t at = (int64_t)row * V;
    const T *in = (const T *)a.in + at;
    T *out = (T *)a.out + at;
    Piece<T> x[PIECES];
    auto first = [&](int i) { return v0 + (i * (int)blockDim.x + (int)threadIdx.x) * E; };
#pragma unroll
    for (int i = 0; i < PIECES; i++) {
        const int v = first(i);
        if (v + E <= V) x[i].load(in + v);
        else
#pragma unroll
            for (int e = 0; e < E; e++) x[i].v[e] = v + e < V ? in[v + e] : (T)0.0f;
    }
    int len = 0;
    if (r.history) {
        len = r.history_len ? r.history_len[row] : r.history_stride;
        len = len < 0 ? 0 : len > r.history_stride ? r.history_stride : len;
    }
    if (len > 0) {
        for (int i = threadIdx.x; i < span; i += blockDim.x) count[i] = 0;
        __syncthreads();
        const int32_t *h = r.history + (int64_t)row * r.history_stride;
        for (int i = threadIdx.x; i < len; i += blockDim.x) {
            const unsigned v = (unsigned)h[i] - (unsigned)v0;
            if (v < (unsigned)span && h[i] < V) atomicAdd(&count[v], 1u);
        }
        __syncthreads();
    }
    const float rep = len > 0 && r.repetition ? r.repetition[row] : 1.0f, pres = len > 0 && r.presence ? r.presence[row] : 0.0f,
                freq = len > 0 && r.frequency ? r.frequency[row] : 0.0f;
    const float *bias = nullptr;
    if (r.bias) {
        const int b = r.bias_row ? r.bias_row[row] : 0;
        if (b >= 0 && b < r.n_bias) bias = r.bias + (int64_t)b * V;
    }
    const uint32_t *mask = nullptr;
    bool nothing = false;
    if (r.mask) {
        const int m = r.mask_row ? r.mask_row[row] : 0;
        if (m >= r.n_masks) nothing = true;
        else if (m >= 0) mask = r.mask + (int64_t)m * ((V + 31) / 32);
    }
#pragma unroll
    for (int i = 0; i < PIECES; i++) {
        const int v = first(i);
        if (v >= V) continue;
        unsigned allowed = nothing ? 0u : ~0u;
        if (mask) allowed = mask[v / 32] >> (v % 32);
        float b[E] = {};
        if (bias) {
            if (v + E <= V) __builtin_memcpy(b, bias + v, E * 4);
            else
#pragma unroll
                for (int e = 0; e < E; e++) b[e] = v + e < V ? bias[v + e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < E; e++) {
            float l = (float)x[i].v[e];
            if (len > 0) {
                const unsigned c = count[v - v0 + e];
                if (c) {
                    if (r.repetition) l = l > 0.0f ? l / rep : l * rep;
                    l -= freq * (float)c + pres;
                }
            }
            if (bias) l += b[e];
            x[i].v[e] = (T)((allowed >> e & 1) ? l : -INFINITY);
        }
        if (v + E <= V) x[i].store(out + v, keep);
        else
#pragma unroll
            for (int e = 0; e < E; e++)
                if (v + e < V) out[v + e] = x[i].v[e];
    }
}

template <typename T> int adjust(const T *in, T *out, int32_t rows, int32_t V, const gr4ad_logit_rules *r, void *stream) {
    if (!in || !out || !r) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: NULL pointer");
    if (rows < 1 || V < 1) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: rows %d and V %d must be positive", rows, V);
    if ((uintptr_t)in % sizeof(T) || (uintptr_t)out % sizeof(T)) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: misaligned logits");
    if (r->history && r->history_stride < 1) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: history_stride %d must be positive", r->history_stride);
    if (!r->history && (r->repetition || r->presence || r->frequency)) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: penalties without a history");
    if (r->bias && r->n_bias < 1) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: n_bias %d must be positive", r->n_bias);
    if (r->mask && r->n_masks < 1) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: n_masks %d must be positive", r->n_masks);
    // Two pieces of 16 bytes per thread, one where the call is short (64 rows of 1024 float32 logits 3.9 us, with one piece 3.2; 16384 of 8192 196, with one 251: each
    // workgroup clears and counts for half as many logits).
    const bool one = (int64_t)rows * V < (8 << 20);
    constexpr int E = Piece<T>::N;
    const int each = one ? E : 2 * E, threads = V <= 64 * each ? 64 : V <= 128 * each ? 128 : 256, span = threads * each;
    const int64_t stretches = ceil_div64(V, span), grid = rows * stretches;
    if (!launchable(grid, threads) || V > (1 << 30)) return gr4ad_set_thread_error(GR4AD_EUNSUPPORTED, "adjust_logits: %d rows of %d logits", rows, V);
    const int keep = (int64_t)rows * V * (int)sizeof(T) < (16 << 20) || V * sizeof(T) % 16 || (uintptr_t)out % 16;
    // (a thread writes only what it has read itself where out is the logits' place, and reads the tables while others write)
    const int64_t bytes = (int64_t)rows * V * (int64_t)sizeof(T), table = (int64_t)V * 4, words = ceil_div64(V, 32) * 4;
    const Span o = {out, bytes}, others[] = {{(const void *)in == (const void *)out ? nullptr : in, bytes}, {r->history, r->history_stride * 4LL, rows, r->history_stride * 4LL},
                                             {r->bias, table * r->n_bias}, {r->mask, words * r->n_masks}, {r->history_len, rows * 4LL}, {r->repetition, rows * 4LL}, {r->presence, rows * 4LL},
                                             {r->frequency, rows * 4LL}, {r->bias_row, rows * 4LL}, {r->mask_row, rows * 4LL}};
    for (const Span &s : others)
        if (overlap(o, s)) return gr4ad_set_thread_error(GR4AD_EINVAL, "adjust_logits: out overlaps another buffer of the call and is not logits itself");
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(KC_ADJUST_LOGITS, st, 0.0, 2.0 * sizeof(T) * rows * (double)V);
    LogitArgs a = {in, out, rows, V, *r};
    const size_t lds = r->history ? span * sizeof(unsigned) : 0;
    if (one) hipLaunchKernelGGL((adjust_logits<T, 1>), dim3((unsigned)grid), dim3(threads), lds, st, a, (int)stretches, keep);
    else hipLaunchKernelGGL((adjust_logits<T, 2>), dim3((unsigned)grid), dim3(threads), lds, st, a, (int)stretches, keep);
    GR4AD_LAUNCH_CHECK_AS("adjust_logits");
    return GR4AD_OK;
}

}  // namespace

extern "C" {

int gr4ad_op_adjust_logits(const float *logits, float *out, int32_t rows, int32_t V, const gr4ad_logit_rules *rules, void *hip_stream) {
    return adjust<float>(logits, out, rows, V, rules, hip_stream);
}

int gr4ad_op_adjust_logits_f16(const void *logits, void *out, int32_t rows, int32_t V, const gr4ad_logit_rules *rules, void *hip_stream) {
    return adjust<_Float16>((const _Float16 *)logits, (_Float16 *)out, rows, V, rules, hip_stream);
}

}  // extern "C"
