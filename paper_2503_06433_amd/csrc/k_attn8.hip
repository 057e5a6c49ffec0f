// Attention over caches in 8 bits (Kv8Layer): causal, paged, grouped query heads; prompts and single tokens.
//
// What is attended to is what the cache holds: full blocks stand for q * (A / 127), the block that is open at the end of a sequence
// is read in the model's type.  Scores are kept in units of log 2.
#include "ss_device.h"
#include "ss_kernels.h"

namespace SS_NS {
using namespace ssk;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---------------------------------------------------------------- any type, any group
// A block per (64 queries, query head, sequence), four threads a query with a quarter of the head dimension each; a page's K and V
// come to LDS as floats.  With `scores` (one query a sequence) the scores and the logarithm of their sum are kept.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn8_generic_kernel(const T* __restrict__ q, int64_t q_stride, T* __restrict__ out, int n_q, int n_kv,
                                                            Kv8Batch b, Kv8Layer kv, float scale_log2e, float* __restrict__ scores,
                                                            float* __restrict__ lse) {
    constexpr int DS = D / 4;
    __shared__ float Ks[16][D];
    __shared__ float Vs[16][D + 1];
    const int sq = blockIdx.z, a = blockIdx.y, tile = blockIdx.x;
    const int q_begin = b.cu_q[sq], q_len = b.cu_q[sq + 1] - q_begin;
    if (tile * 64 >= q_len) return;
    const int before = b.before[sq], full = b.end[sq] / 16;
    const int g = a / (n_q / n_kv);
    const int r = threadIdx.x >> 2, sub = threadIdx.x & 3;
    const int qi = tile * 64 + r;
    const bool valid = qi < q_len;
    const int p = before + (valid ? qi : 0);
    const int last_q = tile * 64 + 63 < q_len ? tile * 64 + 63 : q_len - 1;
    const int n_pages = (before + last_q) / 16 + 1;
    const T* qp = q + (int64_t)(q_begin + (valid ? qi : 0)) * q_stride + (size_t)a * D + sub * DS;
    float qf[DS], acc[DS];
#pragma unroll
    for (int e = 0; e < DS; ++e) { qf[e] = ldf(qp + e) * scale_log2e; acc[e] = 0.f; }
    float m = -INFINITY, l = 0.f;
    const int32_t* pt = b.page_tables + (size_t)sq * b.pt_stride;
    const T* ko = (const T*)kv.open + ((size_t)b.slot[sq] * 2 * n_kv + g) * 16 * D;
    const T* vo = ko + (size_t)n_kv * 16 * D;
    for (int j = 0; j < n_pages; ++j) {
        if (j < full) {
            const size_t page = (size_t)pt[j] * n_kv + g;
            const float sk = kv.amax[page * 2] / 127.f, sv = kv.amax[page * 2 + 1] / 127.f;
            for (int i = threadIdx.x; i < 16 * D; i += 256) {
                Ks[i / D][i % D] = (float)kv.k[page * 16 * D + i] * sk;
                Vs[i % 16][i / 16] = (float)kv.v[page * 16 * D + i] * sv;
            }
        } else {                                            // slots behind the last token hold what was there before
            for (int i = threadIdx.x; i < 16 * D; i += 256) {
                const bool there = j * 16 + i / D <= before + last_q;
                Ks[i / D][i % D] = there ? ldf(ko + i) : 0.f;
                Vs[i / D][i % D] = there ? ldf(vo + i) : 0.f;
            }
        }
        __syncthreads();
        float s[16], mx = m;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            float d = 0.f;
#pragma unroll
            for (int e = 0; e < DS; ++e) d = fmaf(qf[e], Ks[t][sub * DS + e], d);
            d += __shfl_xor(d, 1, 64);
            d += __shfl_xor(d, 2, 64);
            s[t] = j * 16 + t <= p ? d : -INFINITY;
            mx = fmaxf(mx, s[t]);
            if (scores && valid && sub == 0 && j * 16 + t <= p) scores[((size_t)b.tok_off[sq] + j * 16 + t) * n_q + a] = s[t];
        }
        // position 0 is seen by every query: mx is finite from the first page on, unless the scores are not
        const float ref = mx == -INFINITY ? 0.f : mx;
        const float alpha = exp2f(m - ref);
        l *= alpha;
#pragma unroll
        for (int e = 0; e < DS; ++e) acc[e] *= alpha;
#pragma unroll
        for (int t = 0; t < 16; ++t)
            if (j * 16 + t <= p) {                          // a weight of 0 would not keep a value that is not finite out
                const float w = exp2f(s[t] - ref);
                l += w;
#pragma unroll
                for (int e = 0; e < DS; ++e) acc[e] = fmaf(w, Vs[t][sub * DS + e], acc[e]);
            }
        m = mx;
        __syncthreads();
    }
    if (valid) {
        T* op = out + (size_t)(q_begin + qi) * ((size_t)n_q * D) + (size_t)a * D + sub * DS;
        const float inv = 1.0f / l;
#pragma unroll
        for (int e = 0; e < DS; ++e) stf(op + e, acc[e] * inv);
        if (lse && sub == 0) lse[(size_t)sq * n_q + a] = m + log2f(l);
    }
}

static bool attn8_fits(int n_q, int n_kv, int d, const Kv8Batch& b, const void* q, int64_t q_stride, int dt) {
    return (d == 64 || d == 128) && n_kv > 0 && n_q % n_kv == 0 && b.n_seqs <= 65535 && n_q <= 65535 && (uintptr_t)q % 16 == 0 &&
           q_stride % (dt == F32 ? 4 : 8) == 0;
}

static hipError_t attn8_generic(int dt, const void* q, int64_t q_stride, void* out, int n_q, int n_kv, int d, const Kv8Batch& b,
                                const Kv8Layer& kv, float* scores, float* lse, hipStream_t s) {
    const dim3 grid((b.max_q_len + 63) / 64, n_q, b.n_seqs);
    const float sl2 = 1.4426950408889634f / sqrtf((float)d);
#define SS_GO(TT, DD) attn8_generic_kernel<TT, DD><<<grid, 256, 0, s>>>((const TT*)q, q_stride, (TT*)out, n_q, n_kv, b, kv, sl2, scores, lse)
    if (dt == F32) {
        if (d == 64) SS_GO(float, 64); else SS_GO(float, 128);
    } else {
        if (d == 64) SS_GO(bf16_t, 64); else SS_GO(bf16_t, 128);
    }
#undef SS_GO
    return hipGetLastError();
}

hipError_t attn8_prefill(int dt, const void* q, int64_t q_stride, void* out, int n_q, int n_kv, int d, const Kv8Batch& b,
                         const Kv8Layer& kv, bool force_generic, hipStream_t s) {
    if (b.T <= 0 || b.n_seqs <= 0) return hipSuccess;
    if (!attn8_fits(n_q, n_kv, d, b, q, q_stride, dt)) return hipErrorInvalidValue;
    (void)force_generic;
    return attn8_generic(dt, q, q_stride, out, n_q, n_kv, d, b, kv, nullptr, nullptr, s);
}

// ---------------------------------------------------------------- accumulated weights
// A thread per (token, kv head): the weights of the head's G queries, in their order, onto what is there.
__global__ __launch_bounds__(256) void attn8_weights_kernel(const float* __restrict__ scores, const float* __restrict__ lse, int n_q, int n_kv,
                                                            Kv8Batch b, float* __restrict__ w) {
    const int sq = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x, t = i / n_kv, g = i % n_kv;
    if (t > b.before[sq]) return;
    const int G = n_q / n_kv;
    const float* sp = scores + ((size_t)b.tok_off[sq] + t) * n_q + g * G;
    const float* lp = lse + (size_t)sq * n_q + g * G;
    float sum = 0.f;
    for (int j = 0; j < G; ++j) sum += exp2_fast(sp[j] - lp[j]);
    w[((size_t)b.page_tables[(size_t)sq * b.pt_stride + t / 16] * n_kv + g) * 16 + t % 16] += sum;
}

// partial results [n_items][n_q][d + 4], then (weights) the logarithms [n_seqs][n_q] and the scores [tokens seen][n_q]
static size_t partial_floats(const Kv8Batch& b, int n_q, int d) { return (size_t)b.wk.n_items * n_q * (d + 4); }
size_t attn8_decode_scratch_floats(const Kv8Batch& b, int n_q, int d, bool weights) {
    return partial_floats(b, n_q, d) + (weights ? (size_t)b.n_seqs * n_q + (size_t)b.seen * n_q : 0);
}

hipError_t attn8_decode(int dt, const void* q, int64_t q_stride, void* out, int n_q, int n_kv, int d, const Kv8Batch& b,
                        const Kv8Layer& kv, float* scratch, bool force_generic, hipStream_t s) {
    if (b.n_seqs <= 0) return hipSuccess;
    if (!attn8_fits(n_q, n_kv, d, b, q, q_stride, dt) || b.max_q_len != 1 || !scratch) return hipErrorInvalidValue;
    if ((long long)b.max_seen * n_kv > 0x7fffff00ll) return hipErrorInvalidValue;
    (void)force_generic;
    float* lse = kv.w ? scratch + partial_floats(b, n_q, d) : nullptr;
    float* scores = kv.w ? lse + (size_t)b.n_seqs * n_q : nullptr;
    const hipError_t e = attn8_generic(dt, q, q_stride, out, n_q, n_kv, d, b, kv, scores, lse, s);
    if (e != hipSuccess || !kv.w) return e;
    attn8_weights_kernel<<<dim3((unsigned)(((long long)b.max_seen * n_kv + 255) / 256), b.n_seqs), 256, 0, s>>>(scores, lse, n_q, n_kv, b, kv.w);
    return hipGetLastError();
}

}  // namespace SS_NS
