// Attention over caches in 8 bits (Kv8Layer): causal, paged, grouped query heads; prompts and single tokens.
//
// What is attended to is what the cache holds: full blocks stand for q * (A / 127), the block that is open at the end of a sequence
// is read in the model's type.  Scores are kept in units of log 2.
#include <type_traits>

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
            if (scores && valid && sub == 0 && j * 16 + t <= p) scores[(((size_t)b.pg_off[sq] + j) * n_q + a) * 16 + t] = s[t];
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

// ---------------------------------------------------------------- operands of the matrix cores
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
union Frag8 {
    half8_t v;
    vec16 q;
    uint32_t w[4];
};

// Four signed bytes as four numbers of the 16-bit type, exact.  bf16: a conversion that picks its byte, and the upper halves of two
// results put together, six operations; half: 1024 + 128 + byte has the byte in its lowest bits, five.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
#ifdef SS_HALF_F16
    typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
    const uint32_t u = w ^ 0x80808080u;
    const h2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x07010700u)) + off);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x07030702u)) + off);
#else
    const float f0 = (float)(int8_t)w, f1 = (float)(int8_t)(w >> 8), f2 = (float)(int8_t)(w >> 16), f3 = (float)(int8_t)(w >> 24);
    lo = __builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u);
    hi = __builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302u);
#endif
}
__device__ __forceinline__ Frag8 widen8(uint32_t a, uint32_t b) {
    Frag8 f;
    widen4(a, f.w[0], f.w[1]);
    widen4(b, f.w[2], f.w[3]);
    return f;
}

// The weights of a block are kept times its V step: the second product then takes V's whole numbers as they are, and a 16-bit
// weight is rounded relative to what it contributes.  lv: log 2 of the step; inv brings the sum of such weights back.  A block of
// zeros adds to the sum alone: any step serves, this one lies below those of half values and far above underflow.
// The reference r of the exponents follows the largest score + lv, but with an lv of at least LV_REF: the sum, of exp2(score - r), of a cache
// that holds tiny values only would pass the largest float otherwise.  Steps below 2^LV_MIN, of values below 127 * 2^-126, count as that
// (the next smaller ones are no normal floats).
constexpr float LV_ZERO = -40.f, LV_REF = -100.f, LV_MIN = -126.f;
// Half: the largest weight is 2^14 instead of 1, so that those of 2^-28 of it are still in the type's normal range.  With 1 a token
// of weight 2^-16 is rounded to 2^-9 of itself, which shows in outputs whose heavy tokens happen to have a value of 0.
#ifdef SS_HALF_F16
constexpr float TOP_EXP = 14.f;
#else
constexpr float TOP_EXP = 0.f;
#endif
__device__ __forceinline__ float lv_ref(float lv) { return TOP_EXP > 0.f ? lv : fmaxf(lv, LV_REF); }  // half has no steps below 2^-31
// The power of two that an open block's V is divided by, for a largest magnitude of `big`: it then lies below 128, as a full block's whole
// numbers do.  Half has no room for that from 128 on: what is some 2^-16 of the largest would fall below the type's normal range and be
// rounded (0.001 next to 60000 came out as 0.001007).  It is left as it is there; the block's weights are then up to 2^9 further
// below the largest one than they would be.
__device__ __forceinline__ int open_exponent(float big) {
    int e = big > 0.f ? (int)(__float_as_uint(big) >> 23) - 127 - 6 : (int)LV_ZERO;
    if (TOP_EXP > 0.f && e > 0) e = 0;
    return e < (int)LV_REF ? (int)LV_REF : e;
}
// Brain floats: the steps of a head's blocks can lie so far apart that a weight (times its step) underflows although its token has its part in
// the sum: blocks of zeros or of small values beside values 2^90 times as large.  Where a block's largest weight is below 2^FAR its
// sum is formed with exponents of its own, from 0 down.  References that move that far are followed in two steps of half the
// distance, which the sum survives.  Half's steps, 2^-40 to 2^9, are never that far apart, nor are those from 2^-NEAR to 2^NEAR (a token
// that has 2^-30 of the largest score's weight is at 2^-120 there).
constexpr bool WIDE = TOP_EXP == 0.f;
constexpr float FAR = -100.f, NEAR = 45.f;
__device__ __forceinline__ float half_way(float d) { return exp2_fast(WIDE ? 0.5f * d : d); }
__device__ __forceinline__ float twice(float x, float a) { return WIDE ? x * a * a : x * a; }
__device__ __forceinline__ bool far_below(float top) { return WIDE && top < FAR && top > -INFINITY; }
constexpr float ONE_127 = 1.f / 127.f;               // a step is formed with it: one more rounding of 2^-24, ten operations less than the quotient
__device__ __forceinline__ void v_step(float amax, float& lv, float& inv) {
    const float l = __builtin_amdgcn_logf(amax * ONE_127);
    lv = amax == 0.f ? LV_ZERO : l < LV_MIN ? LV_MIN : l;
    inv = exp2_fast(-lv);
}

// ---------------------------------------------------------------- single tokens
// A wave per (work item, kv head, 16 of its query heads).  An item is pages page0, page0 + stride, ... of a sequence.  The transposed
// products S^T = K Q^T and O^T = V^T P^T: the scores of the first are then in the registers where the second wants its weights.
// Four pages a step: row 4 p + v of score product i is token 4 i + v of page p, so that lane group p (16 lanes) ends up with the
// 16 scores of page p, one query a lane: one K and one V step a lane, and 16-byte loads of 16 tokens (V) or 16 elements (K),
// half a cache line a row.  K of the next four pages is requested behind the score products of these, V of these in front of them.
// Bound by the page reads: 256 sequences of 512 - 2560 tokens on 32 heads 533 us, 6.0 TB/s; 1024 of 512 - 4096 on one head 122 us, 4.9 TB/s
// (waves of a few hundred tokens each).  One sequence of 700 tokens: 8 us and 4 for the merge, the chain item -> pages -> sums.
template <int D, bool WEIGHTS>
__global__ __launch_bounds__(64) void attn8_decode_kernel(const bf16_t* __restrict__ q, int64_t q_stride, int n_q, int n_kv, int n_ct,
                                                          Kv8Batch b, Kv8Layer kv, float* __restrict__ scratch, float* __restrict__ scores,
                                                          float scale_log2e) {
    constexpr int HB = D / 64, DT = D / 16;
    const int heads = n_kv * n_ct;
    const int32_t* rec = b.items + (size_t)(blockIdx.x / heads) * 8;
    const int item = rec[0], g = blockIdx.x % heads / n_ct, ct = blockIdx.x % n_ct;
    const int G = n_q / n_kv;
    const int sq = rec[1], page0 = rec[2], np = rec[3];
    const int npg = np & 0xffff, stride = (int)((unsigned)np >> 16);
    const int p = rec[4], full = rec[5] / 16, slot = rec[6], row = rec[7];
    const int lane = threadIdx.x, lq = lane & 15, g4 = lane >> 4;
    const bool open_here = page0 + (npg - 1) * stride >= full;           // the item's last page is the open block
    const int npc = npg - open_here;
    const bool mine = ct * 16 + lq < G;
    const int a = g * G + ct * 16 + lq;

    Frag8 qf[HB][2];
#pragma unroll
    for (int h = 0; h < HB; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            qf[h][j].w[0] = qf[h][j].w[1] = qf[h][j].w[2] = qf[h][j].w[3] = 0u;
            if (mine) qf[h][j].q = *reinterpret_cast<const vec16*>(q + (int64_t)row * q_stride + (size_t)a * D + 64 * h + 16 * g4 + 8 * j);
        }
    f32x4_t o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float r = -INFINITY, l = 0.f;                                        // reference of the exponents, sum in its units
    float* sp = WEIGHTS ? scores + ((size_t)b.pg_off[sq] * n_q + a) * 16 : nullptr;      // [page][n_q][16]

    auto rescale = [&](float top) {
        const float a = r < top ? half_way(r - top) : 1.f;
        const float alpha = twice(1.f, a);
        r = top;
        l = twice(l, a);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) o[t][v] *= alpha;
    };
    auto over_groups = [&](float x) {
        x = fmaxf(x, __shfl_xor(x, 16, 64));
        return fmaxf(x, __shfl_xor(x, 32, 64));
    };

    if (npc > 0) {
        const int32_t* pt = b.page_tables + (size_t)sq * b.pt_stride + page0;
        auto page_at = [&](int j) { return pt[(j < npc ? j : npc - 1) * stride]; };
        struct Ids { int k, v; };
        auto ids = [&](int j0) { return Ids{page_at(j0 + (lq >> 2)), page_at(j0 + g4)}; };
        struct Keys { vec16 k[4][HB]; float2 amax; };
        auto load_k = [&](const Ids& id, Keys& f) {
            const int8_t* kp = kv.k + ((size_t)id.k * n_kv + g) * 16 * D + (lq & 3) * D + 16 * g4;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < HB; ++h) f.k[i][h] = *reinterpret_cast<const vec16*>(kp + 4 * i * D + 64 * h);
            f.amax = *reinterpret_cast<const float2*>(kv.amax + ((size_t)id.v * n_kv + g) * 2);
        };
        auto step = [&](int j0, const Ids& cur, const Keys& f, const Ids& nxt, Keys& fn) {
            const int8_t* vp = kv.v + ((size_t)cur.v * n_kv + g) * 16 * D + lq * 16;
            vec16 vr[DT];
#pragma unroll
            for (int t = 0; t < DT; ++t) vr[t] = *reinterpret_cast<const vec16*>(vp + t * 256);
            __builtin_amdgcn_sched_barrier(0);
            f32x4_t s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < HB; ++h) {
                    s[i] = SS_MFMA_16x16x32(widen8(f.k[i][h].w[0], f.k[i][h].w[1]).v, qf[h][0].v, s[i], 0, 0, 0);
                    s[i] = SS_MFMA_16x16x32(widen8(f.k[i][h].w[2], f.k[i][h].w[3]).v, qf[h][1].v, s[i], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_k(nxt, fn);
            __builtin_amdgcn_sched_barrier(0);
            const float ks = f.amax.x * (ONE_127 * scale_log2e);
            float lv, inv;
            v_step(f.amax.y, lv, inv);
            const int pg = page0 + (j0 + g4) * stride;
            const int seen = j0 + g4 < npc ? p - pg * 16 : -1;           // tokens 0 .. seen of the lane's page
            const bool whole = j0 + 4 < npc;                             // only an item's last step has hidden tokens or pages too few
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    s[i][v] = whole || 4 * i + v <= seen ? s[i][v] * ks : -INFINITY;
                    top = fmaxf(top, s[i][v]);
                }
            if (WEIGHTS && mine && seen >= 0) {                          // those behind the last token are not read
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4_t*>(sp + (size_t)pg * n_q * 16 + 4 * i) = s[i];
            }
            const float own = top;
            top = over_groups(top + lv_ref(lv)) - TOP_EXP;
            if (__any(top > r)) rescale(fmaxf(top, r));
            const float off = lv - r;
            float rs = 0.f, apart = 0.f;
            if (__builtin_expect(__any(far_below(own + off)), 0)) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) apart += exp2_fast(s[i][v] - own);
                apart = twice(apart, half_way(own - r));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float w = exp2_fast(s[i][v] + off);
                    s[i][v] = whole || 4 * i + v <= seen ? w : 0.f;      // the step of a hidden block may not be a number
                    rs += s[i][v];
                }
            l += whole || seen >= 0 ? far_below(own + off) ? apart : rs * inv : 0.f;
            Frag8 pa, pb;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                pa.w[2 * i] = pack_bf16x2(s[i][0], s[i][1]);
                pa.w[2 * i + 1] = pack_bf16x2(s[i][2], s[i][3]);
                pb.w[2 * i] = pack_bf16x2(s[2 + i][0], s[2 + i][1]);
                pb.w[2 * i + 1] = pack_bf16x2(s[2 + i][2], s[2 + i][3]);
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                o[t] = SS_MFMA_16x16x32(widen8(vr[t].w[0], vr[t].w[1]).v, pa.v, o[t], 0, 0, 0);
                o[t] = SS_MFMA_16x16x32(widen8(vr[t].w[2], vr[t].w[3]).v, pb.v, o[t], 0, 0, 0);
            }
        };
        // two steps a trip, the two sets of keys in turn; page numbers are there two steps ahead.  Behind the end the last page is asked
        // for again.
        Ids i0 = ids(0), i1 = ids(4);
        Keys k0, k1;
        load_k(i0, k0);
        for (int j = 0; j < npc; j += 8) {
            const Ids i2 = ids(j + 8);
            step(j, i0, k0, i1, k1);
            const Ids i3 = ids(j + 12);
            if (j + 4 < npc) step(j + 4, i1, k1, i2, k0);
            i0 = i2;
            i1 = i3;
        }
    }
    if (open_here) {
        // Tokens 4 g4 + v of the open block, in the model's type, in the first four of the group's eight slots of the second product.  V is
        // scaled by a power of two (open_exponent).
        const int cnt = p - full * 16 + 1;
        const bf16_t* ko = (const bf16_t*)kv.open + ((size_t)slot * 2 * n_kv + g) * 16 * D;
        const bf16_t* vo = ko + (size_t)n_kv * 16 * D;
        bf16_t raw[DT][4];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) raw[t][v] = vo[(4 * g4 + v) * D + 16 * t + lq];
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                Frag8 kf;
                kf.q = *reinterpret_cast<const vec16*>(ko + lq * D + 64 * h + 16 * g4 + 8 * j);
                s = SS_MFMA_16x16x32(kf.v, qf[h][j].v, s, 0, 0, 0);
            }
        float big = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (4 * g4 + v < cnt) big = fmaxf(big, fabsf(bf2f(raw[t][v])));
        big = wave_max(big);
        const float lv = big < INFINITY ? (float)open_exponent(big) : 0.f;
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            s[v] = 4 * g4 + v < cnt ? s[v] * scale_log2e : -INFINITY;
            top = fmaxf(top, s[v]);
        }
        if (WEIGHTS && mine) *reinterpret_cast<f32x4_t*>(sp + (size_t)full * n_q * 16 + 4 * g4) = s;
        rescale(fmaxf(r, over_groups(top + lv) - TOP_EXP));
        const float off = lv - r;
        float rs = 0.f, apart = 0.f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            apart += 4 * g4 + v < cnt ? exp2_fast(s[v] - top) : 0.f;
            s[v] = 4 * g4 + v < cnt ? exp2_fast(s[v] + off) : 0.f;
            rs += s[v];
        }
        l += far_below(top + off) ? twice(apart, half_way(top - r)) : rs * exp2_fast(-lv);
        Frag8 pf;
        pf.w[0] = pack_bf16x2(s[0], s[1]);
        pf.w[1] = pack_bf16x2(s[2], s[3]);
        pf.w[2] = pf.w[3] = 0u;
        const float down = exp2_fast(-lv);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            float x[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = 4 * g4 + v < cnt ? bf2f(raw[t][v]) * down : 0.f;
            Frag8 vf;
            vf.w[0] = pack_bf16x2(x[0], x[1]);
            vf.w[1] = pack_bf16x2(x[2], x[3]);
            vf.w[2] = vf.w[3] = 0u;
            o[t] = SS_MFMA_16x16x32(vf.v, pf.v, o[t], 0, 0, 0);
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (mine) {
        float* out = scratch + ((size_t)item * n_q + a) * (D + 4);
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4_t*>(out + t * 16 + 4 * g4) = o[t];
        if (g4 == 0) { out[D] = r; out[D + 1] = l; }
    }
}

// Merge of the items' partial results: D / 4 threads (a row) per query head, SPLIT rows of a block share the items of one, four of which
// are requested together.  With 8 rows a head, long caches (70 items) take 6 us less; where a row has few items, one row a head is shorter.
template <int D, int SPLIT>
__global__ __launch_bounds__(256) void attn8_merge_kernel(const float* __restrict__ scratch, bf16_t* __restrict__ out, int n_q, Kv8Batch b,
                                                          float* __restrict__ lse) {
    constexpr int ROWS = 1024 / D;
    static_assert(SPLIT == 1 || SPLIT == ROWS, "");
    __shared__ float part[SPLIT > 1 ? SPLIT : 1][D + 4];
    const int sq = blockIdx.y, e = threadIdx.x % (D / 4) * 4, row = threadIdx.x / (D / 4);
    const int a = SPLIT > 1 ? blockIdx.x : blockIdx.x * ROWS + row, step = SPLIT > 1 ? 4 * SPLIT : 4;
    if (a >= n_q) return;
    const int i0 = b.seq_item0[sq] + (SPLIT > 1 ? row * 4 : 0), i1 = b.seq_item0[sq + 1];
    float M = -INFINITY, den = 0.f;
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    for (int i = i0; i < i1; i += step) {
        float m[4], l[4];
        f32x4_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float* sp = scratch + ((size_t)(i + u < i1 ? i + u : i1 - 1) * n_q + a) * (D + 4);
            m[u] = sp[D];
            l[u] = sp[D + 1];
            v[u] = *reinterpret_cast<const f32x4_t*>(sp + e);
        }
        float mx = M;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i + u >= i1) {                                           // repeated: weight 0 would not keep an infinite one out
                m[u] = -INFINITY;
                l[u] = 0.f;
                v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
            mx = fmaxf(mx, m[u]);
        }
        const float ref = mx == -INFINITY ? 0.f : mx;
        const float a = half_way(M - ref);
        M = mx;
        num *= twice(1.f, a);
        den = twice(den, a);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float w = half_way(m[u] - ref);
            num += twice(1.f, w) * v[u];
            den += twice(l[u], w);
        }
    }
    if constexpr (SPLIT > 1) {
        *reinterpret_cast<f32x4_t*>(&part[row][e]) = num;
        if (e == 0) { part[row][D] = M; part[row][D + 1] = den; }
        __syncthreads();
        if (row > 0) return;
        float mx = M;
#pragma unroll
        for (int u = 1; u < SPLIT; ++u) mx = fmaxf(mx, part[u][D]);
        const float ref = mx == -INFINITY ? 0.f : mx, w0 = half_way(M - ref);
        M = mx;
        num *= twice(1.f, w0);
        den = twice(den, w0);
#pragma unroll
        for (int u = 1; u < SPLIT; ++u) {
            const float w = half_way(part[u][D] - ref);
            num += twice(1.f, w) * *reinterpret_cast<const f32x4_t*>(&part[u][e]);
            den += twice(part[u][D + 1], w);
        }
    }
    vec16 w;
    w.w[0] = pack_bf16x2(num[0] / den, num[1] / den);
    w.w[1] = pack_bf16x2(num[2] / den, num[3] / den);
    *reinterpret_cast<uint2*>(out + (size_t)b.cu_q[sq] * ((size_t)n_q * D) + (size_t)a * D + e) = make_uint2(w.w[0], w.w[1]);
    if (lse && e == 0) lse[(size_t)sq * n_q + a] = M + __builtin_amdgcn_logf(den);
}

template <int D>
static void launch_decode(const void* q, int64_t q_stride, void* out, int n_q, int n_kv, const Kv8Batch& b, const Kv8Layer& kv, float* scratch,
                          float* scores, float* lse, hipStream_t s) {
    const int n_ct = (n_q / n_kv + 15) / 16;
    const float sl2 = 1.4426950408889634f / sqrtf((float)D);
    const unsigned grid = (unsigned)((long long)b.n_items * n_kv * n_ct);
    const auto kernel = scores ? attn8_decode_kernel<D, true> : attn8_decode_kernel<D, false>;
    kernel<<<grid, 64, 0, s>>>((const bf16_t*)q, q_stride, n_q, n_kv, n_ct, b, kv, scratch, scores, sl2);
    constexpr int ROWS = 1024 / D;
    if (b.max_items_per_seq > ROWS) attn8_merge_kernel<D, ROWS><<<dim3(n_q, b.n_seqs), 256, 0, s>>>(scratch, (bf16_t*)out, n_q, b, lse);
    else attn8_merge_kernel<D, 1><<<dim3((n_q + ROWS - 1) / ROWS, b.n_seqs), 256, 0, s>>>(scratch, (bf16_t*)out, n_q, b, lse);
}

// ---------------------------------------------------------------- prompts
// A block of 8 waves takes 256 rows of one (sequence, kv head) at a time; a row is a query of one of the head's G query heads, the
// heads of a token side by side, so that a few tokens of many heads fill a block like many tokens of one.  64 tokens (4 pages) at a
// time come to LDS as numbers of the 16-bit type: every thread widens 16 bytes of K and 16 of V, once for all eight waves (each
// wave widening its own operands would cost 1.5 times the vector operations of the softmax).  The whole numbers stay as they are: K's
// step goes into the exponent's factor, V's into the weight (v_step).  Two stages: while one is multiplied, the next is
// widened from registers and the one behind it requested.
// 24 prompts of 512 - 4096 tokens, 64 heads on 8: 3.0 - 3.3 ms with the clock, 830 - 920 TFLOP/s; a large product reaches 1240 - 1380.  A tile takes a block some 2 us, of which
// the matrix cores work 0.85 and the vector units (exponentials, maxima, sums, conversions) about as long; they overlap in part.
// Not better: the two waves of a SIMD half a tile apart, with a barrier a phase (the vector phase alone takes 2300 cycles), priorities,
// 64 rows a wave and all fragments in registers in front of the products (both spill).
// Row r of a score product is token 4 (r / 8) + r % 4 of the first page of two (r % 8 < 4) or the second: accumulator v of a lane is
// then token v of page 2 h + lane / 32, and a lane needs one K and one V step for its 16 scores.
// K rows are stored with their 16-byte pieces swapped by token and page, V rows (16 tokens of an element) with their halves swapped in
// rows 8 - 15 of 16: reads and writes of 16 lanes fall on all banks.
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16_t;

__device__ __forceinline__ float max_of_halves(float x) {
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// the value of the lane next to it (lanes 0 and 1, 2 and 3, ... swapped)
__device__ __forceinline__ float neighbour(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xb1, 0xf, 0xf, true));
}
// One instruction.  fmaxf would first make its operands from the matrix cores canonical, one by one, because it does not keep a NaN; a
// row with one is NaN whatever this returns.
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

// The reference of a row's exponents follows the largest only when that has grown by more than LAG: the largest weight is 2^TOP_ROW
// to 2^(TOP_ROW + LAG) (half: 2^15, see TOP_EXP).
constexpr float LAG = TOP_EXP > 0.f ? 4.f : 8.f;
constexpr float TOP_ROW = TOP_EXP > 0.f ? 11.f : 0.f;

template <int D> constexpr int prefill_stage = 2 * 64 * D * 2;

template <int D>
__global__ __launch_bounds__(512) void attn8_prefill_kernel(const bf16_t* __restrict__ q, int64_t q_stride, bf16_t* __restrict__ out, int n_q,
                                                            int n_kv, Kv8Batch b, Kv8Layer kv, float scale_log2e, float* __restrict__ scratch) {
    constexpr int KS = D / 16, DT = D / 32, ROW = 2 * D, KBYTES = 64 * ROW, STAGE = prefill_stage<D>;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int G = n_q / n_kv;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lq = lane & 31, g2 = lane >> 5;
    // what a thread widens: of a tile's page pg_w one piece of a K row and one row of V; heads of 64: half of the waves each
    const int pg_w = D == 128 ? wave >> 1 : wave & 3;
    const bool does_k = D == 128 || wave < 4, does_v = D == 128 || wave >= 4;
    const int unit = D == 128 ? threadIdx.x & 127 : lane;                // within the page
    const int k_tok = unit / (D / 16), k_piece = unit % (D / 16);
    auto k_swap = [](int page, int tok) { return D == 128 ? (tok & 7) | (page & 1) << 3 : (tok >> 1 & 3) | (page & 1) << 2; };
    // byte offsets in a stage: where the thread writes its piece of K (the second half 16 bytes on, in the swapped order: ^ 16) and its row
    // of V (likewise), where it reads the fragments of a score product (k-step ks: ^ 32 ks) and of V^T
    const uint32_t k_write = (pg_w * 16 + k_tok) * ROW + (((2 * k_piece) ^ k_swap(pg_w, k_tok)) << 4);
    const uint32_t v_write = KBYTES + pg_w * (D * 32) + unit * 32 + (unit >> 3 & 1) * 16;
    const int r_page = lq >> 2 & 1, r_tok = (lq >> 3) * 4 + (lq & 3);
    const uint32_t k_read = (r_page * 16 + r_tok) * ROW + ((g2 ^ k_swap(r_page, r_tok)) << 4);
    const uint32_t v_read = KBYTES + g2 * (D * 32) + lq * 32 + (lq >> 3 & 1) * 16;
    auto lds = [&](uint32_t at) { return reinterpret_cast<vec16*>(smem + at); };

    // Two walks over the block's items: this one brings tiles, three ahead of the other, which multiplies them, and goes on to the next
    // item's while the other is at the last ones of its own.  Records come one item ahead, an element a lane.
    const int32_t* items = b.pf_items + (size_t)blockIdx.x * b.pf_stride * 16 + (lane & 15);
    auto field = [](int rec, int i) { return __builtin_amdgcn_readlane(rec, i); };
    int rec = items[0], rec_b = rec;
    if (field(rec, 0) < 0) return;
    // a lane holds what belongs to page lane / 32 of a tile or, odd lanes, the second behind it
    const int my_page = g2 + 2 * (lane & 1);
    struct Ids { int page, g; };
    int b_tile = 0, b_pages = 0, b_g = 0, b_next = 0;
    const int32_t* b_pt = nullptr;
    auto b_item = [&] {
        b_pt = b.page_tables + (size_t)field(rec_b, 0) * b.pt_stride;
        b_g = field(rec_b, 1);
        b_pages = field(rec_b, 7);
        b_tile = field(rec_b, 8);
        rec_b = items[++b_next * 16];                                    // behind the last record is one that says so
    };
    b_item();
    auto load_ids = [&] {
        const int j = b_tile * 4 + my_page;
        const Ids r{b_pt[j < b_pages ? j : b_pages - 1], b_g};
        if (++b_tile * 4 >= b_pages) {
            if (field(rec_b, 0) >= 0) b_item();
            else --b_tile;                                               // the last tile again and again, for nobody
        }
        return r;
    };
    struct Raw { vec16 k, v; float2 amax; };
    auto load_raw = [&](const Ids& ids, Raw& w) {
        const size_t page = ((size_t)__builtin_amdgcn_readlane(ids.page, (pg_w & 1) * 32 + (pg_w >> 1)) * n_kv + ids.g) * 16 * D;
        uint32_t at = unit * 16;                                         // 32 bits next to a scalar base, not two 64-bit addresses a lane
        asm volatile("" : "+v"(at));
        if (does_k) w.k = *reinterpret_cast<const vec16*>(kv.k + page + at);
        if (does_v) w.v = *reinterpret_cast<const vec16*>(kv.v + page + at);
        w.amax = *reinterpret_cast<const float2*>(kv.amax + ((size_t)ids.page * n_kv + ids.g) * 2);
    };
    struct Steps { float ks, lv, inv; bool wide; };                      // of the lane's page; whether one of the tile's is not NEAR
    uint32_t stage = 0;                                                  // of the tile that is multiplied; the next one is in the other
    // LDS image of the next tile; returns the steps of its pages
    auto store = [&](uint32_t st, const Raw& w) {
        Steps s;
        s.ks = w.amax.x * (ONE_127 * scale_log2e);
        s.ks = s.ks < 1e-37f ? 1e-37f : s.ks;                            // a block of zeros: any step, but no infinity times zero
        v_step(w.amax.y, s.lv, s.inv);
        s.wide = WIDE && __any(fabsf(s.lv) > NEAR);
        if (does_k) {
            *lds(st + k_write) = widen8(w.k.w[0], w.k.w[1]).q;
            *lds((st + k_write) ^ 16) = widen8(w.k.w[2], w.k.w[3]).q;
        }
        if (does_v) {
            *lds(st + v_write) = widen8(w.v.w[0], w.v.w[1]).q;
            *lds((st + v_write) ^ 16) = widen8(w.v.w[2], w.v.w[3]).q;
        }
        return s;
    };
    auto publish = [] {                                                  // what this wave wrote is there before the others are let on
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // the item that is multiplied
    int g, p, end, full, tile0, n_tiles, open_tile, wave_first, wave_last, sq, bad, part;
    bool valid, active;
    int64_t op;
    half8_t qf[KS];
    int at = 0;
    auto begin = [&] {
        sq = field(rec, 0);
        if (sq < 0) return false;
        g = field(rec, 1);
        const int row0 = field(rec, 2), q_begin = field(rec, 3), rows = field(rec, 4) * G, before = field(rec, 5), n_pages = field(rec, 7);
        end = field(rec, 6);
        tile0 = field(rec, 8);
        part = field(rec, 9);
        rec = items[++at * 16];
        full = end / 16;
        n_tiles = (n_pages + 3) / 4;
        open_tile = full < n_pages ? full >> 2 : -1;
        const int wrow = row0 + wave * 32, row = wrow + lq;
        valid = row < rows;
        active = wrow < rows;
        const int qi = (valid ? row : row0) / G, head = g * G + (valid ? row : row0) - qi * G;
        p = before + qi;
        wave_first = before + wrow / G;
        wave_last = before + (wrow + 31 < rows ? wrow + 31 : rows - 1) / G;
        bad = 0;
        op = part < 0 ? ((int64_t)(q_begin + qi) * n_q + head) * D : ((int64_t)part * 256 + wave * 32 + lq) * (D + 4);
        const bf16_t* qp = q + (int64_t)(q_begin + qi) * q_stride + (size_t)head * D + g2 * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const half8_t*>(qp + ks * 16);
        return true;
    };
    f32x16_t o[DT];
    float r, l;

    // The open block's page of the tile that is multiplied next, over what `store` brought there: the model's type as it is, V divided by
    // a power of two (open_exponent) and without values that are not finite; tokens that have such are marked, their weight is to be NaN.
    auto store_open = [&](uint32_t st, Steps& s) {
        const bf16_t* ko = (const bf16_t*)kv.open + ((size_t)b.slot[sq] * 2 * n_kv + g) * 16 * D;
        const bf16_t* vo = ko + (size_t)n_kv * 16 * D;
        const int cnt = end - full * 16;
        float big = 0.f;
        int mark = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {                           // all of V by every wave: all need its step
            const int at = (i * 64 + lane) * 8, tok = at / D;
            if (tok < cnt) {
                float x[8];
                unpack16<bf16_t>(*reinterpret_cast<const vec16*>(vo + at), x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool fin = fabsf(x[e]) < INFINITY;
                    big = fmaxf(big, fin ? fabsf(x[e]) : 0.f);
                    mark |= fin ? 0 : 1 << tok;
                }
            }
        }
        big = wave_max(big);
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) mark |= __shfl_xor(mark, i, 64);
        bad = mark;
        const int e = open_exponent(big);
        if (my_page == (full & 3)) s = Steps{scale_log2e, (float)e, exp2_fast((float)-e), s.wide};
        if ((full & 3) != pg_w) return;
        if (does_k) {
            const vec16* kr = reinterpret_cast<const vec16*>(ko + k_tok * D + k_piece * 16);
            *lds(st + k_write) = kr[0];
            *lds((st + k_write) ^ 16) = kr[1];
        }
        if (does_v) {
            const float down = exp2_fast((float)-e);
            float x[16];
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                x[t] = t < cnt ? bf2f(vo[t * D + unit]) : 0.f;
                x[t] = fabsf(x[t]) < INFINITY ? x[t] * down : 0.f;
            }
            Frag8 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo.w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
                hi.w[i] = pack_bf16x2(x[8 + 2 * i], x[9 + 2 * i]);
            }
            *lds(st + v_write) = lo.q;
            *lds((st + v_write) ^ 16) = hi.q;
        }
    };

    // 32 tokens of scores, of the lane's page 16, become weights.  `hidden`: some of them are not to be seen by every row, or the steps that
    // the row has met need not be NEAR each other.
    auto softmax = [&](auto hidden_c, f32x16_t& s, float ks, float lv, float inv, int t0, Frag8& pA, Frag8& pB) {
        constexpr bool hidden = decltype(hidden_c)::value;
        if constexpr (hidden) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = t0 + v <= p ? s[v] : -INFINITY;
        }
        float m = max3(s[0], s[1], s[2]);
#pragma unroll
        for (int v = 3; v < 15; v += 2) m = max3(m, s[v], s[v + 1]);
        m = fmaxf(m, s[15]);
        const float top = max_of_halves(fmaf(m, ks, hidden ? lv_ref(lv) : lv)) - TOP_ROW;
        const bool moved = top - r > LAG;                            // also in the first step (r = -infinity)
        const float a = !moved ? 1.f : hidden ? half_way(r - top) : exp2_fast(r - top), alpha = hidden ? twice(1.f, a) : a;
        r = moved ? top : r;
        const float off = lv - r;
        float sum = 0.f, apart = 0.f;
        bool far = false;
        if constexpr (hidden && WIDE) {
            const float own = fmaf(m, ks, off);                      // exponent of the largest weight
            far = far_below(own);
            if (__builtin_expect(__any(far), 0)) {
#pragma unroll
                for (int v = 0; v < 16; ++v) apart += exp2_fast((s[v] - m) * ks);
                apart = twice(apart, half_way(fmaf(m, ks, -r)));
            }
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            s[v] = exp2_fast(fmaf(s[v], ks, off));
            if constexpr (hidden) {                                  // the steps of a block that is not seen may not be numbers
                s[v] = t0 + v <= p ? s[v] : 0.f;
                if (bad && t0 + v >= full * 16 && t0 + v <= p && (bad >> (t0 + v - full * 16) & 1)) s[v] = __uint_as_float(0x7fc00000u);
            }
            sum += s[v];
        }
        sum = far ? apart : sum * inv;
        l = (hidden ? twice(l, a) : l * a) + (hidden && t0 > p ? 0.f : sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            pA.w[i] = pack_bf16x2(s[2 * i], s[2 * i + 1]);
            pB.w[i] = pack_bf16x2(s[8 + 2 * i], s[9 + 2 * i]);
        }
        // complete here, not wherever their first use is moved to
        asm volatile("" : "+v"(pA.w[0]), "+v"(pA.w[1]), "+v"(pA.w[2]), "+v"(pA.w[3]), "+v"(pB.w[0]), "+v"(pB.w[1]), "+v"(pB.w[2]), "+v"(pB.w[3]));
        return alpha;
    };
    auto rescale = [&](float alpha) {
        if (__builtin_expect(__any(alpha != 1.f), 0)) {              // said to be rare, so that the other path needs no copies of o
#pragma unroll
            for (int u = 0; u < DT; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[u][v] *= alpha;
        }
    };
    // One tile; the scores of its second half are asked for in front of the softmax of the first, so that products and vector
    // operations can stand side by side.
    auto tile = [&](auto hidden_c, int it, const Steps& st) {
        constexpr bool hidden = decltype(hidden_c)::value;
        const uint32_t kp = stage + k_read, vp = stage + v_read;
        auto read_k = [&](int h, int ks) { return *reinterpret_cast<const half8_t*>(lds((kp ^ (ks * 32)) + h * 32 * ROW)); };
        auto read_v = [&](int h, int i) { return *reinterpret_cast<const half8_t*>(lds((vp ^ (i & 1) * 16) + h * D * 64 + (i >> 1) * 1024)); };
        const float ks_n = neighbour(st.ks), lv_n = neighbour(st.lv), inv_n = neighbour(st.inv);
        const bool odd = lane & 1;
        const int t0 = it * 64 + g2 * 16;
        f32x16_t s0, s1;
#pragma unroll
        for (int v = 0; v < 16; ++v) s0[v] = s1[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s0 = SS_MFMA_32x32x16(read_k(0, ks), qf[ks], s0, 0, 0, 0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s1 = SS_MFMA_32x32x16(read_k(1, ks), qf[ks], s1, 0, 0, 0);
        // Fragments are requested four products ahead, not right in front of their own, and the first of V in front of the softmax: chunks
        // behind long caches take 4 % less, long prompts 1 %.  (Six ahead and four of V: the same, and 8 registers more.)
        half8_t va[2], vb[2];
        auto held = [](half8_t (&v)[2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(v[i]));
        };
#pragma unroll
        for (int i = 0; i < 2; ++i) va[i] = read_v(0, i);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);               // reads of LDS
#pragma unroll
        for (int i = 0; i < 2 * KS - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);             // products
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        Frag8 pA, pB;
        float alpha = softmax(hidden_c, s0, odd ? ks_n : st.ks, odd ? lv_n : st.lv, odd ? inv_n : st.inv, t0, pA, pB);
        held(va);
        rescale(alpha);
#pragma unroll
        for (int i = 0; i < KS; ++i) o[i >> 1] = SS_MFMA_32x32x16(i < 2 ? va[i < 2 ? i : 0] : read_v(0, i), i & 1 ? pB.v : pA.v, o[i >> 1], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) vb[i] = read_v(1, i);
        __builtin_amdgcn_sched_group_barrier(0x100, KS - 2, 0);
        Frag8 pC, pD;
        alpha = softmax(hidden_c, s1, odd ? st.ks : ks_n, odd ? st.lv : lv_n, odd ? st.inv : inv_n, t0 + 32, pC, pD);
        held(vb);
        rescale(alpha);
#pragma unroll
        for (int i = 0; i < KS; ++i) o[i >> 1] = SS_MFMA_32x32x16(i < 2 ? vb[i < 2 ? i : 0] : read_v(1, i), i & 1 ? pD.v : pC.v, o[i >> 1], 0, 0, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, KS - 2, 0);
    };

    Ids ids = load_ids();
    Raw raw;
    load_raw(ids, raw);
    ids = load_ids();
    begin();
    Steps cur = store(0, raw);
    load_raw(ids, raw);
    ids = load_ids();
    publish();
    for (;;) {
#pragma unroll
        for (int u = 0; u < DT; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[u][v] = 0.f;
        r = -INFINITY;
        l = 0.f;
        Steps nxt;
        auto bring = [&] {
            nxt = store(stage ^ STAGE, raw);
            load_raw(ids, raw);
            ids = load_ids();
        };
        auto next = [&] {
            cur = nxt;
            stage ^= STAGE;
            publish();
        };
        // first the tiles that every row of the wave sees all of, while all steps are NEAR
        int it = tile0;
        for (; it < n_tiles && active && it * 64 + 63 <= wave_first && !cur.wide; ++it) {
            bring();
            tile(std::false_type{}, it, cur);
            next();
        }
        for (; it < n_tiles; ++it) {
            bring();
            if (it == open_tile) {
                store_open(stage, cur);
                publish();
            }
            if (active && it * 64 <= wave_last) tile(std::true_type{}, it, cur);
            next();
        }
        l += __shfl_xor(l, 32, 64);
        const float inv = 1.f / l;
        const int64_t to = op;
        const bool whole = part < 0, stores = valid, more = begin();     // the next item's queries are requested
        if (stores && !whole) {
            float* po = scratch + to;
#pragma unroll
            for (int u = 0; u < DT; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<f32x4_t*>(po + u * 32 + 8 * j + 4 * g2) = f32x4_t{o[u][4 * j], o[u][4 * j + 1], o[u][4 * j + 2], o[u][4 * j + 3]};
            if (g2 == 0) { po[D] = r; po[D + 1] = l; }
        } else if (stores) {
#pragma unroll
            for (int u = 0; u < DT; ++u)
#pragma unroll
                for (int j = 0; j < 4; j += 2) {                         // lane halves hold 4 elements each of 8: one takes the even 8, one the odd
                    vec16 w;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[u][4 * j + 2 * i] * inv, o[u][4 * j + 2 * i + 1] * inv),
                                                                        pack_bf16x2(o[u][4 * j + 4 + 2 * i] * inv, o[u][4 * j + 5 + 2 * i] * inv), false, false);
                        w.w[i] = x[0];
                        w.w[2 + i] = x[1];
                    }
                    *reinterpret_cast<vec16*>(out + to + u * 32 + 8 * (j + g2)) = w;
                }
        }
        if (!more) break;
    }
}

// Items that were cut: their parts' sums (o, reference, l of 256 rows each) together.  D / 4 threads a row.
template <int D>
__global__ __launch_bounds__(256) void attn8_join_kernel(const float* __restrict__ scratch, bf16_t* __restrict__ out, int n_q, int n_kv, Kv8Batch b) {
    constexpr int ROWS = 1024 / D;
    const int32_t* rec = b.pf_cuts + blockIdx.x * 8;                     // sequence, kv head, first row, first query, rows, first part, parts
    const int G = n_q / n_kv, e = threadIdx.x % (D / 4) * 4, i = blockIdx.y * ROWS + threadIdx.x / (D / 4), row = rec[2] + i;
    if (row >= rec[4] * G) return;
    const float* sp = scratch + ((size_t)rec[5] * 256 + i) * (D + 4);
    float M = -INFINITY, den = 0.f;
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    const int parts = rec[6];
    for (int i0 = 0; i0 < parts; i0 += 4) {                              // four are requested together
        float m[4], l[4], mx = M;
        f32x4_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float* p = sp + (size_t)(i0 + u < parts ? i0 + u : parts - 1) * 256 * (D + 4);
            m[u] = p[D];
            l[u] = p[D + 1];
            v[u] = *reinterpret_cast<const f32x4_t*>(p + e);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + u >= parts) {                                       // repeated: weight 0 would not keep an infinite one out
                m[u] = -INFINITY;
                l[u] = 0.f;
                v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
            mx = fmaxf(mx, m[u]);
        }
        const float ref = mx == -INFINITY ? 0.f : mx, a = half_way(M - ref);
        M = mx;
        num *= twice(1.f, a);
        den = twice(den, a);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float w = half_way(m[u] - ref);
            num += twice(1.f, w) * v[u];
            den += twice(l[u], w);
        }
    }
    *reinterpret_cast<uint2*>(out + ((int64_t)(rec[3] + row / G) * n_q + rec[1] * G + row % G) * D + e) =
        make_uint2(pack_bf16x2(num[0] / den, num[1] / den), pack_bf16x2(num[2] / den, num[3] / den));
}

template <int D>
static hipError_t launch_prefill(const void* q, int64_t q_stride, void* out, int n_q, int n_kv, const Kv8Batch& b, const Kv8Layer& kv, float* scratch,
                                 hipStream_t s) {
    constexpr int LDS = 2 * prefill_stage<D>;
    const float sl2 = 1.4426950408889634f / sqrtf((float)D);
    attn8_prefill_kernel<D><<<(unsigned)b.pf_blocks, 512, LDS, s>>>((const bf16_t*)q, q_stride, (bf16_t*)out, n_q, n_kv, b, kv, sl2, scratch);
    if (b.n_cuts > 0) attn8_join_kernel<D><<<dim3((unsigned)b.n_cuts, D / 4), 256, 0, s>>>(scratch, (bf16_t*)out, n_q, n_kv, b);
    return hipGetLastError();
}

size_t attn8_prefill_scratch_floats(const Kv8Batch& b, int d) { return (size_t)b.n_parts * 256 * (d + 4); }

bool attn8_takes(int dt, int n_q, int n_kv, int d, const Kv8Batch& b, bool decode, bool force_generic) {
    if (!attn8_fits(n_q, n_kv, d, b, nullptr, 0, dt)) return false;
    if (!decode) return true;
    return (long long)b.max_seen * n_kv <= 0x7fffff00ll && (dt == F32 || force_generic || (long long)b.n_items * n_kv * ((n_q / n_kv + 15) / 16) <= 0x7fffffffll);
}

hipError_t attn8_prefill(int dt, const void* q, int64_t q_stride, void* out, int n_q, int n_kv, int d, const Kv8Batch& b,
                         const Kv8Layer& kv, float* scratch, bool force_generic, hipStream_t s) {
    if (b.T <= 0 || b.n_seqs <= 0) return hipSuccess;
    if (!attn8_fits(n_q, n_kv, d, b, q, q_stride, dt)) return hipErrorInvalidValue;
    if (dt == F32 || force_generic) return attn8_generic(dt, q, q_stride, out, n_q, n_kv, d, b, kv, nullptr, nullptr, s);
    if (!b.pf_items || b.pf_blocks <= 0 || (b.n_parts > 0 && !scratch)) return hipErrorInvalidValue;
    return d == 64 ? launch_prefill<64>(q, q_stride, out, n_q, n_kv, b, kv, scratch, s)
                   : launch_prefill<128>(q, q_stride, out, n_q, n_kv, b, kv, scratch, s);
}

// ---------------------------------------------------------------- accumulated weights
// A thread per (four tokens, kv head): the weights of the head's G queries, in their order, onto what is there.
__global__ __launch_bounds__(256) void attn8_weights_kernel(const float* __restrict__ scores, const float* __restrict__ lse, int n_q, int n_kv,
                                                            Kv8Batch b, float* __restrict__ w) {
    const int sq = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x, t4 = i % 4 * 4, g = i / 4 % n_kv, pg = i / 4 / n_kv, before = b.before[sq];
    if (pg * 16 + t4 > before) return;
    const int G = n_q / n_kv;
    const float* sp = scores + (((size_t)b.pg_off[sq] + pg) * n_q + g * G) * 16 + t4;
    const float* lp = lse + (size_t)sq * n_q + g * G;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int j = 0; j < G; ++j) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(sp + j * 16);
#pragma unroll
        for (int v = 0; v < 4; ++v) sum[v] += exp2_fast(x[v] - lp[j]);
    }
    f32x4_t* wp = reinterpret_cast<f32x4_t*>(w + ((size_t)b.page_tables[(size_t)sq * b.pt_stride + pg] * n_kv + g) * 16 + t4);
    f32x4_t x = *wp;
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (pg * 16 + t4 + v <= before) x[v] += sum[v];
    *wp = x;
}

// partial results [n_items][n_q][d + 4], then (weights) the scores [pages seen][n_q][16] and the logarithms [n_seqs][n_q]
static size_t partial_floats(const Kv8Batch& b, int n_q, int d) { return (size_t)b.n_items * n_q * (d + 4); }
size_t attn8_decode_scratch_floats(const Kv8Batch& b, int n_q, int d, bool weights) {
    return partial_floats(b, n_q, d) + (weights ? (size_t)b.n_seqs * n_q + (size_t)b.seen_pages * n_q * 16 : 0);
}

hipError_t attn8_decode(int dt, const void* q, int64_t q_stride, void* out, int n_q, int n_kv, int d, const Kv8Batch& b,
                        const Kv8Layer& kv, float* scratch, bool force_generic, hipStream_t s) {
    if (b.n_seqs <= 0) return hipSuccess;
    if (!attn8_fits(n_q, n_kv, d, b, q, q_stride, dt) || b.max_q_len != 1 || !scratch || !attn8_takes(dt, n_q, n_kv, d, b, true, force_generic))
        return hipErrorInvalidValue;
    float* scores = kv.w ? scratch + partial_floats(b, n_q, d) : nullptr;
    float* lse = kv.w ? scores + (size_t)b.seen_pages * n_q * 16 : nullptr;
    hipError_t e = hipSuccess;
    if (dt == F32 || force_generic) {
        e = attn8_generic(dt, q, q_stride, out, n_q, n_kv, d, b, kv, scores, lse, s);
    } else {
        if (b.n_items <= 0) return hipErrorInvalidValue;
        if (d == 64) launch_decode<64>(q, q_stride, out, n_q, n_kv, b, kv, scratch, scores, lse, s);
        else launch_decode<128>(q, q_stride, out, n_q, n_kv, b, kv, scratch, scores, lse, s);
        e = hipGetLastError();
    }
    if (e != hipSuccess || !kv.w) return e;
    attn8_weights_kernel<<<dim3((unsigned)(((long long)(b.max_seen + 15) / 16 * 4 * n_kv + 255) / 256), b.n_seqs), 256, 0, s>>>(scores, lse, n_q, n_kv, b, kv.w);
    return hipGetLastError();
}

}  // namespace SS_NS
