// Cache in 8 bits: what fills it, reads it back, keeps the accumulated attention weights and evicts by them.  Everything here moves
// data: bound by HBM (32 prompts of 512 - 4096 tokens on 8 heads written in 107 us, 4.3 TB/s, and read back in 82, 5.6 TB/s).
// The arithmetic of a block (see Kv8Layer): A = max |v|, q = rint(v * 127 / A).  For 16-bit v the product v * 127 is exact, the quotient
// correctly rounded, and q the one of real arithmetic: with whole numbers m, M < 2^11 for v = m 2^-j (j >= 0) and A = M >= 2^10, the quotient
// is (254 m - (2 k + 1) M 2^j) / (2 M 2^j) away from half a step k + 1 / 2, which is 0 or more than 2^-(12 + j); it is below 2^(8 - j), so its
// rounding moves it by 2^-(16 + j) at most.  For 32-bit v a quotient close to half a step is formed again in 64 bits (25 bits decide there).
#include "ss_device.h"
#include "ss_kernels.h"

namespace SS_NS {
using namespace ssk;

// Where 127 times a value would pass the largest float both sides of the quotient are scaled; a power of two leaves it as it is.
__device__ __forceinline__ float kv8_fit(float amax) { return amax > 1e36f ? 0.00390625f : 1.f; }
template <typename T> __device__ __forceinline__ int kv8_round(float v, float amax) {
    if (!(amax > 0.f && amax < INFINITY)) return 0;
    const float t = v * 127.f / amax, r = rintf(t);
    if (sizeof(T) == 4 && fabsf(t - r) > 0.499f) return (int)rint((double)v * 127.0 / (double)amax);
    return (int)r;
}
// N of them: by the reciprocal (rc = 1 / amax), off from the quotient by at most 127 * 3 * 2^-24 < 2.3e-5; where that could decide, by the
// division, which is ten times the instructions.
template <typename T, int N>
__device__ __forceinline__ void kv8_round_n(const float* v, float amax, float rc, int* q) {
    constexpr float FAR = sizeof(T) == 4 ? 0.4989f : 0.4999f;
    float off = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float t = v[j] * 127.f * rc, r = rintf(t);
        q[j] = (int)r;
        off = fmaxf(off, fabsf(t - r));
    }
    if (!(off < FAR && amax > 1e-30f && amax < INFINITY)) {              // (a smaller one's reciprocal may not be finite)
#pragma unroll
        for (int j = 0; j < N; ++j) q[j] = kv8_round<T>(v[j], amax);
    }
}
__device__ __forceinline__ float kv8_step(float amax) { return amax / 127.f; }
// a value that is not finite makes the block's magnitude NaN, and no other way round (fmaxf would drop a NaN)
__device__ __forceinline__ float kv8_mag(float v) { const float a = fabsf(v); return a < INFINITY ? a : INFINITY; }
__device__ __forceinline__ float kv8_amax(float m) { return m < INFINITY ? m : __uint_as_float(0x7fc00000u); }

__device__ __forceinline__ uint32_t kv8_pack4(const int* q) {
    return (uint32_t)(q[0] & 255) | (uint32_t)(q[1] & 255) << 8 | (uint32_t)(q[2] & 255) << 16 | (uint32_t)(q[3] & 255) << 24;
}
__device__ __forceinline__ int kv8_byte(uint32_t w, int i) { return (int)(int8_t)(w >> (8 * i)); }

// One wave's share of a block of 16 tokens x D elements: lane l has rows 4 * (l / 16) + i, i = 0 .. 3, and of each the 16-byte
// pieces l % 16, l % 16 + 16, ... (one or two, half the lanes idle where a row has only 8 pieces).  Four tokens of one element are
// then in one lane: a dword of the transposed V page.
template <typename T, int D> struct Kv8Tile {
    static constexpr int EV = 16 / (int)sizeof(T);
    static constexpr int PIECES = D / EV;                       // 16-byte pieces of a row: 8, 16 or 32
    static constexpr int NP = PIECES > 16 ? PIECES / 16 : 1;
    float x[4][NP * EV];
    __device__ static bool idle(int lane) { return PIECES < 16 && (lane & 15) >= PIECES; }
    __device__ static int col(int lane, int p) { return ((lane & 15) + 16 * p) * EV; }
};

// LDS image of a V page, 4 tokens a dword: element e, tokens 4 * r .. + 3.  Rows of 8 elements are padded so that what 16 lanes
// write falls on all banks.
__device__ __forceinline__ int kv8_vword(int e, int r) { return e * 4 + r + (e >> 3) * 4; }
template <int D> constexpr int kv8_vwords = D * 4 + (D / 8) * 4;

// Quantises the tile into K rows and, through `lds` (kv8_vwords of this wave), V rows.
template <typename T, int D>
__device__ __forceinline__ void kv8_store_block(const Kv8Tile<T, D>& k, const Kv8Tile<T, D>& v, int8_t* kp, int8_t* vp, float* amax,
                                                uint32_t* lds, int lane) {
    using Tile = Kv8Tile<T, D>;
    float mk = 0.f, mv = 0.f;
    if (!Tile::idle(lane)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < Tile::NP * Tile::EV; ++e) {
                mk = fmaxf(mk, kv8_mag(k.x[i][e]));
                mv = fmaxf(mv, kv8_mag(v.x[i][e]));
            }
    }
    mk = wave_max(mk);
    mv = wave_max(mv);
    if (lane == 0) {
        amax[0] = kv8_amax(mk);
        amax[1] = kv8_amax(mv);
    }
    const float fk = kv8_fit(mk), fv = kv8_fit(mv), ak = mk * fk, av = mv * fv, rk = 1.f / ak, rv = 1.f / av;
    if (!Tile::idle(lane)) {
#pragma unroll
        for (int p = 0; p < Tile::NP; ++p) {
            const int c = Tile::col(lane, p);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int e = 0; e < Tile::EV; e += 4) {
                    float x[4];
                    int q[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = k.x[i][p * Tile::EV + e + j] * fk;
                    kv8_round_n<T, 4>(x, ak, rk, q);
                    *reinterpret_cast<uint32_t*>(kp + (4 * (lane >> 4) + i) * D + c + e) = kv8_pack4(q);
                }
            }
#pragma unroll
            for (int e = 0; e < Tile::EV; ++e) {
                float x[4];
                int q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = v.x[i][p * Tile::EV + e] * fv;
                kv8_round_n<T, 4>(x, av, rv, q);
                lds[kv8_vword(c + e, lane >> 4)] = kv8_pack4(q);
            }
        }
    }
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
#pragma unroll
    for (int r = 0; r < D / 64; ++r) {
        const int e = r * 64 + lane;
        vec16 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.w[i] = lds[kv8_vword(e, i)];
        *reinterpret_cast<vec16*>(vp + e * 16) = o;
    }
}

// rows [0, slot0) of the open block, then cnt rows of src
template <typename T, int D>
__device__ __forceinline__ void kv8_load_tile(Kv8Tile<T, D>& t, const T* src, int64_t stride, const T* open, int slot0, int lane) {
    using Tile = Kv8Tile<T, D>;
    if (Tile::idle(lane)) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 4 * (lane >> 4) + i;
        const T* p = row < slot0 ? open + row * D : src + (row - slot0) * stride;
#pragma unroll
        for (int j = 0; j < Tile::NP; ++j) unpack16<T>(*reinterpret_cast<const vec16*>(p + Tile::col(lane, j)), t.x[i] + j * Tile::EV);
    }
}

// n rows of D elements into the open block from slot `at` on
template <typename T, int D>
__device__ __forceinline__ void kv8_copy_rows(const T* src, int64_t stride, T* open, int at, int n, int lane) {
    constexpr int EV = 16 / (int)sizeof(T), PIECES = D / EV;
    for (int i = lane; i < n * PIECES; i += 64)
        *reinterpret_cast<vec16*>(open + (at + i / PIECES) * D + i % PIECES * EV) =
            *reinterpret_cast<const vec16*>(src + (i / PIECES) * stride + i % PIECES * EV);
}

// New tokens.  One wave per (page unit, kv head): a unit is the tokens of a sequence that fall into one block.  A unit that
// fills its block quantises it.  The tokens of a sequence's last block go to its open block; the wave of the sequence's FIRST unit
// brings them there, because that unit may begin inside the block that was open before and has to read that one first.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_write_kernel(const T* k, int64_t k_stride, const T* v, int64_t v_stride, int n_heads,
                                                        Kv8Batch b, Kv8Layer kv) {
    __shared__ uint32_t lds[4][kv8_vwords<D>];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t id = (int64_t)blockIdx.x * 4 + wave;
    if (id >= (int64_t)b.n_units * n_heads) return;
    const int u = (int)(id / n_heads), g = (int)(id % n_heads);
    const int sq = b.unit_seq[u], tok0 = b.unit_tok0[u], pos0 = b.unit_pos0[u], cnt = b.unit_cnt[u];
    const int before = b.before[sq], end = b.end[sq];
    const size_t page = (size_t)b.page_tables[(size_t)sq * b.pt_stride + pos0 / 16] * n_heads + g;
    T* ko = (T*)kv.open + ((size_t)b.slot[sq] * 2 * n_heads + g) * 16 * D;
    T* vo = ko + (size_t)n_heads * 16 * D;
    const int slot0 = pos0 & 15;
    k += (size_t)g * D;
    v += (size_t)g * D;
    if (kv.w && lane < cnt) kv.w[page * 16 + slot0 + lane] = 0.f;
    if (slot0 + cnt == 16) {
        Kv8Tile<T, D> tk, tv;
        kv8_load_tile<T, D>(tk, k + tok0 * k_stride, k_stride, ko, slot0, lane);
        kv8_load_tile<T, D>(tv, v + tok0 * v_stride, v_stride, vo, slot0, lane);
        kv8_store_block<T, D>(tk, tv, kv.k + page * 16 * D, kv.v + page * 16 * D, kv.amax + page * 2, lds[wave], lane);
    }
    if (pos0 == before) {
        const int last = (end - 1) & ~15, from = last > before ? last : before, n = end - from;
        const int64_t t = (int64_t)b.cu_q[sq] + from - before;
        kv8_copy_rows<T, D>(k + t * k_stride, k_stride, ko, from & 15, n, lane);
        kv8_copy_rows<T, D>(v + t * v_stride, v_stride, vo, from & 15, n, lane);
    }
}

// Whole sequences from staging [K | V][head][position][D]: a wave per (page, unit, head).
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_scatter_kernel(const Kv8Layer* __restrict__ layers, int n_heads, RepackUnits u,
                                                          const T* __restrict__ staging) {
    __shared__ uint32_t lds[4][kv8_vwords<D>];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int unit = blockIdx.y, g = blockIdx.z, pg = blockIdx.x * 4 + wave, len = u.unit_len[unit];
    if (pg * 16 >= len) return;
    const Kv8Layer kv = layers[u.unit_layer[unit]];
    const size_t page = (size_t)u.pages[u.unit_pt[unit] + pg] * n_heads + g;
    const T* k = staging + u.unit_off[unit] + ((size_t)g * len + pg * 16) * D;
    const T* v = k + (size_t)n_heads * len * D;
    const int n = len - pg * 16 < 16 ? len - pg * 16 : 16;
    if (kv.w && lane < n) kv.w[page * 16 + lane] = 0.f;
    if (n == 16) {
        Kv8Tile<T, D> tk, tv;
        kv8_load_tile<T, D>(tk, k, D, nullptr, 0, lane);
        kv8_load_tile<T, D>(tv, v, D, nullptr, 0, lane);
        kv8_store_block<T, D>(tk, tv, kv.k + page * 16 * D, kv.v + page * 16 * D, kv.amax + page * 2, lds[wave], lane);
    }
    if (pg * 16 + n == len) {
        T* ko = (T*)kv.open + ((size_t)u.unit_slot[unit] * 2 * n_heads + g) * 16 * D;
        kv8_copy_rows<T, D>(k, D, ko, 0, n, lane);
        kv8_copy_rows<T, D>(v, D, ko + (size_t)n_heads * 16 * D, 0, n, lane);
    }
}

// ... and into it: full blocks as what they stand for, rounded once to the model's type, the open block as it is.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_gather_kernel(const Kv8Layer* __restrict__ layers, int n_heads, RepackUnits u,
                                                         T* __restrict__ staging) {
    using Tile = Kv8Tile<T, D>;
    __shared__ uint32_t lds[4][kv8_vwords<D>];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int unit = blockIdx.y, g = blockIdx.z, pg = blockIdx.x * 4 + wave, len = u.unit_len[unit];
    if (pg * 16 >= len) return;
    const Kv8Layer kv = layers[u.unit_layer[unit]];
    T* k = staging + u.unit_off[unit] + ((size_t)g * len + pg * 16) * D;
    T* v = k + (size_t)n_heads * len * D;
    const int n = len - pg * 16;
    if (n < 16) {
        const T* ko = (const T*)kv.open + ((size_t)u.unit_slot[unit] * 2 * n_heads + g) * 16 * D;
        kv8_copy_rows<T, D>(ko, D, k, 0, n, lane);
        kv8_copy_rows<T, D>(ko + (size_t)n_heads * 16 * D, D, v, 0, n, lane);
        return;
    }
    const size_t page = (size_t)u.pages[u.unit_pt[unit] + pg] * n_heads + g;
    const int8_t *kp = kv.k + page * 16 * D, *vp = kv.v + page * 16 * D;
    const float sk = kv8_step(kv.amax[page * 2]), sv = kv8_step(kv.amax[page * 2 + 1]);
    uint32_t* l = lds[wave];
#pragma unroll
    for (int r = 0; r < D / 64; ++r) {
        const vec16 w = *reinterpret_cast<const vec16*>(vp + (r * 64 + lane) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) l[kv8_vword(r * 64 + lane, i)] = w.w[i];
    }
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
    if (Tile::idle(lane)) return;
#pragma unroll
    for (int p = 0; p < Tile::NP; ++p) {
        const int c = Tile::col(lane, p);
        uint32_t vw[Tile::EV];
#pragma unroll
        for (int e = 0; e < Tile::EV; ++e) vw[e] = l[kv8_vword(c + e, lane >> 4)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * (lane >> 4) + i;
            float f[Tile::EV];
#pragma unroll
            for (int e = 0; e < Tile::EV; e += 4) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(kp + row * D + c + e);
#pragma unroll
                for (int j = 0; j < 4; ++j) f[e + j] = (float)kv8_byte(w, j) * sk;
            }
            *reinterpret_cast<vec16*>(k + row * D + c) = pack16<T>(f);
#pragma unroll
            for (int e = 0; e < Tile::EV; ++e) f[e] = (float)kv8_byte(vw[e], i) * sv;
            *reinterpret_cast<vec16*>(v + row * D + c) = pack16<T>(f);
        }
    }
}

#define SS_TYPED(dt, d, KERNEL, ...)                                        \
    do {                                                                    \
        if ((dt) == F32) {                                                  \
            if ((d) == 64) KERNEL<float, 64> __VA_ARGS__;                   \
            else KERNEL<float, 128> __VA_ARGS__;                            \
        } else {                                                            \
            if ((d) == 64) KERNEL<bf16_t, 64> __VA_ARGS__;                  \
            else KERNEL<bf16_t, 128> __VA_ARGS__;                           \
        }                                                                   \
    } while (0)

template <typename T, int D>
static void launch_write(const void* k, int64_t ks, const void* v, int64_t vs, int n_heads, const Kv8Batch& b, const Kv8Layer& kv, hipStream_t s) {
    const long long waves = (long long)b.n_units * n_heads;
    kv8_write_kernel<T, D><<<(unsigned)((waves + 3) / 4), 256, 0, s>>>((const T*)k, ks, (const T*)v, vs, n_heads, b, kv);
}

hipError_t kv8_write(int dt, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int n_heads, int d, const Kv8Batch& b,
                     const Kv8Layer& kv, hipStream_t s) {
    if (b.n_units <= 0) return hipSuccess;
    const int ev = dt == F32 ? 4 : 8;
    if ((d != 64 && d != 128) || n_heads <= 0 || (long long)b.n_units * n_heads > 0x7fffffffll) return hipErrorInvalidValue;
    if (((uintptr_t)k | (uintptr_t)v) % 16 || k_stride % ev || v_stride % ev) return hipErrorInvalidValue;
    SS_TYPED(dt, d, launch_write, (k, k_stride, v, v_stride, n_heads, b, kv, s));
    return hipGetLastError();
}

template <typename T, int D>
static void launch_gather(const Kv8Layer* layers, int n_heads, const RepackUnits& u, void* staging, dim3 grid, hipStream_t s) {
    kv8_gather_kernel<T, D><<<grid, 256, 0, s>>>(layers, n_heads, u, (T*)staging);
}
template <typename T, int D>
static void launch_scatter(const Kv8Layer* layers, int n_heads, const RepackUnits& u, const void* staging, dim3 grid, hipStream_t s) {
    kv8_scatter_kernel<T, D><<<grid, 256, 0, s>>>(layers, n_heads, u, (const T*)staging);
}

static bool repack_fits(int n_heads, int d, const RepackUnits& u) {
    return (d == 64 || d == 128) && n_heads > 0 && n_heads <= 65535 && u.n_units <= 65535 && u.unit_slot;
}

hipError_t kv8_gather(int dt, const Kv8Layer* layers, int n_heads, int d, const RepackUnits& u, void* staging, hipStream_t s) {
    if (u.n_units <= 0 || u.max_pages <= 0) return hipSuccess;
    if (!repack_fits(n_heads, d, u)) return hipErrorInvalidValue;
    SS_TYPED(dt, d, launch_gather, (layers, n_heads, u, staging, dim3((u.max_pages + 3) / 4, u.n_units, n_heads), s));
    return hipGetLastError();
}

hipError_t kv8_scatter(int dt, const Kv8Layer* layers, int n_heads, int d, const RepackUnits& u, const void* staging, hipStream_t s) {
    if (u.n_units <= 0 || u.max_pages <= 0) return hipSuccess;
    if (!repack_fits(n_heads, d, u)) return hipErrorInvalidValue;
    SS_TYPED(dt, d, launch_scatter, (layers, n_heads, u, staging, dim3((u.max_pages + 3) / 4, u.n_units, n_heads), s));
    return hipGetLastError();
}

// ---------------------------------------------------------------- rotary embedding of a batch's q and k, in place
// A thread per (token, head, 16-byte piece of the first half): it has the pairs of both halves.
template <typename T>
__global__ __launch_bounds__(256) void kv8_rope_kernel(T* __restrict__ qkv, int heads, int64_t row_stride, int d, const float* __restrict__ rope,
                                                       Kv8Batch b) {
    constexpr int V = VecOf<T>::N;
    const int u = blockIdx.x, sq = b.unit_seq[u], cnt = b.unit_cnt[u];
    const int pos0 = b.unit_pos0[u] - b.before[sq] + b.pos[sq];
    const int cph = d / 2 / V;
    for (int i = threadIdx.x; i < cnt * heads * cph; i += 256) {
        const int c = i % cph * V, h = i / cph % heads, t = i / (cph * heads);
        T* lo_p = qkv + (size_t)(b.unit_tok0[u] + t) * row_stride + (size_t)h * d + c;
        T* hi_p = lo_p + d / 2;
        const float* cs = rope + (size_t)(pos0 + t) * d + 2 * c;
        float lo[V], hi[V], olo[V], ohi[V];
        unpack16<T>(*reinterpret_cast<const vec16*>(lo_p), lo);
        unpack16<T>(*reinterpret_cast<const vec16*>(hi_p), hi);
#pragma unroll
        for (int j = 0; j < V; ++j) rope_rotate(lo[j], hi[j], cs[2 * j], cs[2 * j + 1], olo[j], ohi[j]);
        *reinterpret_cast<vec16*>(lo_p) = pack16<T>(olo);
        *reinterpret_cast<vec16*>(hi_p) = pack16<T>(ohi);
    }
}

hipError_t kv8_rope(int dt, void* qkv, int n_q, int n_kv, int d, const float* rope_table, const Kv8Batch& b, hipStream_t s) {
    if (b.n_units <= 0) return hipSuccess;
    if (d % 16 || n_q <= 0 || n_kv <= 0) return hipErrorInvalidValue;
    const int64_t stride = (int64_t)(n_q + 2 * n_kv) * d;
    if (dt == F32) kv8_rope_kernel<float><<<b.n_units, 256, 0, s>>>((float*)qkv, n_q + n_kv, stride, d, rope_table, b);
    else kv8_rope_kernel<bf16_t><<<b.n_units, 256, 0, s>>>((bf16_t*)qkv, n_q + n_kv, stride, d, rope_table, b);
    return hipGetLastError();
}

// A decode step's one launch for both: queries rotated in place, the new token's key (rotated) and value into the open block, and that
// quantised where it is full now.  One token a sequence, a unit of its own each.  A wave per (sequence, kv head), and one for every few query heads.
// Rotation and write as two launches took 4 us more a layer, of 115 for eight sequences.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_step_kernel(T* __restrict__ qkv, int n_q, int n_kv, const float* __restrict__ rope, Kv8Batch b, Kv8Layer kv) {
    constexpr int V = VecOf<T>::N, HALF = D / 2 / V, HEADS = 64 / HALF;  // 16-byte pieces of half a head; query heads of a wave
    __shared__ uint32_t lds[4][kv8_vwords<D>];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = n_kv + (n_q + HEADS - 1) / HEADS;
    const int64_t id = (int64_t)blockIdx.x * 4 + wave;
    if (id >= (int64_t)b.n_seqs * per) return;
    const int sq = (int)(id / per), part = (int)(id % per), pos0 = b.before[sq], slot0 = pos0 & 15;
    T* row = qkv + (size_t)b.cu_q[sq] * (n_q + 2 * n_kv) * D;
    const int c = lane % HALF * V;
    auto rotated = [&](const T* head, vec16& lo, vec16& hi) {
        const float* cs = rope + (size_t)b.pos[sq] * D + 2 * c;
        float x[V], y[V], ox[V], oy[V];
        unpack16<T>(*reinterpret_cast<const vec16*>(head + c), x);
        unpack16<T>(*reinterpret_cast<const vec16*>(head + D / 2 + c), y);
#pragma unroll
        for (int j = 0; j < V; ++j) rope_rotate(x[j], y[j], cs[2 * j], cs[2 * j + 1], ox[j], oy[j]);
        lo = pack16<T>(ox);
        hi = pack16<T>(oy);
    };
    vec16 lo, hi;
    if (part >= n_kv) {
        const int a = (part - n_kv) * HEADS + lane / HALF;
        if (a >= n_q) return;
        T* head = row + (size_t)a * D;
        rotated(head, lo, hi);
        *reinterpret_cast<vec16*>(head + c) = lo;
        *reinterpret_cast<vec16*>(head + D / 2 + c) = hi;
        return;
    }
    const int g = part;
    const T *k = row + (size_t)(n_q + g) * D, *v = row + (size_t)(n_q + n_kv + g) * D;
    T* ko = (T*)kv.open + ((size_t)b.slot[sq] * 2 * n_kv + g) * 16 * D;
    T* vo = ko + (size_t)n_kv * 16 * D;
    const size_t page = (size_t)b.page_tables[(size_t)sq * b.pt_stride + pos0 / 16] * n_kv + g;
    if (lane < HALF) {
        rotated(k, lo, hi);
        *reinterpret_cast<vec16*>(ko + slot0 * D + c) = lo;
        *reinterpret_cast<vec16*>(ko + slot0 * D + D / 2 + c) = hi;
    }
    if (lane < 2 * HALF) *reinterpret_cast<vec16*>(vo + slot0 * D + lane * V) = *reinterpret_cast<const vec16*>(v + lane * V);
    if (kv.w && lane == 0) kv.w[page * 16 + slot0] = 0.f;
    if (slot0 == 15) {
        // the rows that were just stored are read back by other lanes of the wave
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __threadfence_block();
        Kv8Tile<T, D> tk, tv;
        kv8_load_tile<T, D>(tk, nullptr, 0, ko, 16, lane);
        kv8_load_tile<T, D>(tv, nullptr, 0, vo, 16, lane);
        kv8_store_block<T, D>(tk, tv, kv.k + page * 16 * D, kv.v + page * 16 * D, kv.amax + page * 2, lds[wave], lane);
    }
}

template <typename T, int D>
static void launch_step(void* qkv, int n_q, int n_kv, const float* rope, const Kv8Batch& b, const Kv8Layer& kv, unsigned blocks, hipStream_t s) {
    kv8_step_kernel<T, D><<<blocks, 256, 0, s>>>((T*)qkv, n_q, n_kv, rope, b, kv);
}

hipError_t kv8_step(int dt, void* qkv, int n_q, int n_kv, int d, const float* rope_table, const Kv8Batch& b, const Kv8Layer& kv, hipStream_t s) {
    if (b.n_seqs <= 0) return hipSuccess;
    if ((d != 64 && d != 128) || n_q <= 0 || n_kv <= 0 || b.max_q_len != 1 || b.n_units != b.n_seqs || (uintptr_t)qkv % 16) return hipErrorInvalidValue;
    const int heads = 64 / (d / 2 / (dt == F32 ? 4 : 8));
    const long long waves = (long long)b.n_seqs * (n_kv + (n_q + heads - 1) / heads);
    if (waves > 0x7fffffffll) return hipErrorInvalidValue;
    SS_TYPED(dt, d, launch_step, (qkv, n_q, n_kv, rope_table, b, kv, (unsigned)((waves + 3) / 4), s));
    return hipGetLastError();
}

// ---------------------------------------------------------------- accumulated weights of whole sequences
__global__ __launch_bounds__(256) void kv8_weights_kernel(const Kv8Layer* __restrict__ layers, int n_heads, RepackUnits u, float* __restrict__ buf,
                                                          bool in) {
    const int unit = blockIdx.y, len = u.unit_len[unit], t = blockIdx.x * 256 + threadIdx.x;
    if (t >= len) return;
    float* w = layers[u.unit_layer[unit]].w + ((size_t)u.pages[u.unit_pt[unit] + t / 16] * n_heads) * 16 + t % 16;
    float* p = buf + u.unit_off[unit] + t;
    for (int g = blockIdx.z; g < n_heads; g += gridDim.z) {
        if (in) w[(size_t)g * 16] = p[(size_t)g * len];
        else p[(size_t)g * len] = w[(size_t)g * 16];
    }
}

hipError_t kv8_weights(const Kv8Layer* layers, int n_heads, const RepackUnits& u, float* buf, bool in, hipStream_t s) {
    if (u.n_units <= 0 || u.max_pages <= 0) return hipSuccess;
    if (n_heads <= 0 || u.n_units > 65535) return hipErrorInvalidValue;
    kv8_weights_kernel<<<dim3((u.max_pages + 15) / 16, u.n_units, n_heads < 64 ? n_heads : 64), 256, 0, s>>>(layers, n_heads, u, buf, in);
    return hipGetLastError();
}

// ---------------------------------------------------------------- eviction
// Order of the weights as unsigned numbers: larger weight, larger number; -0 is 0, NaN is above everything.
__device__ __forceinline__ uint32_t evict_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t b = __float_as_uint(w + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Which tokens stay.  A block per (head, layer, sequence).  The key of the last token that stays among the older ones is found digit
// by digit (four histograms of 256), then one ordered pass lists the positions: all above that key, and of those
// equal to it the first ones.
// Keys are read from the cache once, to LDS, those behind the EV_KEYS first ones for every pass again.  256 lists of 1500 - 9000 keys: 22 us
// (57 with keys read for every pass and the digit looked for by one lane).
constexpr int EV_T = 1024, EV_KEYS = 36 * 1024;
__global__ __launch_bounds__(EV_T) void kv8_select_kernel(const Kv8Layer* __restrict__ layers, int n_heads, Kv8Evict e, int32_t* __restrict__ lists) {
    __shared__ int hist[256], digit_s, left_s, eq_w[EV_T / 64], out_w[EV_T / 64];
    const int g = blockIdx.x, layer = blockIdx.y, sq = blockIdx.z;
    const int len = e.len[sq], keep = e.keep[sq];
    if (len <= keep) return;
    const int recent = e.recent < keep ? e.recent : keep;
    const int n = len - recent, k = keep - recent;
    const float* w = layers[layer].w;
    const int32_t* pt = e.page_tables + (size_t)sq * e.pt_stride;
    int32_t* list = lists + e.list_off[sq] + ((size_t)layer * n_heads + g) * keep;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < recent; i += EV_T) list[k + i] = n + i;
    if (k == 0) return;
    extern __shared__ uint32_t keys[];
    auto fetch = [&](int t) { return evict_key(w[((size_t)pt[t >> 4] * n_heads + g) * 16 + (t & 15)]); };
    auto key_at = [&](int t) { return t < EV_KEYS ? keys[t] : fetch(t); };
#pragma unroll 4
    for (int t = tid; t < n && t < EV_KEYS; t += EV_T) keys[t] = fetch(t);
    uint32_t prefix = 0;
    int left = k;                         // how many of those with the prefix stay
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += EV_T) hist[i] = 0;
        __syncthreads();
        for (int t = tid; t < n; t += EV_T) {
            const uint32_t key = key_at(t);
            if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[key >> shift & 255], 1);
        }
        __syncthreads();
        if (wave == 0) {                  // lane l counts what lies above its digits 255 - 4 l .. 252 - 4 l; the digit where `left` is passed
            int h[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += h[i] = hist[255 - 4 * lane - i];
            int above = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int x = __shfl_up(above, o, 64);
                if (lane >= o) above += x;
            }
            above -= sum;
            if (above < left && left <= above + sum) {
                int i = 0, rest = left - above;
                while (h[i] < rest) rest -= h[i++];
                digit_s = 255 - 4 * lane - i;
                left_s = rest;
            }
        }
        __syncthreads();
        prefix |= (uint32_t)digit_s << shift;
        left = left_s;
        __syncthreads();
    }
    int n_eq = 0, n_out = 0;              // found in front of this stretch
    for (int t0 = 0; t0 < n; t0 += EV_T) {
        const int t = t0 + tid;
        const uint32_t key = t < n ? key_at(t) : 0;
        const bool eq = t < n && key == prefix, above = t < n && key > prefix;
        const uint64_t eqm = __ballot(eq), lower = (1ull << lane) - 1;
        if (lane == 0) eq_w[wave] = __popcll(eqm);
        __syncthreads();
        int eq_before = n_eq, eq_all = 0;
        for (int i = 0; i < EV_T / 64; ++i) {
            if (i < wave) eq_before += eq_w[i];
            eq_all += eq_w[i];
        }
        const bool stays = above || (eq && eq_before + __popcll(eqm & lower) < left);
        const uint64_t sm = __ballot(stays);
        if (lane == 0) out_w[wave] = __popcll(sm);
        __syncthreads();
        int out_before = n_out, out_all = 0;
        for (int i = 0; i < EV_T / 64; ++i) {
            if (i < wave) out_before += out_w[i];
            out_all += out_w[i];
        }
        if (stays) list[out_before + __popcll(sm & lower)] = t;
        n_eq += eq_all;
        n_out += out_all;
        __syncthreads();
    }
}

// Moves the kept tokens to the front, in place.  A block per (head, layer, sequence), a wave per new block of 16 tokens, EM_WAVES of
// them a round.  Token s of the new cache comes from position list[s] >= s, so that a new block reads from pages at or behind its own:
// when all waves of a round have what they move, they store, and what later rounds read is still there.  What bounds it is the chain
// position -> page -> bytes, so a round's bytes are requested before the round in front of it stores (its pages lie behind),
// page numbers one round and positions two rounds ahead.
// A token's V is a byte of every row of its page: the page's rows are brought once, 16 bytes a lane, for all tokens that come from
// it, and v_perm puts the bytes where they go (one load a token and row instead took twice the time).  Eight pages are requested ahead,
// which is enough where half of a page or more stays; what lies behind them is waited for.  256 lists of 2048 tokens from up to 9000:
// 130 us, 8 a round; with a wave a half of a block's elements and twice the waves 141, one load a byte 197.
// In units of A / 127 the old values are q * A, exact in fp32 where A has the 16 bits of the model's type; those of the open
// block are 127 * v.  The new block's magnitude in those units is W: A' = W / 127, q' = rint(value * 127 / W).  All in 32 bits,
// for 32-bit models and blocks that were evicted before too, whose products are rounded.
constexpr int EM_WAVES = 8;
template <typename T, int D>
__global__ __launch_bounds__(64 * EM_WAVES) void kv8_move_kernel(const Kv8Layer* __restrict__ layers, int n_heads, Kv8Evict e,
                                                                 const int32_t* __restrict__ lists) {
    const int g = blockIdx.x, layer = blockIdx.y, sq = blockIdx.z;
    const int len = e.len[sq], keep = e.keep[sq];
    if (len <= keep) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Kv8Layer kv = layers[layer];
    const int32_t* pt = e.page_tables + (size_t)sq * e.pt_stride;
    const int32_t* list = lists + e.list_off[sq] + ((size_t)layer * n_heads + g) * keep;
    T* ko = (T*)kv.open + ((size_t)e.slot[sq] * 2 * n_heads + g) * 16 * D;
    T* vo = ko + (size_t)n_heads * 16 * D;
    const int full = len / 16;                               // full blocks of the old cache
    const int blocks = (keep + 15) / 16;
    constexpr int R = D / 64;                                // a lane has elements R * lane + r of every token
    // lane t (of 16): position and page of token t of a wave's block; behind the end the last token again
    auto position = [&](int blk) {
        const int i = blk * 16 + (lane & 15);
        return list[i < keep ? i : keep - 1];
    };
    constexpr int AHEAD = 8;
    struct Raw { uint32_t k[16]; vec16 v[AHEAD][R]; float ak, av, w; };
    // first tokens of the pages that a block comes from
    auto starts = [&](int pos) { return (uint32_t)__ballot(lane == 0 || pos >> 4 != __shfl_up(pos, 1, 64) >> 4) & 0xffffu; };
    auto fetch_rows = [&](uint32_t from, int page, vec16 (&rows)[AHEAD][R]) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (from) {
                const size_t at = ((size_t)__builtin_amdgcn_readlane(page, __builtin_ctz(from)) * n_heads + g) * 16 * D;
                from &= from - 1;
#pragma unroll
                for (int r = 0; r < R; ++r) rows[j][r] = *reinterpret_cast<const vec16*>(kv.v + at + (R * lane + r) * 16);
            }
        }
    };
    auto fetch = [&](int pos, int page, Raw& x) {
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const size_t at = ((size_t)__builtin_amdgcn_readlane(page, t) * n_heads + g) * 16 * D;
            const int tok = __builtin_amdgcn_readlane(pos, t) & 15;
            const int8_t* kp = kv.k + at + tok * D;
            x.k[t] = R == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(kp + 2 * lane) : (uint32_t)*reinterpret_cast<const uint8_t*>(kp + lane);
        }
        fetch_rows(starts(pos), page, x.v);
        const size_t at = (size_t)page * n_heads + g;
        const float2 a = *reinterpret_cast<const float2*>(kv.amax + at * 2);
        x.ak = a.x;
        x.av = a.y;
        x.w = kv.w[at * 16 + (pos & 15)];
    };
    int pos = position(wave), page = pt[pos >> 4], pos_n = position(wave + EM_WAVES);
    Raw raw;
    fetch(pos, page, raw);
    for (int b0 = 0; b0 < blocks; b0 += EM_WAVES) {
        const int blk = b0 + wave;
        const int cnt = blk < blocks ? (keep - blk * 16 < 16 ? keep - blk * 16 : 16) : 0;
        const int page_n = pt[pos_n >> 4], pos_nn = position(blk + 2 * EM_WAVES);
        const int page_to = blk < blocks ? pt[blk] : 0;
        // an open block's token: the value is itself, its magnitude stands for 127
        const bool open_mine = (lane & 15) < cnt && pos >= full * 16;
        const uint32_t opens = (uint32_t)__ballot(open_mine) & 0xffffu;
        const float ak = (lane & 15) >= cnt ? 0.f : open_mine ? 127.f : raw.ak, av = (lane & 15) >= cnt ? 0.f : open_mine ? 127.f : raw.av, w = raw.w;
        // lane 4 j + i: where tokens 4 i .. + 3 come from in a row of the block's j-th page, as selectors of its lower and its upper 8
        // bytes; 12 is a byte of zeros
        uint32_t from = starts(pos), sel_lo = 0, sel_hi = 0;
        const int mine = (__popc(from & ((2u << (lane & 15)) - 1)) - 1) << 4 | (pos & 15);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int x = __shfl(mine, (lane & 3) * 4 + u, 64);
            const bool here = x >> 4 == lane >> 2;
            sel_lo |= (here && !(x & 8) ? x & 7 : 12) << (8 * u);
            sel_hi |= (here && (x & 8) ? x & 7 : 12) << (8 * u);
        }
        uint32_t vw[4][R];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) vw[i][r] = 0;
        auto take = [&](int j0, int n, const vec16 (&rows)[AHEAD][R]) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (j < n) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t lo = __builtin_amdgcn_readlane(sel_lo, 4 * (j0 + j) + i), hi = __builtin_amdgcn_readlane(sel_hi, 4 * (j0 + j) + i);
#pragma unroll
                        for (int r = 0; r < R; ++r)
                            vw[i][r] |= __builtin_amdgcn_perm(rows[j][r].w[1], rows[j][r].w[0], lo) | __builtin_amdgcn_perm(rows[j][r].w[3], rows[j][r].w[2], hi);
                    }
                }
            }
        };
        const int n_from = __popc(from);
        take(0, n_from, raw.v);
        if (n_from > AHEAD) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) from &= from - 1;
            fetch_rows(from, page, raw.v);
            take(AHEAD, n_from - AHEAD, raw.v);
        }
        float xk[16][R], xv[16][R];
#pragma unroll
        for (int t = 0; t < 16; ++t)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                xk[t][r] = (float)(int8_t)(raw.k[t] >> (8 * r));
                xv[t][r] = (float)(int8_t)(vw[t / 4][r] >> (8 * (t & 3)));
            }
        float top_k = open_mine ? 0.f : ak, top_v = open_mine ? 0.f : av;
        if (opens) {
#pragma unroll
            for (int t = 0; t < 16; ++t)
                if (opens >> t & 1) {
                    const int p = __builtin_amdgcn_readlane(pos, t) & 15;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        xk[t][r] = ldf(ko + p * D + R * lane + r);
                        xv[t][r] = ldf(vo + p * D + R * lane + r);
                        top_k = fmaxf(top_k, fabsf(xk[t][r]));
                        top_v = fmaxf(top_v, fabsf(xv[t][r]));
                    }
                }
        }
        // scaled where a product could pass the largest float
        const float fk = kv8_fit(wave_max(top_k)), fv = kv8_fit(wave_max(top_v));
        float mk = 0.f, mv = 0.f;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const float sk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ak * fk), t));
            const float sv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(av * fv), t));
#pragma unroll
            for (int r = 0; r < R; ++r) {
                xk[t][r] *= sk;
                xv[t][r] *= sv;
                mk = fmaxf(mk, fabsf(xk[t][r]));
                mv = fmaxf(mv, fabsf(xv[t][r]));
            }
        }
        // What fmaxf does not keep: a NaN, of a block whose magnitude is one or of the open block.  In a block that is not full no
        // magnitude is asked for, and tokens behind the end (0 times whatever is there) are not stored.
        if (__any(ak != ak)) mk = INFINITY;
        if (__any(av != av)) mv = INFINITY;
        if (opens) {
#pragma unroll
            for (int t = 0; t < 16; ++t)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    mk = fmaxf(mk, kv8_mag(xk[t][r]));
                    mv = fmaxf(mv, kv8_mag(xv[t][r]));
                }
        }
        mk = wave_max(mk);
        mv = wave_max(mv);
        // Complete here: only then are the others let on to store.
#pragma unroll
        for (int t = 0; t < 16; ++t)
#pragma unroll
            for (int r = 0; r < R; ++r) asm volatile("" : "+v"(xk[t][r]), "+v"(xv[t][r]));
        float w_to = w;
        asm volatile("" : "+v"(w_to));
        pos = pos_n;
        page = page_n;
        pos_n = pos_nn;
        if (b0 + EM_WAVES < blocks) fetch(pos, page, raw);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (cnt > 0) {
            const size_t to = (size_t)page_to * n_heads + g;
            if (lane < cnt) kv.w[to * 16 + lane] = w_to;
            if (cnt == 16) {
                if (lane == 0) {
                    kv.amax[to * 2] = kv8_amax(mk) / 127.f / fk;
                    kv.amax[to * 2 + 1] = kv8_amax(mv) / 127.f / fv;
                }
                const float gk = kv8_fit(mk), gv = kv8_fit(mv), wk = mk * gk, wv = mv * gv, rk = 1.f / wk, rv = 1.f / wv;
                if (gk * gv != 1.f) {
#pragma unroll
                    for (int t = 0; t < 16; ++t)
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            xk[t][r] *= gk;
                            xv[t][r] *= gv;
                        }
                }
                int q[R][4];
#pragma unroll
                for (int t = 0; t < 16; t += 4) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float x[4] = {xk[t][r], xk[t + 1][r], xk[t + 2][r], xk[t + 3][r]};
                        kv8_round_n<bf16_t, 4>(x, wk, rk, q[r]);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        int8_t* kp = kv.k + to * 16 * D + (t + j) * D + R * lane;
                        if constexpr (R == 2) *reinterpret_cast<uint16_t*>(kp) = (uint16_t)((q[0][j] & 255) | q[R - 1][j] << 8);
                        else *kp = (int8_t)q[0][j];
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    vec16 o;
#pragma unroll
                    for (int t = 0; t < 16; t += 4) {
                        const float x[4] = {xv[t][r], xv[t + 1][r], xv[t + 2][r], xv[t + 3][r]};
                        kv8_round_n<bf16_t, 4>(x, wv, rv, q[r]);
                        o.w[t / 4] = kv8_pack4(q[r]);
                    }
                    *reinterpret_cast<vec16*>(kv.v + to * 16 * D + (size_t)(R * lane + r) * 16) = o;
                }
            } else {
#pragma unroll
                for (int t = 0; t < 16; ++t)
                    if (t < cnt)
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            stf(ko + t * D + R * lane + r, xk[t][r] / 127.f / fk);
                            stf(vo + t * D + R * lane + r, xv[t][r] / 127.f / fv);
                        }
            }
        }
    }
}

template <typename T, int D>
static void launch_move(const Kv8Layer* layers, int n_heads, const Kv8Evict& e, const int32_t* lists, dim3 grid, hipStream_t s) {
    kv8_move_kernel<T, D><<<grid, 64 * EM_WAVES, 0, s>>>(layers, n_heads, e, lists);
}

hipError_t kv8_evict(int dt, const Kv8Layer* layers, int n_heads, int d, const Kv8Evict& e, int32_t* lists, hipStream_t s) {
    if (e.n_seqs <= 0) return hipSuccess;
    if ((d != 64 && d != 128) || n_heads <= 0 || e.n_layers <= 0 || e.n_layers > 65535 || e.n_seqs > 65535 || !lists || e.recent < 0)
        return hipErrorInvalidValue;
    const dim3 grid(n_heads, e.n_layers, e.n_seqs);
    kv8_select_kernel<<<grid, EV_T, sizeof(uint32_t) * (e.max_len < EV_KEYS ? e.max_len : EV_KEYS), s>>>(layers, n_heads, e, lists);
    SS_TYPED(dt, d, launch_move, (layers, n_heads, e, lists, grid, s));
    return hipGetLastError();
}

}  // namespace SS_NS
