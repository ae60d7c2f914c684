// Decode over the 8-bit cache (cart_cache_decode): one query token per request, keys = [shared segments ; the request's own
// tokens], all visible, codes in blocks of 64 tokens with a scale per block and head.
//
// Codes go from memory to the matrix cores without passing through LDS.  A step is 32 keys of one KV head:
//   S^T (key x query) = K Q^T,  v_mfma_f32_16x16x32_bf16, A = K (lane l: key l%16, 8 dims), B = Q^T (lane l: query l%16)
//   O^T (dim x query) += V^T P^T, A = V^T (lane l: a dim, 8 keys), B = P^T (lane l: query l%16, 8 keys)
// A result tile has lane l holding query l%16 and rows 4 (l/16) + r, r = 0..3: of two score tiles (keys 0..15, 16..31) a lane
// has the 8 keys {4g + r, 16 + 4g + r}, g = l/16, of its query, and those are the 8 contracted keys of lane group g in the
// second product, so P never leaves its lane; V's rows are read in that order.  A lane reads D/16 neighbouring dims of each
// of its 8 rows (whole rows a wavefront, coalesced); byte j of each row makes the operand of the j-th product, whose
// row m is dim (D/16) m + j, and in the end a lane owns D/4 neighbouring dims of its query.  K's dims are taken in whatever
// order 16-byte loads bring them, Q's in the same one.
// Codes become bf16 exactly; the block's K scale goes into the exponent's factor, its V scale onto the weights before they
// are rounded to bf16 (the operand type: 2^-9 of each weight, as in the 16-bit decode; sums, maxima and O are fp32).
#include <math.h>

#include "cache.h"

namespace cart {
using namespace cache;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int STEP = 32;                // keys per step
// A weight may exceed 1 by this power of two before the sums are brought down: the reference is moved when a score passes
// it by so much, not at every new maximum.
constexpr float SLACK = 8.f;

struct DecodeArgs {
    const bf16_t* q;
    const char *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *seg[CART_MAX_SEGMENTS];
    int seg_p[CART_MAX_SEGMENTS], n_seg;
    const int32_t *table, *cu;
    int B, Hq, Hkv, G, max_blocks, max_own, n_blocks;
    float c;                            // softmax scale x log2 e
    bf16_t* o;
    float* lse;
};

// two codes of a word (0: the lower) as bf16
template <int FMT> __device__ __forceinline__ uint32_t two_bf16(uint32_t w, bool upper);
template <> __device__ __forceinline__ uint32_t two_bf16<CART_E4M3>(uint32_t w, bool upper) {
    return __builtin_bit_cast(uint32_t, upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)
                                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
}
// (integers up to 127 in magnitude: fp32's upper half is the bf16)
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
template <> __device__ __forceinline__ uint32_t two_bf16<CART_I8>(uint32_t w, bool upper) {
    return upper ? upper_halves(static_cast<float>(static_cast<int8_t>(w >> 16)), static_cast<float>(static_cast<int8_t>(w >> 24)))
                 : upper_halves(static_cast<float>(static_cast<int8_t>(w)), static_cast<float>(static_cast<int8_t>(w >> 8)));
}

// The codes of a step as they were read.
template <int D> struct Codes {
    u32x4 k[2][D / 64];                 // key 16 t + l%16, bytes 64 i + 16 g
    uint32_t v[8][D / 64];              // key 16 (x/4) + 4 g + x%4, bytes (D/16) (l%16)
    __device__ __forceinline__ void load(const char* kp, const char* vp, int lane) {
        const int g = lane >> 4, c = lane & 15;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) k[t][i] = *reinterpret_cast<const u32x4*>(kp + (16 * t + c) * D + 64 * i + 16 * g);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const char* const p = vp + (16 * (x >> 2) + 4 * g + (x & 3)) * D + (D / 16) * c;
            if constexpr (D == 128) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                v[x][0] = w[0];
                v[x][1] = w[1];
            } else {
                v[x][0] = *reinterpret_cast<const uint32_t*>(p);
            }
        }
    }
    // rows from `valid` on may hold anything: a weight of 0 does not silence a NaN
    __device__ __forceinline__ void clear_v(int valid, int lane) {
        const int g = lane >> 4;
#pragma unroll
        for (int x = 0; x < 8; ++x)
            if (16 * (x >> 2) + 4 * g + (x & 3) >= valid)
#pragma unroll
                for (int i = 0; i < D / 64; ++i) v[x][i] = 0;
    }
};

// N groups of 16 queries against the keys that pass: O, the reference of the softmax (log2 units) and the sum of the lane's
// own keys' weights.
template <int FMT, int D, int N>
struct Rows {
    bf16x8 q[N][D / 32];
    f32x4 o[N][D / 16];
    float m[N], l[N];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // row: the lane's query of group n
    __device__ __forceinline__ void load_q(int n, const bf16_t* row, int lane) {
        const int g = lane >> 4;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            q[n][2 * i] = *reinterpret_cast<const bf16x8*>(row + 64 * i + 16 * g);
            q[n][2 * i + 1] = *reinterpret_cast<const bf16x8*>(row + 64 * i + 16 * g + 8);
        }
    }
    // valid: keys of the step that exist, 1..32
    __device__ __forceinline__ void step(Codes<D>& x, float c, float vs, int valid, int lane) {
        const int g = lane >> 4;
        f32x4 s[N][2];
#pragma unroll
        for (int n = 0; n < N; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int h = 0; h < D / 32; ++h) {
                const uint32_t w0 = x.k[t][h >> 1][2 * (h & 1)], w1 = x.k[t][h >> 1][2 * (h & 1) + 1];
                const u32x4 a = {two_bf16<FMT>(w0, false), two_bf16<FMT>(w0, true), two_bf16<FMT>(w1, false), two_bf16<FMT>(w1, true)};
#pragma unroll
                for (int n = 0; n < N; ++n) s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), q[n][h], s[n][t], 0, 0, 0);
            }
        if (valid < STEP) {
            x.clear_v(valid, lane);
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[n][t][r] = 16 * t + 4 * g + r < valid ? s[n][t][r] * c : -INFINITY;
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int t = 0; t < 2; ++t) s[n][t] *= c;
        }
        bf16x8 p[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float top = fmaxf(fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3])),
                              fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3])));
            if (__any(top > m[n] + SLACK)) {        // (the first step of all: the reference is -inf)
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                top = fmaxf(top, m[n]);
                const float down = fast_exp2(m[n] - top);
                m[n] = top;
                l[n] *= down;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[n][j] *= down;
            }
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = fast_exp2(s[n][i >> 2][i & 3] - m[n]);
                l[n] += w[i];
            }
            const u32x4 b = {pack_bf16x2(w[0] * vs, w[1] * vs), pack_bf16x2(w[2] * vs, w[3] * vs), pack_bf16x2(w[4] * vs, w[5] * vs),
                             pack_bf16x2(w[6] * vs, w[7] * vs)};
            p[n] = __builtin_bit_cast(bf16x8, b);
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const int i = j >> 2, at = j & 3;
            u32x4 a;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const uint32_t w0 = x.v[2 * y][i], w1 = x.v[2 * y + 1][i];
                if constexpr (FMT == CART_E4M3) {
                    // bytes 0 and 1 of both rows next to each other, or 2 and 3
                    const uint32_t both = __builtin_amdgcn_perm(w1, w0, at < 2 ? 0x05010400u : 0x07030602u);
                    a[y] = two_bf16<FMT>(both, at & 1);
                } else {
                    a[y] = upper_halves(static_cast<float>(static_cast<int8_t>(w0 >> (8 * at))), static_cast<float>(static_cast<int8_t>(w1 >> (8 * at))));
                }
            }
#pragma unroll
            for (int n = 0; n < N; ++n) o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), p[n], o[n][j], 0, 0, 0);
        }
    }
};

// A workgroup per (request, KV head); its four wavefronts take the steps in turn and join their results in LDS.
template <int FMT, int D, int N>
__global__ __launch_bounds__(256) void cache_decode_kernel(const DecodeArgs a) {
    __shared__ __align__(16) float part_o[4][16 * N][D];
    __shared__ float part_m[4][16 * N], part_l[4][16 * N];
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int id = workgroup_id();
    const int b = id / a.Hkv, hk = id % a.Hkv;
    if (b >= a.B) return;
    const size_t row0 = static_cast<size_t>(b) * a.Hq + hk * a.G;

    Rows<FMT, D, N> rows;
    rows.clear();
#pragma unroll
    for (int n = 0; n < N; ++n) rows.load_q(n, a.q + (row0 + min(16 * n + col, a.G - 1)) * D, lane);

    auto run = [&](const int32_t* blocks, int n_keys) {
        for (int s = wv; s * STEP < n_keys; s += 4) {
            const int blk = blocks[s >> 1];
            if (blk < 0 || blk >= a.n_blocks) continue;
            const size_t at = static_cast<size_t>(blk) * a.Hkv + hk;
            Codes<D> x;
            x.load(a.k + at * (BLOCK * D) + (s & 1) * (STEP * D), a.v + at * (BLOCK * D) + (s & 1) * (STEP * D), lane);
            rows.step(x, a.c * a.k_scale[at], a.v_scale[at], min(STEP, n_keys - s * STEP), lane);
        }
    };
    for (int s = 0; s < a.n_seg; ++s) run(a.seg[s], a.seg_p[s]);
    if (a.max_own > 0) {
        const int n = a.cu[b + 1] - a.cu[b];
        run(a.table + static_cast<size_t>(b) * a.max_blocks, min(n, a.max_own));
    }

#pragma unroll
    for (int n = 0; n < N; ++n) {
        float l = rows.l[n];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) {
            part_m[wv][16 * n + col] = rows.m[n];
            part_l[wv][16 * n + col] = l;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) part_o[wv][16 * n + col][(D / 16) * (4 * g + r) + j] = rows.o[n][j][r];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.G * (D / 4); i += 256) {
        const int h = i / (D / 4), d = i % (D / 4) * 4;
        float m = part_m[0][h];
        for (int w = 1; w < 4; ++w) m = fmaxf(m, part_m[w][h]);
        float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < 4; ++w) {
            const float f = part_m[w][h] == -INFINITY ? 0.f : fast_exp2(part_m[w][h] - m);
            l += f * part_l[w][h];
            for (int e = 0; e < 4; ++e) o[e] += f * part_o[w][h][d + e];
        }
        const float inv = l != 0.f ? 1.f / l : 0.f;
        const u32x2 out = {pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
        *reinterpret_cast<u32x2*>(a.o + (row0 + h) * D + d) = out;
        if (a.lse && d == 0) a.lse[row0 + h] = l != 0.f ? (m + fast_log2(l)) * CART_LN2 : -INFINITY;
    }
}

template <int FMT, int D>
void launch(const DecodeArgs& a, hipStream_t st) {
    const dim3 grid = grid_of(static_cast<long>(a.B) * a.Hkv);
    if (a.G <= 16) cache_decode_kernel<FMT, D, 1><<<grid, 256, 0, st>>>(a);
    else cache_decode_kernel<FMT, D, 2><<<grid, 256, 0, st>>>(a);
}

}  // namespace

size_t cache_decode_workspace(const cart_cache_decode_desc&, const cart_cache&, const cart_cache_segment*) { return 0; }

int launch_cache_decode(const cart_cache_decode_desc& d, const cart_cache& c, float scale, const void* q,
                        const cart_cache_segment* shared, const int32_t* table, const int32_t* cu, void* o, float* lse, void*,
                        hipStream_t st) {
    DecodeArgs a = {};
    a.q = static_cast<const bf16_t*>(q);
    a.k = static_cast<const char*>(c.k); a.v = static_cast<const char*>(c.v);
    a.k_scale = c.k_scale; a.v_scale = c.v_scale;
    for (int s = 0; s < d.n_shared; ++s) {
        if (shared[s].p == 0) continue;
        a.seg[a.n_seg] = shared[s].blocks;
        a.seg_p[a.n_seg++] = shared[s].p;
    }
    a.table = table; a.cu = cu;
    a.B = d.B; a.Hq = d.Hq; a.Hkv = c.Hkv; a.G = d.Hq / c.Hkv;
    a.max_blocks = d.max_blocks; a.max_own = d.max_own_len; a.n_blocks = c.n_blocks;
    a.c = scale * CART_LOG2E;
    a.o = static_cast<bf16_t*>(o); a.lse = lse;
    if (c.D == 64) {
        if (c.format == CART_I8) launch<CART_I8, 64>(a, st);
        else launch<CART_E4M3, 64>(a, st);
    } else {
        if (c.format == CART_I8) launch<CART_I8, 128>(a, st);
        else launch<CART_E4M3, 128>(a, st);
    }
    return static_cast<int>(hipGetLastError());
}

}  // namespace cart
