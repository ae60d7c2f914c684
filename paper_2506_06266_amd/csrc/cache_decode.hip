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
constexpr int MIN_RANGE = 2;            // fewest steps of a range

struct DecodeArgs {
    const bf16_t* q;
    const char *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *seg[CART_MAX_SEGMENTS];
    int seg_p[CART_MAX_SEGMENTS], seg_s0[CART_MAX_SEGMENTS + 1], n_seg;     // seg_s0: steps before each segment, and of all
    const int32_t *table, *cu;
    int B, Hq, Hkv, G, max_blocks, max_own, n_blocks;
    float c;                            // softmax scale x log2 e
    bf16_t* o;
    float* lse;
    // the split form: row blocks and parts of the shared segments, workgroups of that role, ranges of the own tokens per KV
    // head, where the partial results go (O as summed, {reference, sum of weights})
    int n_rb, n_parts, n_shared_wg, n_ranges;
    float *shared_o, *own_o;
    float2 *shared_ml, *own_ml;
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

// The codes of a step as they were read.  Through buffer descriptors of the step's rows: what lies behind them -- rows that do
// not exist, or no step at all -- reads as 0 and costs no memory traffic, so the loads of the steps ahead need no branch.
template <int D> struct Codes {
    u32x4 k[2][D / 64];                 // key 16 t + l%16, bytes 64 i + 16 g
    uint32_t v[8][D / 64];              // key 16 (x/4) + 4 g + x%4, bytes (D/16) (l%16)
    __device__ __forceinline__ void load(const char* kp, const char* vp, int n_rows, int lane) {
        const int g = lane >> 4, c = lane & 15;
        const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kp), 0, n_rows * D, 0x20000);
        const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vp), 0, n_rows * D, 0x20000);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) k[t][i] = __builtin_amdgcn_raw_buffer_load_b128(kb, (16 * t + c) * D + 64 * i + 16 * g, 0, 0);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int at = (16 * (x >> 2) + 4 * g + (x & 3)) * D + (D / 16) * c;
            if constexpr (D == 128) {
                const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(vb, at, 0, 0);
                v[x][0] = w[0];
                v[x][1] = w[1];
            } else {
                v[x][0] = __builtin_amdgcn_raw_buffer_load_b32(vb, at, 0, 0);
            }
        }
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
    // the sum of all keys' weights of the lane's query
    __device__ __forceinline__ float sum(int n) const {
        const float s = l[n] + __shfl_xor(l[n], 16);
        return s + __shfl_xor(s, 32);
    }
    // c: softmax scale x log2 e x K scale; lv: log2 of the V scale, which goes into the weights' exponent (a factor of each block
    // that the sum of weights is freed of again); valid: keys of the step that exist, 1..32
    __device__ __forceinline__ void step(const Codes<D>& x, float c, float lv, int valid, int lane) {
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
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[n][t][r] = 16 * t + 4 * g + r < valid ? s[n][t][r] : -INFINITY;
        }
        if (lv != lv) {                             // a V scale of NaN is O's, not the weights'
            lv = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[n][j] += __uint_as_float(0x7fc00000u);
        }
        const float unscale = fast_exp2(-lv);
        bf16x8 p[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float top = c * fmaxf(fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3])),
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
            const float shift = lv - m[n];
            float w[8], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = fast_exp2(fmaf(s[n][i >> 2][i & 3], c, shift));
                sum += w[i];
            }
            l[n] = fmaf(sum, unscale, l[n]);
            const u32x4 b = {pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])};
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

// Up to 64 steps in the order they are taken, one a lane.
struct Steps {
    int id = -1;                        // block (-1: none of the pool)
    int rows = 0, half = 0;             // keys that exist (0: there is no such step); the upper half of the block
    int request = 0;
    float c = 0.f, lv = 0.f;            // factors of the block: see Rows::step

    __device__ __forceinline__ void of_block(const DecodeArgs& a, int hk, int block, int local, int n_keys) {
        rows = min(STEP, n_keys - local * STEP);
        half = local & 1;
        if (block < 0 || block >= a.n_blocks) return;
        id = block;
        const size_t at = static_cast<size_t>(block) * a.Hkv + hk;
        c = a.c * a.k_scale[at];
        lv = fast_log2(a.v_scale[at]);
    }
    // step s of the shared segments, one after the other
    __device__ __forceinline__ void of_segments(const DecodeArgs& a, int hk, int s) {
        int i = 0;
        for (int k = 1; k < a.n_seg; ++k) i = s >= a.seg_s0[k] ? k : i;
        const int local = s - a.seg_s0[i];
        of_block(a, hk, a.seg[i][local >> 1], local, a.seg_p[i]);
    }
    // step `local` of request b's n own tokens
    __device__ __forceinline__ void of_request(const DecodeArgs& a, int hk, int b, int local, int n) {
        request = b;
        if (local >= 0 && local * STEP < n) of_block(a, hk, a.table[static_cast<size_t>(b) * a.max_blocks + (local >> 1)], local, n);
    }
};
__device__ __forceinline__ float lane_of(float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); }
__device__ __forceinline__ int lane_of(int x, int i) { return __builtin_amdgcn_readlane(x, i); }

__device__ __forceinline__ int own_len(const DecodeArgs& a, int c0, int c1) { return min(max(c1 - c0, 0), a.max_own); }

// Takes steps 0 .. n-1 of the list, DEPTH of them in flight.  begin(request): called where the request changes.
template <int FMT, int D, int N, int DEPTH, bool MANY, typename F>
__device__ __forceinline__ void run(const DecodeArgs& a, const Steps& st, int n, int hk, Rows<FMT, D, N>& rows, int& current, F&& begin, int lane) {
    if (n <= 0) return;
    Codes<D> x[DEPTH];
    auto load = [&](Codes<D>& y, int i) __attribute__((always_inline)) {
        const int at = min(i, n - 1), id = lane_of(st.id, at);
        const size_t block = (static_cast<size_t>(max(id, 0)) * a.Hkv + hk) * (BLOCK * D) + lane_of(st.half, at) * (STEP * D);
        y.load(a.k + block, a.v + block, i < n && id >= 0 ? lane_of(st.rows, at) : 0, lane);
    };
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) load(x[j], j);
    for (int i = 0; i < n; i += DEPTH) {
#pragma unroll
        for (int j = 0; j < DEPTH; ++j) {
            const int at = min(i + j, n - 1), n_rows = i + j < n ? lane_of(st.rows, at) : 0;
            if (n_rows > 0) {
                if constexpr (MANY) {
                    const int request = lane_of(st.request, at);
                    if (request != current) {
                        begin(request);
                        current = request;
                    }
                }
                if (lane_of(st.id, at) >= 0) rows.step(x[j], lane_of(st.c, at), lane_of(st.lv, at), n_rows, lane);
            }
            load(x[j], i + j + DEPTH);
        }
    }
}

// The results of a workgroup's W wavefronts for the same queries, joined in LDS.
template <int D, int N, int W> struct Join {
    float o[W][16 * N][D];
    float m[W][16 * N], l[W][16 * N];

    template <int FMT>
    __device__ __forceinline__ void put(int w, const Rows<FMT, D, N>& rows, int lane) {
        const int g = lane >> 4, col = lane & 15;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float sum = rows.sum(n);
            if (g == 0) {
                m[w][16 * n + col] = rows.m[n];
                l[w][16 * n + col] = sum;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[w][16 * n + col][(D / 16) * (4 * g + r) + j] = rows.o[n][j][r];
        }
    }
    // dims d .. d+3 of query h of all wavefronts
    __device__ __forceinline__ void get(int h, int d, float (&x)[4], float& ref, float& sum) const {
        ref = m[0][h];
#pragma unroll
        for (int w = 1; w < W; ++w) ref = fmaxf(ref, m[w][h]);
        sum = x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = l[w][h] == 0.f ? 0.f : fast_exp2(m[w][h] - ref);
            sum += f * l[w][h];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += f * o[w][h][d + e];
        }
    }
};

// a finished query's output: D / 4 lanes a row
__device__ __forceinline__ void finish(const DecodeArgs& a, size_t row, int D, int d, const float (&x)[4], float ref, float sum) {
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const u32x2 out = {pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
    *reinterpret_cast<u32x2*>(a.o + row * D + d) = out;
    if (a.lse && d == 0) a.lse[row] = sum != 0.f ? (ref + fast_log2(sum)) * CART_LN2 : -INFINITY;
}

// ---- one launch: a workgroup per (request, KV head), its W wavefronts each take a part of the steps
template <int FMT, int D, int N, int W, int DEPTH>
__global__ __launch_bounds__(64 * W) void cache_decode_one_kernel(const DecodeArgs a) {
    __shared__ Join<D, N, W> join;
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int id = workgroup_id();
    const int b = id / a.Hkv, hk = id % a.Hkv;
    if (b >= a.B) return;
    const size_t row0 = static_cast<size_t>(b) * a.Hq + hk * a.G;

    Rows<FMT, D, N> rows;
    rows.clear();
#pragma unroll
    for (int n = 0; n < N; ++n) rows.load_q(n, a.q + (row0 + min(16 * n + (lane & 15), a.G - 1)) * D, lane);
    const int n_own = a.max_own > 0 ? own_len(a, a.cu[b], a.cu[b + 1]) : 0;
    const int n_shared = a.seg_s0[a.n_seg], total = n_shared + (n_own + STEP - 1) / STEP;
    const int each = (total + W - 1) / W, s0 = wv * each, s1 = min(total, s0 + each);
    int current = 0;
    for (int s = s0; s < s1; s += 64) {
        const int n = min(64, s1 - s);
        Steps st;
        if (lane < n) {
            if (s + lane < n_shared) st.of_segments(a, hk, s + lane);
            else st.of_request(a, hk, b, s + lane - n_shared, n_own);
        }
        run<FMT, D, N, DEPTH, false>(a, st, n, hk, rows, current, [](int) {}, lane);
    }
    join.put(wv, rows, lane);
    __syncthreads();
    for (int i = threadIdx.x; i < a.G * (D / 4); i += 64 * W) {
        const int h = i / (D / 4), d = i % (D / 4) * 4;
        float x[4], ref, sum;
        join.get(h, d, x, ref, sum);
        finish(a, row0 + h, D, d, x, ref, sum);
    }
}

// ---- split: the shared segments and the requests' own tokens in one launch, partial results, a second launch that joins them
//
// Shared role: a workgroup takes 16 NS of the B G query rows that read one KV head and one part of the segments' steps, its four
// wavefronts a quarter of it each.  Own role: the axis of all requests' steps (request b from cu[b] / 32 + b on: one place to spare
// each makes it a function of its own offset) is cut into equal ranges, whatever the requests' lengths; a wavefront takes a
// range of one KV head.  Range r leaves the partial result of request b in slot r + b: pairs of neighbours never share one.
__device__ __forceinline__ int range_len(const DecodeArgs& a) {
    const int places = (a.cu[a.B] >> 5) + a.B;
    return max((max(places, 1) + a.n_ranges - 1) / a.n_ranges, MIN_RANGE);
}

template <int FMT, int D, int NS, int NO, int DEPTH>
__global__ __launch_bounds__(256, 2) void cache_decode_parts_kernel(const DecodeArgs a) {
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int id = workgroup_id();
    if (id < a.n_shared_wg) {
        __shared__ Join<D, NS, 4> join;
        const int hk = id % a.Hkv; id /= a.Hkv;
        const int rb = id % a.n_rb, part = id / a.n_rb;
        const int n_rows = a.B * a.G;
        Rows<FMT, D, NS> rows;
        rows.clear();
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const int r = min(rb * 16 * NS + 16 * n + col, n_rows - 1);
            rows.load_q(n, a.q + (static_cast<size_t>(r / a.G) * a.Hq + hk * a.G + r % a.G) * D, lane);
        }
        const int total = a.seg_s0[a.n_seg];
        const int p0 = static_cast<int>(static_cast<long>(total) * part / a.n_parts), p1 = static_cast<int>(static_cast<long>(total) * (part + 1) / a.n_parts);
        const int s0 = p0 + (p1 - p0) * wv / 4, s1 = p0 + (p1 - p0) * (wv + 1) / 4;
        int current = 0;
        for (int s = s0; s < s1; s += 64) {
            const int n = min(64, s1 - s);
            Steps st;
            if (lane < n) st.of_segments(a, hk, s + lane);
            run<FMT, D, NS, DEPTH, false>(a, st, n, hk, rows, current, [](int) {}, lane);
        }
        join.put(wv, rows, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * NS * (D / 4); i += 256) {
            const int h = i / (D / 4), d = i % (D / 4) * 4, r = rb * 16 * NS + h;
            if (r >= n_rows) break;
            float x[4], ref, sum;
            join.get(h, d, x, ref, sum);
            const size_t at = static_cast<size_t>(part) * a.B * a.Hq + static_cast<size_t>(r / a.G) * a.Hq + hk * a.G + r % a.G;
            *reinterpret_cast<float4*>(a.shared_o + at * D + d) = float4{x[0], x[1], x[2], x[3]};
            if (d == 0) a.shared_ml[at] = float2{ref, sum};
        }
        return;
    }
    const long w = static_cast<long>(id - a.n_shared_wg) * 4 + wv;
    const int hk = static_cast<int>(w % a.Hkv), range = static_cast<int>(w / a.Hkv);
    if (range >= a.n_ranges) return;
    const int len = range_len(a), places = (a.cu[a.B] >> 5) + a.B;
    const long from = static_cast<long>(range) * len;
    if (from >= places) return;
    const int to = static_cast<int>(min(from + len, static_cast<long>(places)));

    Rows<FMT, D, NO> rows;
    rows.clear();
    int current = -1;
    auto flush = [&](int b) __attribute__((always_inline)) {
        const int c0 = a.cu[b], steps = (own_len(a, c0, a.cu[b + 1]) + STEP - 1) / STEP, p0 = (c0 >> 5) + b;
        const bool whole = a.n_parts == 0 && p0 >= from && p0 + steps <= to;        // nothing to join
#pragma unroll
        for (int n = 0; n < NO; ++n) {
            const float sum = rows.sum(n);
            const int h = 16 * n + col;
            if (h >= a.G) continue;
            if (whole) {
                const size_t row = static_cast<size_t>(b) * a.Hq + hk * a.G + h;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < D / 16; j += 4) {
                        const float x[4] = {rows.o[n][j][r], rows.o[n][j + 1][r], rows.o[n][j + 2][r], rows.o[n][j + 3][r]};
                        finish(a, row, D, (D / 16) * (4 * g + r) + j, x, rows.m[n], sum);
                    }
            } else {
                const size_t at = (static_cast<size_t>(range + b) * a.Hkv + hk) * a.G + h;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < D / 16; j += 4)
                        *reinterpret_cast<float4*>(a.own_o + at * D + (D / 16) * (4 * g + r) + j) =
                            float4{rows.o[n][j][r], rows.o[n][j + 1][r], rows.o[n][j + 2][r], rows.o[n][j + 3][r]};
                if (g == 0) a.own_ml[at] = float2{rows.m[n], sum};
            }
        }
    };
    auto begin = [&](int b) __attribute__((always_inline)) {
        if (current >= 0) {
            flush(current);
            rows.clear();
        }
#pragma unroll
        for (int n = 0; n < NO; ++n) rows.load_q(n, a.q + (static_cast<size_t>(b) * a.Hq + hk * a.G + min(16 * n + col, a.G - 1)) * D, lane);
    };
    for (int p = static_cast<int>(from); p < to; p += 64) {
        const int n = min(64, to - p);
        const int b0 = request_of(a.cu, a.B, 0x7fffffff, 5, 1, p, lane);
        // the requests of these places: lane k looks at b0 + k, and a lane's place belongs to the last one that begins there or before
        const int bk = min(b0 + lane, a.B - 1), c0 = offset_at(a.cu, bk, 0x7fffffff), c1 = offset_at(a.cu, bk + 1, 0x7fffffff);
        const long start = static_cast<long>(c0 >> 5) + bk - p;
        uint64_t begins = lane > 0 && b0 + lane < a.B && start > 0 && start < 64 ? 1ull << start : 0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint32_t lo = static_cast<uint32_t>(__shfl_xor(static_cast<int>(begins), o)), hi = static_cast<uint32_t>(__shfl_xor(static_cast<int>(begins >> 32), o));
            begins |= static_cast<uint64_t>(hi) << 32 | lo;
        }
        const int k = __builtin_popcountll(begins & ((2ull << lane) - 1));
        const int r0 = __shfl(c0, k), r1 = __shfl(c1, k), b = b0 + k;
        Steps st;
        if (lane < n) st.of_request(a, hk, b, p + lane - (r0 >> 5) - b, own_len(a, r0, r1));
        run<FMT, D, NO, DEPTH, true>(a, st, n, hk, rows, current, begin, lane);
    }
    if (current >= 0) flush(current);
}

// joins the partial results of a query: D / 4 lanes each
template <int D>
__global__ __launch_bounds__(256) void cache_decode_join_kernel(const DecodeArgs a) {
    constexpr int LANES = D / 4;
    const long row = static_cast<long>(workgroup_id()) * (256 / LANES) + threadIdx.x / LANES;
    if (row >= static_cast<long>(a.B) * a.Hq) return;
    const int d = threadIdx.x % LANES * 4;
    const int b = static_cast<int>(row / a.Hq), h = static_cast<int>(row % a.Hq), hk = h / a.G;
    int r0 = 0, n_own = 0;
    if (a.n_ranges > 0) {
        const int c0 = a.cu[b], steps = (own_len(a, c0, a.cu[b + 1]) + STEP - 1) / STEP, p0 = (max(c0, 0) >> 5) + b, len = range_len(a);
        if (steps > 0) {
            r0 = min(p0 / len, a.n_ranges - 1);
            n_own = min((p0 + steps - 1) / len, a.n_ranges - 1) - r0 + 1;
        }
        if (a.n_parts == 0 && n_own == 1) return;           // the range that holds the whole request has finished it
    }
    const size_t all = static_cast<size_t>(a.B) * a.Hq;
    auto ml = [&](int i) { return i < a.n_parts ? a.shared_ml[i * all + row] : a.own_ml[(static_cast<size_t>(r0 + i - a.n_parts + b) * a.Hkv + hk) * a.G + h % a.G]; };
    auto part = [&](int i) {
        const float* p = i < a.n_parts ? a.shared_o + (i * all + row) * D : a.own_o + ((static_cast<size_t>(r0 + i - a.n_parts + b) * a.Hkv + hk) * a.G + h % a.G) * D;
        return *reinterpret_cast<const float4*>(p + d);
    };
    const int n = a.n_parts + n_own;
    float ref = -INFINITY, sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; ++i) ref = fmaxf(ref, ml(i).x);
    for (int i = 0; i < n; ++i) {
        const float2 s = ml(i);
        const float4 y = part(i);
        const float f = s.y == 0.f ? 0.f : fast_exp2(s.x - ref);
        sum += f * s.y;
        x[0] += f * y.x; x[1] += f * y.y; x[2] += f * y.z; x[3] += f * y.w;
    }
    finish(a, static_cast<size_t>(row), D, d, x, ref, sum);
}

struct Plan {
    bool split;
    int n_rb, n_parts, n_shared_wg, n_ranges;
    size_t shared_rows, own_rows;       // partial results
};
int steps_of(const cart_cache_decode_desc& d, const cart_cache_segment* shared) {
    long n = 0;
    for (int s = 0; s < d.n_shared; ++s) n += (shared[s].p + STEP - 1) / STEP;
    return static_cast<int>(n);
}
#ifndef CACHE_FORM
#define CACHE_FORM -1
#endif
Plan plan_of(const cart_cache_decode_desc& d, const cart_cache& c, const cart_cache_segment* shared) {
    Plan p = {};
    const int G = d.Hq / c.Hkv, cus = device_cus(), steps = steps_of(d, shared);
    const long rows = static_cast<long>(d.B) * G;
    const int per = rows > 16 ? 32 : 16;
    p.split = CACHE_FORM != 0;
    if (steps > 0) {
        p.n_rb = static_cast<int>((rows + per - 1) / per);
        const long one = static_cast<long>(p.n_rb) * c.Hkv;
        const long want = (cus + one - 1) / one, most = (steps + 3) / 4;
        p.n_parts = static_cast<int>(want < most ? want : most);
        p.n_shared_wg = static_cast<int>(one * p.n_parts);
    }
    if (d.max_own_len > 0) {
        const long room = 2L * cus - p.n_shared_wg, waves = 4 * (room > cus / 2 ? room : cus / 2);
        const long places = static_cast<long>(d.B) * ((d.max_own_len + STEP - 1) / STEP + 1);
        long r = waves / c.Hkv;
        r = r < 1 ? 1 : r > places ? places : r;
        p.n_ranges = static_cast<int>(r);
    }
    p.shared_rows = static_cast<size_t>(p.n_parts) * d.B * d.Hq;
    p.own_rows = p.n_ranges ? static_cast<size_t>(p.n_ranges + d.B) * d.Hq : 0;
    return p;
}

template <int FMT, int D>
void launch(const DecodeArgs& a, const Plan& p, hipStream_t st) {
    const long pairs = static_cast<long>(a.B) * a.Hkv;
    if (!p.split) {
        if (a.G <= 16) cache_decode_one_kernel<FMT, D, 1, 4, 2><<<grid_of(pairs), 256, 0, st>>>(a);
        else cache_decode_one_kernel<FMT, D, 2, 4, 2><<<grid_of(pairs), 256, 0, st>>>(a);
        return;
    }
    const long wgs = p.n_shared_wg + (static_cast<long>(p.n_ranges) * a.Hkv + 3) / 4;
    const dim3 grid = grid_of(wgs);
    if (wgs == 0) {}                                        // no key at all: the join writes what there is to write
    else if (a.G > 16) cache_decode_parts_kernel<FMT, D, 2, 2, 2><<<grid, 256, 0, st>>>(a);
    else if (static_cast<long>(a.B) * a.G > 16) cache_decode_parts_kernel<FMT, D, 2, 1, 2><<<grid, 256, 0, st>>>(a);
    else cache_decode_parts_kernel<FMT, D, 1, 1, 2><<<grid, 256, 0, st>>>(a);
    cache_decode_join_kernel<D><<<grid_of((static_cast<long>(a.B) * a.Hq + 1024 / D - 1) / (1024 / D)), 256, 0, st>>>(a);
}

}  // namespace

size_t cache_decode_workspace(const cart_cache_decode_desc& d, const cart_cache& c, const cart_cache_segment* shared) {
    const Plan p = plan_of(d, c, shared);
    return p.split ? (p.shared_rows + p.own_rows) * (c.D + 2) * sizeof(float) + 64 : 0;
}

int launch_cache_decode(const cart_cache_decode_desc& d, const cart_cache& c, float scale, const void* q,
                        const cart_cache_segment* shared, const int32_t* table, const int32_t* cu, void* o, float* lse, void* ws,
                        hipStream_t st) {
    const Plan p = plan_of(d, c, shared);
    DecodeArgs a = {};
    a.q = static_cast<const bf16_t*>(q);
    a.k = static_cast<const char*>(c.k); a.v = static_cast<const char*>(c.v);
    a.k_scale = c.k_scale; a.v_scale = c.v_scale;
    for (int s = 0; s < d.n_shared; ++s) {
        if (shared[s].p == 0) continue;
        a.seg[a.n_seg] = shared[s].blocks;
        a.seg_p[a.n_seg] = shared[s].p;
        a.seg_s0[a.n_seg + 1] = a.seg_s0[a.n_seg] + (shared[s].p + STEP - 1) / STEP;
        ++a.n_seg;
    }
    a.table = table; a.cu = cu;
    a.B = d.B; a.Hq = d.Hq; a.Hkv = c.Hkv; a.G = d.Hq / c.Hkv;
    a.max_blocks = d.max_blocks; a.max_own = d.max_own_len; a.n_blocks = c.n_blocks;
    a.c = scale * CART_LOG2E;
    a.o = static_cast<bf16_t*>(o); a.lse = lse;
    a.n_rb = p.n_rb; a.n_parts = p.n_parts; a.n_shared_wg = p.n_shared_wg; a.n_ranges = p.n_ranges;
    // O first: its rows are multiples of 16 bytes
    a.shared_o = static_cast<float*>(ws);
    a.own_o = a.shared_o + p.shared_rows * c.D;
    a.shared_ml = reinterpret_cast<float2*>(a.own_o + p.own_rows * c.D);
    a.own_ml = a.shared_ml + p.shared_rows;
    if (c.D == 64) {
        if (c.format == CART_I8) launch<CART_I8, 64>(a, p, st);
        else launch<CART_E4M3, 64>(a, p, st);
    } else {
        if (c.format == CART_I8) launch<CART_I8, 128>(a, p, st);
        else launch<CART_E4M3, 128>(a, p, st);
    }
    return static_cast<int>(hipGetLastError());
}

}  // namespace cart
