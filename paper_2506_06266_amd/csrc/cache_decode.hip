// Decode over the 8-bit cache (cart_cache_decode): one query token per request, keys = [shared segments ; the request's own
// tokens], all visible, codes in blocks of 64 tokens with a scale per block and head.
//
// A step is 32 keys of one KV head against Q = 16 or 32 queries, by v_mfma_f32_16x16x32_bf16 or v_mfma_f32_32x32x16_bf16:
//   S^T (key x query) = K Q^T      A = K   (lane l: key l%Q, 8 dims)    B = Q^T (lane l: query l%Q)
//   O^T (dim x query) += V^T P^T   A = V^T (lane l: a dim, 8 keys)      B = P^T (lane l: query l%Q, 8 keys)
// A result tile has lane l holding query l%Q and, with g = l/Q, rows 4g + r (16) or 8x + 4g + r (32), r = 0..3.  So a lane's score
// entries 0..7 (and 8..15 with 32) are 8 keys of its query, and those are the 8 contracted keys of its lane group in a second
// product: P never leaves its lane, and V's rows are read in that order.  A lane reads D/Q neighbouring dims of each of its
// rows (whole rows a wavefront, coalesced); byte j of 8 rows makes the operand of product j, whose row m is dim
// (D/Q) m + j.  K's dims are taken in whatever order 16-byte pieces bring them, Q's in the same one.
// The larger shape keeps the vector ALU waiting for less of its length (an MFMA holds it off for 12 to 20 clocks of its 32, or most of its
// 16), so 32 queries take it where there are more than 16.
// Codes become bf16 exactly; the block's K scale goes into the exponent's factor, its V scale into the exponent.  The weights are
// rounded to bf16, the second product's operand type (2^-9 of each, as in the 16-bit decode); sums, references and O are fp32.
#include <float.h>
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "cache.h"

namespace cart {
using namespace cache;

// How a call is cut (host only: the planner is tested without a GPU)
struct CachePlan {
    int n_rb, n_parts, n_ranges;        // the segments by their own (n_cuts == 0)
    int n_cuts, cut;                    // every (request, KV head) by itself
    long n_shared_wg, n_wg;
    long slots;                         // partial results of Hq rows
};
CachePlan cache_decode_plan(const cart_cache_decode_desc& d, const cart_cache& c, const cart_cache_segment* shared);

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int STEP = 32;                // keys per step
// The softmax's reference is the largest score of a query's first step; it is moved where the weights of a later step add up to
// more than this in a lane (fp32 and bf16 have room for far more; no maximum is formed otherwise).
constexpr float LIMIT = 65536.f;
// Own tokens' bytes, half the lengths' bound, from which the codes are read non-temporal: a model's layers have a cache each, and
// what eight of them read is no longer in the memory-side cache (256 MB) when the next token comes.  us with and without, the cache not
// read shortly before / read by the call before: 17 MB 9.5 10.4 / 8.4 7.7, 69 MB 17.9 19.8 / 16.0 16.8, 138 MB 29.5 33.2 / 27.5 26.6,
// 1074 MB 164 185; beside 8192 common slots, which stay in the L2 for it, 128 requests of up to 1024 tokens 48.6 52.1.
constexpr double NT_BYTES = 32e6;
constexpr int FEW_ROWS = 2048;          // output rows up to which the join takes four wavefronts a row

struct Sums;
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
    int n_rb, n_parts, n_ranges, n_cuts, cut;       // see the kernels; partial results: [slot][Hq]
    long n_shared_wg;
    float *part_o;
    Sums *part_sums;
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

// 8 codes of a row as an operand
template <int FMT> __device__ __forceinline__ u32x4 eight_of_row(uint32_t w0, uint32_t w1) {
    return u32x4{two_bf16<FMT>(w0, false), two_bf16<FMT>(w0, true), two_bf16<FMT>(w1, false), two_bf16<FMT>(w1, true)};
}
// byte j of two rows as bf16, the first row's below
template <int FMT> __device__ __forceinline__ uint32_t two_rows(uint32_t w0, uint32_t w1, int j) {
    // (bytes 0 and 1 of both rows next to each other, or 2 and 3: one permutation serves two j)
    if constexpr (FMT == CART_E4M3) return two_bf16<FMT>(__builtin_amdgcn_perm(w1, w0, j < 2 ? 0x05010400u : 0x07030602u), j & 1);
    else return upper_halves(static_cast<float>(static_cast<int8_t>(w0 >> (8 * j))), static_cast<float>(static_cast<int8_t>(w1 >> (8 * j))));
}

// The codes of a step as they were read.  Through buffer descriptors of the step's rows: what lies behind them -- rows that do
// not exist, or no step at all -- reads as 0 and costs no memory traffic, so the loads of the steps ahead need no branch.
template <int D, int Q> struct Codes {
    static constexpr int CHUNKS = D / 16, PER = 64 / CHUNKS;    // 16-byte pieces of a row, rows a load of K brings
    static constexpr int BYTES = D / Q, OWN = Q / 2;            // of a row of V, and rows, that a lane reads
    u32x4 k[STEP / PER];                // key PER x + l/CHUNKS, piece l%CHUNKS: whole rows, as they lie in memory
    uint32_t v[OWN][BYTES > 4 ? 2 : 1]; // key of(x, g), bytes BYTES (l%Q)
    static __device__ __forceinline__ int of(int x, int g) { return (x >> 2) * (Q == 16 ? 16 : 8) + 4 * g + (x & 3); }
    // AUX: 2 for non-temporal
    template <int AUX>
    __device__ __forceinline__ void load(const char* kp, const char* vp, int n_rows, int lane) {
        const int g = lane / Q, c = lane % Q;
        const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kp), 0, n_rows * D, 0x20000);
        const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vp), 0, n_rows * D, 0x20000);
#pragma unroll
        for (int x = 0; x < STEP / PER; ++x) k[x] = __builtin_amdgcn_raw_buffer_load_b128(kb, x * PER * D + 16 * lane, 0, AUX);
#pragma unroll
        for (int x = 0; x < OWN; ++x) {
            const int at = of(x, g) * D + BYTES * c;
            if constexpr (BYTES == 8) {
                const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(vb, at, 0, AUX);
                v[x][0] = w[0];
                v[x][1] = w[1];
            } else if constexpr (BYTES == 4) {
                v[x][0] = __builtin_amdgcn_raw_buffer_load_b32(vb, at, 0, AUX);
            } else {
                v[x][0] = __builtin_amdgcn_raw_buffer_load_b16(vb, at, 0, AUX);
            }
        }
    }
};

// K's way from whole rows to matrix operands: a wavefront's own 32 rows in LDS.  (Loaded as operands, 16 lanes next to each other
// touch 16 rows, and the address path is busy for longer: 5 to 18 % of a call.)  Piece c of row r lies at c ^ f(r), so that both the
// 16 lanes that write one or several whole rows and the 16 that read one piece of 16 rows cover all banks.
template <int D> struct Keys {
    static constexpr int CHUNKS = D / 16, PER = 64 / CHUNKS;
    u32x4 piece[STEP * CHUNKS];
    static __device__ __forceinline__ int at(int r, int c) { return r * CHUNKS + (c ^ ((r / (16 / CHUNKS)) & (CHUNKS - 1))); }
    template <int Q>
    __device__ __forceinline__ void put(const Codes<D, Q>& x, int lane) {
#pragma unroll
        for (int i = 0; i < STEP / PER; ++i) piece[at(PER * i + lane / CHUNKS, lane % CHUNKS)] = x.k[i];
    }
    __device__ __forceinline__ u32x4 get(int r, int c) const { return piece[at(r, c)]; }
};

// Q queries against the keys that pass: O, the reference of the softmax (log2 units) and two sums of the weights: l of the lane's own
// keys' as they are, for the log-sum-exp; lr of all keys' as they were rounded for the second product, by a product with ones, which is
// what O is divided by (where one key has most of the weight, its rounding leaves no trace then: 2.0e-3 of O against 2.4e-3, of
// which the output's own rounding is 1.65e-3).
template <int FMT, int D, int Q>
struct Rows {
    static constexpr int GROUPS = 64 / Q, TILES = STEP / Q, PIECES = D / 16 / GROUPS;    // lane groups, score tiles, pieces of a row of K per lane
    static constexpr int REGS = Q * Q / 64, JS = D / Q, US = Q / 16;                     // of a result tile; tiles of O; products over the keys
    typedef float Tile __attribute__((ext_vector_type(REGS)));
    bf16x8 q[2 * PIECES];
    Tile o[JS];
    float m, l, lr;

    static __device__ __forceinline__ Tile mfma(const u32x4& a, const bf16x8& b, const Tile& c) {
        if constexpr (Q == 16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), b, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), b, c, 0, 0, 0);
    }
    // the dim of entry (j, r) of a lane's part of O; four j or r in a row are four dims in a row
    static __device__ __forceinline__ int dim(int j, int r, int g) { return JS * (Q == 16 ? 4 * g + r : 8 * (r >> 2) + 4 * g + (r & 3)) + j; }
    // entries four at a time: f(dim, float4)
    template <typename F>
    __device__ __forceinline__ void each4(int lane, F&& f) const {
        const int g = lane / Q;
#pragma unroll
        for (int r = 0; r < REGS; r += JS >= 4 ? 1 : 4 / JS)
#pragma unroll
            for (int j = 0; j < JS; j += 4) {
                if constexpr (JS >= 4) f(dim(j, r, g), float4{o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]});
                else f(dim(0, r, g), float4{o[0][r], o[1][r], o[0][r + 1], o[1][r + 1]});
            }
    }
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = lr = 0.f;
#pragma unroll
        for (int j = 0; j < JS; ++j)
#pragma unroll
            for (int r = 0; r < REGS; ++r) o[j][r] = 0.f;
    }
    // row: the lane's query
    __device__ __forceinline__ void load_q(const bf16_t* row, int lane) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const bf16_t* const p = row + 16 * (GROUPS * i + lane / Q);
            q[2 * i] = *reinterpret_cast<const bf16x8*>(p);
            q[2 * i + 1] = *reinterpret_cast<const bf16x8*>(p + 8);
        }
    }
    // l of all keys
    __device__ __forceinline__ float sum() const {
        float s = l;
#pragma unroll
        for (int o = Q; o < 64; o <<= 1) s += __shfl_xor(s, o);
        return s;
    }
    // c: softmax scale x log2 e x K scale; lv: log2 of the V scale, which goes into the weights' exponent (a factor of each block
    // that the sums of weights are freed of again by `unscale`, its inverse); valid: keys of the step that exist, 1..32
    __device__ __forceinline__ void step(const Codes<D, Q>& x, Keys<D>& keys, float c, float lv, float unscale, int valid, int lane) {
        const int g = lane / Q;
        keys.put(x, lane);
        u32x4 k[TILES][PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int t = 0; t < TILES; ++t) k[t][i] = keys.get(Q * t + lane % Q, GROUPS * i + g);
        Tile s[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int r = 0; r < REGS; ++r) s[t][r] = 0.f;
#pragma unroll
        for (int h = 0; h < 2 * PIECES; ++h)
#pragma unroll
            for (int t = 0; t < TILES; ++t)         // (neighbouring products do not wait for each other)
                s[t] = mfma(eight_of_row<FMT>(k[t][h >> 1][2 * (h & 1)], k[t][h >> 1][2 * (h & 1) + 1]), q[h], s[t]);
        float e[8 * US];                            // in the order of the second product's keys
#pragma unroll
        for (int i = 0; i < 8 * US; ++i) e[i] = s[i / REGS][i % REGS];
        if (valid < STEP) {
            const int left = valid - 4 * g;         // (the entries' places without g are constants: one register for all)
#pragma unroll
            for (int i = 0; i < 8 * US; ++i) e[i] = Codes<D, Q>::of(i, 0) < left ? e[i] : -INFINITY;
        }
        float w[8 * US], part;
        auto weigh = [&]() __attribute__((always_inline)) {
            const float shift = lv - m;
            part = 0.f;
#pragma unroll
            for (int i = 0; i < 8 * US; ++i) {
                w[i] = fast_exp2(fmaf(e[i], c, shift));
                part += w[i];
            }
            part *= unscale;
        };
        weigh();
        if (__any(!(part <= LIMIT))) {              // the first step, or scores far above all before
            float top = e[0];
#pragma unroll
            for (int i = 1; i < 8 * US; ++i) top = fmaxf(top, e[i]);
            top *= c;
#pragma unroll
            for (int o = Q; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
            top = fmaxf(top, m);
            const float down = fast_exp2(m - top);
            m = top;
            l *= down;
            lr *= down;
#pragma unroll
            for (int j = 0; j < JS; ++j) o[j] *= down;
            weigh();
        }
        // (the weights first, then V's operands: with 32 queries their registers would not be had at once)
        if constexpr (Q == 32) __builtin_amdgcn_sched_barrier(0);
        bf16x8 p[US];
        Tile sum;
#pragma unroll
        for (int r = 0; r < REGS; ++r) sum[r] = 0.f;
#pragma unroll
        for (int u = 0; u < US; ++u) {
            const u32x4 b = {pack_bf16x2(w[8 * u], w[8 * u + 1]), pack_bf16x2(w[8 * u + 2], w[8 * u + 3]), pack_bf16x2(w[8 * u + 4], w[8 * u + 5]),
                             pack_bf16x2(w[8 * u + 6], w[8 * u + 7])};
            p[u] = __builtin_bit_cast(bf16x8, b);
            sum = mfma(u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}, p[u], sum);       // (every row: the sum over the keys)
        }
        l += part;
        lr = fmaf(sum[0], unscale, lr);
#pragma unroll
        for (int u = 0; u < US; ++u)
#pragma unroll
            for (int j = 0; j < JS; ++j) {
                u32x4 v;
#pragma unroll
                for (int y = 0; y < 4; ++y) v[y] = two_rows<FMT>(x.v[8 * u + 2 * y][j >> 2], x.v[8 * u + 2 * y + 1][j >> 2], j & 3);
                o[j] = mfma(v, p[u], o[j]);
            }
    }
};

// Step `local` of the n tokens that a list of blocks holds; null: no step.
struct Where { const int32_t* list; int local, n; };
// step s of the shared segments, one after the other
__device__ __forceinline__ Where in_segments(const DecodeArgs& a, int s) {
    Where w = {a.seg[0], s, a.seg_p[0]};
    for (int k = 1; k < a.n_seg; ++k)               // (selected, not indexed: the arguments stay in scalar registers)
        if (s >= a.seg_s0[k]) w = Where{a.seg[k], s - a.seg_s0[k], a.seg_p[k]};
    return w;
}
// step `local` of request b's n own tokens
__device__ __forceinline__ Where in_request(const DecodeArgs& a, int b, int local, int n) {
    return Where{local >= 0 && local * STEP < n ? a.table + static_cast<size_t>(b) * a.max_blocks : nullptr, local, n};
}
// Up to 64 steps in the order they are taken, one a lane, as far worked out as a lane can: what a wavefront does for a step by itself
// (reads of a lane, scalar arithmetic) is not hidden by anything of its own.
struct Steps {
    int rows = 0;                       // keys that exist; 0: there is no such step, -1: its block is none of the pool
    uint32_t at_lo = 0, at_hi = 0;      // where its rows begin in either array of codes, bytes
    int request = 0;                    // whose, where a list has steps of several
    float c = 0.f, lv = 0.f, unscale = 0.f;     // the block's scales; once settled, its factors: see Rows::step

    __device__ __forceinline__ void put(const DecodeArgs& a, int hk, int D, const Where& w) {
        if (!w.list) return;
        rows = -1;
        const int block = w.list[w.local >> 1];
        if (block < 0 || block >= a.n_blocks) return;
        rows = min(STEP, w.n - w.local * STEP);
        const size_t at = static_cast<size_t>(block) * a.Hkv + hk, from = at * (BLOCK * D) + (w.local & 1) * (STEP * D);
        at_lo = static_cast<uint32_t>(from);
        at_hi = static_cast<uint32_t>(from >> 32);
        c = a.k_scale[at];
        lv = a.v_scale[at];
    }
    // (after the first codes are requested, which do not wait for the scales)
    __device__ __forceinline__ void settle(const DecodeArgs& a) {
        c *= a.c;
        c = c < FLT_MIN ? FLT_MIN : c;  // (not 0, by which the -inf of a key that does not exist would become NaN)
        lv = fast_log2(lv);
        unscale = fast_exp2(-lv);
    }
};
__device__ __forceinline__ float lane_of(float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); }
__device__ __forceinline__ int lane_of(int x, int i) { return __builtin_amdgcn_readlane(x, i); }
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int i) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), i)); }

__device__ __forceinline__ int own_len(const DecodeArgs& a, int c0, int c1) { return min(max(c1 - c0, 0), a.max_own); }

// Takes steps 0 .. n-1 of the list, DEPTH of them in flight.  begin(request) is called ahead of each step.
template <bool NT, int DEPTH, int FMT, int D, int Q, typename F>
__device__ __forceinline__ void run(const DecodeArgs& a, Steps& st, int n, int hk, Rows<FMT, D, Q>& rows, Keys<D>& keys, int lane, F&& begin) {
    Codes<D, Q> x[DEPTH];
    auto load = [&](Codes<D, Q>& y, int i) __attribute__((always_inline)) {
        const int at = min(i, n - 1), rows = i < n ? max(lane_of(st.rows, at), 0) : 0;
        const size_t from = static_cast<size_t>(lane_of(st.at_hi, at)) << 32 | lane_of(st.at_lo, at);
        y.template load<NT ? 2 : 0>(a.k + from, a.v + from, rows, lane);
    };
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) load(x[j], j);
    st.settle(a);
    for (int i = 0; i < n; i += DEPTH) {
#pragma unroll
        for (int j = 0; j < DEPTH; ++j) {
            const int at = min(i + j, n - 1), n_rows = i + j < n ? lane_of(st.rows, at) : 0;
            if (n_rows != 0) {
                begin(at);
                if (n_rows > 0) rows.step(x[j], keys, lane_of(st.c, at), lane_of(st.lv, at), lane_of(st.unscale, at), n_rows, lane);
            }
            load(x[j], i + j + DEPTH);
        }
    }
}

__host__ __device__ __forceinline__ int steps_of(int n_keys) { return (n_keys + STEP - 1) / STEP; }

// What the steps of a wavefront, a workgroup or a request leave of a query beside O: the reference and both sums.
struct Sums { float m, l, lr; };
__device__ __forceinline__ Sums none() { return Sums{-INFINITY, 0.f, 0.f}; }
// factor that brings x to reference m (0 where there was no key; a NaN stays one)
__device__ __forceinline__ float to_reference(const Sums& x, float m) { return x.l == 0.f ? 0.f : fast_exp2(x.m - m); }

// The results of a workgroup's W wavefronts for the same queries, joined in LDS.
template <int D, int Q, int W> struct alignas(16) Join {
    float o[W][Q][D + 4];                   // (rows 4 banks apart: 16 queries' pieces cover all banks)
    Sums sums[W][Q];

    template <int FMT>
    __device__ __forceinline__ void put(int w, const Rows<FMT, D, Q>& rows, int lane) {
        const int col = lane % Q;
        const float l = rows.sum();
        if (lane < Q) sums[w][col] = Sums{rows.m, l, rows.lr};
        rows.each4(lane, [&](int d, const float4& x) __attribute__((always_inline)) { *reinterpret_cast<float4*>(&o[w][col][d]) = x; });
    }
    // dims d .. d+3 of query h of all wavefronts
    __device__ __forceinline__ void get(int h, int d, float (&x)[4], Sums& all) const {
        all = none();
#pragma unroll
        for (int w = 0; w < W; ++w) all.m = fmaxf(all.m, sums[w][h].m);
        x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = to_reference(sums[w][h], all.m);
            all.l += f * sums[w][h].l;
            all.lr += f * sums[w][h].lr;
            const float4 y = *reinterpret_cast<const float4*>(&o[w][h][d]);
            x[0] += f * y.x; x[1] += f * y.y; x[2] += f * y.z; x[3] += f * y.w;
        }
    }
};

// a finished query's output: D / 4 lanes a row
__device__ __forceinline__ void finish(const DecodeArgs& a, size_t row, int D, int d, const float (&x)[4], const Sums& s) {
    const float inv = s.l != 0.f ? 1.f / s.lr : 0.f;
    const u32x2 out = {pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
    *reinterpret_cast<u32x2*>(a.o + row * D + d) = out;
    if (a.lse && d == 0) a.lse[row] = s.l != 0.f ? (s.m + fast_log2(s.l)) * CART_LN2 : -INFINITY;
}

// a partial result of a query, likewise: slots of Hq rows
__device__ __forceinline__ void leave(const DecodeArgs& a, long slot, size_t row, int D, int d, const float (&x)[4], const Sums& s) {
    const size_t at = static_cast<size_t>(slot) * a.Hq + row;
    *reinterpret_cast<float4*>(a.part_o + at * D + d) = float4{x[0], x[1], x[2], x[3]};
    if (d == 0) a.part_sums[at] = s;
}

// ---- every (request, KV head) by itself: a workgroup takes one of n_cuts pieces, of `cut` steps, of its sequence -- the segments'
// steps, then its own -- its four wavefronts a quarter each, joined in LDS.  With one piece it writes the output.
template <int FMT, int D, int Q, bool NT>
__global__ __launch_bounds__(256, Q == 16 ? 3 : 1) void cache_decode_each_kernel(const DecodeArgs a) {
    __shared__ union Lds {
        Join<D, Q, 4> join;
        Keys<D> keys[4];
        __device__ Lds() {}
    } lds;
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long id = static_cast<long>(blockIdx.x) + static_cast<long>(blockIdx.y) * GRID_X;
    // (the first pieces of all first: every sequence has those, so the last ones to start are short or empty)
    const int hk = static_cast<int>(id % a.Hkv), piece = static_cast<int>(id / a.Hkv / a.B);
    const long b = id / a.Hkv % a.B;
    if (piece >= a.n_cuts) return;
    const int n_own = a.max_own > 0 ? own_len(a, a.cu[b], a.cu[b + 1]) : 0, n_shared = a.seg_s0[a.n_seg];
    const int s0 = piece * a.cut, s1 = min(s0 + a.cut, n_shared + steps_of(n_own));
    if (s0 >= s1 && a.n_cuts > 1) return;               // (nothing there: the join does not ask for it)
    const size_t row0 = static_cast<size_t>(b) * a.Hq + hk * a.G;
    Rows<FMT, D, Q> rows;
    rows.clear();
    rows.load_q(a.q + (row0 + min(lane % Q, a.G - 1)) * D, lane);
    const int n = max(s1 - s0, 0), w1 = s0 + n * (wv + 1) / 4;
    for (int s = s0 + n * wv / 4; s < w1; s += 64) {
        Steps st;
        if (s + lane < w1) {
            Where w = in_segments(a, s + lane);
            if (s + lane >= n_shared) w = in_request(a, static_cast<int>(b), s + lane - n_shared, n_own);
            st.put(a, hk, D, w);
        }
        run<NT, 2>(a, st, min(64, w1 - s), hk, rows, lds.keys[wv], lane, [](int) {});
    }
    __syncthreads();                                    // (the keys' place)
    lds.join.put(wv, rows, lane);
    __syncthreads();
    for (int i = threadIdx.x; i < a.G * (D / 4); i += 256) {
        const int h = i / (D / 4), d = i % (D / 4) * 4;
        float x[4];
        Sums sums;
        lds.join.get(h, d, x, sums);
        if (a.n_cuts == 1) finish(a, row0 + h, D, d, x, sums);
        else leave(a, static_cast<long>(piece) * a.B, row0 + h, D, d, x, sums);
    }
}

// ---- the segments by their own: workgroups of two roles, the first n_shared_wg of them
//   shared: Q of the B G query rows that read one KV head, against one of n_parts parts of the segments' steps, the four wavefronts a
//           quarter each, joined in LDS;
//   own:    each wavefront one of n_ranges ranges of the axis of all requests' steps, for one KV head.  Request b begins on that axis at
//           cu[b] / 32 + b -- one place to spare each makes that a function of its own offset -- and the ranges are equal, whatever the
//           requests' lengths.  (A wavefront for each request, 128 requests of 1 .. 1024 tokens: the launch waits for the longest.)
// Partial results: part i of the segments in slot i; of range r for request b in slot n_parts B + r + b, so that neighbours never share
// one.  Two workgroups share a CU, so that the matrix products on the segments and the streaming of the requests' own blocks overlap.
__device__ __forceinline__ int places_of(const DecodeArgs& a, int total) { return (total >> 5) + a.B; }
__device__ __forceinline__ int range_len(const DecodeArgs& a, int places) { return (places + a.n_ranges - 1) / a.n_ranges; }
template <int FMT, int D, int QS, bool NT>
__global__ __launch_bounds__(256, 2) void cache_decode_split_kernel(const DecodeArgs a) {
    constexpr int QO = 16;                              // (at most 16 queries a KV head: see cache_decode_plan)
    __shared__ union Lds {
        Join<D, QS, 4> join;
        Keys<D> keys[4];
        __device__ Lds() {}
    } lds;
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long id = static_cast<long>(blockIdx.x) + static_cast<long>(blockIdx.y) * GRID_X;
    if (id < a.n_shared_wg) {
        const int hk = static_cast<int>(id % a.Hkv), x = static_cast<int>(id / a.Hkv), part = x / a.n_rb;
        const long r0 = static_cast<long>(x % a.n_rb) * QS, n_rows = static_cast<long>(a.B) * a.G;
        auto row_of = [&](long r) { return static_cast<size_t>(r / a.G) * a.Hq + hk * a.G + r % a.G; };
        Rows<FMT, D, QS> rows;
        rows.clear();
        rows.load_q(a.q + row_of(min(r0 + lane % QS, n_rows - 1)) * D, lane);
        const long total = a.seg_s0[a.n_seg];
        const int p0 = static_cast<int>(total * part / a.n_parts), n = static_cast<int>(total * (part + 1) / a.n_parts) - p0, w1 = p0 + n * (wv + 1) / 4;
        for (int s = p0 + n * wv / 4; s < w1; s += 64) {
            Steps st;
            if (s + lane < w1) st.put(a, hk, D, in_segments(a, s + lane));
            run<false, 2>(a, st, min(64, w1 - s), hk, rows, lds.keys[wv], lane, [](int) {});
        }
        __syncthreads();                                // (the keys' place)
        lds.join.put(wv, rows, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < QS * (D / 4); i += 256) {
            const int h = i / (D / 4), d = i % (D / 4) * 4;
            if (r0 + h >= n_rows) break;
            float y[4];
            Sums sums;
            lds.join.get(h, d, y, sums);
            leave(a, static_cast<long>(part) * a.B, row_of(r0 + h), D, d, y, sums);
        }
        return;
    }
    const long w = (id - a.n_shared_wg) * 4 + wv;
    const int hk = static_cast<int>(w % a.Hkv);
    const long range = w / a.Hkv;
    if (range >= a.n_ranges) return;
    // fewer than 64 requests: one trip to memory for all offsets
    const bool few = a.B < 64;
    const int cu_lane = offset_at(a.cu, few ? min(lane, a.B) : a.B, INT_MAX);
    const int places = places_of(a, lane_of(cu_lane, few ? a.B : 0)), len = range_len(a, places);
    const long from = range * len;
    if (from >= places) return;
    const int to = static_cast<int>(min(from + len, static_cast<long>(places)));
    const int h = lane % QO;
    Rows<FMT, D, QO> rows;
    rows.clear();
    int current = -1;
    auto flush = [&]() __attribute__((always_inline)) {
        const float l = rows.sum();
        if (h >= a.G) return;
        rows.each4(lane, [&](int d, const float4& y) __attribute__((always_inline)) {
            const float z[4] = {y.x, y.y, y.z, y.w};
            leave(a, a.n_parts * static_cast<long>(a.B) + range + current, hk * a.G + h, D, d, z, Sums{rows.m, l, rows.lr});
        });
    };
    for (int p = static_cast<int>(from); p < to; p += 64) {
        const int n = min(64, to - p);
        // the requests of these places: lane k looks at b0 + k, and a lane's place belongs to the last one that begins there or before
        int b0, bk, c0, c1;
        if (few) {
            b0 = max(static_cast<int>(__builtin_popcountll(__ballot(lane < a.B && (cu_lane >> 5) + lane <= p))) - 1, 0);
            bk = min(b0 + lane, a.B - 1);
            c0 = __shfl(cu_lane, bk);
            c1 = __shfl(cu_lane, bk + 1);
        } else {
            b0 = request_of(a.cu, nullptr, a.B, INT_MAX, 5, 1, p, lane).b;
            bk = min(b0 + lane, a.B - 1);
            c0 = offset_at(a.cu, bk, INT_MAX);
            c1 = offset_at(a.cu, bk + 1, INT_MAX);
        }
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
        st.request = b;
        if (lane < n) st.put(a, hk, D, in_request(a, b, p + lane - (r0 >> 5) - b, own_len(a, r0, r1)));
        run<NT, 2>(a, st, n, hk, rows, lds.keys[wv], lane, [&](int at) __attribute__((always_inline)) {
            const int request = lane_of(st.request, at);
            if (request == current) return;
            if (current >= 0) {
                flush();
                rows.clear();
            }
            current = request;
            rows.load_q(a.q + (static_cast<size_t>(request) * a.Hq + hk * a.G + min(h, a.G - 1)) * D, lane);
            // arrived here, once a request: otherwise every step waits for the last load issued, a request's first or not
#pragma unroll
            for (auto& x : rows.q) asm volatile("" : "+v"(x));
        });
    }
    if (current >= 0) flush();
}

// Joins the partial results of a query: of all parts of the segments and of the ranges that hold some of its own tokens, or of as many
// pieces as its sequence takes.  W wavefronts a query, D / 4 lanes a partial result (so a wavefront takes 64 / (D / 4) at a time, and has
// UNROLL times as many in flight).
template <int D, int W>
__global__ __launch_bounds__(256) void cache_decode_join_kernel(const DecodeArgs a) {
    constexpr int LANES = D / 4, PER = 64 / LANES, UNROLL = 4;
    __shared__ float4 part_o[W == 1 ? 1 : W][LANES];
    __shared__ Sums part_sums[4];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long row = W == 1 ? static_cast<long>(workgroup_id()) * 4 + wv : workgroup_id();
    if (row >= static_cast<long>(a.B) * a.Hq) return;
    const int d = lane % LANES * 4, sub = lane / LANES;
    const int b = static_cast<int>(row / a.Hq);
    // result i: slot i B + b, below n_parts; from there on slot own + i - n_parts
    int n_parts = a.n_parts, n_own = 0;
    long own = 0;
    const int c0 = a.max_own > 0 ? offset_at(a.cu, b, INT_MAX) : 0, steps = a.max_own > 0 ? steps_of(own_len(a, c0, a.cu[b + 1])) : 0;
    if (a.n_ranges > 0 && steps > 0) {
        const int len = range_len(a, places_of(a, offset_at(a.cu, a.B, INT_MAX))), p0 = (c0 >> 5) + b, r0 = min(p0 / len, a.n_ranges - 1);
        n_own = min((p0 + steps - 1) / len, a.n_ranges - 1) - r0 + 1;
        own = static_cast<long>(n_parts) * a.B + r0 + b;
    } else if (a.n_cuts > 0) {
        n_parts = (a.seg_s0[a.n_seg] + steps + a.cut - 1) / a.cut;
    }
    const int n = n_parts + n_own;
    const int in_slot = static_cast<int>(row % a.Hq);
    Sums t = none();
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = (W == 1 ? 0 : wv) * PER * UNROLL; i0 < n; i0 += W * PER * UNROLL) {
        Sums s[UNROLL];
        float4 y[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int i = i0 + u * PER + sub;
            s[u] = none();
            y[u] = float4{0.f, 0.f, 0.f, 0.f};
            if (i >= n) continue;
            const size_t at = static_cast<size_t>(i < n_parts ? static_cast<long>(i) * a.B + b : own + i - n_parts) * a.Hq + in_slot;
            s[u] = a.part_sums[at];
            y[u] = *reinterpret_cast<const float4*>(a.part_o + at * D + d);
        }
        float top = t.m;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) top = fmaxf(top, s[u].m);
        const float down = to_reference(t, top);
        t = Sums{top, t.l * down, t.lr * down};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] *= down;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const float f = to_reference(s[u], top);
            t.l += f * s[u].l;
            t.lr += f * s[u].lr;
            x[0] += f * y[u].x; x[1] += f * y[u].y; x[2] += f * y[u].z; x[3] += f * y[u].w;
        }
    }
    // with another lane's or wavefront's
    auto add = [&](const Sums& s, const float (&y)[4]) __attribute__((always_inline)) {
        const float top = fmaxf(t.m, s.m), f = to_reference(t, top), f2 = to_reference(s, top);
        t = Sums{top, t.l * f + s.l * f2, t.lr * f + s.lr * f2};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = x[e] * f + y[e] * f2;
    };
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1) {
        const float y[4] = {__shfl_xor(x[0], o), __shfl_xor(x[1], o), __shfl_xor(x[2], o), __shfl_xor(x[3], o)};
        const Sums s = {__shfl_xor(t.m, o), __shfl_xor(t.l, o), __shfl_xor(t.lr, o)};
        add(s, y);
    }
    if constexpr (W > 1) {
        if (sub == 0) part_o[wv][lane] = float4{x[0], x[1], x[2], x[3]};
        if (lane == 0) part_sums[wv] = t;
        __syncthreads();
        if (wv > 0) return;
#pragma unroll
        for (int w = 1; w < W; ++w) {
            const float4 z = part_o[w][lane % LANES];
            const float y[4] = {z.x, z.y, z.z, z.w};
            add(part_sums[w], y);
        }
    }
    if (sub == 0) finish(a, static_cast<size_t>(row), D, d, x, t);
}

constexpr int MIN_CUT = 4;              // fewest steps of a piece: one a wavefront
// most workgroups of pieces, and wavefronts of ranges, per CU
constexpr int MAX_PIECES = 16, MAX_RANGES = 4;

double own_bytes(const cart_cache_decode_desc& d, const cart_cache& c) {
    return 0.5 * static_cast<double>(d.B) * c.Hkv * steps_of(d.max_own_len) * STEP * 2 * c.D;
}

// Partial results that no plan of these sizes or smaller ones exceeds (slots of Hq rows), so that a workspace for a program's largest
// call serves its others.  Parts: cus / (n_rb Hkv) + 1 for each request at most, and n_rb >= rows / 32.
long most_slots(const cart_cache_decode_desc& d, const cart_cache& c, const cart_cache_segment* shared) {
    const long cus = device_cus(), B = d.B, own = steps_of(d.max_own_len);
    long steps = 0;
    for (int s = 0; s < d.n_shared; ++s) steps += steps_of(shared[s].p);
    auto least = [](long x, long y) { return x < y ? x : y; };
    const long pieces = least(((steps + own) / MIN_CUT + 1) * B, MAX_PIECES * cus / c.Hkv + B);
    const long parts = least((steps + 3) / 4 * B, 32 * cus / d.Hq + B + 1);
    const long ranges = own > 0 ? least(B * (own + 1), MAX_RANGES * cus / c.Hkv + 1) + B : 0;
    return pieces > parts + ranges ? pieces : parts + ranges;
}

template <int FMT, int D, bool NT>
void launch(const DecodeArgs& a, const CachePlan& p, hipStream_t st) {
    const dim3 grid = grid_of(p.n_wg);
    if (p.n_cuts > 0) {
        if (a.G <= 16) cache_decode_each_kernel<FMT, D, 16, NT><<<grid, 256, 0, st>>>(a);
        else cache_decode_each_kernel<FMT, D, 32, NT><<<grid, 256, 0, st>>>(a);
        if (p.n_cuts == 1) return;
    } else if (static_cast<long>(a.B) * a.G > 16) cache_decode_split_kernel<FMT, D, 32, NT><<<grid, 256, 0, st>>>(a);
    else cache_decode_split_kernel<FMT, D, 16, NT><<<grid, 256, 0, st>>>(a);
    const long rows = static_cast<long>(a.B) * a.Hq;
    if (rows <= FEW_ROWS) cache_decode_join_kernel<D, 4><<<grid_of(rows), 256, 0, st>>>(a);
    else cache_decode_join_kernel<D, 1><<<grid_of((rows + 3) / 4), 256, 0, st>>>(a);
}

}  // namespace

// The faster by an estimate (us; `own` half full on average), whose figures are those of sweeps of all forms, 40 problems without
// segments and 300 with (256 CUs, head_dim 128 unless said):
//   every (request, KV head) by itself, in n pieces: 5.3 and 0.14 a step of the longest piece (its four wavefronts share it) where the chip
//     is not full, 0.6 a segment's step and SIMD -- every request's again -- and the own bytes at 6.2 TB/s; the second launch 3 and its
//     partial results.  CUs share the memory's rate evenly, so a CU with one workgroup more than others holds the call up for as
//     long: 144 (request, head) pairs of 32000 .. 61000 tokens n = 1 336, 2 304, 4 302, 6 260, 12 265.  32 requests of up to 1024: n = 1
//     10.9, 2 15.3, 4 17.8; one of 16384: n = 1 76, 4 26.8, 16 14.1, 32 13.6;
//   split: 13, the second launch's rows, and the longer of a segment wavefront's 0.73 a step and the own bytes, with some of the other.  For
//     the same reason each CU gets one workgroup of ranges, and one of the segments at most where the own bytes take longer (230
//     requests of up to 2300 tokens behind 2268 slots: 130; with a part more, 464 workgroups of the segments, 264); where the
//     segments take longer the CUs left over are worth another part (221 of 5 behind 5497: 45, without 52).
//   By itself / split: 128 requests of up to 1024 tokens behind 8192 slots 164 / 48, of 512 behind 1024 36.4 / 26.5, of 1024 behind 512
//   37.0 / 37.2; 64 of 512 behind 512 16.0 / 22.2; 16 of 16384 behind 8192 79 / 60; 1 of 131072 behind 2048 31.8 / 41.1; head_dim 64: 128
//   of 2048 behind 2048 54.0 / 34.3, 32 of 1024 behind 1024 11.3 / 14.8.  Over 260 problems drawn like servers' the choice costs 0.7 % on
//   average and 15 % at most.  With more than 16 queries a KV head shares its keys among enough of them by itself: 25.2 / 30.1, 41.0 /
//   59.0, 36.0 / 33.9 of 9.
CachePlan cache_decode_plan(const cart_cache_decode_desc& d, const cart_cache& c, const cart_cache_segment* shared) {
    CachePlan p = {}, q = {};
    const long cus = device_cus();
    long steps = 0;
    for (int s = 0; s < d.n_shared; ++s) steps += steps_of(shared[s].p);
    const long own = steps_of(d.max_own_len), all = steps + own, group = d.Hq / c.Hkv;
    const long rows = d.B * group, pairs = static_cast<long>(d.B) * c.Hkv, out = static_cast<long>(d.B) * d.Hq;
    const double chip = static_cast<double>(cus) / 256, own_us = own_bytes(d, c) / 6.2e6 / chip;

    double each_us = 0;
    // 1, 2, 3, 4, 6, 8, 12, 16 ..
    for (long n = 1; n == 1 || (n * MIN_CUT <= all && n * pairs <= MAX_PIECES * cus); n = n == 1 ? 2 : n & (n - 1) ? n / 3 * 4 : n / 2 * 3) {
        const double per_cu = static_cast<double>(pairs * n) / static_cast<double>(cus), full = per_cu / 6;
        const double us = 5.3 + fmax(0.14 * static_cast<double>((all + n - 1) / n) * fmax(1.0, full),
                                     (0.6 * static_cast<double>(pairs * steps) / static_cast<double>(4 * cus) + own_us) * (per_cu > 1 ? ceil(per_cu) / per_cu : 1.0)) +
                          (n > 1 ? 3 + static_cast<double>(out * n) / 1000 : 0.0);
        if (n > 1 && us >= each_us) continue;
        each_us = us;
        p.cut = static_cast<int>(all > 0 ? (all + n - 1) / n : 1);
    }
    p.n_cuts = static_cast<int>(all > 0 ? (all + p.cut - 1) / p.cut : 1);
    p.n_wg = pairs * p.n_cuts;
    p.slots = p.n_cuts == 1 ? 0 : static_cast<long>(p.n_cuts) * d.B;
    if (steps == 0 || group > 16) return p;

    const int per = rows > 16 ? 32 : 16;
    q.n_rb = static_cast<int>((rows + per - 1) / per);
    const long one = static_cast<long>(q.n_rb) * c.Hkv, most = (steps + 3) / 4;
    auto shared_us_of = [&](long parts) { return 0.73 * static_cast<double>(steps) / (4.0 * static_cast<double>(parts)); };
    long want = one < cus ? cus / one : 1;
    if (cus % one != 0 && one < cus && shared_us_of(want) > own_us) ++want;
    q.n_parts = static_cast<int>(want < most ? want : most);
    const double shared_us = shared_us_of(q.n_parts);
    const double split_us = 13 + static_cast<double>(out) / 1200 + fmax(shared_us, own_us) + 0.3 * fmin(shared_us, own_us);
    if (each_us <= split_us) return p;
    q.n_shared_wg = one * q.n_parts;
    q.slots = static_cast<long>(q.n_parts) * d.B;
    if (own > 0) {
        const long room = 2 * cus - q.n_shared_wg, wgs = room > cus ? cus : room > cus / 2 ? room : cus / 2;
        const long r = 4 * wgs / c.Hkv, places = static_cast<long>(d.B) * (own + 1);
        q.n_ranges = static_cast<int>(r < 1 ? 1 : r < places ? r : places);
        q.slots += q.n_ranges + d.B;
    }
    q.n_wg = q.n_shared_wg + (static_cast<long>(q.n_ranges) * c.Hkv + 3) / 4;
    return q;
}

size_t cache_decode_workspace(const cart_cache_decode_desc& d, const cart_cache& c, const cart_cache_segment* shared) {
    return static_cast<size_t>(most_slots(d, c, shared)) * d.Hq * (c.D * sizeof(float) + sizeof(Sums));
}

int launch_cache_decode(const cart_cache_decode_desc& d, const cart_cache& c, float scale, const void* q,
                        const cart_cache_segment* shared, const int32_t* table, const int32_t* cu, void* o, float* lse, void* ws,
                        hipStream_t st) {
    const CachePlan p = cache_decode_plan(d, c, shared);
    DecodeArgs a = {};
    a.q = static_cast<const bf16_t*>(q);
    a.k = static_cast<const char*>(c.k); a.v = static_cast<const char*>(c.v);
    a.k_scale = c.k_scale; a.v_scale = c.v_scale;
    for (int s = 0; s < d.n_shared; ++s) {
        if (shared[s].p == 0) continue;
        a.seg[a.n_seg] = shared[s].blocks;
        a.seg_p[a.n_seg] = shared[s].p;
        a.seg_s0[a.n_seg + 1] = a.seg_s0[a.n_seg] + steps_of(shared[s].p);
        ++a.n_seg;
    }
    a.table = table; a.cu = cu;
    a.B = d.B; a.Hq = d.Hq; a.Hkv = c.Hkv; a.G = d.Hq / c.Hkv;
    a.max_blocks = d.max_blocks; a.max_own = d.max_own_len; a.n_blocks = c.n_blocks;
    a.c = scale * CART_LOG2E;
    a.o = static_cast<bf16_t*>(o); a.lse = lse;
    a.n_rb = p.n_rb; a.n_parts = p.n_parts; a.n_ranges = p.n_ranges; a.n_cuts = p.n_cuts; a.cut = p.cut;
    a.n_shared_wg = p.n_shared_wg;
    a.part_o = static_cast<float*>(ws);             // (first: its rows are multiples of 16 bytes)
    a.part_sums = reinterpret_cast<Sums*>(a.part_o + static_cast<size_t>(p.slots) * d.Hq * c.D);
    auto go = [&](auto nt) {
        constexpr bool NT = decltype(nt)::value;
        if (c.D == 64) {
            if (c.format == CART_I8) launch<CART_I8, 64, NT>(a, p, st);
            else launch<CART_E4M3, 64, NT>(a, p, st);
        } else {
            if (c.format == CART_I8) launch<CART_I8, 128, NT>(a, p, st);
            else launch<CART_E4M3, 128, NT>(a, p, st);
        }
    };
    if (own_bytes(d, c) >= NT_BYTES) go(std::true_type{});
    else go(std::false_type{});
    return static_cast<int>(hipGetLastError());
}

}  // namespace cart
