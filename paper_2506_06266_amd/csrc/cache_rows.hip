// Rows into and out of the 8-bit cache (cart_cache_write, cart_cache_read).
//
// A block of 64 tokens of one head and one of K and V is a wavefront's work in either direction: its scale needs the
// largest magnitude of all its rows, which stay in registers between the search for it and the rounding, so memory is
// passed over once and no wavefront waits for another.  Bound: HBM, 2 T Hkv D (element size + 1) bytes.
#include "cache.h"

namespace cart {
using namespace cache;

namespace {

// Rows of a call past what the memory-side cache keeps of them are moved non-temporally (NT), so that the codes stay in it.  us a call:
// writing 64 prompts (150 MB of rows) 48.2, so 40.7; 537 MB 153.8, 155.0; a cartridge of 67 MB 17.3, 20.3; reading back 537 MB
// 160.8, 155.7, a cartridge of 34 MB 10.4, 10.1 (and whoever reads it next would find less of it).
constexpr long NT_BYTES = 100000000;
template <bool NT, typename V> __device__ __forceinline__ V load_as(const char* p) {
    const V* const q = reinterpret_cast<const V*>(p);
    if constexpr (NT) return __builtin_nontemporal_load(q);
    else return *q;
}
template <bool NT, typename V> __device__ __forceinline__ void store_as(char* p, V v) {
    V* const q = reinterpret_cast<V*>(p);
    if constexpr (NT) __builtin_nontemporal_store(v, q);
    else *q = v;
}

struct RowsArgs {
    const int32_t *cu, *first, *table;
    int T, B, max_blocks, n_blocks, Hkv;
    int each, places;           // rows of each request and places it gets, where cu is null
    long n_waves;
    char *codes_k, *codes_v;
    float *scale_k, *scale_v;
    char *k, *v;
    int64_t k_row, k_head, v_row, v_head;       // strides in elements
};

// What a wavefront works on: rows [row, row + n) of the call, tokens from `pos` on of their request, all in one block.
struct Piece {
    int row, n, in_block;       // in_block: the first one's place in the block
    long block;                 // block id, -1: none
};

__device__ __forceinline__ Piece piece_of(const RowsArgs& a, int place, int lane) {
    Piece p = {0, 0, 0, -1};
    int b, j, row0, n, first;
    if (a.cu) {
        const Request r = request_of(a.cu, a.first, a.B, a.T, 6, 2, place, lane);
        b = r.b;
        row0 = r.from;
        n = r.to - r.from;
        first = r.first;
        j = place - (row0 >> 6) - 2 * b;
    } else {
        b = place / a.places;
        j = place - b * a.places;
        row0 = b * a.each;
        n = a.each;
        first = a.first ? a.first[b] : 0;
    }
    if (n <= 0 || j < 0) return p;
    // (a negative `first` has no blocks; its rows are counted from 0 so that a reader clears them)
    const long f = first < 0 ? 0 : first, blk = f / BLOCK + j;
    const long lo = blk * BLOCK > f ? blk * BLOCK : f, hi = blk * BLOCK + BLOCK < f + n ? blk * BLOCK + BLOCK : f + n;
    if (hi <= lo) return p;
    p.row = row0 + static_cast<int>(lo - f);
    p.n = static_cast<int>(hi - lo);
    p.in_block = static_cast<int>(lo - blk * BLOCK);
    if (first >= 0 && blk < a.max_blocks) {
        const int id = a.table[static_cast<size_t>(b) * a.max_blocks + blk];
        if (id >= 0 && id < a.n_blocks) p.block = id;
    }
    return p;
}

// 8 elements of a row as fp32 bits or values
template <typename T, bool NT> struct Eight;
template <bool NT> struct Eight<float, NT> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const char* p) {
        a = load_as<NT, u32x4>(p);
        b = load_as<NT, u32x4>(p + 16);
    }
    __device__ __forceinline__ uint32_t bits(int i) const { return i < 4 ? a[i] : b[i - 4]; }
    static __device__ __forceinline__ void store(char* p, const float (&x)[8]) {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        store_as<NT>(p, f32x4{x[0], x[1], x[2], x[3]});
        store_as<NT>(p + 16, f32x4{x[4], x[5], x[6], x[7]});
    }
};
template <bool NT> struct Eight<bf16_t, NT> {
    u32x4 a;
    __device__ __forceinline__ void load(const char* p) { a = load_as<NT, u32x4>(p); }
    __device__ __forceinline__ uint32_t bits(int i) const { return i & 1 ? a[i >> 1] & 0xffff0000u : a[i >> 1] << 16; }
    static __device__ __forceinline__ void store(char* p, const float (&x)[8]) {
        const u32x4 w = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        store_as<NT>(p, w);
    }
};

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint32_t u = static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o, CART_WAVE));
        v = v > u ? v : u;
    }
    return v;
}

// A lane holds 8 elements of a row at a time, so D / 8 lanes a row and 64 / (D / 8) rows a step.
template <typename T, int FMT, int D, bool NT, int STEPS>
__device__ __forceinline__ void write_rows(const Piece& p, const char* rows, int64_t stride_b, char* codes, float* scale, int lane) {
    constexpr int LANES = D / 8, PER = 64 / LANES;
    const int sub = lane / LANES, col = lane % LANES;
    const float old = p.in_block > 0 ? *scale : 0.f;
    Eight<T, NT> x[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int r = i * PER + sub;        // (rows past the last are that one again: they change no maximum)
        x[i].load(rows + (r < p.n ? r : p.n - 1) * stride_b + col * 8 * sizeof(T));
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = x[i].bits(e) & 0x7fffffffu;
            m = m > b ? m : b;
        }
    float s = scale_for<FMT>(wave_umax(m));
    if (p.in_block > 0) s = old != old || s != s ? __uint_as_float(0x7fc00000u) : fmaxf(s, old);
    if (p.in_block > 0 && s > old) {        // the rows before these, in the larger scale
        const float f = old / s;
        for (int r = sub; r < p.in_block; r += PER) {
            uint32_t* const c = reinterpret_cast<uint32_t*>(codes + r * D + col * 8);
            const u32x2 w = *reinterpret_cast<const u32x2*>(c);
            float y[4], z[4];
            Code<FMT>::decode4(w[0], y);
            Code<FMT>::decode4(w[1], z);
            const u32x2 n = {Code<FMT>::encode4(y[0] * f, y[1] * f, y[2] * f, y[3] * f), Code<FMT>::encode4(z[0] * f, z[1] * f, z[2] * f, z[3] * f)};
            *reinterpret_cast<u32x2*>(c) = n;
        }
    }
    const float inv = 1.f / s;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int r = i * PER + sub;
        if (r >= p.n) continue;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __uint_as_float(x[i].bits(e)) * inv;
        const u32x2 n = {Code<FMT>::encode4(y[0], y[1], y[2], y[3]), Code<FMT>::encode4(y[4], y[5], y[6], y[7])};
        *reinterpret_cast<u32x2*>(codes + (p.in_block + r) * D + col * 8) = n;
    }
    if (lane == 0) *scale = s;
}

template <typename T, int FMT, int D, bool NT>
__global__ __launch_bounds__(256) void cache_write_kernel(const RowsArgs a) {
    const int lane = threadIdx.x & 63;
    const long w = static_cast<long>(workgroup_id()) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= a.n_waves) return;
    const int hk = static_cast<int>(w % a.Hkv), kv = static_cast<int>(w / a.Hkv % 2), place = static_cast<int>(w / a.Hkv / 2);
    const Piece p = piece_of(a, place, lane);
    if (p.n == 0 || p.block < 0) return;
    const int64_t stride = (kv ? a.v_row : a.k_row) * static_cast<int64_t>(sizeof(T));
    const char* const rows = (kv ? a.v : a.k) + p.row * stride + hk * (kv ? a.v_head : a.k_head) * static_cast<int64_t>(sizeof(T));
    const size_t at = static_cast<size_t>(p.block) * a.Hkv + hk;
    char* const codes = (kv ? a.codes_v : a.codes_k) + at * (BLOCK * D);
    float* const scale = (kv ? a.scale_v : a.scale_k) + at;
    // few rows (a generated token, the ends of a prompt) in as many steps as they take
    constexpr int PER = 512 / D;
    if (p.n <= PER) write_rows<T, FMT, D, NT, 1>(p, rows, stride, codes, scale, lane);
    else if (p.n <= D / 32 * PER) write_rows<T, FMT, D, NT, D / 32>(p, rows, stride, codes, scale, lane);
    else write_rows<T, FMT, D, NT, D / 8>(p, rows, stride, codes, scale, lane);
}

template <typename T, int FMT, int D, bool NT>
__global__ __launch_bounds__(256) void cache_read_kernel(const RowsArgs a) {
    const int lane = threadIdx.x & 63;
    const long w = static_cast<long>(workgroup_id()) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= a.n_waves) return;
    const int hk = static_cast<int>(w % a.Hkv), kv = static_cast<int>(w / a.Hkv % 2), place = static_cast<int>(w / a.Hkv / 2);
    const Piece p = piece_of(a, place, lane);
    if (p.n == 0) return;
    constexpr int LANES = D / 8, PER = 64 / LANES, STEPS = D / 8;
    const int sub = lane / LANES, col = lane % LANES;
    const int64_t stride = (kv ? a.v_row : a.k_row) * static_cast<int64_t>(sizeof(T));
    char* const rows = (kv ? a.v : a.k) + p.row * stride + hk * (kv ? a.v_head : a.k_head) * static_cast<int64_t>(sizeof(T));
    const size_t at = static_cast<size_t>(p.block < 0 ? 0 : p.block) * a.Hkv + hk;
    const char* const codes = (kv ? a.codes_v : a.codes_k) + at * (BLOCK * D) + p.in_block * D;
    const float s = (kv ? a.scale_v : a.scale_k)[at];
    u32x2 c[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {           // (rows past the last are that one again, so that no load waits for a branch)
        const int r = i * PER + sub;
        c[i] = load_as<NT, u32x2>(codes + (r < p.n ? r : p.n - 1) * D + col * 8);
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int r = i * PER + sub;
        if (r >= p.n) continue;
        float lo[4], hi[4], y[8];
        Code<FMT>::decode4(c[i][0], lo);
        Code<FMT>::decode4(c[i][1], hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = p.block < 0 ? 0.f : lo[e] * s;
            y[e + 4] = p.block < 0 ? 0.f : hi[e] * s;
        }
        Eight<T, NT>::store(rows + r * stride + col * 8 * sizeof(T), y);
    }
}

template <typename T, int FMT, int D, bool NT>
void launch(const RowsArgs& a, bool write, hipStream_t st) {
    const dim3 grid = grid_of((a.n_waves + 3) / 4);
    if (write) cache_write_kernel<T, FMT, D, NT><<<grid, 256, 0, st>>>(a);
    else cache_read_kernel<T, FMT, D, NT><<<grid, 256, 0, st>>>(a);
}
template <typename T, int FMT, int D>
void launch(const RowsArgs& a, bool write, hipStream_t st) {
    if (2L * a.T * a.Hkv * D * static_cast<long>(sizeof(T)) > NT_BYTES) launch<T, FMT, D, true>(a, write, st);
    else launch<T, FMT, D, false>(a, write, st);
}
template <typename T, int FMT>
void launch(const RowsArgs& a, int D, bool write, hipStream_t st) {
    if (D == 64) launch<T, FMT, 64>(a, write, st);
    else launch<T, FMT, 128>(a, write, st);
}

}  // namespace

int launch_cache_rows(const cart_cache& c, const cart_cache_rows& r, void* k, void* v, const int32_t* cu, const int32_t* first,
                      const int32_t* table, bool write, hipStream_t st) {
    RowsArgs a;
    a.cu = cu; a.first = first; a.table = table;
    a.T = r.T; a.B = r.B; a.max_blocks = r.max_blocks; a.n_blocks = c.n_blocks; a.Hkv = c.Hkv;
    a.each = r.T / r.B;
    a.places = (a.each + BLOCK - 2) / BLOCK + 1;        // blocks that `each` rows reach into, wherever they begin
    a.codes_k = static_cast<char*>(c.k); a.codes_v = static_cast<char*>(c.v);
    a.scale_k = c.k_scale; a.scale_v = c.v_scale;
    a.k = static_cast<char*>(k); a.v = static_cast<char*>(v);
    a.k_row = r.k_row_stride; a.k_head = r.k_head_stride; a.v_row = r.v_row_stride; a.v_head = r.v_head_stride;
    const long places = cu ? r.T / BLOCK + 2L * r.B : static_cast<long>(a.places) * r.B;
    a.n_waves = places * 2 * c.Hkv;
    if (r.dtype == CART_F32) {
        if (c.format == CART_I8) launch<float, CART_I8>(a, c.D, write, st);
        else launch<float, CART_E4M3>(a, c.D, write, st);
    } else {
        if (c.format == CART_I8) launch<bf16_t, CART_I8>(a, c.D, write, st);
        else launch<bf16_t, CART_E4M3>(a, c.D, write, st);
    }
    return static_cast<int>(hipGetLastError());
}

}  // namespace cart
