// A paged cache of keys and values in 8 bits: new tokens into their pages, and back.  Layout and format stand in
// include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit_pages.hpp"

namespace enec {
namespace lowbit {

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t o = __shfl_xor(v, k);
        v = v > o ? v : o;
    }
    return v;
}

// four values as E4M3 codes of v / 2^e; the scale is a power of two, so the division is exact, and nearest even is the rounding
// of the definition.  Finite values fit by the choice of e; an infinity is cut to the largest value, a NaN is not touched.
__device__ __forceinline__ float cut(float v, float inverse)
{
    const float s = v * inverse;
    return __builtin_isinf(s) ? __builtin_copysignf(448.0f, s) : s;
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inverse)
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_pk_fp8_f32(cut(a, inverse), cut(b, inverse), r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(cut(c, inverse), cut(d, inverse), r, true);
    return r;
}
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float by)
{
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, r, true);
    return r;
}
// magnitude bits of a finite value, 0 of others
__device__ __forceinline__ uint32_t finite_bits(float v)
{
    const uint32_t b = bits_of(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0;
}
// what an item's workgroup knows of its page
struct Page {
    uint32_t first, end;        // slots of the page that the call's tokens have
    uint32_t token;             // the call's token in slot 0 (may lie before the sequence's first one: mod 2^32)
    int32_t position;           // of slot 0
    const int32_t *entry;       // where its number is; null: it has none
    bool good;
};
__device__ __forceinline__ Page page_of_item(const Pages &c, uint32_t item, int32_t most = MAX_SEQUENCE)
{
    const Found f = sequence_of_item(c, item);
    const Sequence &s = f.s;
    Page p{};
    if (f.b < 0) return p;
    if (!s.good || s.length > most) {
        complain(c);
        return p;
    }
    const int32_t begin = s.length - (int32_t)s.count;           // position of the sequence's first token in the call; may be negative
    const int32_t slot = ((begin >> c.log_page) + (int32_t)(item - f.first));
    p.position = slot << c.log_page;
    const int32_t lo = begin > p.position ? begin : p.position;
    const int32_t hi = s.length < p.position + (1 << c.log_page) ? s.length : p.position + (1 << c.log_page);
    if (lo >= hi || slot >= (int32_t)c.table_stride) return p;
    p.first = (uint32_t)(lo - p.position);
    p.end = (uint32_t)(hi - p.position);
    p.token = s.start + (uint32_t)(p.position - begin);
    p.entry = slot >= 0 ? c.table + (size_t)f.b * c.table_stride + (uint32_t)slot : nullptr;
    p.good = true;
    return p;
}
// its number; -1: none, or none of the cache's
__device__ __forceinline__ int32_t number_of(const Pages &c, const Page &p)
{
    if (!p.entry) return -1;
    const int32_t n = *p.entry;
    if ((uint32_t)n < c.n_pages) return n;
    complain(c);
    return -1;
}

// Rotation by positions: pairs (j, half + j), or neighbours (2 j, 2 j + 1), of a head's first 2 half values.
enum { STAY = 0, HALVES = 1, NEIGHBOURS = 2 };
using f32x4_a8 = f32x4 __attribute__((aligned(8)));
struct Turns {
    const float *table;         // positions x half pairs
    uint32_t half;
    int32_t positions;
};
// cosines and sines of N pairs from pair j on
template <int N> __device__ __forceinline__ void load_turns(const Turns &t, int32_t position, uint32_t j, float (&c)[N], float (&s)[N])
{
    const f32x4_a8 *p = reinterpret_cast<const f32x4_a8 *>(t.table + ((size_t)(uint32_t)position * t.half + j) * 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const f32x4 v = p[i];
        c[2 * i] = v[0], s[2 * i] = v[1], c[2 * i + 1] = v[2], s[2 * i + 1] = v[3];
    }
}
// eight neighbours, four pairs
__device__ __forceinline__ void turn_neighbours(const float (&c)[4], const float (&s)[4], float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        x[2 * i] = a * c[i] - b * s[i], x[2 * i + 1] = b * c[i] + a * s[i];
    }
}
// the eight values from element i + dim on, of a head that begins at element i
template <int DT, int ROTATION>
__device__ __forceinline__ void load8_turned(const void *in, size_t i, uint32_t dim, int32_t position, const Turns &t, float (&x)[8])
{
    load8<DT>(in, i + dim, x);
    if (dim >= 2 * t.half) return;
    if constexpr (ROTATION == NEIGHBOURS) {
        float c[4], s[4];
        load_turns(t, position, dim / 2, c, s);
        turn_neighbours(c, s, x);
    } else {
        const bool second = dim >= t.half;
        float y[8], c[8], s[8];
        load8<DT>(in, second ? i + dim - t.half : i + dim + t.half, y);
        load_turns(t, position, second ? dim - t.half : dim, c, s);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float own = x[k] * c[k], other = y[k] * s[k];
            x[k] = second ? own + other : own - other;
        }
    }
}

// A workgroup has one page of one head, keys or values: it alone knows all tokens that the scale depends on, and nothing is
// shared between workgroups.  Tiles of 32 values: keys 2 tokens x 16 dimensions, values 16 tokens x 2 dimensions, so that
// both ways a thread's codes are two runs of 16 bytes; consecutive threads have consecutive dimensions, so that the loads of a
// token are one run.  The tiles stay in registers between finding the scale and writing; pages of more than 8192 values are read
// twice (the second time from the cache).
// Bound by HBM for prompts (3 bytes a bf16 value) and by its chain of dependent reads for single tokens: starts and lengths, table
// beside the new values, old scale, old codes.  (The last two need not wait for one another: asked for together they would shorten it; before the new values
// they cost prompts 19 -> 25 us.)  A workgroup has a thread for each tile, 64 to 256.
// Eight prompts of up to 2047 tokens, 8 heads of 128, fp16, pages of 16: 18.7 us, 14.5 back.  One token for each of 32 sequences, pages of 64: 7.9 us.
template <int DT, bool V, int ROTATION = STAY> struct Tile {
    uint32_t slot, dim;         // first slot and dimension
    float x[32];
    static constexpr int SLOTS = V ? 16 : 2, DIMS = V ? 2 : 16;
    __device__ __forceinline__ void at(uint32_t t, uint32_t log_dims)         // log_dims: of the tiles side by side
    {
        dim = (t & ((1u << log_dims) - 1)) * DIMS;
        slot = (t >> log_dims) * SLOTS;
    }
    __device__ __forceinline__ void load(const void *in, size_t token_stride, size_t head, const Page &p, const Turns &turns)
    {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const bool has = slot + s >= p.first && slot + s < p.end;
            const size_t i = (size_t)(p.token + slot + s) * token_stride + head + dim;
            if constexpr (V) {
                const uint32_t w = has ? *reinterpret_cast<const u32_a2 *>(static_cast<const uint16_t *>(in) + i) : 0;
                const f32x2 u = unpack2<DT>(w);
                x[s] = u[0], x[16 + s] = u[1];
            } else {
                float u[16] = {};
                if (has) {
#pragma unroll
                    for (int r = 0; r < 16; r += 8) {
                        float(&v)[8] = *reinterpret_cast<float(*)[8]>(u + r);
                        if constexpr (ROTATION == STAY) load8<DT>(in, i + r, v);
                        else load8_turned<DT, ROTATION>(in, i - dim, dim + r, p.position + (int32_t)(slot + s), turns, v);
                    }
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) x[16 * s + j] = u[j];
            }
        }
    }
    __device__ __forceinline__ uint32_t largest() const
    {
        uint32_t a = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const uint32_t b = finite_bits(x[j]);
            a = a > b ? a : b;
        }
        return a;
    }
    __device__ __forceinline__ size_t run_at(int r, uint32_t log_page, uint32_t head_dim) const
    {
        return V ? ((size_t)(dim + r) << log_page) + slot : (size_t)(slot + r) * head_dim + dim;
    }
    // the 16-byte runs: keys, of each token; values, of each dimension.  `move`: earlier codes of the page follow a larger scale.
    __device__ __forceinline__ void store(uint8_t *codes, uint32_t log_page, uint32_t head_dim, const Page &p, float inverse, bool move, float by) const
    {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const size_t i = run_at(r, log_page, head_dim);
            // slots of the run: one (keys) or sixteen (values)
            const uint32_t lo = V ? slot : slot + r, hi = lo + (V ? 16 : 1);
            const bool fresh = hi > p.first && lo < p.end, whole = lo >= p.first && hi <= p.end, older = move && lo < p.first;
            if (!fresh && !older) continue;
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = codes4(x[16 * r + 4 * j], x[16 * r + 4 * j + 1], x[16 * r + 4 * j + 2], x[16 * r + 4 * j + 3], inverse);
            u32x4 *at = reinterpret_cast<u32x4 *>(codes + i);
            if (!whole) {
                const u32x4 old = *at;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t moved = move ? rescale4(old[j], by) : old[j];
                    uint32_t word = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t s = V ? slot + 4 * j + k : lo, mask = 255u << (8 * k);
                        word |= (s < p.first ? moved : s < p.end ? w[j] : old[j]) & mask;
                    }
                    w[j] = word;
                }
            }
            *at = w;
        }
    }
};

template <int DT, bool V, int ROTATION = STAY>
__device__ __forceinline__ void write_page(const Pages &c, const Page &p, uint32_t head, const void *in, size_t token_stride, size_t head_stride,
                                           uint32_t *shared, const Turns &turns = Turns{})
{
    const size_t values = (size_t)c.head_dim << c.log_page;
    const uint32_t log_dims = (uint32_t)__builtin_ctz(c.head_dim / (V ? 2u : 16u)), tiles = (uint32_t)(values / 32);
    Tile<DT, V, ROTATION> t;
    uint32_t a = 0;
    const int32_t number = number_of(c, p);
    if (ROTATION != STAY && p.position < 0) return;         // (there are no turns for negative positions, and nothing is stored)
    for (uint32_t i = threadIdx.x; i < tiles; i += blockDim.x) {
        t.at(i, log_dims);
        t.load(in, token_stride, head * head_stride, p, turns);
        const uint32_t b = t.largest();
        a = a > b ? a : b;
    }
    if (number < 0) return;
    const size_t page_head = (size_t)(uint32_t)number * c.heads + head;
    uint8_t *codes = (V ? c.v_codes : c.k_codes) + page_head * values;
    uint8_t *scales = (V ? c.v_scales : c.k_scales) + page_head;
    const uint32_t kept = *scales, old = kept < 255 ? kept : 254;
    a = wave_max(a);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = a;
    __syncthreads();
    for (uint32_t i = 0; i < blockDim.x / 64; ++i) a = a > shared[i] ? a : shared[i];
    uint32_t byte = scale_byte(a);
    // slots before the first new one hold earlier tokens of the sequence, unless they are slots of negative positions
    const bool held = p.first > 0 && p.position >= 0;
    const bool move = held && byte > old;
    if (held && old > byte) byte = old;
    const float inverse = power_of(254 - byte), by = move ? power_of(127 - (byte - old > 126 ? 126 : byte - old)) : 1.0f;
    if (threadIdx.x == 0) *scales = (uint8_t)byte;
    for (uint32_t i = threadIdx.x; i < tiles; i += blockDim.x) {
        if (tiles > blockDim.x) {
            t.at(i, log_dims);
            t.load(in, token_stride, head * head_stride, p, turns);
        }
        t.store(codes, c.log_page, c.head_dim, p, inverse, move, by);
    }
}

struct NewTokens {
    const void *k, *v;
    size_t k_token, k_head, v_token, v_head;
};

template <int DT>
__global__ void __launch_bounds__(256) cache_write_kernel(Pages c, NewTokens n)
{
    __shared__ uint32_t shared[4];
    const Page p = page_of_item(c, blockIdx.x);
    if (!p.good) return;
    if (blockIdx.z == 0) write_page<DT, false>(c, p, blockIdx.y, n.k, n.k_token, n.k_head, shared);
    else write_page<DT, true>(c, p, blockIdx.y, n.v, n.v_token, n.v_head, shared);
}

// Queries of a page's tokens, a few heads to a workgroup.  A thread has a unit: both ends of eight pairs, so that a call may write where it reads, or eight
// values that stay; or, of neighbours, eight values.
struct Queries {
    const void *in;
    void *out;
    size_t in_token, in_head, out_token, out_head;
    uint32_t per_group;                     // heads that share a key
    Divide units;                           // of a head
};
constexpr uint32_t QUERY_HEADS = 4;         // of a workgroup
template <int DT, int ROTATION, int U>
__device__ __forceinline__ void turn_queries(const Pages &c, const Page &p, const Queries &q, const Turns &turns, uint32_t head, uint32_t heads)
{
    constexpr int PAIRS = ROTATION == HALVES ? 8 : 4;
    const uint32_t count = (p.end - p.first) * q.units.by * heads, half = turns.half;
    for (uint32_t first = threadIdx.x; first < count; first += U * blockDim.x) {
        float x[U][8], y[U][8], co[U][PAIRS], si[U][PAIRS];
        size_t to[U];
        uint32_t dim[U];
        bool turned[U];             // the unit is turned; of halves, both ends are the unit's
        // (loads that do not wait for one another, turns among them: asked for behind the values they cost 10 us of 45)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = first + u * blockDim.x < count ? first + u * blockDim.x : first, rest = quotient(i, q.units), unit = i - rest * q.units.by;
            const uint32_t token = rest / heads, h = head + rest - token * heads;
            const size_t from = (size_t)(p.token + p.first + token) * q.in_token + h * q.in_head;
            const int32_t position = p.position + (int32_t)(p.first + token);
            to[u] = (size_t)(p.token + p.first + token) * q.out_token + h * q.out_head;
            turned[u] = 8 * unit < (ROTATION == HALVES ? half : 2 * half);
            dim[u] = ROTATION == NEIGHBOURS || turned[u] ? 8 * unit : 8 * unit + half;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[u][k] = y[u][k] = 0;
#pragma unroll
            for (int k = 0; k < PAIRS; ++k) co[u][k] = si[u][k] = 0;
            if (position < 0) continue;                     // (zeros, turned or not)
            load8<DT>(q.in, from + dim[u], x[u]);
            if (turned[u]) {
                if (ROTATION == HALVES) load8<DT>(q.in, from + dim[u] + half, y[u]);
                load_turns(turns, position, ROTATION == HALVES ? dim[u] : dim[u] / 2, co[u], si[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (first + u * blockDim.x >= count) break;
            if (turned[u]) {
                if constexpr (ROTATION == NEIGHBOURS) {
                    turn_neighbours(co[u], si[u], x[u]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float a = x[u][k], b = y[u][k];
                        x[u][k] = a * co[u][k] - b * si[u][k], y[u][k] = b * co[u][k] + a * si[u][k];
                    }
                }
            }
            store8<DT>(q.out, to[u] + dim[u], x[u]);
            if (ROTATION == HALVES && turned[u]) store8<DT>(q.out, to[u] + dim[u] + half, y[u]);
        }
    }
}

// Keys, values and queries side by side in one launch: a page's heads follow one another, and for each of them its keys, its values, and the queries that share
// it, a few heads to a workgroup; so workgroups that run together have neighbouring memory (with the heads a grid's second axis prompts took 61.4 us instead of 59.1).
// Bound by HBM, and where few tokens are new by a chain of reads as in cache_write: starts, table, values and turns, scale and codes.  Prompts of up to 2047 tokens of eight sequences,
// 32 heads over 8 of 128, half of a head rotated, fp16, pages of 16: 58 us, of which the queries alone are 39 (26 at the rate of a large copy) and keys and values 20.  One token for each of
// 32 sequences, pages of 64: 7.8 us.
struct Order {
    Divide per_page, per_head;
    uint32_t blocks, per_row;       // all workgroups, and those of a row of the grid
};
template <int DT, int ROTATION>
__global__ void __launch_bounds__(256) cache_write_rotated_kernel(Pages c, NewTokens n, Queries q, Turns turns, Order order)
{
    __shared__ uint32_t shared[4];
    const uint32_t block = blockIdx.y * order.per_row + blockIdx.x;
    if (block >= order.blocks) return;
    const uint32_t item = quotient(block, order.per_page), within = block - item * order.per_page.by;
    const uint32_t head = quotient(within, order.per_head), part = within - head * order.per_head.by;
    const Page p = page_of_item(c, item, turns.positions);
    if (!p.good) return;
    if (part == 0) {
        write_page<DT, false, ROTATION>(c, p, head, n.k, n.k_token, n.k_head, shared, turns);
    } else if (part == 1) {
        write_page<DT, true>(c, p, head, n.v, n.v_token, n.v_head, shared);
    } else {
        const uint32_t first = (part - 2) * QUERY_HEADS, left = q.per_group - first;
        turn_queries<DT, ROTATION, 2>(c, p, q, turns, head * q.per_group + first, left < QUERY_HEADS ? left : QUERY_HEADS);
    }
}

// The way back, with the same tiles: two runs of 16 codes in, 32 values out, those of a token side by side over the threads.
template <int DT, bool V>
__device__ __forceinline__ void read_page(const Pages &c, const Page &p, uint32_t head, void *out, size_t token_stride, size_t head_stride)
{
    const int32_t number = number_of(c, p);
    const size_t page_head = (size_t)(uint32_t)(number < 0 ? 0 : number) * c.heads + head, values = (size_t)c.head_dim << c.log_page;
    const uint8_t *codes = (V ? c.v_codes : c.k_codes) + page_head * values;
    const float scale = number < 0 ? 0.0f : power_of((V ? c.v_scales : c.k_scales)[page_head]);
    const uint32_t log_dims = (uint32_t)__builtin_ctz(c.head_dim / (V ? 2u : 16u)), tiles = (uint32_t)(values / 32);
    for (uint32_t i = threadIdx.x; i < tiles; i += blockDim.x) {
        const uint32_t dim = (i & ((1u << log_dims) - 1)) * (V ? 2 : 16), slot = (i >> log_dims) * (V ? 16 : 2);
        if (slot >= p.end || slot + (V ? 16 : 2) <= p.first) continue;
        float x[2][16];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const size_t at = V ? ((size_t)(dim + r) << c.log_page) + slot : (size_t)(slot + r) * c.head_dim + dim;
            const u32x4 w = number < 0 ? u32x4{} : *reinterpret_cast<const u32x4 *>(codes + at);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], true);
                x[r][4 * j] = lo[0] * scale, x[r][4 * j + 1] = lo[1] * scale, x[r][4 * j + 2] = hi[0] * scale, x[r][4 * j + 3] = hi[1] * scale;
            }
        }
#pragma unroll
        for (int s = 0; s < (V ? 16 : 2); ++s) {
            if (slot + s < p.first || slot + s >= p.end) continue;
            const size_t at = (size_t)(p.token + slot + s) * token_stride + head * head_stride + dim;
            if constexpr (!V) {
                store8<DT>(out, at, *reinterpret_cast<const float(*)[8]>(x[s]));
                store8<DT>(out, at + 8, *reinterpret_cast<const float(*)[8]>(x[s] + 8));
            } else if constexpr (DT == FP32) {
                store1<DT>(out, at, x[0][s]);
                store1<DT>(out, at + 1, x[1][s]);
            } else {
                *reinterpret_cast<u32_a2 *>(static_cast<uint16_t *>(out) + at) = pack2<DT>(x[0][s], x[1][s]);
            }
        }
    }
}

struct Returned {
    void *k, *v;
    size_t k_token, k_head, v_token, v_head;
};

template <int DT>
__global__ void __launch_bounds__(256) cache_read_kernel(Pages c, Returned n)
{
    const Page p = page_of_item(c, blockIdx.x);
    if (!p.good) return;
    if (blockIdx.z == 0) read_page<DT, false>(c, p, blockIdx.y, n.k, n.k_token, n.k_head);
    else read_page<DT, true>(c, p, blockIdx.y, n.v, n.v_token, n.v_head);
}

}  // namespace lowbit
}  // namespace enec

using namespace enec::lowbit;

namespace enec {
namespace lowbit {

// argument checks that the calls on a cache share, and what its kernels take
int pages_of(const enec_cache *cache, const enec_cache_batch *batch, Pages &p)
{
    if (!cache || !batch) return ENEC_E_ARG;
    const uint32_t P = cache->page_tokens, D = cache->head_dim;
    if (P < 16 || P > 256 || (P & (P - 1)) || (D != 64 && D != 128 && D != 256)) return ENEC_E_BLOCK;
    if (cache->kv_heads == 0 || cache->kv_heads > 65535 || cache->n_pages == 0 || cache->n_pages > 0x7FFFFFFFu || batch->batch > 65535 || batch->n_tokens >= MAX_TOKENS)
        return ENEC_E_ARG;
    // (an empty batch needs no arrays)
    if (batch->batch && batch->n_tokens) {
        if (!cache->k_codes || !cache->v_codes || !cache->k_scales || !cache->v_scales || !batch->table || !batch->starts || !batch->lengths)
            return ENEC_E_ARG;
        if (((uintptr_t)cache->k_codes | (uintptr_t)cache->v_codes) & 15) return ENEC_E_ARG;
        if (((uintptr_t)batch->table | (uintptr_t)batch->starts | (uintptr_t)batch->lengths | (uintptr_t)batch->status) & 3) return ENEC_E_ARG;
        if (batch->table_stride == 0 || batch->table_stride > 0x7FFFFFFFu) return ENEC_E_ARG;
    }
    p.k_codes = static_cast<uint8_t *>(cache->k_codes), p.v_codes = static_cast<uint8_t *>(cache->v_codes);
    p.k_scales = static_cast<uint8_t *>(cache->k_scales), p.v_scales = static_cast<uint8_t *>(cache->v_scales);
    p.table = batch->table, p.starts = batch->starts, p.lengths = batch->lengths, p.status = batch->status;
    p.n_pages = cache->n_pages, p.log_page = (uint32_t)__builtin_ctz(P), p.heads = cache->kv_heads, p.head_dim = D;
    p.table_stride = batch->table_stride, p.batch = batch->batch, p.n_tokens = batch->n_tokens;
    return ENEC_OK;
}

}  // namespace lowbit
}  // namespace enec

// a thread for each tile of a page, in whole waves
static unsigned threads_of(const Pages &p)
{
    const unsigned tiles = (p.head_dim << p.log_page) / 32;
    return tiles < 64 ? 64 : tiles > 256 ? 256 : tiles;
}

extern "C" {

int enec_cache_write(const enec_cache *cache, const enec_cache_batch *batch, const void *k, size_t k_token_stride, size_t k_head_stride,
                     const void *v, size_t v_token_stride, size_t v_head_stride, int dtype, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16) return ENEC_E_DTYPE;
    Pages p;
    if (const int rc = pages_of(cache, batch, p)) return rc;
    if (p.batch == 0 || p.n_tokens == 0) return ENEC_OK;
    if (!k || !v || (((uintptr_t)k | (uintptr_t)v) & 1)) return ENEC_E_ARG;
    const dim3 grid((p.n_tokens >> p.log_page) + 2 * p.batch, p.heads, 2);
    auto kernel = dtype == ENEC_BF16 ? cache_write_kernel<BF16> : cache_write_kernel<FP16>;
    kernel<<<grid, threads_of(p), 0, (hipStream_t)stream>>>(p, NewTokens{k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride});
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

int enec_cache_write_rotated(const enec_cache *cache, const enec_cache_batch *batch, const void *k, size_t k_token_stride, size_t k_head_stride,
                             const void *v, size_t v_token_stride, size_t v_head_stride, const void *q, size_t q_token_stride, size_t q_head_stride,
                             void *q_out, size_t q_out_token_stride, size_t q_out_head_stride, uint32_t q_heads, int dtype, const void *turns,
                             uint32_t positions, uint32_t rotary, int interleaved, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16) return ENEC_E_DTYPE;
    Pages p;
    if (const int rc = pages_of(cache, batch, p)) return rc;
    if (rotary == 0 || rotary % 16 || rotary > p.head_dim) return ENEC_E_ARG;
    if (q_heads % p.heads || q_heads / p.heads > 65535 || (q_heads != 0) != (q != nullptr) || (q_heads != 0) != (q_out != nullptr)) return ENEC_E_ARG;
    if (q_heads && (((uintptr_t)q | (uintptr_t)q_out) & 1)) return ENEC_E_ARG;
    // in place a unit's thread has read what it writes; with other strides it would write what another reads
    if (q_heads && q == q_out && (q_token_stride != q_out_token_stride || q_head_stride != q_out_head_stride)) return ENEC_E_ARG;
    if (p.batch == 0 || p.n_tokens == 0) return ENEC_OK;
    if (!k || !v || !turns || (((uintptr_t)k | (uintptr_t)v) & 1) || ((uintptr_t)turns & 7)) return ENEC_E_ARG;
    const uint32_t group = q_heads / p.heads, units = interleaved ? p.head_dim / 8 : (p.head_dim - rotary / 2) / 8;
    const uint32_t parts = 2 + (group + QUERY_HEADS - 1) / QUERY_HEADS;
    const uint64_t blocks = ((uint64_t)(p.n_tokens >> p.log_page) + 2 * p.batch) * p.heads * parts;
    if (blocks >= (uint64_t)1 << 31) return ENEC_E_ARG;
    // (a grid's axis holds fewer than 2^32 threads, 256 a workgroup: what is more goes into further rows)
    constexpr uint32_t MOST_PER_ROW = (1u << 24) - 1;
    const uint32_t rows = (uint32_t)((blocks + MOST_PER_ROW - 1) / MOST_PER_ROW), per_row = (uint32_t)((blocks + rows - 1) / rows);
    auto kernel = dtype == ENEC_BF16 ? (interleaved ? cache_write_rotated_kernel<BF16, NEIGHBOURS> : cache_write_rotated_kernel<BF16, HALVES>)
                                     : (interleaved ? cache_write_rotated_kernel<FP16, NEIGHBOURS> : cache_write_rotated_kernel<FP16, HALVES>);
    kernel<<<dim3(per_row, rows), threads_of(p), 0, (hipStream_t)stream>>>(
        p, NewTokens{k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride},
        Queries{q, q_out, q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride, group, divide_by(units)},
        Turns{static_cast<const float *>(turns), rotary / 2, positions < (uint32_t)MAX_SEQUENCE ? (int32_t)positions : MAX_SEQUENCE},
        Order{divide_by(p.heads * parts), divide_by(parts), (uint32_t)blocks, per_row});
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

int enec_cache_read(const enec_cache *cache, const enec_cache_batch *batch, void *k, size_t k_token_stride, size_t k_head_stride, void *v,
                    size_t v_token_stride, size_t v_head_stride, int dtype, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    Pages p;
    if (const int rc = pages_of(cache, batch, p)) return rc;
    if (p.batch == 0 || p.n_tokens == 0) return ENEC_OK;
    if (!k || !v || (((uintptr_t)k | (uintptr_t)v) & (dtype == ENEC_FP32 ? 3 : 1))) return ENEC_E_ARG;
    const dim3 grid((p.n_tokens >> p.log_page) + 2 * p.batch, p.heads, 2);
    auto kernel = dtype == ENEC_BF16 ? cache_read_kernel<BF16> : dtype == ENEC_FP16 ? cache_read_kernel<FP16> : cache_read_kernel<FP32>;
    kernel<<<grid, threads_of(p), 0, (hipStream_t)stream>>>(p, Returned{k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride});
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
