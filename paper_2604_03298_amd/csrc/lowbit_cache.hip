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
// the byte of the smallest power of two 2^e with a <= 448 2^e, 448 = 1.75 * 2^8: one exponent more where the mantissa is over 1.75.
// Below 2^-126 the exponent field says 0 where the exponent is smaller still; both give the least scale.
__device__ __forceinline__ uint32_t scale_byte(uint32_t a)
{
    const int32_t e = (int32_t)(a >> 23) - 8 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e > 0 ? (uint32_t)e : 0;
}

// what an item's workgroup knows of its page
struct Page {
    uint32_t first, end;        // slots of the page that the call's tokens have
    uint32_t token;             // the call's token in slot 0 (may lie before the sequence's first one: mod 2^32)
    int32_t position;           // of slot 0
    const int32_t *entry;       // where its number is; null: it has none
    bool good;
};
__device__ __forceinline__ Page page_of_item(const Pages &c, uint32_t item)
{
    const Found f = sequence_of_item(c, item);
    const Sequence &s = f.s;
    Page p{};
    if (f.b < 0) return p;
    if (!s.good) {
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

// A workgroup has one page of one head, keys or values: it alone knows all tokens that the scale depends on, and nothing is
// shared between workgroups.  Tiles of 32 values: keys 2 tokens x 16 dimensions, values 16 tokens x 2 dimensions, so that
// both ways a thread's codes are two runs of 16 bytes; consecutive threads have consecutive dimensions, so that the loads of a
// token are one run.  The tiles stay in registers between finding the scale and writing; pages of more than 8192 values are read
// twice (the second time from the cache).
// Bound by HBM for prompts (3 bytes a bf16 value) and by its chain of dependent reads for single tokens: starts and lengths, table
// beside the new values, old scale, old codes.  (The last two need not wait for one another: asked for together they would shorten it; before the new values
// they cost prompts 19 -> 25 us.)  A workgroup has a thread for each tile, 64 to 256.
// Eight prompts of up to 2047 tokens, 8 heads of 128, fp16, pages of 16: 18.7 us, 14.5 back.  One token for each of 32 sequences, pages of 64: 7.9 us.
template <int DT, bool V> struct Tile {
    uint32_t slot, dim;         // first slot and dimension
    float x[32];
    static constexpr int SLOTS = V ? 16 : 2, DIMS = V ? 2 : 16;
    __device__ __forceinline__ void at(uint32_t t, uint32_t log_dims)         // log_dims: of the tiles side by side
    {
        dim = (t & ((1u << log_dims) - 1)) * DIMS;
        slot = (t >> log_dims) * SLOTS;
    }
    __device__ __forceinline__ void load(const void *in, size_t token_stride, size_t head, const Page &p)
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
                    load8<DT>(in, i, *reinterpret_cast<float(*)[8]>(u));
                    load8<DT>(in, i + 8, *reinterpret_cast<float(*)[8]>(u + 8));
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

template <int DT, bool V>
__device__ __forceinline__ void write_page(const Pages &c, const Page &p, uint32_t head, const void *in, size_t token_stride, size_t head_stride,
                                           uint32_t *shared)
{
    const size_t values = (size_t)c.head_dim << c.log_page;
    const uint32_t log_dims = (uint32_t)__builtin_ctz(c.head_dim / (V ? 2u : 16u)), tiles = (uint32_t)(values / 32);
    Tile<DT, V> t;
    uint32_t a = 0;
    const int32_t number = number_of(c, p);
    for (uint32_t i = threadIdx.x; i < tiles; i += blockDim.x) {
        t.at(i, log_dims);
        t.load(in, token_stride, head * head_stride, p);
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
            t.load(in, token_stride, head * head_stride, p);
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
