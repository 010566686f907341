// Attention over the paged 8-bit cache.  The definition stands in include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit_pages.hpp"

namespace enec {
namespace lowbit {

int pages_of(const enec_cache *cache, const enec_cache_batch *batch, Pages &p);

struct Attend {
    Pages c;
    const void *q;
    void *out;
    size_t q_token, q_head, out_token, out_head;
    uint32_t q_heads;
    Divide group;                       // query heads of a key head
    float scale;                        // with log2 e: exponentials are powers of two
    uint32_t max_new, max_length, chunk, splits, row_tiles;
    float *part, *part_stat;            // per split, token and head: a sum over its tokens, and (maximum, sum of weights)
};

__device__ __forceinline__ Sequence sequence_of(const Attend &a, uint32_t b)
{
    Sequence s = sequence_of(a.c, b, (int32_t)a.max_length);
    s.good = s.good && s.count <= a.max_new;
    return s;
}

__device__ __forceinline__ float over_groups_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_groups_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

template <int DT> __device__ __forceinline__ f32x4 mfma16(const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    if constexpr (DT == BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// eight E4M3 codes as values of the 16-bit format: all of them are numbers of it (bf16: also with a power of two)
template <int DT> __device__ __forceinline__ u32x4 values8(uint32_t lo, uint32_t hi, float scale)
{
    u32x4 r;
    if constexpr (DT == BF16) {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
    } else {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true));
    }
    return r;
}

// bytes of a word of codes that are NaN, as 0xFF
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w)
{
    uint32_t r = 0;
    for (int k = 0; k < 4; ++k) r |= (w >> (8 * k) & 0x7F) == 0x7F ? 255u << (8 * k) : 0;
    return r;
}

// Scores are computed transposed: tokens are the rows of the matrix instruction (left operand: keys), query rows its columns.  A lane then
// holds scores of one query row, and with the tokens of a tile of 64 dealt out as
//     instruction j, row r: token 16 (r / 4) + 4 j + r mod 4
// lane group g has tokens 16 g ... 16 g + 15, which is what the product with the values wants of it as right operand: weights
// go from one product to the next without leaving their lane.  Left operand there are the transposed values, 16 dimensions x
// 16 consecutive tokens a lane: one run of 16 bytes.  A run of 16 keys' bytes is two steps of the first product, whose order of
// dimensions is the same for the queries.
// Query rows are pairs of (token, head of the key head's group), 16 to a workgroup; its four waves take every fourth tile and
// meet in LDS.
template <int DT, int D>
__global__ void __launch_bounds__(256) attend_kernel(Attend a)
{
    constexpr int KC = D / 64, VT = D / 16;
    __shared__ float stat[2][4][16];
    __shared__ f32x4 sums[4][16][17];
    const Pages &c = a.c;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const uint32_t split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits, b = rest / a.row_tiles, head = blockIdx.y;
    const Sequence s = sequence_of(a, b);
    if (!s.good) {
        complain(c);
        return;
    }
    const uint32_t rows = s.count * a.group.by, row0 = rest % a.row_tiles * 16;
    if (row0 >= rows) return;
    const int32_t begin = s.length - (int32_t)s.count;
    const uint32_t row = row0 + col;
    const uint32_t token = quotient(row, a.group), q_head = head * a.group.by + (row - token * a.group.by);
    const int32_t limit = row < rows ? begin + (int32_t)token : -1;           // the last position that the row sees
    const int32_t least = begin + (int32_t)quotient(row0, a.group);           // of all rows here
    const uint32_t last_row = row0 + 15 < rows ? row0 + 15 : rows - 1;
    const int32_t end = begin + (int32_t)quotient(last_row, a.group) + 1;     // none sees a position from here on
    const int32_t from = (int32_t)(split * a.chunk), to = end - from < (int32_t)a.chunk ? end : from + (int32_t)a.chunk;
    if (split > 0 && from >= to) return;

    u32x4 q[KC][2] = {};
    if (row < rows) {
        const uint16_t *p = static_cast<const uint16_t *>(a.q) + (size_t)(s.start + token) * a.q_token + (size_t)q_head * a.q_head;
#pragma unroll
        for (int i = 0; i < KC; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) q[i][h] = *reinterpret_cast<const u32x4_a2 *>(p + 64 * i + 16 * g + 8 * h);
    }
    f32x4 o[VT] = {};
    float most = -__builtin_inff(), total = 0;
    const uint32_t page_mask = (1u << c.log_page) - 1;
    const size_t head_values = (size_t)D << c.log_page;
    const int32_t *table = c.table + (size_t)b * c.table_stride;

    for (int32_t t0 = from + 64 * (int32_t)wave; t0 < to; t0 += 256) {
        // the pages of the 16 tokens that this lane loads keys of, and of those that it loads values of
        const int32_t tk = t0 + 16 * (int32_t)(col >> 2), tv = t0 + 16 * (int32_t)g;
        int32_t pk = tk < s.length ? table[tk >> c.log_page] : -1, pv = tv < s.length ? table[tv >> c.log_page] : -1;
        if ((uint32_t)pk >= c.n_pages) {
            if (tk < s.length) complain(c);
            pk = -1;
        }
        if ((uint32_t)pv >= c.n_pages) pv = -1;
        const uint8_t *kp = c.k_codes + ((size_t)(uint32_t)(pk < 0 ? 0 : pk) * c.heads + head) * head_values + (size_t)((tk & page_mask) + (col & 3)) * D + 16 * g;
        const uint8_t *vp = c.v_codes + ((size_t)(uint32_t)(pv < 0 ? 0 : pv) * c.heads + head) * head_values + ((size_t)col << c.log_page) + (tv & page_mask);
        u32x4 k[4][KC] = {}, v[VT] = {};
        float ks = 0, vs = 0;
        if (pk >= 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < KC; ++i) k[j][i] = *reinterpret_cast<const u32x4 *>(kp + 4 * j * D + 64 * i);
        }
        if (pv >= 0) {
            ks = power_of(c.k_scales[(size_t)pv * c.heads + head]);
            vs = power_of(c.v_scales[(size_t)pv * c.heads + head]);
#pragma unroll
            for (int i = 0; i < VT; ++i) v[i] = *reinterpret_cast<const u32x4 *>(vp + ((size_t)(16 * i) << c.log_page));
        }
        f32x4 x[4] = {};
#pragma unroll
        for (int i = 0; i < KC; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = mfma16<DT>(values8<DT>(k[j][i][2 * h], k[j][i][2 * h + 1], 1.0f), q[i][h], x[j]);
        // what a row does not see takes no part, whatever its codes are
        ks *= a.scale;
        float high = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[j][i] = pv >= 0 && tv + 4 * j + i <= limit ? x[j][i] * ks : -__builtin_inff();
                high = fmaxf(high, x[j][i]);
            }
        const float now = fmaxf(most, over_groups_max(high)), base = now == -__builtin_inff() ? 0.0f : now;
        const float fade = exp2_of(most - base);
        most = now;
        total *= fade;
#pragma unroll
        for (int i = 0; i < VT; ++i) o[i] *= fade;
        float w[16];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[4 * j + i] = exp2_of(x[j][i] - base);
                total += w[4 * j + i];
            }
        // codes behind the sequence's end are anyone's
        if (t0 + 64 > s.length) {
            const int32_t n = s.length - tv;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t here = n - 4 * j;
                const uint32_t mask = here >= 4 ? 0xFFFFFFFFu : here <= 0 ? 0 : (1u << (8 * here)) - 1;
#pragma unroll
                for (int i = 0; i < VT; ++i) v[i][j] &= mask;
            }
        }
        // A value that is NaN has to reach the rows that see it, and no other: 0 * NaN would.  Where some rows do not see the whole tile,
        // such values are taken out and the rows that see one are told.
        if (t0 + 63 > least) {
            uint32_t any = 0;
#pragma unroll
            for (int i = 0; i < VT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) any |= nan_bytes(v[i][j]);
            if (__any(any)) {
                u32x4 sees[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int32_t at = tv + 8 * h + 2 * j;
                        sees[h][j] = (at <= limit ? 0x3F80u : 0) | (at + 1 <= limit ? 0x3F800000u : 0);
                    }
#pragma unroll
                for (int i = 0; i < VT; ++i) {
                    f32x4 seen = {};
                    u32x4 bad;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t n = nan_bytes(v[i][j]);
                        v[i][j] &= ~n;
                        bad[j] = n & 0x38383838u;            // 1.0 as E4M3
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) seen = mfma16<BF16>(values8<BF16>(bad[2 * h], bad[2 * h + 1], 1.0f), sees[h], seen);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][e] = seen[e] > 0 ? __builtin_nanf("") : o[i][e];
                }
            }
        }
        u32x4 p[2], rest_of[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float lo = w[8 * h + 2 * j], hi = w[8 * h + 2 * j + 1];
                p[h][j] = pack2<BF16>(lo, hi);
                if constexpr (DT == FP16) {
                    const f32x2 r = unpack2<BF16>(p[h][j]);
                    rest_of[h][j] = pack2<BF16>(lo - r[0], hi - r[1]);
                }
            }
#pragma unroll
        for (int i = 0; i < VT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 values = values8<BF16>(v[i][2 * h], v[i][2 * h + 1], vs);
                o[i] = mfma16<BF16>(values, p[h], o[i]);
                if constexpr (DT == FP16) o[i] = mfma16<BF16>(values, rest_of[h], o[i]);
            }
    }

    // the waves' sums, in their order
    total = over_groups_sum(total);
    if (g == 0) stat[0][wave][col] = most, stat[1][wave][col] = total;
    __syncthreads();
    float top = stat[0][0][col];
    for (int i = 1; i < 4; ++i) top = fmaxf(top, stat[0][i][col]);
    const float mine = most == -__builtin_inff() ? 0.0f : exp2_of(most - top);
    // thread: row r of the tile, four dimensions of every 64
    const uint32_t r = threadIdx.x >> 4, d4 = threadIdx.x & 15;
    float row_top = stat[0][0][r], row_total = 0;
    for (int i = 1; i < 4; ++i) row_top = fmaxf(row_top, stat[0][i][r]);
    for (int i = 0; i < 4; ++i) row_total += stat[0][i][r] == -__builtin_inff() ? 0.0f : stat[1][i][r] * exp2_of(stat[0][i][r] - row_top);
    const uint32_t out_row = row0 + r, out_token = quotient(out_row, a.group), out_head = head * a.group.by + (out_row - out_token * a.group.by);
#pragma unroll
    for (int i = 0; i < KC; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[wave][col][4 * e + g] = o[4 * i + e] * mine;
        __syncthreads();
        f32x4 v = sums[0][r][d4];
        for (int w = 1; w < 4; ++w) v += sums[w][r][d4];
        if (out_row >= rows) continue;
        const uint32_t d = 64 * i + 4 * d4;
        if (a.splits == 1) {
            const float by = row_total == 0 ? 0.0f : 1.0f / row_total;
            uint16_t *p = static_cast<uint16_t *>(a.out) + (size_t)(s.start + out_token) * a.out_token + (size_t)out_head * a.out_head + d;
            *reinterpret_cast<u32x2_a2 *>(p) = u32x2{pack2<DT>(v[0] * by, v[1] * by), pack2<DT>(v[2] * by, v[3] * by)};
        } else {
            const size_t at = ((size_t)split * c.n_tokens + s.start + out_token) * a.q_heads + out_head;
            *reinterpret_cast<f32x4 *>(a.part + at * D + d) = v;
            if (i == 0 && d4 == 0) *reinterpret_cast<f32x2 *>(a.part_stat + 2 * at) = f32x2{row_top, row_total};
        }
    }
}

// The splits of a row, in their order: one wave a row.
template <int DT, int D>
__global__ void __launch_bounds__(64) attend_join_kernel(Attend a)
{
    constexpr int N = D / 64;
    const uint32_t lane = threadIdx.x, token = blockIdx.x, q_head = blockIdx.y;
    // the token's sequence: the last one that starts at or before it
    uint32_t n = 0;
    for (uint32_t b = 0; b < a.c.batch; b += 64) n += (uint32_t)__popcll(__ballot(b + lane < a.c.batch && a.c.starts[b + lane] <= (int32_t)token));
    if (n == 0) return;
    const Sequence s = sequence_of(a, n - 1);
    if (!s.good || token - s.start >= s.count) return;
    const int32_t sees = s.length - (int32_t)s.count + (int32_t)(token - s.start) + 1;
    const uint32_t splits = sees <= 0 ? 1 : ((uint32_t)sees + a.chunk - 1) / a.chunk;
    const size_t at = (size_t)token * a.q_heads + q_head, step = (size_t)a.c.n_tokens * a.q_heads;
    float top = -__builtin_inff(), total = 0, o[N] = {};
    for (uint32_t i = 0; i < splits; ++i) top = fmaxf(top, a.part_stat[2 * (at + i * step)]);
    for (uint32_t i = 0; i < splits; ++i) {
        const size_t j = at + i * step;
        const float high = a.part_stat[2 * j], w = high == -__builtin_inff() ? 0.0f : exp2_of(high - top);
        total += w * a.part_stat[2 * j + 1];
        for (int e = 0; e < N; ++e) o[e] += w * a.part[j * D + N * lane + e];
    }
    const float by = total == 0 ? 0.0f : 1.0f / total;
    for (int e = 0; e < N; ++e)
        store1<DT>(a.out, (size_t)token * a.out_token + (size_t)q_head * a.out_head + N * lane + e, o[e] * by);
}

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

struct Plan {
    uint32_t row_tiles, chunk, splits;
};
// How a call is cut up.  A sequence's cached tokens are split where rows and heads alone leave the card empty.
Plan plan_of(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t max_new, uint32_t max_length)
{
    Plan p;
    p.row_tiles = (uint32_t)(((uint64_t)max_new * group + 15) / 16);
    const uint64_t others = (uint64_t)batch * kv_heads * p.row_tiles;
    const uint64_t want = others >= 1024 ? 1 : (1024 + others - 1) / others;
    const uint64_t tokens = (max_length + want - 1) / want;
    p.chunk = (uint32_t)(tokens <= 256 ? 256 : (tokens + 255) / 256 * 256);
    p.splits = max_length <= p.chunk ? 1 : (max_length + p.chunk - 1) / p.chunk;
    return p;
}

template <int DT, int D> void launch(const Attend &a, hipStream_t s)
{
    attend_kernel<DT, D><<<dim3(a.splits * a.c.batch * a.row_tiles, a.c.heads), 256, 0, s>>>(a);
    if (a.splits > 1) attend_join_kernel<DT, D><<<dim3(a.c.n_tokens, a.q_heads), 64, 0, s>>>(a);
}
template <int DT> void launch(const Attend &a, hipStream_t s)
{
    if (a.c.head_dim == 64) launch<DT, 64>(a, s);
    else if (a.c.head_dim == 128) launch<DT, 128>(a, s);
    else launch<DT, 256>(a, s);
}

// one call's arguments; 0 = none of its kernels can count with these
bool shape_ok(const enec_cache *cache, uint32_t batch, uint32_t n_tokens, uint32_t q_heads, uint32_t max_new, uint32_t max_length)
{
    if (cache->kv_heads == 0 || q_heads == 0 || q_heads > 65535 || q_heads % cache->kv_heads || max_length > (uint32_t)MAX_SEQUENCE) return false;
    const uint64_t rows = (uint64_t)max_new * (q_heads / cache->kv_heads);
    return rows < (1u << 30) && n_tokens <= 0x7FFFFFFFu && batch <= 65535;
}

}  // namespace

extern "C" {

size_t enec_cache_attention_workspace(const enec_cache *cache, uint32_t batch, uint32_t n_tokens, uint32_t q_heads, uint32_t max_new, uint32_t max_length)
{
    if (!cache || !shape_ok(cache, batch, n_tokens, q_heads, max_new, max_length) || batch == 0 || n_tokens == 0 || max_new == 0) return 0;
    const Plan p = plan_of(batch, cache->kv_heads, q_heads / cache->kv_heads, max_new, max_length);
    return p.splits == 1 ? 0 : (size_t)p.splits * n_tokens * q_heads * (cache->head_dim + 2) * sizeof(float);
}

int enec_cache_attention(const enec_cache *cache, const enec_cache_batch *batch, const void *q, size_t q_token_stride, size_t q_head_stride, void *out,
                         size_t out_token_stride, size_t out_head_stride, int dtype, uint32_t q_heads, uint32_t max_new, uint32_t max_length,
                         float scale, void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16) return ENEC_E_DTYPE;
    Attend a;
    if (const int rc = pages_of(cache, batch, a.c)) return rc;
    if (!shape_ok(cache, a.c.batch, a.c.n_tokens, q_heads, max_new, max_length)) return ENEC_E_ARG;
    if (a.c.batch == 0 || a.c.n_tokens == 0) return ENEC_OK;
    if (!q || !out || (((uintptr_t)q | (uintptr_t)out) & 1) || max_new == 0) return ENEC_E_ARG;
    const uint32_t group = q_heads / a.c.heads;
    const Plan p = plan_of(a.c.batch, a.c.heads, group, max_new, max_length);
    if ((uint64_t)p.splits * a.c.batch * p.row_tiles > 0x7FFFFFFFu) return ENEC_E_ARG;
    const size_t need = enec_cache_attention_workspace(cache, a.c.batch, a.c.n_tokens, q_heads, max_new, max_length);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && ((uintptr_t)workspace & 15)) return ENEC_E_ARG;
    a.q = q, a.out = out;
    a.q_token = q_token_stride, a.q_head = q_head_stride, a.out_token = out_token_stride, a.out_head = out_head_stride;
    a.q_heads = q_heads, a.group = divide_by(group), a.scale = scale * 1.44269504088896340736f;
    a.max_new = max_new, a.max_length = max_length, a.chunk = p.chunk, a.splits = p.splits, a.row_tiles = p.row_tiles;
    a.part = static_cast<float *>(workspace);
    a.part_stat = a.part + (size_t)p.splits * a.c.n_tokens * q_heads * a.c.head_dim;
    if (dtype == ENEC_BF16) launch<BF16>(a, (hipStream_t)stream);
    else launch<FP16>(a, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
