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

// ---- many rows ---------------------------------------------------------------------------------------------------------

// Keys and values of a tile of 64 tokens in LDS, two tiles in turn, as codes: a token's keys are a row of D / 16 chunks of 16 bytes, a
// dimension's values a row of four.  Chunk i of a row lies at place i ^ turn: the sixteen lanes whose 16 bytes are read in one go (rows {0-3, 12-15} of a
// lane group and rows {4-11} of its neighbour) find theirs in sixteen different places of 256 bytes.
template <int D> __device__ __forceinline__ uint32_t key_turn(uint32_t token)
{
    const uint32_t half = token >> 5 & 1;
    if constexpr (D == 64) return 2 * half;
    if constexpr (D == 128) return (token & 2) + 4 * half;
    return 2 * (token & 3) + 8 * half;
}
__device__ __forceinline__ uint32_t value_turn(uint32_t dim) { return 2 * (dim >> 3 & 1); }

// The same arrangement as above, with 16 NT query rows to each of the four waves, which share the tiles: a wave has all of them, so nothing is
// joined in the end.  The memory unit copies the codes of a tile into LDS while the one before is worked on.  Every wave makes
// 16-bit values of the codes by itself: a conversion makes two of them in the time of any vector instruction, and NT tiles of rows use each.
template <int DT, int D, int NT>
__global__ void __launch_bounds__(256, 2) attend_many_kernel(Attend a)
{
    constexpr int KC = D / 64, VT = D / 16, COPIES = D / 64, ROWS = 64 * NT;
    __shared__ __attribute__((aligned(16))) uint8_t keys[2][64 * D], values[2][64 * D];
    const Pages &c = a.c;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    // Workgroups are dealt out to the eight dies one by one.  Each die takes a run of (sequence, head)s, whose keys and values stay in its cache,
    // and of their rows the last ones first: they see most.
    const uint32_t groups = c.batch * c.heads, each = a.row_tiles * a.splits, total_tiles = groups * each, per_die = (total_tiles + 7) / 8;
    const uint32_t tile = blockIdx.x % 8 * per_die + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per_die || tile >= total_tiles) return;
    const uint32_t group = tile / each, within = tile % each, b = group / c.heads, head = group % c.heads;
    const uint32_t split = within % a.splits, row_tile = a.row_tiles - 1 - within / a.splits;
    const Sequence s = sequence_of(a, b);
    if (!s.good) {
        complain(c);
        return;
    }
    const uint32_t rows = s.count * a.group.by, first_row = row_tile * ROWS;
    if (first_row >= rows) return;
    const int32_t begin = s.length - (int32_t)s.count;
    const uint32_t last_row = first_row + ROWS < rows ? first_row + ROWS - 1 : rows - 1;
    const int32_t end = begin + (int32_t)quotient(last_row, a.group) + 1;     // no row here sees a position from here on
    const int32_t from = (int32_t)(split * a.chunk), to = end - from < (int32_t)a.chunk ? end : from + (int32_t)a.chunk;
    if (split > 0 && from >= to) return;

    const uint32_t row0 = first_row + wave * (16 * NT);
    uint32_t token[NT], q_head[NT];
    int32_t limit[NT];                                                        // the last position that the row sees
    u32x4 q[NT][KC][2] = {};
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t row = row0 + 16 * n + col;
        token[n] = quotient(row, a.group), q_head[n] = head * a.group.by + (row - token[n] * a.group.by);
        limit[n] = row < rows ? begin + (int32_t)token[n] : -1;
        if (row < rows) {
            const uint16_t *p = static_cast<const uint16_t *>(a.q) + (size_t)(s.start + token[n]) * a.q_token + (size_t)q_head[n] * a.q_head;
#pragma unroll
            for (int i = 0; i < KC; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) q[n][i][h] = *reinterpret_cast<const u32x4_a2 *>(p + 64 * i + 16 * g + 8 * h);
        }
    }
    // of this wave's rows: what the first sees, and where the last one's view ends (none: nothing)
    const int32_t least = row0 < rows ? begin + (int32_t)quotient(row0, a.group) : 0;
    const uint32_t my_last = row0 + 16 * NT - 1 < last_row ? row0 + 16 * NT - 1 : last_row;
    const int32_t my_end = row0 < rows ? begin + (int32_t)quotient(my_last, a.group) + 1 : 0;

    f32x4 o[NT][VT] = {};
    float most[NT], total[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) most[n] = -__builtin_inff(), total[n] = 0;
    const uint32_t page_mask = (1u << c.log_page) - 1;
    const size_t head_values = (size_t)D << c.log_page;
    const int32_t *table = c.table + (size_t)b * c.table_stride;

    // The page of 16 tokens from position t on, -1 where there is none.  Copies from no page take page 0, which exists, and are not looked at.
    auto page_at = [&](int32_t t) {
        const int32_t p = t < s.length ? table[t >> c.log_page] : -1;
        if ((uint32_t)p < c.n_pages) return p;
        if (t < s.length) complain(c);
        return -1;
    };
    // wave w copies the keys of 16 tokens and a quarter of the dimensions' values
    const uint32_t value_group = (lane & 3) ^ value_turn(lane >> 2);
    auto copy = [&](int32_t t0, int buffer, int32_t key_page, int32_t value_page) {
        using from_t = const __attribute__((address_space(1))) void *;
        using to_t = __attribute__((address_space(3))) void *;
        const uint8_t *k = c.k_codes + ((size_t)(uint32_t)(key_page < 0 ? 0 : key_page) * c.heads + head) * head_values + (size_t)((t0 + 16 * wave) & page_mask) * D;
        const uint8_t *v = c.v_codes + ((size_t)(uint32_t)(value_page < 0 ? 0 : value_page) * c.heads + head) * head_values + ((t0 + 16 * value_group) & page_mask);
#pragma unroll
        for (int r = 0; r < COPIES; ++r) {
            const uint32_t place = r * 64 + lane, row = place / (D / 16), chunk = place % (D / 16) ^ key_turn<D>(16 * wave + row);
            __builtin_amdgcn_global_load_lds((from_t)(k + row * D + 16 * chunk), (to_t)(keys[buffer] + 16 * wave * D + r * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < COPIES; ++r) {
            const uint32_t dim = (wave * COPIES + r) * 16 + (lane >> 2);
            __builtin_amdgcn_global_load_lds((from_t)(v + ((size_t)dim << c.log_page)), (to_t)(values[buffer] + (wave * COPIES + r) * 1024), 16, 0, 0);
        }
    };
    uint32_t key_at[4], value_at = col * 64 + ((g ^ value_turn(col)) << 4);
#pragma unroll
    for (int i = 0; i < KC; ++i) {
        const uint32_t t = 16 * (col >> 2) + (col & 3);                       // (+ 4 j, which does not turn)
        key_at[i] = t * D + (((4 * i + g) ^ key_turn<D>(t)) << 4);
    }

    int32_t page = page_at(from + 16 * (int32_t)g), next_page = -1;           // of the tokens that this lane has weights of
    {
        const int32_t kp = page_at(from + 16 * (int32_t)wave), vp = page_at(from + 16 * (int32_t)value_group);
        if (from < to) copy(from, 0, kp, vp);
    }
    auto scales_of = [&](int32_t p, float &k, float &v) {
        const size_t at = (size_t)(uint32_t)(p < 0 ? 0 : p) * c.heads + head;
        k = power_of(c.k_scales[at]), v = power_of(c.v_scales[at]);
    };
    float ks, vs, next_ks = 0, next_vs = 0;
    scales_of(page, ks, vs);
    int32_t next_kp = page_at(from + 64 + 16 * (int32_t)wave), next_vp = page_at(from + 64 + 16 * (int32_t)value_group);
    next_page = page_at(from + 64 + 16 * (int32_t)g);

    int buffer = 0;
    for (int32_t t0 = from; t0 < to; t0 += 64, buffer ^= 1) {
        __builtin_amdgcn_sched_barrier(0);
        // this wave's copies are in LDS, then all waves' are, and nobody reads the tile before any more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        int32_t far_page = -1, far_kp = -1, far_vp = -1;
        if (t0 + 64 < to) {
            copy(t0 + 64, buffer ^ 1, next_kp, next_vp);
            scales_of(next_page, next_ks, next_vs);
            far_page = page_at(t0 + 128 + 16 * (int32_t)g);
            far_kp = page_at(t0 + 128 + 16 * (int32_t)wave);
            far_vp = page_at(t0 + 128 + 16 * (int32_t)value_group);
        }
        if (t0 < my_end) {
            const int32_t tv = t0 + 16 * (int32_t)g;
            const bool partial = t0 + 63 > least || t0 + 64 > s.length || __any(page < 0);
            f32x4 x[NT][4] = {};
#pragma unroll
            for (int i = 0; i < KC; ++i) {
                u32x4 k[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const u32x4 *>(keys[buffer] + key_at[i] + 4 * j * D);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const u32x4 v = values8<DT>(k[j][2 * h], k[j][2 * h + 1], 1.0f);
#pragma unroll
                        for (int n = 0; n < NT; ++n) x[n][j] = mfma16<DT>(v, q[n][i][h], x[n][j]);
                    }
            }
            const float by = ks * a.scale;
            u32x4 p[NT][2], rest_of[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (partial) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[n][j][i] = page >= 0 && tv + 4 * j + i <= limit[n] ? x[n][j][i] * by : -__builtin_inff();
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[n][j] *= by;
                }
                float high = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) high = fmaxf(high, x[n][j][i]);
                high = over_groups_max(high);
                // Weights are taken relative to a maximum that may lag behind by up to 2^8, which costs nothing in 32 bits: most tiles need no
                // change of what is summed already.
                if (__any(high > most[n] + 8.0f)) {
                    const float now = fmaxf(most[n], high), fade = now == -__builtin_inff() ? 1.0f : exp2_of(most[n] - now);
                    most[n] = now;
                    total[n] *= fade;
#pragma unroll
                    for (int i = 0; i < VT; ++i) o[n][i] *= fade;
                }
                const float base = most[n] == -__builtin_inff() ? 0.0f : most[n];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float lo = exp2_of(x[n][2 * h + j / 2][2 * (j & 1)] - base), hi = exp2_of(x[n][2 * h + j / 2][2 * (j & 1) + 1] - base);
                        total[n] += lo;
                        total[n] += hi;
                        p[n][h][j] = pack2<BF16>(lo, hi);
                        if constexpr (DT == FP16) {
                            const f32x2 r = unpack2<BF16>(p[n][h][j]);
                            rest_of[n][h][j] = pack2<BF16>(lo - r[0], hi - r[1]);
                        }
                    }
            }
            // in a tile that not every row sees whole: bytes behind the sequence's end and of no page are anyone's, and a NaN is
            // told to the rows that see it, as above
            uint32_t mask[4] = {~0u, ~0u, ~0u, ~0u};
            bool careful = false;
            if (partial) {
                uint32_t any = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int32_t here = s.length - tv - 4 * j;
                    mask[j] = page < 0 || here <= 0 ? 0 : here >= 4 ? ~0u : (1u << (8 * here)) - 1;
                }
                for (int i = 0; i < VT; ++i) {
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(values[buffer] + value_at + i * 1024);
                    for (int j = 0; j < 4; ++j) any |= nan_bytes(v[j] & mask[j]);
                }
                careful = __any(any);
            }
#pragma unroll
            for (int i = 0; i < VT; ++i) {
                u32x4 v = *reinterpret_cast<const u32x4 *>(values[buffer] + value_at + i * 1024);
                if (partial) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] &= mask[j];
                    if (careful) {
                        u32x4 bad;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t nan = nan_bytes(v[j]);
                            v[j] &= ~nan;
                            bad[j] = nan & 0x38383838u;              // 1.0 as E4M3
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            f32x4 seen = {};
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                u32x4 sees;
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const int32_t at = tv + 8 * h + 2 * j;
                                    sees[j] = (at <= limit[n] ? 0x3F80u : 0) | (at + 1 <= limit[n] ? 0x3F800000u : 0);
                                }
                                seen = mfma16<BF16>(values8<BF16>(bad[2 * h], bad[2 * h + 1], 1.0f), sees, seen);
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[n][i][e] = seen[e] > 0 ? __builtin_nanf("") : o[n][i][e];
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u32x4 vv = values8<BF16>(v[2 * h], v[2 * h + 1], vs);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        o[n][i] = mfma16<BF16>(vv, p[n][h], o[n][i]);
                        if constexpr (DT == FP16) o[n][i] = mfma16<BF16>(vv, rest_of[n][h], o[n][i]);
                    }
                }
            }
        }
        page = next_page, ks = next_ks, vs = next_vs;
        next_page = far_page, next_kp = far_kp, next_vp = far_vp;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float sum = over_groups_sum(total[n]);
        if (row0 + 16 * n + col >= rows) continue;
        const float by = sum == 0 ? 0.0f : 1.0f / sum;
        const size_t at = ((size_t)split * c.n_tokens + s.start + token[n]) * a.q_heads + q_head[n];
        uint16_t *out = static_cast<uint16_t *>(a.out) + (size_t)(s.start + token[n]) * a.out_token + (size_t)q_head[n] * a.out_head;
#pragma unroll
        for (int i = 0; i < VT; ++i) {
            const uint32_t d = 16 * i + 4 * g;
            if (a.splits == 1) *reinterpret_cast<u32x2_a2 *>(out + d) = u32x2{pack2<DT>(o[n][i][0] * by, o[n][i][1] * by), pack2<DT>(o[n][i][2] * by, o[n][i][3] * by)};
            else *reinterpret_cast<f32x4 *>(a.part + at * D + d) = o[n][i];
        }
        if (a.splits > 1 && g == 0) *reinterpret_cast<f32x2 *>(a.part_stat + 2 * at) = f32x2{most[n], sum};
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
    bool many;                          // the kernel for many rows
    uint32_t row_tiles, chunk, splits;
};

inline uint32_t rows_of_many(uint32_t head_dim) { return head_dim == 256 ? 64 : 128; }

// How a call is cut up.  A sequence's cached tokens are split where rows and heads alone leave the card empty.
Plan plan_of(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t head_dim, uint32_t max_new, uint32_t max_length)
{
    Plan p;
    const uint64_t rows = (uint64_t)max_new * group;
    p.many = rows > 32;
    const uint32_t tile = p.many ? rows_of_many(head_dim) : 16, slots = p.many ? 512 : 1024;
    p.row_tiles = (uint32_t)((rows + tile - 1) / tile);
    const uint64_t others = (uint64_t)batch * kv_heads * p.row_tiles;
    const uint64_t want = others >= slots ? 1 : (slots + others - 1) / others;
    const uint64_t tokens = (max_length + want - 1) / want;
    p.chunk = (uint32_t)(tokens <= 256 ? 256 : (tokens + 255) / 256 * 256);
    p.splits = max_length <= p.chunk ? 1 : (max_length + p.chunk - 1) / p.chunk;
    return p;
}

template <int DT, int D> void launch(const Attend &a, bool many, hipStream_t s)
{
    const uint32_t tiles = a.splits * a.c.batch * a.row_tiles;
    if (many) attend_many_kernel<DT, D, D == 256 ? 1 : 2><<<(tiles * a.c.heads + 7) / 8 * 8, 256, 0, s>>>(a);
    else attend_kernel<DT, D><<<dim3(tiles, a.c.heads), 256, 0, s>>>(a);
    if (a.splits > 1) attend_join_kernel<DT, D><<<dim3(a.c.n_tokens, a.q_heads), 64, 0, s>>>(a);
}
template <int DT> void launch(const Attend &a, bool many, hipStream_t s)
{
    if (a.c.head_dim == 64) launch<DT, 64>(a, many, s);
    else if (a.c.head_dim == 128) launch<DT, 128>(a, many, s);
    else launch<DT, 256>(a, many, s);
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
    const Plan p = plan_of(batch, cache->kv_heads, q_heads / cache->kv_heads, cache->head_dim, max_new, max_length);
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
    const Plan p = plan_of(a.c.batch, a.c.heads, group, a.c.head_dim, max_new, max_length);
    if ((uint64_t)p.splits * a.c.batch * p.row_tiles > 0x3FFFFFFFu / a.c.heads) return ENEC_E_ARG;
    const size_t need = enec_cache_attention_workspace(cache, a.c.batch, a.c.n_tokens, q_heads, max_new, max_length);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && ((uintptr_t)workspace & 15)) return ENEC_E_ARG;
    a.q = q, a.out = out;
    a.q_token = q_token_stride, a.q_head = q_head_stride, a.out_token = out_token_stride, a.out_head = out_head_stride;
    a.q_heads = q_heads, a.group = divide_by(group), a.scale = scale * 1.44269504088896340736f;
    a.max_new = max_new, a.max_length = max_length, a.chunk = p.chunk, a.splits = p.splits, a.row_tiles = p.row_tiles;
    a.part = static_cast<float *>(workspace);
    a.part_stat = a.part + (size_t)p.splits * a.c.n_tokens * q_heads * a.c.head_dim;
    if (dtype == ENEC_BF16) launch<BF16>(a, p.many, (hipStream_t)stream);
    else launch<FP16>(a, p.many, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
