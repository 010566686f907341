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

// What a row's sum is multiplied with in the end.  The weights' sum is zero where no score is above minus infinity: such a row has no softmax (NaN), unless
// it sees no token at all.
__device__ __forceinline__ float share_of(const Attend &a, const Sequence &s, uint32_t b, uint32_t token, float total)
{
    if (total != 0) return 1.0f / total;                     // (NaN too)
    const int32_t *table = a.c.table + (size_t)b * a.c.table_stride;
    for (int32_t at = s.length - (int32_t)s.count + (int32_t)token; at >= 0; at -= 1 << a.c.log_page)
        if ((uint32_t)table[at >> a.c.log_page] < a.c.n_pages) return __builtin_nanf("");
    return 0;
}

// The largest of four lanes sixteen apart.  The exchanges swap rows of lanes of two registers that hold the same; as instructions of their own, since the
// compiler takes the two results for equal.
// (`maximum` is one instruction for three operands; fmaxf passes each through an instruction of its own first.  It gives NaN where one of them is, which is the
// row's result.)
__device__ __forceinline__ float over_groups_max(float v)
{
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    a = b = __builtin_elementwise_maximum(a, b);
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return __builtin_elementwise_maximum(a, b);
}
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
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

// bytes of a word of codes that are NaN, as 0xFF; whether there are any
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w)
{
    uint32_t r = 0;
    for (int k = 0; k < 4; ++k) r |= (w >> (8 * k) & 0x7F) == 0x7F ? 255u << (8 * k) : 0;
    return r;
}
__device__ __forceinline__ uint32_t any_nan(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

__device__ __forceinline__ void copy_to_lds(const uint8_t *from, uint8_t *to)
{
    using from_t = const __attribute__((address_space(1))) void *;
    using to_t = __attribute__((address_space(3))) void *;
    __builtin_amdgcn_global_load_lds((from_t)from, (to_t)to, 16, 0, 0);
}

// ---- a tile of 64 tokens ----------------------------------------------------------------------------------------------------
// Keys and values of a tile lie in LDS as codes: a token's keys are a row of D / 16 chunks of 16 bytes, a dimension's values a row of four.
// Chunk i of a row lies at place i ^ turn: the sixteen lanes whose 16 bytes are read in one go (rows {0-3, 12-15} of a lane group and rows {4-11} of
// its neighbour) find theirs in sixteen different places of 256 bytes.
template <int D> __device__ __forceinline__ uint32_t key_turn(uint32_t token)
{
    const uint32_t half = token >> 5 & 1;
    if constexpr (D == 64) return 2 * half;
    if constexpr (D == 128) return (token & 2) + 4 * half;
    return 2 * (token & 3) + 8 * half;
}
__device__ __forceinline__ uint32_t value_turn(uint32_t dim) { return 2 * (dim >> 3 & 1); }

template <int D> struct Tile {
    uint8_t keys[64 * D], values[64 * D];
};

// The pages of a tile's four runs of 16 tokens, the same for all lanes; -1: none.
struct Runs {
    int32_t page[4];
};
struct Cached {
    const Pages *c;
    const __attribute__((address_space(4))) int32_t *table;       // (read through the scalar cache: it does not change under the kernel)
    int32_t length;
    uint32_t head;
    bool bad;                                                      // a page number outside the cache was met

    // (pages of 64 tokens and more hold whole tiles: one entry is all)
    __device__ __forceinline__ bool one() const { return c->log_page >= 6; }
    __device__ __forceinline__ void table_entries(int32_t t0, int32_t (&raw)[4]) const
    {
        if (one()) {
            raw[0] = table[(t0 < length ? t0 : length - 1) >> c->log_page];                 // (a length of zero has no tiles)
            return;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) raw[r] = table[(t0 + 16 * r < length ? t0 + 16 * r : length - 1) >> c->log_page];
    }
    __device__ __forceinline__ Runs runs(int32_t t0, const int32_t (&raw)[4])
    {
        Runs p;
        if (one()) {
            const bool in = (uint32_t)raw[0] < c->n_pages;
            bad |= !in;
            p.page[0] = p.page[1] = p.page[2] = p.page[3] = in ? raw[0] : -1;
            return p;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const bool in = (uint32_t)raw[r] < c->n_pages, there = t0 + 16 * r < length;
            bad |= there && !in;
            p.page[r] = in && there ? raw[r] : -1;
        }
        return p;
    }
    // where a page's keys, or values, of the head begin: in page 0, which exists, where there is none
    __device__ __forceinline__ size_t place_of(int32_t page, uint32_t log_values) const
    {
        return ((size_t)(uint32_t)(page < 0 ? 0 : page) * c->heads + head) << log_values;
    }
};
__device__ __forceinline__ int32_t select4(const Runs &p, uint32_t i)
{
    const int32_t p0 = p.page[0], p1 = p.page[1], p2 = p.page[2], p3 = p.page[3];
    const int32_t lo = i & 1 ? p1 : p0, hi = i & 1 ? p3 : p2;
    return i & 2 ? hi : lo;
}

// Copies of a tile's keys, or values, into LDS, 1024 bytes an instruction: PARTS waves share them, or one takes all.  What is copied of no page is not
// looked at.
template <int D, int PARTS> __device__ __forceinline__ void copy_keys(const Cached &s, const Runs &p, int32_t t0, Tile<D> &to, uint32_t part)
{
    constexpr int COPIES = D / 16 / PARTS, TOKENS = 1024 / D, OF_RUN = 16 / TOKENS;      // tokens of a copy, copies of a run
    constexpr uint32_t LOG_D = D == 64 ? 6 : D == 128 ? 7 : 8;
    const Pages &c = *s.c;
    const uint32_t lane = threadIdx.x & 63, mask = (1u << c.log_page) - 1;
    if (s.one()) {
        const uint8_t *k = c.k_codes + s.place_of(p.page[0], LOG_D + c.log_page) + (size_t)((t0 & mask) + part * COPIES * TOKENS) * D;
#pragma unroll
        for (int r = 0; r < COPIES; ++r) {
            const uint32_t token = TOKENS * r + lane / (D / 16), chunk = lane % (D / 16) ^ key_turn<D>(part * COPIES * TOKENS + token);
            copy_to_lds(k + (token * D + 16 * chunk), to.keys + (part * COPIES + r) * 1024);
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < (COPIES + OF_RUN - 1) / OF_RUN; ++q) {
        const uint32_t run = PARTS == 1 ? q : part * COPIES / OF_RUN + q;
        const uint8_t *k = c.k_codes + s.place_of(PARTS == 1 ? p.page[q & 3] : select4(p, run), LOG_D + c.log_page) + (size_t)((t0 + 16 * run) & mask) * D;
#pragma unroll
        for (int r = 0; r < OF_RUN && r < COPIES; ++r) {
            const uint32_t token = TOKENS * r + lane / (D / 16), chunk = lane % (D / 16) ^ key_turn<D>(16 * run + token);
            copy_to_lds(k + (token * D + 16 * chunk), to.keys + (16 * run + TOKENS * r) * D);
        }
    }
}
template <int D, int PARTS> __device__ __forceinline__ void copy_values(const Cached &s, const Runs &p, int32_t t0, Tile<D> &to, uint32_t part)
{
    constexpr int COPIES = D / 16 / PARTS;
    constexpr uint32_t LOG_D = D == 64 ? 6 : D == 128 ? 7 : 8;
    const Pages &c = *s.c;
    const uint32_t lane = threadIdx.x & 63, mask = (1u << c.log_page) - 1;
    const uint32_t run = (lane & 3) ^ value_turn(lane >> 2), own = ((lane >> 2) << c.log_page) + (s.one() ? 16 * run : 0);
    const uint8_t *v = c.v_codes;
    if (s.one()) v += s.place_of(p.page[0], LOG_D + c.log_page) + (t0 & mask);
    else v += s.place_of(select4(p, run), LOG_D + c.log_page) + ((t0 + 16 * run) & mask);
#pragma unroll
    for (int r = 0; r < COPIES; ++r) {
        const uint32_t n = part * COPIES + r;
        copy_to_lds(v + ((size_t)(n * 16) << c.log_page) + own, to.values + n * 1024);
    }
}

// Scores are computed transposed: tokens are the rows of the matrix instruction (left operand: keys), query rows its columns.  A lane then
// holds scores of one query row, and with the tokens of a tile dealt out as
//     instruction j, row r: token 16 (r / 4) + 4 j + r mod 4
// lane group g has tokens 16 g ... 16 g + 15, which is what the product with the values wants of it as right operand: weights
// go from one product to the next without leaving their lane.  Left operand there are the transposed values, 16 dimensions x
// 16 consecutive tokens a lane: one run of 16 bytes.  A run of 16 keys' bytes is two steps of the first product, whose order of
// dimensions is the same for the queries.
// Query rows are pairs of (token, head of the key head's group).  A wave has 16 NT of them.
//
// Keys become 16-bit values for the product with the queries, whose bits all count.  (bf16 queries as the sum of two E4M3 numbers against the codes as they are
// took two prompts of 4000 tokens over 5003 from 457 to 435 us, but such a sum does not hold what is 2^-14 of a row's largest value or less, and
// it is the keys that decide whether that counts.)
template <int DT, int D, int NT, bool MANY> struct Rows {
    static constexpr float LAG = MANY ? 8 : 0;
    static constexpr int KC = D / 64, VT = D / 16;
    u32x4 q[NT][KC][2];                 // eight values each
    // Weights go into the product with the values as the sum of two bf16 numbers each, 16 significant bits: with one the error is of the order of the
    // output's own rounding (bf16, against 64 bits: 0.0018, many rows 0.0022; with two 0.00166, which is that rounding alone).  It costs 64 sequences of up
    // to 8191 tokens 135 us instead of 132, and two prompts of 4000 tokens over 5003 457 instead of 350.
    // The weights' sum is a product too, with a row of ones: every register of `total` has it, and it is that of the rounded weights, whose
    // errors the division takes out again where one weight outdoes the others.
    f32x4 o[NT][VT], total[NT];
    float most[NT];
    int32_t limit[NT];                  // the last position that the row sees; -1: nothing
    int32_t least;                      // of all of the wave's rows: every tile that ends there is seen whole
    uint32_t key_at[KC], value_at;

    __device__ __forceinline__ void begin(const Attend &a, const Sequence &s, uint32_t row0, uint32_t rows, uint32_t head)
    {
        const uint32_t lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
        const int32_t first = s.length - (int32_t)s.count;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t row = row0 + 16 * n + col, token = quotient(row, a.group), q_head = head * a.group.by + (row - token * a.group.by);
            limit[n] = row < rows ? first + (int32_t)token : -1;
            const uint16_t *p = static_cast<const uint16_t *>(a.q) + (size_t)(s.start + token) * a.q_token + (size_t)q_head * a.q_head;
#pragma unroll
            for (int i = 0; i < KC; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) q[n][i][h] = row < rows ? *reinterpret_cast<const u32x4_a2 *>(p + 64 * i + 16 * g + 8 * h) : u32x4{};
#pragma unroll
            for (int i = 0; i < VT; ++i) o[n][i] = f32x4{};
            total[n] = f32x4{};
            most[n] = -__builtin_inff();
        }
        least = row0 < rows ? first + (int32_t)quotient(row0, a.group) : -1;
#pragma unroll
        for (int i = 0; i < KC; ++i) {
            const uint32_t t = 16 * (col >> 2) + (col & 3);               // (+ 4 j, which does not turn)
            key_at[i] = t * D + (((4 * i + g) ^ key_turn<D>(t)) << 4);
        }
        value_at = col * 64 + ((g ^ value_turn(col)) << 4);
    }

    static constexpr int EARLY = KC < 2 ? KC : 2;            // keys that fit registers before they are needed
    __device__ __forceinline__ u32x4 keys_of(const Tile<D> &tile, int i, int j) const { return *reinterpret_cast<const u32x4 *>(tile.keys + key_at[i] + 4 * j * D); }
    __device__ __forceinline__ void load_keys(const Tile<D> &tile, u32x4 (&k)[EARLY][4]) const
    {
#pragma unroll
        for (int i = 0; i < EARLY; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) k[i][j] = keys_of(tile, i, j);
    }
    // early: what load_keys read
    __device__ __forceinline__ void scores(const Tile<D> &tile, const u32x4 (&early)[EARLY][4], f32x4 (&x)[NT][4]) const
    {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[n][j] = f32x4{};
#pragma unroll
        for (int i = 0; i < KC; ++i) {
            u32x4 k[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = i < EARLY ? early[i][j] : keys_of(tile, i, j);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x4 v = values8<DT>(k[j][2 * h], k[j][2 * h + 1], 1.0f);
#pragma unroll
                    for (int n = 0; n < NT; ++n) x[n][j] = mfma16<DT>(v, q[n][i][h], x[n][j]);
                }
        }
    }

    // page, ks, vs: of the lane group's run, ks its keys' scale.  by: the call's scale and log2 e.  arrived(): waits for the tile's values.
    template <typename F>
    __device__ __forceinline__ void add(const Tile<D> &tile, f32x4 (&x)[NT][4], int32_t t0, int32_t length, bool whole_pages, int32_t page, float ks, float by, float vs,
                                        F arrived)
    {
        const uint32_t g = threadIdx.x >> 4 & 3;
        const int32_t tv = t0 + 16 * (int32_t)g;
        // What a row does not see takes no part, whatever its codes are.  (The empty instructions keep what few tiles need out of the others' way, where
        // the compiler would compute both and select.)
        constexpr int AHEAD = MANY ? VT / 2 : 0;             // values on their way while the weights are computed
        u32x4 v[VT];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) v[i] = *reinterpret_cast<const u32x4 *>(tile.values + value_at + i * 1024);
        if (AHEAD) __builtin_amdgcn_sched_barrier(0);
        const bool partial = t0 + 63 > least || t0 + 64 > length || !whole_pages;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[n][j] *= ks;
        if (partial) {
            asm volatile("");
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int32_t sees = page >= 0 ? limit[n] - tv : -1;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[n][j][i] = 4 * j + i <= sees ? x[n][j][i] : -__builtin_inff();
            }
        }
        u32x4 p[NT][2], rest_of[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float high = x[n][0][0];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                high = max3(high, x[n][j][0], x[n][j][1]);
                high = max3(high, x[n][j][2], x[n][j][3]);
            }
            high = over_groups_max(high) * by;
            // Weights are taken relative to a maximum that may lag behind by up to 2^LAG, which costs no bits of theirs, and most tiles need no change of
            // what is summed already (two prompts of 4000 tokens over 5003, fp16: 457 us with a lag of 8, 480 with none; where time is the memory's it is the
            // same).  (A row goes by its own scores only, so that its bits do not depend on the other rows of the wave.)
            const bool moves = high > most[n] + LAG;
            if (__any(moves)) {
                const float now = moves ? high : most[n], fade = moves ? exp2_of(most[n] - now) : 1.0f;
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
                    const float lo = exp2_of(__builtin_fmaf(x[n][2 * h + j / 2][2 * (j & 1)], by, -base));
                    const float hi = exp2_of(__builtin_fmaf(x[n][2 * h + j / 2][2 * (j & 1) + 1], by, -base));
                    p[n][h][j] = pack2<BF16>(lo, hi);
                    const f32x2 r = unpack2<BF16>(p[n][h][j]);
                    rest_of[n][h][j] = pack2<BF16>(lo - r[0], hi - r[1]);
                }
        }
        const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                total[n] = mfma16<BF16>(ones, p[n][h], total[n]);
                total[n] = mfma16<BF16>(ones, rest_of[n][h], total[n]);
            }
        arrived();
#pragma unroll
        for (int i = AHEAD; i < VT; ++i) v[i] = *reinterpret_cast<const u32x4 *>(tile.values + value_at + i * 1024);
        if (partial) {
            asm volatile("");
            // Bytes behind the sequence's end and of no page are anyone's.  A value that is NaN has to reach the rows that see it, and no other:
            // 0 * NaN would.  Such values are taken out, and the rows that see one are told.
            u32x4 mask;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t here = page >= 0 ? length - tv - 4 * j : 0;
                mask[j] = here <= 0 ? 0 : here >= 4 ? ~0u : (1u << (8 * here)) - 1;
            }
            uint32_t any = 0;
#pragma unroll
            for (int i = 0; i < VT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[i][j] &= mask[j];
                    any |= any_nan(v[i][j]);
                }
            if (__any(any)) {
                asm volatile("");
#pragma unroll
                for (int i = 0; i < VT; ++i) {
                    u32x4 bad;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t nan = nan_bytes(v[i][j]);
                        v[i][j] &= ~nan;
                        bad[j] = nan & 0x38383838u;              // 1.0 as E4M3
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        f32x4 seen = {};
                        const int32_t sees = limit[n] - tv;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            u32x4 visible;
#pragma unroll
                            for (int j = 0; j < 4; ++j) visible[j] = (8 * h + 2 * j <= sees ? 0x3F80u : 0) | (8 * h + 2 * j + 1 <= sees ? 0x3F800000u : 0);
                            seen = mfma16<BF16>(values8<BF16>(bad[2 * h], bad[2 * h + 1], 1.0f), visible, seen);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][i][e] = seen[e] > 0 ? __builtin_nanf("") : o[n][i][e];
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < VT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 vv = values8<BF16>(v[i][2 * h], v[i][2 * h + 1], vs);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    o[n][i] = mfma16<BF16>(vv, p[n][h], o[n][i]);
                    o[n][i] = mfma16<BF16>(vv, rest_of[n][h], o[n][i]);
                }
            }
    }
};

// what both kernels know of a workgroup's rows: `end` is where the view of the last of them ends
struct Span {
    uint32_t rows;
    int32_t from, to, end;
};
__device__ __forceinline__ Span span_of(const Attend &a, const Sequence &s, uint32_t first_row, uint32_t count, uint32_t split)
{
    Span v;
    v.rows = s.count * a.group.by;
    const uint32_t last = first_row + count < v.rows ? first_row + count - 1 : v.rows - 1;
    v.end = s.length - (int32_t)s.count + (int32_t)quotient(last, a.group) + 1;
    v.from = (int32_t)(split * a.chunk);
    v.to = v.end - v.from < (int32_t)a.chunk ? v.end : v.from + (int32_t)a.chunk;
    return v;
}
__device__ __forceinline__ Cached cached_of(const Attend &a, const Sequence &s, uint32_t b, uint32_t head)
{
    return {&a.c, (const __attribute__((address_space(4))) int32_t *)(a.c.table + (size_t)b * a.c.table_stride), s.length, head, false};
}

// ---- few rows: the card reads the cache, everything else is small ----------------------------------------------------------------

// A workgroup has 16 NT rows; its WAVES waves take tiles in turn and meet in LDS in the end.  A wave has LDS for one tile of its own: when its keys have
// been multiplied, the next tile's are copied there while the weights are computed and the values multiplied, and the next values while the next keys are.
// It waits for its own copies only: no barrier until the end.  Two waves to a SIMD (head_dim 256: one) did more than copies further ahead: a tile's
// chain of steps leaves half of a wave's cycles idle (64 sequences of up to 8191 tokens: 4 waves with two tiles each 150 us).
// Bound by the way of the cached codes into LDS: 64 sequences of up to 8191 tokens, 8 heads of 128, bf16 135 us (4.95 TB/s; reads alone reach 7.0 on this
// card), of which the copies and their waits take 128 without any arithmetic; two of 131072, fp16, pages of 16, 84 to 88 us and the join 4.7.  One sequence of
// 1000 tokens: 10.3 us, a chain of dependent reads (7.9 without the arithmetic).  Heads of 64 72 us, of 256 150 (16 over 4 heads).
template <int DT, int D, int NT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, D == 256 ? 1 : 2) attend_few_kernel(Attend a)
{
    constexpr int KC = D / 64, COPIES = D / 16;              // of a tile's keys, and of its values
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    const Pages &c = a.c;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const uint32_t split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits, b = rest / a.row_tiles, head = blockIdx.y, row0 = rest % a.row_tiles * (16 * NT);
    const Sequence s = sequence_of(a, b);
    if (!s.good) {
        complain(c);
        return;
    }
    if (row0 >= s.count * a.group.by) return;
    const Span v = span_of(a, s, row0, 16 * NT, split);
    if (split > 0 && v.from >= v.to) return;
    Cached cache = cached_of(a, s, b, head);
    Tile<D> &tile = reinterpret_cast<Tile<D> *>(shared)[wave];
    constexpr int32_t STEP = 64 * WAVES;
    const int32_t first = v.from + 64 * (int32_t)wave;
    int32_t raw[4];
    Runs runs{};
    uint32_t k_byte = 0, v_byte = 0;
    auto ask_keys = [&](int32_t t0) {                        // and the scales, before them
        const Runs next = cache.runs(t0, raw);
        runs = next;
        const int32_t page = select4(next, g);
        const size_t scale = (size_t)(uint32_t)(page < 0 ? 0 : page) * c.heads + head;
        k_byte = c.k_scales[scale], v_byte = c.v_scales[scale];
        __builtin_amdgcn_sched_barrier(0);
        copy_keys<D, 1>(cache, next, t0, tile, 0);
        cache.table_entries(t0 + STEP, raw);
    };
    if (first < v.to) {
        cache.table_entries(first, raw);
        ask_keys(first);
        __builtin_amdgcn_sched_barrier(0);
        copy_values<D, 1>(cache, runs, first, tile, 0);
    }
    Rows<DT, D, NT, false> r;
    r.begin(a, s, row0, v.rows, head);
    for (int32_t t0 = first; t0 < v.to; t0 += STEP) {
        const Runs now = runs;
        const int32_t page = select4(now, g);
        const bool whole = (now.page[0] | now.page[1] | now.page[2] | now.page[3]) >= 0, more = t0 + STEP < v.to;
        // Copies and loads come back in the order in which they were issued: with as many left as were issued of the values behind the keys, the keys are
        // in LDS.
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
        __builtin_amdgcn_sched_barrier(0);
        f32x4 x[NT][4];
        u32x4 k[Rows<DT, D, NT, false>::EARLY][4];
        r.load_keys(tile, k);
        r.scores(tile, k, x);
        const float ks = power_of(k_byte), vs = page >= 0 ? power_of(v_byte) : 1.0f;       // (no page: another one's, and 0 * NaN would be one)
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the keys have been read)
        if (more) ask_keys(t0 + STEP);
        __builtin_amdgcn_sched_barrier(0);
        r.add(tile, x, t0, s.length, whole, page, ks, a.scale, vs, [&] {
            // the same for the values, with the next keys behind them
            __builtin_amdgcn_sched_barrier(0);
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) copy_values<D, 1>(cache, runs, t0 + STEP, tile, 0);
    }
    if (cache.bad && lane == 0) complain(c);

    // the waves' sums, in their order; the tiles' LDS is free now
    __syncthreads();
    float *most_of = reinterpret_cast<float *>(shared), *total_of = most_of + WAVES * 16 * NT;
    f32x4 *sums = reinterpret_cast<f32x4 *>(shared + 2 * WAVES * 16 * NT * sizeof(float));       // [WAVES][16 NT][17]
    if (g == 0) {
#pragma unroll
        for (int n = 0; n < NT; ++n) most_of[(wave * NT + n) * 16 + col] = r.most[n], total_of[(wave * NT + n) * 16 + col] = r.total[n][0];
    }
    __syncthreads();
    float mine[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float top = -__builtin_inff();
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, most_of[(w * NT + n) * 16 + col]);
        mine[n] = r.most[n] == -__builtin_inff() ? 0.0f : exp2_of(r.most[n] - top);
    }
#pragma unroll
    for (int i = 0; i < KC; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(wave * 16 * NT + 16 * n + col) * 17 + 4 * e + g] = r.o[n][4 * i + e] * mine[n];
        __syncthreads();
        for (uint32_t at = threadIdx.x; at < 16 * NT * 16; at += 64 * WAVES) {
            const uint32_t row = at >> 4, d4 = at & 15, out_row = row0 + row;
            if (out_row >= v.rows) continue;
            float top = -__builtin_inff(), total = 0;
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, most_of[(w * NT + row / 16) * 16 + row % 16]);
            for (int w = 0; w < WAVES; ++w) {
                const float m = most_of[(w * NT + row / 16) * 16 + row % 16];
                total += m == -__builtin_inff() ? 0.0f : total_of[(w * NT + row / 16) * 16 + row % 16] * exp2_of(m - top);
            }
            f32x4 sum = sums[row * 17 + d4];
            for (int w = 1; w < WAVES; ++w) sum += sums[(w * 16 * NT + row) * 17 + d4];
            const uint32_t token = quotient(out_row, a.group), q_head = head * a.group.by + (out_row - token * a.group.by), d = 64 * i + 4 * d4;
            if (a.splits == 1) {
                const float by = share_of(a, s, b, token, total);
                uint16_t *p = static_cast<uint16_t *>(a.out) + (size_t)(s.start + token) * a.out_token + (size_t)q_head * a.out_head + d;
                *reinterpret_cast<u32x2_a2 *>(p) = u32x2{pack2<DT>(sum[0] * by, sum[1] * by), pack2<DT>(sum[2] * by, sum[3] * by)};
            } else {
                const size_t to = ((size_t)split * c.n_tokens + s.start + token) * a.q_heads + q_head;
                *reinterpret_cast<f32x4 *>(a.part + to * D + d) = sum;
                if (i == 0 && d4 == 0) *reinterpret_cast<f32x2 *>(a.part_stat + 2 * to) = f32x2{top, total};
            }
        }
    }
}

// ---- many rows: the matrix and vector units work, the cache's codes come from the die's own cache ---------------------------------------

// 16 NT rows to each of four waves, which share the tiles: a wave has all of them, so nothing is joined in the end.  The memory unit copies the codes
// of a tile into LDS while the one before is worked on.  Every wave makes 16-bit values of the codes by itself, where it needs them: a conversion makes two of
// them in the time of any vector instruction, and NT tiles of rows use each.
// Bound by the vector and the matrix unit together: two prompts of 4000 tokens over 5003, 32 heads of 128, 457 to 472 us (630 to 650 TFLOP/s) in either format;
// matrix instructions take 45 % of the cycles, vector instructions 65 % (the issue of the former among them).  32 heads of 64 take 306 us, 16 of 256 541 to
// 547.  Multiplying a tile's values while the next tile's weights are computed, instruction by instruction, did not help, nor did four tiles of rows to a wave,
// which do not fit the registers.  Rows fill the tiles of 128 only where there are many: 5 new tokens of 8 heads a group, 40 rows, over 4000 cached of 32
// sequences take 125 us, 8 tokens of one head a group, 8 rows of the kernel above, over four times the codes 144.
template <int DT, int D, int NT>
__global__ void __launch_bounds__(256, 2) attend_many_kernel(Attend a)
{
    constexpr int VT = D / 16, ROWS = 64 * NT;
    __shared__ __attribute__((aligned(16))) Tile<D> tiles[2];
    const Pages &c = a.c;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    // The last rows first, as they see most; workgroups are dealt out to the eight dies one by one, so where (sequence, head)s are a multiple of
    // eight each of them stays with one die and its cache.
    const uint32_t groups = c.batch * c.heads, split = blockIdx.x / groups, within = blockIdx.x - split * groups, b = within / c.heads, head = within - b * c.heads;
    const uint32_t first_row = (a.row_tiles - 1 - blockIdx.y) * ROWS;
    const Sequence s = sequence_of(a, b);
    if (!s.good) {
        complain(c);
        return;
    }
    if (first_row >= s.count * a.group.by) return;
    const Span v = span_of(a, s, first_row, ROWS, split);
    if (split > 0 && v.from >= v.to) return;
    const uint32_t row0 = first_row + wave * (16 * NT);
    Cached cache = cached_of(a, s, b, head);
    int32_t raw[4], page = -1, next_page = -1;
    uint32_t kb = 0, vb = 0, next_kb = 0, next_vb = 0;
    bool whole = true, next_whole = true;
    auto ask = [&](int32_t t0, Tile<D> &to, int32_t &pg, bool &all, uint32_t &k, uint32_t &w) {
        const Runs p = cache.runs(t0, raw);
        all = (p.page[0] | p.page[1] | p.page[2] | p.page[3]) >= 0;
        copy_keys<D, 4>(cache, p, t0, to, wave);
        copy_values<D, 4>(cache, p, t0, to, wave);
        pg = select4(p, g);
        const size_t scale = (size_t)(uint32_t)(pg < 0 ? 0 : pg) * c.heads + head;
        k = c.k_scales[scale], w = c.v_scales[scale];
    };
    if (v.from < v.to) {
        cache.table_entries(v.from, raw);
        ask(v.from, tiles[0], page, whole, kb, vb);
        cache.table_entries(v.from + 64, raw);
    }
    Rows<DT, D, NT, true> r;
    r.begin(a, s, row0, v.rows, head);
    int buffer = 0;
    for (int32_t t0 = v.from; t0 < v.to; t0 += 64, buffer ^= 1) {
        __builtin_amdgcn_sched_barrier(0);
        // this wave's copies are in LDS, then all waves' are, and nobody reads the tile before any more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        u32x4 k[Rows<DT, D, NT, true>::EARLY][4];            // (on their way while the next tile is asked for)
        r.load_keys(tiles[buffer], k);
        __builtin_amdgcn_sched_barrier(0);
        if (t0 + 64 < v.to) {
            ask(t0 + 64, tiles[buffer ^ 1], next_page, next_whole, next_kb, next_vb);
            cache.table_entries(t0 + 128, raw);
        }
        // (also the last tiles, of which the first waves' rows see nothing: a branch around them cost every tile a copy of all sums)
        f32x4 x[NT][4];
        r.scores(tiles[buffer], k, x);
        // (a wave between its products goes first: the other one of its SIMD has matrix instructions running meanwhile; 400 -> 378 us for two prompts of
        // 4000 tokens over 5003, with one bf16 number a weight)
        __builtin_amdgcn_s_setprio(1);
        r.add(tiles[buffer], x, t0, s.length, whole, page, power_of(kb), a.scale, page >= 0 ? power_of(vb) : 1.0f, [] { __builtin_amdgcn_s_setprio(0); });
        page = next_page, whole = next_whole, kb = next_kb, vb = next_vb;
    }
    if (cache.bad && threadIdx.x == 0) complain(c);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t row = row0 + 16 * n + col;
        if (row >= v.rows) continue;
        const uint32_t token = quotient(row, a.group), q_head = head * a.group.by + (row - token * a.group.by);
        const float sum = r.total[n][0], by = a.splits == 1 ? share_of(a, s, b, token, sum) : 0;
        const size_t at = ((size_t)split * c.n_tokens + s.start + token) * a.q_heads + q_head;
        uint16_t *out = static_cast<uint16_t *>(a.out) + (size_t)(s.start + token) * a.out_token + (size_t)q_head * a.out_head;
#pragma unroll
        for (int i = 0; i < VT; ++i) {
            const uint32_t d = 16 * i + 4 * g;
            const f32x4 &o = r.o[n][i];
            if (a.splits == 1) *reinterpret_cast<u32x2_a2 *>(out + d) = u32x2{pack2<DT>(o[0] * by, o[1] * by), pack2<DT>(o[2] * by, o[3] * by)};
            else *reinterpret_cast<f32x4 *>(a.part + at * D + d) = o;
        }
        if (a.splits > 1 && g == 0) *reinterpret_cast<f32x2 *>(a.part_stat + 2 * at) = f32x2{r.most[n], sum};
    }
}

// The splits of a row: a workgroup a row, D / 4 threads to a split, 1024 / D splits at a time; each thread's sums in the order of the splits, then theirs.
template <int DT, int D>
__global__ void __launch_bounds__(256) attend_join_kernel(Attend a)
{
    constexpr uint32_t LANES = D / 4, AT_ONCE = 256 / LANES;
    __shared__ f32x4 sums[AT_ONCE][LANES];
    __shared__ float tops[4], totals[AT_ONCE];
    const uint32_t token = blockIdx.x, q_head = blockIdx.y, lane = threadIdx.x & 63, d4 = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    // the token's sequence: the one that starts at or before it and ends behind it
    uint32_t b = 0;
    for (;; b += 64) {
        if (b >= a.c.batch) return;
        const uint32_t i = b + lane < a.c.batch ? b + lane : a.c.batch - 1;
        const int32_t start = a.c.starts[i], next = a.c.starts[i + 1];
        const uint64_t has = __ballot(in_order(a.c, start, next) && start <= (int32_t)token && (int32_t)token < next);
        if (has == 0) continue;
        b += (uint32_t)__builtin_ctzll(has);
        break;
    }
    const Sequence s = sequence_of(a, b);
    if (!s.good) return;
    const int32_t sees = s.length - (int32_t)s.count + (int32_t)(token - s.start) + 1;
    const uint32_t splits = sees <= 0 ? 1 : ((uint32_t)sees + a.chunk - 1) / a.chunk;
    const size_t at = (size_t)token * a.q_heads + q_head, step = (size_t)a.c.n_tokens * a.q_heads;
    float top = -__builtin_inff();
    for (uint32_t i = threadIdx.x; i < splits; i += 256) top = fmaxf(top, a.part_stat[2 * (at + i * step)]);
    for (int k = 1; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
    if (lane == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    f32x4 o = {};
    float total = 0;
#pragma unroll 4
    for (uint32_t i = mine; i < splits; i += AT_ONCE) {
        const size_t j = at + i * step;
        const f32x2 stat = *reinterpret_cast<const f32x2 *>(a.part_stat + 2 * j);
        const f32x4 part = *reinterpret_cast<const f32x4 *>(a.part + j * D + 4 * d4);
        const float w = stat[0] == -__builtin_inff() ? 0.0f : exp2_of(stat[0] - top);
        total += w * stat[1];
        o += w * part;
    }
    sums[mine][d4] = o;
    if (d4 == 0) totals[mine] = total;
    __syncthreads();
    if (mine != 0) return;
    for (uint32_t i = 1; i < AT_ONCE; ++i) o += sums[i][d4], total += totals[i];
    const float by = share_of(a, s, b, token - s.start, total);
    uint16_t *p = static_cast<uint16_t *>(a.out) + (size_t)token * a.out_token + (size_t)q_head * a.out_head + 4 * d4;
    *reinterpret_cast<u32x2_a2 *>(p) = u32x2{pack2<DT>(o[0] * by, o[1] * by), pack2<DT>(o[2] * by, o[3] * by)};
}

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

struct Plan {
    bool many;                          // the kernel for many rows
    uint32_t rows, row_tiles, chunk, splits;      // rows of a workgroup
};

inline uint32_t rows_of_many(uint32_t head_dim) { return head_dim == 256 ? 64 : 128; }

// One round of workgroups, as many as the card holds, each with at least `least` tokens: a workgroup's start and end, and joining, cost as much as
// some hundred tokens.
inline uint32_t slots_of(bool many, uint32_t head_dim) { return many || head_dim == 64 ? 512 : 256; }
inline uint32_t least_of(bool many) { return many ? 512 : 1024; }
constexpr uint32_t FEW_ROWS = 32;       // more take the kernel for many

// How a call is cut up.  A sequence's cached tokens are split where rows and heads alone leave the card empty.
Plan plan_of(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t head_dim, uint32_t max_new, uint32_t max_length)
{
    Plan p;
    const uint64_t rows = (uint64_t)max_new * group;
    p.many = rows > FEW_ROWS;
    p.rows = p.many ? rows_of_many(head_dim) : rows > 16 && head_dim < 256 ? 32 : 16;       // (32 rows of 256 dimensions do not fit the registers)
    p.row_tiles = (uint32_t)((rows + p.rows - 1) / p.rows);
    const uint32_t slots = slots_of(p.many, head_dim), least = least_of(p.many);
    const uint64_t others = (uint64_t)batch * kv_heads * p.row_tiles;
    const uint64_t want = others >= slots ? 1 : slots / others;
    const uint64_t tokens = (max_length + want - 1) / want;
    p.chunk = (uint32_t)(tokens <= least ? least : (tokens + 255) / 256 * 256);
    p.splits = max_length <= p.chunk ? 1 : (max_length + p.chunk - 1) / p.chunk;
    return p;
}

// The rows of parts, each of a token, that no call exceeds with at most so many of all these.  Smaller calls may be split more, but a kernel's splits,
// sequences, heads and tiles of rows multiply to `slots` at most, a tile has the tokens of so many rows, and a split has `least` tokens.
uint64_t most_parts(uint32_t n_tokens, uint32_t q_heads, uint32_t group, uint32_t head_dim, uint32_t max_new, uint32_t max_length)
{
    const uint64_t rows = (uint64_t)max_new * group;
    uint64_t most = 0;
    for (const bool many : {false, true}) {
        if (many ? rows <= FEW_ROWS : group > FEW_ROWS) continue;             // not met by any of them
        const uint64_t of_tile = many ? rows_of_many(head_dim) : FEW_ROWS, splits = ((uint64_t)max_length + least_of(many) - 1) / least_of(many);
        if (splits < 2) continue;
        const uint64_t by_slots = slots_of(many, head_dim) * (rows < of_tile ? rows : of_tile) / q_heads, by_length = splits * n_tokens;
        const uint64_t parts = by_slots < by_length ? by_slots : by_length;
        most = most > parts ? most : parts;
    }
    return most;
}

template <int DT, int D, int NT> bool launch_few(const Attend &a, uint32_t tiles, hipStream_t s)
{
    constexpr int WAVES = D == 256 ? 4 : 8;
    // what is joined in the end takes the tiles' place
    constexpr size_t JOINED = 2 * WAVES * 16 * NT * sizeof(float) + WAVES * 16 * NT * 17 * sizeof(f32x4), TILES = WAVES * sizeof(Tile<D>);
    constexpr size_t LDS = JOINED > TILES ? JOINED : TILES;
    static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
    const auto kernel = attend_few_kernel<DT, D, NT, WAVES>;
    static std::atomic<uint64_t> allowed{0};
    if (LDS > 65536 && !allow_lds((const void *)kernel, LDS, allowed)) return false;
    kernel<<<dim3(tiles, a.c.heads), 64 * WAVES, LDS, s>>>(a);
    return true;
}
template <int DT, int D> bool launch(const Attend &a, const Plan &p, hipStream_t s)
{
    const uint32_t tiles = a.splits * a.c.batch * a.row_tiles;
    bool ok = true;
    if (p.many) attend_many_kernel<DT, D, D == 256 ? 1 : 2><<<dim3(a.splits * a.c.batch * a.c.heads, a.row_tiles), 256, 0, s>>>(a);
    else if (D == 256 || p.rows == 16) ok = launch_few<DT, D, 1>(a, tiles, s);
    else ok = launch_few<DT, D, D == 256 ? 1 : 2>(a, tiles, s);
    if (ok && a.splits > 1) attend_join_kernel<DT, D><<<dim3(a.c.n_tokens, a.q_heads), 256, 0, s>>>(a);
    return ok;
}
template <int DT> bool launch(const Attend &a, const Plan &p, hipStream_t s)
{
    return a.c.head_dim == 64 ? launch<DT, 64>(a, p, s) : a.c.head_dim == 128 ? launch<DT, 128>(a, p, s) : launch<DT, 256>(a, p, s);
}

constexpr float MAX_SCALE = 0x1p127f;              // times log2 e it is still finite
constexpr uint32_t MAX_ROWS = 1u << 21, MAX_GROUPS = 1u << 23;      // what a launch holds: 65535 tiles of rows, 2^32 threads side by side

// one call's arguments; 0 = none of its kernels can count with these
bool shape_ok(const enec_cache *cache, uint32_t batch, uint32_t n_tokens, uint32_t q_heads, uint32_t max_new, uint32_t max_length)
{
    if (cache->kv_heads == 0 || q_heads == 0 || q_heads > 65535 || q_heads % cache->kv_heads || max_length > (uint32_t)MAX_SEQUENCE) return false;
    const uint64_t rows = (uint64_t)max_new * (q_heads / cache->kv_heads);
    return rows < MAX_ROWS && n_tokens < MAX_TOKENS && (uint64_t)batch * cache->kv_heads < MAX_GROUPS;
}

}  // namespace

extern "C" {

size_t enec_cache_attention_workspace(const enec_cache *cache, uint32_t batch, uint32_t n_tokens, uint32_t q_heads, uint32_t max_new, uint32_t max_length)
{
    if (!cache || !shape_ok(cache, batch, n_tokens, q_heads, max_new, max_length) || batch == 0 || n_tokens == 0 || max_new == 0) return 0;
    const Plan p = plan_of(batch, cache->kv_heads, q_heads / cache->kv_heads, cache->head_dim, max_new, max_length);
    const uint64_t own = p.splits == 1 ? 0 : (uint64_t)p.splits * n_tokens, most = most_parts(n_tokens, q_heads, q_heads / cache->kv_heads, cache->head_dim, max_new, max_length);
    return (size_t)(own > most ? own : most) * q_heads * (cache->head_dim + 2) * sizeof(float);
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
    if (!q || !out || (((uintptr_t)q | (uintptr_t)out) & 1) || max_new == 0 || !(scale > 0) || !(scale <= MAX_SCALE)) return ENEC_E_ARG;
    const uint32_t group = q_heads / a.c.heads;
    const Plan p = plan_of(a.c.batch, a.c.heads, group, a.c.head_dim, max_new, max_length);
    const size_t need = enec_cache_attention_workspace(cache, a.c.batch, a.c.n_tokens, q_heads, max_new, max_length);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && ((uintptr_t)workspace & 15)) return ENEC_E_ARG;
    a.q = q, a.out = out;
    a.q_token = q_token_stride, a.q_head = q_head_stride, a.out_token = out_token_stride, a.out_head = out_head_stride;
    a.q_heads = q_heads, a.group = divide_by(group), a.scale = scale * 1.44269504088896340736f;
    a.max_new = max_new, a.max_length = max_length, a.chunk = p.chunk, a.splits = p.splits, a.row_tiles = p.row_tiles;
    a.part = static_cast<float *>(workspace);
    a.part_stat = a.part + (size_t)p.splits * a.c.n_tokens * q_heads * a.c.head_dim;
    const bool ok = dtype == ENEC_BF16 ? launch<BF16>(a, p, (hipStream_t)stream) : launch<FP16>(a, p, (hipStream_t)stream);
    return ok && hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
