// A token for each row of logits.  The definition stands in include/enec_sampling.h.
#include "enec_sampling.h"
#include "lowbit.hpp"

namespace enec {
namespace sampling {

using namespace lowbit;

constexpr uint32_t THREADS = 1024, WAVES = THREADS / 64, VEC = 8, CHUNK = THREADS * VEC;
constexpr uint32_t MAX_VOCAB = 1u << 22;
constexpr uint32_t BINS = 2048;

struct Rows {
    const void *logits;
    size_t stride;
    uint32_t vocab, log_unit;           // weights are multiples of 2^-log_unit
    enec_sampling how;
    int32_t *tokens;
    float *log_probs;
};

// Floats order as these whole numbers do; 0 and -0 are one.  No float has 0.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = bits_of(v + 0.0f), k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return k > 0 ? k : 1;
}
__device__ __forceinline__ float value_of(uint32_t key) { return f32_of_bits(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t LEAST_KEY = 0x007FFFFFu;             // minus infinity's
constexpr uint32_t INFINITY_KEY = 0xFF800000u;

// this thread's eight logits of a chunk, as keys; 0 behind the row's end
template <int DT> __device__ __forceinline__ void load_keys(const Rows &a, size_t row, uint32_t chunk, uint32_t (&k)[VEC])
{
    const uint32_t first = chunk * CHUNK + threadIdx.x * VEC;
    const size_t i = row * a.stride + first;
    if (first + VEC <= a.vocab) {
        float v[VEC];
        load8<DT>(a.logits, i, v);
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) k[j] = key_of(v[j]);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) k[j] = first + j < a.vocab ? key_of(load1<DT>(a.logits, i + j)) : 0;
    }
}

// Weights as whole numbers: adding 2^(52 - log_unit) to a number up to one leaves its multiple of 2^-log_unit in the low bits, rounded to nearest.
struct Weights {
    double largest, inverse, magic;     // the largest logit, 1 / T
    bool infinite;                      // the largest is
    __device__ __forceinline__ double value(uint32_t key) const
    {
        const double d = ((double)value_of(key) - largest) * inverse;
        const double w = exp(d < -800.0 ? -800.0 : d);
        return infinite ? (key == INFINITY_KEY ? 1.0 : 0.0) : key <= LEAST_KEY ? 0.0 : w;
    }
    __device__ __forceinline__ uint64_t whole(double w) const { return __builtin_bit_cast(uint64_t, w + magic) - __builtin_bit_cast(uint64_t, magic); }
};

// The order's elements up to one: keys above `key`, and `key` itself up to index `last`.
struct Cut {
    uint32_t key, last;
    __device__ __forceinline__ bool keeps(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= last); }
};

struct Shared {
    uint64_t mass[BINS];
    uint32_t count[BINS];
    uint64_t wave_mass[WAVES];
    uint32_t wave_a[WAVES], wave_b[WAVES];
    uint64_t found_mass, found_before;
    uint32_t found, found_count;
};

template <class T> __device__ __forceinline__ T wave_sum(T v)
{
#pragma unroll
    for (int k = 1; k < 64; k *= 2) v += __shfl_xor(v, k);
    return v;
}
// sum over the lanes before this one
template <class T> __device__ __forceinline__ T wave_before(T v)
{
    const uint32_t lane = threadIdx.x & 63;
    T s = v;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const T o = __shfl_up(s, k);
        s += lane >= (uint32_t)k ? o : 0;
    }
    return s - v;
}
// sum over the threads before this one, and over all
template <class T> __device__ __forceinline__ T block_before(T v, T *waves, T &total)
{
    const uint32_t wave = threadIdx.x >> 6;
    const T before = wave_before(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) waves[wave] = before + v;
    __syncthreads();
    T sum = 0, mine = 0;
#pragma unroll
    for (uint32_t i = 0; i < WAVES; ++i) {
        mine = i == wave ? sum : mine;
        sum += waves[i];
    }
    total = sum;
    return mine + before;
}

// The index of the `nth` (from 1) token with this key, in ascending order; all of them: the last index.
template <int DT> __device__ uint32_t index_of_tie(const Rows &a, size_t row, uint32_t key, uint32_t nth, Shared &s)
{
    const uint32_t chunks = (a.vocab + CHUNK - 1) / CHUNK;
    for (uint32_t c = 0; c < chunks; ++c) {
        uint32_t k[VEC], n = 0, total;
        load_keys<DT>(a, row, c, k);
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) n += k[j] == key;
        const uint32_t before = block_before(n, s.wave_a, total);
        if (before < nth && nth <= before + n) {
            uint32_t seen = before;
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                seen += k[j] == key;
                if (k[j] == key && seen == nth) s.found = c * CHUNK + threadIdx.x * VEC + j;
            }
        }
        __syncthreads();
        if (nth <= total) return s.found;
        nth -= total;
    }
    return a.vocab - 1;
}

// Where the order is cut by a number of tokens (MASS: by a sum of weights): the last token before which there are fewer than `target`, among those that `within` keeps.
// The key's bits are found from the top, 11 at a time.
template <int DT, bool MASS> __device__ Cut select(const Rows &a, size_t row, const Weights &w, const Cut &within, uint64_t target, Shared &s)
{
    const uint32_t chunks = (a.vocab + CHUNK - 1) / CHUNK;
    uint32_t prefix = 0;
    for (int shift = 21; shift >= -1; shift -= 11) {
        const int low = shift < 0 ? 0 : shift, bits = shift < 0 ? 10 : 11;
        for (uint32_t i = threadIdx.x; i < BINS; i += THREADS) s.count[i] = 0, s.mass[i] = 0;
        __syncthreads();
        for (uint32_t c = 0; c < chunks; ++c) {
            uint32_t k[VEC];
            load_keys<DT>(a, row, c, k);
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                if (k[j] == 0 || (shift != 21 && (k[j] ^ prefix) >> (low + bits) != 0)) continue;
                const uint32_t digit = k[j] >> low & ((1u << bits) - 1);
                if constexpr (MASS) {
                    if (!within.keeps(k[j], c * CHUNK + threadIdx.x * VEC + j)) continue;
                    atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[digit]), (unsigned long long)w.whole(w.value(k[j])));
                }
                atomicAdd(&s.count[digit], 1u);
            }
        }
        __syncthreads();
        // two bins a thread, in descending order
        uint64_t m[2], total;
        uint32_t bin[2];
        for (uint32_t j = 0; j < 2; ++j) {
            bin[j] = BINS - 1 - (2 * threadIdx.x + j);
            m[j] = MASS ? s.mass[bin[j]] : s.count[bin[j]];
        }
        uint64_t before = block_before<uint64_t>(m[0] + m[1], s.wave_mass, total);
        for (uint32_t j = 0; j < 2; ++j) {
            if (before < target && target <= before + m[j]) s.found = bin[j], s.found_before = before, s.found_count = s.count[bin[j]];
            before += m[j];
        }
        __syncthreads();
        prefix |= s.found << low;
        target -= s.found_before;
        __syncthreads();
    }
    const uint64_t each = MASS ? w.whole(w.value(prefix)) : 1, nth = (target + each - 1) / each;
    const uint32_t ties = s.found_count;
    __syncthreads();
    return {prefix, nth >= ties ? within.key == prefix ? within.last : a.vocab - 1 : index_of_tie<DT>(a, row, prefix, (uint32_t)nth, s)};
}

template <int DT> __global__ void __launch_bounds__(THREADS) sample_kernel(Rows a)
{
    __shared__ Shared s;
    __shared__ uint64_t chunk_mass[MAX_VOCAB / CHUNK];
    const size_t row = blockIdx.x;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, chunks = (a.vocab + CHUNK - 1) / CHUNK;
    const float temperature = a.how.temperature ? a.how.temperature[row] : 1.0f, u = a.how.uniform[row];
    const float top_p = a.how.top_p ? a.how.top_p[row] : 1.0f, min_p = a.how.min_p ? a.how.min_p[row] : 0.0f;
    const int32_t top_k = a.how.top_k ? a.how.top_k[row] : 0;

    // the first of the order; a NaN's key lies above infinity's, or below minus infinity's
    uint32_t best = 0, at = 0;
    bool nan = false;
    for (uint32_t c = 0; c < chunks; ++c) {
        uint32_t k[VEC];
        load_keys<DT>(a, row, c, k);
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) {
            if (k[j] > best) best = k[j], at = c * CHUNK + threadIdx.x * VEC + j;
            nan |= k[j] > INFINITY_KEY || (k[j] != 0 && k[j] < LEAST_KEY);
        }
    }
    if (nan) best = 0xFFFFFFFFu;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t b = __shfl_xor(best, k), i = __shfl_xor(at, k);
        if (b > best || (b == best && i < at)) best = b, at = i;
    }
    if (lane == 0) s.wave_a[wave] = best, s.wave_b[wave] = at;
    __syncthreads();
    for (uint32_t i = 0; i < WAVES; ++i)
        if (s.wave_a[i] > best || (s.wave_a[i] == best && s.wave_b[i] < at)) best = s.wave_a[i], at = s.wave_b[i];
    __syncthreads();
    const bool good = best > LEAST_KEY && best <= INFINITY_KEY && temperature >= 0.0f && temperature <= 3.4028234663852886e38f && u >= 0.0f && u < 1.0f && top_p == top_p &&
                      min_p == min_p;
    if (!good || temperature == 0.0f) {
        if (threadIdx.x == 0) {
            a.tokens[row] = good ? (int32_t)at : -1;
            if (a.log_probs) a.log_probs[row] = good ? 0.0f : __builtin_nanf("");
        }
        return;
    }
    const Weights w{(double)value_of(best), 1.0 / (double)temperature, __builtin_bit_cast(double, (uint64_t)(1023 + 52 - a.log_unit) << 52), best == INFINITY_KEY};
    Cut cut{0, a.vocab - 1};
    if (top_k > 0 && (uint32_t)top_k < a.vocab) cut = select<DT, false>(a, row, w, cut, (uint64_t)top_k, s);

    // the kept weights of each chunk; with top_p first all that top_k leaves
    uint64_t total = 0;
    for (int round = top_p < 1.0f ? 0 : 1; round < 2; ++round) {
        for (uint32_t c = threadIdx.x; c < chunks; c += THREADS) chunk_mass[c] = 0;
        __syncthreads();
        for (uint32_t c = 0; c < chunks; ++c) {
            uint32_t k[VEC];
            uint64_t m = 0;
            load_keys<DT>(a, row, c, k);
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                const uint32_t i = c * CHUNK + threadIdx.x * VEC + j;
                if (!cut.keeps(k[j], i)) continue;
                const double v = w.value(k[j]);
                if (round == 0 || v >= (double)min_p || i == at) m += w.whole(v);
            }
            m = wave_sum(m);
            if (lane == 0 && m) atomicAdd(reinterpret_cast<unsigned long long *>(&chunk_mass[c]), (unsigned long long)m);
        }
        __syncthreads();
        total = 0;
        for (uint32_t c = 0; c < chunks; ++c) total += chunk_mass[c];
        __syncthreads();
        if (round == 0) {
            const double wanted = __builtin_ceil((double)top_p * (double)total);
            cut = select<DT, true>(a, row, w, cut, wanted < 1.0 ? 1 : (uint64_t)wanted, s);
        }
    }
    uint64_t left = (uint64_t)((double)u * (double)total);
    left = left < total ? left : total - 1;
    uint32_t c = 0;
    while (chunk_mass[c] <= left) left -= chunk_mass[c++];
    uint32_t k[VEC];
    uint64_t m[VEC], sum = 0, all;
    load_keys<DT>(a, row, c, k);
#pragma unroll
    for (uint32_t j = 0; j < VEC; ++j) {
        const uint32_t i = c * CHUNK + threadIdx.x * VEC + j;
        const double v = w.value(k[j]);
        m[j] = cut.keeps(k[j], i) && (v >= (double)min_p || i == at) ? w.whole(v) : 0;
        sum += m[j];
    }
    uint64_t before = block_before<uint64_t>(sum, s.wave_mass, all);
#pragma unroll
    for (uint32_t j = 0; j < VEC; ++j) {
        if (before <= left && left < before + m[j]) {
            a.tokens[row] = (int32_t)(c * CHUNK + threadIdx.x * VEC + j);
            if (a.log_probs) a.log_probs[row] = (float)-log1p((double)(total - m[j]) / (double)m[j]);
        }
        before += m[j];
    }
}

}  // namespace sampling
}  // namespace enec

using namespace enec::sampling;

static inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

extern "C" {

size_t enec_sample_workspace(size_t rows, size_t vocab)
{
    (void)rows, (void)vocab;
    return 0;
}

int enec_sample(const void *logits, size_t rows, size_t vocab, size_t row_stride, int dtype, const enec_sampling *how, int32_t *tokens, float *log_probs,
                void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (vocab == 0 || vocab > MAX_VOCAB || rows > (1u << 24) || !how) return ENEC_E_ARG;
    if (rows == 0) return ENEC_OK;
    if (!logits || !aligned(logits, dtype == ENEC_FP32 ? 4 : 2) || row_stride < vocab || !tokens || !how->uniform) return ENEC_E_ARG;
    for (const void *p : {(const void *)tokens, (const void *)log_probs, (const void *)how->temperature, (const void *)how->top_k, (const void *)how->top_p,
                          (const void *)how->min_p, (const void *)how->uniform})
        if (!aligned(p, 4)) return ENEC_E_ARG;
    const size_t need = enec_sample_workspace(rows, vocab);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && !aligned(workspace, 16)) return ENEC_E_ARG;
    uint32_t log_vocab = 0;
    while (((size_t)1 << log_vocab) < vocab) ++log_vocab;
    const Rows a{logits, row_stride, (uint32_t)vocab, log_vocab > 16 ? 62 - log_vocab : 46, *how, tokens, log_probs};
    auto kernel = dtype == ENEC_BF16 ? sample_kernel<BF16> : dtype == ENEC_FP16 ? sample_kernel<FP16> : sample_kernel<FP32>;
    kernel<<<dim3((unsigned)rows), THREADS, 0, (hipStream_t)stream>>>(a);
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
