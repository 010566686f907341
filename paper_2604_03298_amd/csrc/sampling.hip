// A token for each row of logits.  The definition stands in include/enec_sampling.h.
#include "enec_sampling.h"
#include "lowbit.hpp"

namespace enec {
namespace sampling {

using namespace lowbit;

// The order of a row is never made.  Three launches, the first two with a workgroup for each part of a row, the last with one for each row:
//   1. survey: each part's largest logit, and a histogram of its logits in bins that ascend with them.  Logits well over the others are counted all, of the
//      others one in eight, as atomics on LDS are what this launch would spend its time on (256 rows of 131072 in two parts each: all counted 123 us, one in four 52, one in eight
//      42, in four parts 37; without cuts 30, 4.5 TB/s);
//   2. weigh: the histogram says about where a cut lies, and how far off that may be.  Weights of logits above are summed in 64 bits and their tokens counted, and
//      the tokens in between, some tens to some thousands, are listed.  Bound by the vector unit, 21 instructions for a weight and some 10 around it: 64 us of those rows;
//   3. draw: the cuts are picked from the list; then the token is drawn by the kept weights of each run of logits, and of one run's.  Bound by the latency of one workgroup:
//      26 us of those rows, 11 of one row of 32003 with every filter, whose other launches take 4.6 and 9.3.
// Where a cut turns out to lie outside the list, or the list is too short, the third launch finds the cut's key from its highest bits down instead, which takes up to three passes over
// the row a cut and is always right.  That happens with many ties, and with top_k to rows whose bins do not fit the logits about the cut: bins as wide as a sample's spread, which finite
// mask values (-1e4, -65504, the format's lowest) stretch where minus infinity does not, and bins that begin at a lone logit far over the others and end above the cut.  64 rows of 32000 with
// top_k 50 take 60 us with 2 % of the logits at -1e4 and 57 with a lone logit at 14 deviations, 25 otherwise; 256 of 131072 285, 256 and 75; top_p alone is as fast as ever.
// Threads of the third launch: with 1024 one row took 26.6 instead of 24.3 us with every filter, 64 rows with top_p, whose lists are long, 43.1 instead of 44.3.
constexpr uint32_t PART_THREADS = 512, PART_WAVES = PART_THREADS / 64, DRAW_THREADS = 512, DRAW_WAVES = DRAW_THREADS / 64;
constexpr uint32_t VEC = 8, PIECE = 64 * VEC, CHUNK = DRAW_THREADS * VEC;
constexpr uint32_t MAX_VOCAB = 1u << 22, MAX_PARTS = 16, MOST_PART = 65536;
constexpr uint32_t FULLY_COUNTED = 16384;               // a vocabulary up to that
constexpr uint32_t BINS = 2048, DIGITS = 2048, LISTED = 6144, PART_LISTED = LISTED, SAMPLE = 128;

struct Part {
    uint32_t key, first;                // its largest logit's, and that logit's index
    int32_t base;                       // the grid's bin that its histogram begins with; it goes down from there
    float width;                        // of the row's bins
    float counted;                      // from this logit on all are counted
    uint32_t over, listed;              // tokens over top_k's listed ones, and how many are listed
    uint32_t unused;
    uint64_t low, all;                  // weights over top_p's listed ones, and all down to the end of top_k's
    uint64_t kept[PART_WAVES];          // of what lies over the list what min_p keeps, of each wave's run
};
struct Row {
    float p_high, p_low, k_high, k_low;             // top_p's listed logits, from p_low to below p_high, and top_k's
};
struct Listed {
    uint32_t key, index;
};

struct Rows {
    const void *logits;
    size_t stride;
    uint32_t vocab, log_unit;           // weights are multiples of 2^-log_unit
    uint32_t parts, run;                // of a row; logits of a wave's run
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    uint32_t has;                       // which of them are there (the others point somewhere that may be read)
    int32_t *tokens;
    float *log_probs;
    Part *part;
    Row *rows;
    Listed *list;
    uint32_t *bins;
};
enum { HAS_TEMPERATURE = 1, HAS_TOP_K = 2, HAS_TOP_P = 4, HAS_MIN_P = 8 };

// Floats order as these whole numbers do; 0 and -0 are one.  No float has 0.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = bits_of(v + 0.0f), k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return k > 0 ? k : 1;
}
__device__ __forceinline__ float value_of(uint32_t key) { return f32_of_bits(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t LEAST_KEY = 0x007FFFFFu;             // minus infinity's
constexpr uint32_t INFINITY_KEY = 0xFF800000u;

// What a row is drawn with.
struct How {
    float temperature, top_p, min_p, uniform;
    uint32_t top_k;                     // 0: all
    bool good, by_mass;
    __device__ __forceinline__ How(const Rows &a, size_t row)
    {
        const float t = a.temperature[row], p = a.top_p[row], m = a.min_p[row];
        const int32_t k = a.top_k[row];
        uniform = a.uniform[row];
        temperature = a.has & HAS_TEMPERATURE ? t : 1.0f, top_p = a.has & HAS_TOP_P ? p : 1.0f, min_p = a.has & HAS_MIN_P ? m : 0.0f;
        top_k = a.has & HAS_TOP_K && k > 0 && (uint32_t)k < a.vocab ? (uint32_t)k : 0;
        good = temperature >= 0.0f && temperature <= 3.4028234663852886e38f && uniform >= 0.0f && uniform < 1.0f && top_p == top_p && min_p == min_p;
        by_mass = top_p < 1.0f;
    }
    __device__ __forceinline__ bool greedy() const { return temperature == 0.0f; }
    __device__ __forceinline__ bool cuts() const { return good && !greedy() && (top_k || by_mass); }
    __device__ __forceinline__ bool wants_first() const { return greedy() || min_p > 1.0f; }
};

// A grid of bins over all numbers, ascending with them, of which a row's are those from `base` down.
struct Grid {
    float each;                         // 1 / width
    int32_t base;
    // the lower end of bin b
    __device__ __forceinline__ float end(uint32_t b, float width) const { return (float)(((double)base - (double)b) * (double)width); }
    __device__ __forceinline__ int32_t of(float v) const
    {
        return (int32_t)__builtin_amdgcn_fmed3f(__builtin_floorf(v * each), -2147483648.0f, 2147483520.0f);
    }
    __device__ __forceinline__ uint32_t bin(float v) const
    {
        const uint32_t b = (uint32_t)base - (uint32_t)of(v);
        return b < BINS - 1 ? b : BINS - 1;
    }
};

// exp(d / T) for d <= 0, as 2^n 2^r with |r| <= 1/2, the second by its series, whose twelfth term is below 2^-47.  Adding 1.5 2^52 rounds to a whole number,
// which then stands in the low bits.  Weights are whole numbers: adding 2^(52 - log_unit) to a number up to one leaves its multiple of 2^-log_unit in
// the low bits, rounded to nearest.
constexpr double LN2 = 0.693147180559945309417;
template <int K> constexpr double TERM = TERM<K - 1> * LN2 / K;
template <> constexpr double TERM<0> = 1.0;
template <int K> __device__ __forceinline__ double series(double p, double r)
{
    if constexpr (K < 0) return p;
    else return series<K - 1>(__builtin_fma(p, r, TERM<K>), r);
}
struct Weights {
    double top, scale, least, magic;    // the largest logit, 1 / (T ln 2), and -60 of that (2^-60 is rounded to nothing)
    // (infinities stand for 2^128, over all other floats, and are so far over them that these weigh nothing)
    __device__ __forceinline__ Weights(const Rows &a, const How &how, uint32_t most)
    {
        const bool infinite = most == INFINITY_KEY;
        top = infinite ? 0x1p128 : (double)value_of(most), scale = infinite ? 1.0 : 1.0 / LN2 / (double)how.temperature;
        least = infinite ? -60.0 : -60.0 * LN2 * (double)how.temperature;
        magic = __builtin_bit_cast(double, (uint64_t)(1023 + 52 - a.log_unit) << 52);
    }
    __device__ __forceinline__ double value(float v) const
    {
        constexpr double WHOLE = 6755399441055744.0;
        const double d = __builtin_fmax(__builtin_fmin((double)v, top) - top, least);
        const double shifted = __builtin_fma(d, scale, WHOLE), r = __builtin_fma(d, scale, WHOLE - shifted);
        u32x2 p = __builtin_bit_cast(u32x2, series<10>(TERM<11>, r));
        p[1] += __builtin_bit_cast(u32x2, shifted)[0] << 20;
        return __builtin_bit_cast(double, p);
    }
    // as a whole number, and that on top of a constant, which sums take off in one go
    __device__ __forceinline__ uint64_t raised(double w) const { return __builtin_bit_cast(uint64_t, w + magic); }
    __device__ __forceinline__ uint64_t whole(double w) const { return raised(w) - __builtin_bit_cast(uint64_t, magic); }
};

// The order's elements up to one: keys above `key`, and `key` itself up to index `last`.
struct Cut {
    uint32_t key, last;
    __device__ __forceinline__ bool keeps(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= last); }
};
// min_p's: the first token is kept whatever it says (up to one it keeps all of the largest logit)
struct Least {
    double min_p;
    uint32_t first;
    __device__ __forceinline__ bool keeps(double w, uint32_t i) const { return w >= min_p || i == first; }
};

// eight logits from index `first` on; n of them are there, the others zeros
template <int DT> __device__ __forceinline__ uint32_t load_chunk(const Rows &a, size_t row, uint32_t first, uint32_t end, float (&v)[VEC])
{
    const size_t i = row * a.stride + first;
#pragma unroll
    for (uint32_t j = 0; j < VEC; ++j) v[j] = 0;
    if (first + VEC <= end) {
        load8<DT>(a.logits, i, v);
        return VEC;
    }
    if (first >= end) return 0;
#pragma unroll
    for (uint32_t j = 0; j + 1 < VEC; ++j)
        if (first + j < end) v[j] = load1<DT>(a.logits, i + j);
    return end - first;
}

// A wave's run of a row: pieces of eight logits a lane, and, in the last run, up to seven that are one a lane.
template <int DT> struct Run {
    const Rows &a;
    size_t row;
    uint32_t begin, end, rest;
    bool has_rest;
    float v0[VEC], rest_value;                              // the first piece
    __device__ __forceinline__ Run(const Rows &rows, size_t r, uint32_t run) : a(rows), row(r), v0{}, rest_value(0)
    {
        const uint32_t lane = threadIdx.x & 63, whole = a.vocab / VEC * VEC;
        begin = run * a.run, end = begin + a.run < whole ? begin + a.run : whole;
        if (begin + lane * VEC < end) load8<DT>(a.logits, row * a.stride + begin + lane * VEC, v0);
        rest = whole + lane;
        has_rest = run == whole / a.run && rest < a.vocab;
        if (has_rest) rest_value = load1<DT>(a.logits, row * a.stride + rest);
    }
    // f(eight logits, index of the first) for every piece; its logits are asked for before those of the piece before are used
    template <class F> __device__ __forceinline__ void pieces(F &&f) const
    {
        float v[VEC], next[VEC];
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) v[j] = next[j] = v0[j];
#pragma unroll 1
        for (uint32_t first = begin + (threadIdx.x & 63) * VEC; first < end; first += PIECE) {
            if (first + PIECE < end) load8<DT>(a.logits, row * a.stride + first + PIECE, next);
            f(v, first);
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) v[j] = next[j];
        }
    }
    // f(logit, index, number in its piece) for every token.  Says how many a lane had.
    template <class F> __device__ __forceinline__ uint32_t each(F &&f) const
    {
        uint32_t n = has_rest ? 1 : 0;
        pieces([&](const float (&v)[VEC], uint32_t first) {
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) f(v[j], first + j, j);
            n += VEC;
        });
        if (has_rest) f(rest_value, rest, 1u);
        return n;
    }
};

// A value of another lane: 32 or 64 bits by lane moves.  Lanes that have no such neighbour, or whose rows are not in ROWS, get `none`.
template <int CONTROL, int ROWS, class T> __device__ __forceinline__ T moved(T v, T none)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CONTROL, ROWS, 15, false));
    } else {
        const uint64_t a = __builtin_bit_cast(uint64_t, v), b = __builtin_bit_cast(uint64_t, none);
        const uint32_t low = moved<CONTROL, ROWS>((uint32_t)a, (uint32_t)b), high = moved<CONTROL, ROWS>((uint32_t)(a >> 32), (uint32_t)(b >> 32));
        return __builtin_bit_cast(T, (uint64_t)high << 32 | low);
    }
}
template <class T> __device__ __forceinline__ T of_lane(T v, uint32_t lane)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), (int)lane));
    } else {
        const uint64_t a = __builtin_bit_cast(uint64_t, v);
        return __builtin_bit_cast(T, (uint64_t)of_lane((uint32_t)(a >> 32), lane) << 32 | of_lane((uint32_t)a, lane));
    }
}
// f over the lanes up to this one, in six steps: 1, 2, 4 and 8 to the right in each row of sixteen, a row's last to the next row, the second row's last to the upper half
template <class T, class F> __device__ __forceinline__ T wave_scan(T v, T none, F &&f)
{
    v = f(v, moved<0x111, 15>(v, none));
    v = f(v, moved<0x112, 15>(v, none));
    v = f(v, moved<0x114, 15>(v, none));
    v = f(v, moved<0x118, 15>(v, none));
    v = f(v, moved<0x142, 10>(v, none));
    return f(v, moved<0x143, 12>(v, none));
}
template <class T> __device__ __forceinline__ T wave_up_to(T v)
{
    return wave_scan(v, (T)0, [](T x, T y) { return x + y; });
}
template <class T> __device__ __forceinline__ T wave_sum(T v) { return of_lane(wave_up_to(v), 63); }
template <class T> __device__ __forceinline__ T wave_max(T v, T none)
{
    return of_lane(wave_scan(v, none, [](T x, T y) { return x > y ? x : y; }), 63);
}
template <class T> __device__ __forceinline__ T wave_min(T v, T none)
{
    return of_lane(wave_scan(v, none, [](T x, T y) { return x < y ? x : y; }), 63);
}
// sum over the threads before this one, and over all; `waves` has sixteen entries
template <uint32_t WAVES, class T> __device__ __forceinline__ T block_before(T v, T *waves, T &total)
{
    static_assert(WAVES <= 16, "a row of lanes");
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const T up_to = wave_up_to(v);
    __syncthreads();
    if (lane == 63) waves[wave] = up_to;
    __syncthreads();
    T sums = lane < WAVES ? waves[lane & 15] : (T)0;
    sums += moved<0x111, 15>(sums, (T)0), sums += moved<0x112, 15>(sums, (T)0), sums += moved<0x114, 15>(sums, (T)0);
    if constexpr (WAVES > 8) sums += moved<0x118, 15>(sums, (T)0);
    total = of_lane(sums, WAVES - 1);
    return (wave ? of_lane(sums, wave - 1) : (T)0) + (up_to - v);
}
__device__ __forceinline__ void add(uint64_t &to, uint64_t v) { atomicAdd(reinterpret_cast<unsigned long long *>(&to), (unsigned long long)v); }

// The grid's bins that histograms begin with are whole numbers of a thread's bins, so that one part's are another's moved by whole threads.
__device__ __forceinline__ int32_t base_over(int32_t bin, int32_t free)
{
    const int64_t b = ((int64_t)bin + free + 3) & ~(int64_t)3;
    return (int32_t)(b < 2147483640 ? b : 2147483640);
}

// ---- 1 ------------------------------------------------------------------------------

template <int DT> __global__ void __launch_bounds__(PART_THREADS) survey_kernel(Rows a)
{
    __shared__ uint32_t count[BINS], first[PART_WAVES];
    __shared__ float high[PART_WAVES], low[PART_WAVES], begins[PART_WAVES];
    __shared__ bool nans;
    const size_t row = blockIdx.x / a.parts;
    const uint32_t part = blockIdx.x % a.parts, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Run<DT> run(a, row, part * PART_WAVES + wave);
    const uint32_t sample = a.vocab < SAMPLE ? threadIdx.x : (uint32_t)((uint64_t)threadIdx.x * a.vocab / SAMPLE);
    float some = threadIdx.x < SAMPLE && sample < a.vocab ? load1<DT>(a.logits, row * a.stride + sample) : __builtin_nanf("");
    const How how(a, row);
    const bool cuts = how.cuts();
    constexpr float INF = __builtin_inff();
    Grid grid{1.0f, 0};
    float width = 1.0f, counted = -INF;
    if (threadIdx.x == 0) nans = false;
    if (cuts) {
        // The bins' width by the spread of some logits of the row: twice that down from the largest, or 24 T, beyond which weights are below 2^-34.  And the largest of
        // the waves' first pieces, over which a tenth of the bins are left free.
        some = some > -INF && some < INF ? some : __builtin_nanf("");
        float h = some, l = some, b = -INF;
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j)
            if (run.begin + lane * VEC < run.end) b = fmaxf(b, run.v0[j]);
        if (run.has_rest) b = fmaxf(b, run.rest_value);
        h = wave_max(h == h ? h : -INF, -INF), l = wave_min(l == l ? l : INF, INF), b = wave_max(b, -INF);
        if (lane == 0) high[wave] = h, low[wave] = l, begins[wave] = b;
        for (uint32_t i = threadIdx.x; i < BINS; i += PART_THREADS) count[i] = 0;
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < PART_WAVES; ++i) h = fmaxf(h, high[i]), l = fminf(l, low[i]), b = fmaxf(b, begins[i]);
        const float spread = h - l > 0.0f ? 2.0f * (h - l) : 16.0f, reach = 24.0f * how.temperature;
        width = (how.top_k || spread < reach ? spread : reach) / BINS;
        width = width > 1e-30f ? width < 1e30f ? width : 1e30f : 1e-30f;
        counted = a.vocab > FULLY_COUNTED ? h - 0.25f * (h - l) : -INF;
        grid.each = 1.0f / width;
        grid.base = base_over(grid.of(b), BINS / 10);
    }
    float most = -INF;
    bool nan = false;
    auto count_one = [&](float v, uint32_t, uint32_t j) {
        const bool one = v >= counted;
        // (what lies over the free bins is put right below)
        if (one || j == 0) atomicAdd(&count[grid.bin(v)], one ? 1u : VEC);
    };
    if (cuts) run.each([&](float v, uint32_t i, uint32_t j) { most = fmaxf(most, v), nan |= v != v, count_one(v, i, j); });
    else run.each([&](float v, uint32_t, uint32_t) { most = fmaxf(most, v), nan |= v != v; });
    most = wave_max(most, -INF);
    __syncthreads();
    if (lane == 0) high[wave] = most;
    if (nan) nans = true;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < PART_WAVES; ++i) most = fmaxf(most, high[i]);
    if (cuts && grid.of(most) > grid.base) {                // once more, from the largest down
        grid.base = base_over(grid.of(most), 0);
        for (uint32_t i = threadIdx.x; i < BINS; i += PART_THREADS) count[i] = 0;
        __syncthreads();
        run.each(count_one);
    }
    uint32_t at = 0xFFFFFFFFu;
    if (how.wants_first()) {
        run.each([&](float v, uint32_t i, uint32_t) { at = v == most && i < at ? i : at; });
        at = wave_min(at, 0xFFFFFFFFu);
        if (lane == 0) first[wave] = at;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        if (how.wants_first())
            for (uint32_t i = 1; i < PART_WAVES; ++i) at = first[i] < at ? first[i] : at;
        Part &p = a.part[blockIdx.x];
        p.key = nans ? 0xFFFFFFFFu : key_of(most), p.first = at, p.base = grid.base, p.width = width, p.counted = counted;
    }
    if (cuts) {
        u32x4 *to = reinterpret_cast<u32x4 *>(a.bins + (size_t)blockIdx.x * BINS);
        for (uint32_t i = threadIdx.x; i < BINS / 4; i += PART_THREADS) to[i] = reinterpret_cast<const u32x4 *>(count)[i];
    }
}

// What a row's parts say together: the largest logit, its key and its first token, and the row's bins.  Lane p of a wave has part p's.
struct Top {
    uint32_t key, first;
    Grid grid;
    float width;
    int32_t base;                       // this lane's part's
    __device__ __forceinline__ Top(const Rows &a, size_t row)
    {
        const uint32_t lane = threadIdx.x & 63;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(a.part + row * a.parts + (lane < a.parts ? lane : 0));
        key = v[0], first = v[1], base = (int32_t)v[2];
        int32_t most = base;
#pragma unroll
        for (uint32_t k = 1; k < MAX_PARTS; k *= 2) {
            const uint32_t o = __shfl_xor(key, k), i = __shfl_xor(first, k);
            const int32_t b = __shfl_xor(most, k);
            first = o > key || (o == key && i < first) ? i : first, key = o > key ? o : key, most = b > most ? b : most;
        }
        key = __builtin_amdgcn_readfirstlane(key), first = __builtin_amdgcn_readfirstlane(first);
        width = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(v[3]));
        grid = Grid{1.0f / width, __builtin_amdgcn_readfirstlane(most)};
    }
    __device__ __forceinline__ bool good() const { return key > LEAST_KEY && key <= INFINITY_KEY; }
};

// ---- 2 ------------------------------------------------------------------------------

template <int DT> __global__ void __launch_bounds__(PART_THREADS) weigh_kernel(Rows a)
{
    __shared__ uint32_t n_listed, over_of[PART_WAVES];
    __shared__ float k_mass, k_off, p_off;
    __shared__ f32x4 sums_of[PART_WAVES];
    __shared__ uint64_t low_of[PART_WAVES], all_of[PART_WAVES];
    __shared__ uint32_t k_first, k_last, p_first, p_last, p_wide, few;
    __shared__ Listed list[PART_LISTED];
    const size_t row = blockIdx.x / a.parts;
    const uint32_t part = blockIdx.x % a.parts, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Run<DT> run(a, row, part * PART_WAVES + wave);
    const Top top(a, row);
    const float counted = a.part[row * a.parts].counted;
    const How how(a, row);
    if (!how.good || how.greedy() || !top.good()) return;
    const Weights w(a, how, top.key);
    const Least least{(double)how.min_p, how.min_p > 1.0f ? top.first : 0xFFFFFFFFu};
    const uint64_t magic = __builtin_bit_cast(uint64_t, w.magic);
    Part &mine = a.part[blockIdx.x];
    if (!how.cuts()) {
        uint64_t kept = 0;
        uint32_t n;
        if (how.min_p > 0.0f) {
            n = run.each([&](float v, uint32_t i, uint32_t) {
                const double x = w.value(v);
                kept += w.raised(least.keeps(x, i) ? x : 0.0);
            });
        } else {
            n = run.each([&](float v, uint32_t, uint32_t) { kept += w.raised(w.value(v)); });
        }
        kept = wave_sum(kept - n * magic);
        if (lane == 0) mine.kept[wave] = kept;
        return;
    }
    // Four bins a thread: the parts' histograms, each as far below this row's as its base; what is below all bins is in the last.
    constexpr uint32_t EACH = BINS / PART_THREADS;
    static_assert(EACH == 4, "a vector");
    uint32_t n[EACH] = {};
    const uint32_t b0 = threadIdx.x * EACH;
#pragma unroll 1
    for (uint32_t p = 0; p < a.parts; p += 4) {
        u32x4 v[4];
        uint32_t shift[4];
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {                      // (loads that do not wait for one another)
            const uint32_t o = p + q < a.parts ? p + q : p;
            shift[q] = (uint32_t)top.grid.base - (uint32_t)of_lane(top.base, o);
            v[q] = *reinterpret_cast<const u32x4 *>(a.bins + (row * a.parts + o) * BINS + (shift[q] <= b0 ? b0 - shift[q] : 0));
            shift[q] = p + q < a.parts ? shift[q] : 0xFFFFFFFFu;
        }
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) n[j] += shift[q] <= b0 ? v[q][j] : 0;
    }
    // Tokens and weights up to each bin, the latter by the bins' middles, and the variance of what one in eight was counted of (the last bin has no weight to speak of).
    const uint32_t exact = a.vocab > FULLY_COUNTED ? top.grid.bin(counted) : BINS;
    const float cold = 1.0f / how.temperature, step = top.width * cold;
    const float middle_of_0 = (float)((((double)top.grid.base + 0.5) * (double)top.width - (double)value_of(top.key)) * (double)cold);
    float e[EACH], e_sum = 0, v_sum = 0, c_sum = 0;
    uint32_t n_sum = 0;
#pragma unroll
    for (uint32_t j = 0; j < EACH; ++j) {
        const float d = middle_of_0 - (float)(b0 + j) * step, each = b0 + j == BINS - 1 ? 0.0f : d > 0.0f ? 1.0f : __expf(d);
        e[j] = (float)n[j] * each;
        n_sum += n[j], e_sum += e[j];
        if (b0 + j >= exact) v_sum += (VEC - 1) * e[j] * each, c_sum += (VEC - 1) * (float)n[j];
    }
    if (threadIdx.x == 0) {
        k_first = k_last = p_first = p_last = p_wide = BINS - 1, few = 0xFFFFFFFFu;
        n_listed = 0, k_mass = k_off = p_off = 0;
    }
    // (the four sums over the threads before this one meet once)
    const uint32_t n_to = wave_up_to(n_sum);
    const float e_to = wave_up_to(e_sum), v_to = wave_up_to(v_sum), c_to = wave_up_to(c_sum);
    if (lane == 63) sums_of[wave] = f32x4{f32_of_bits(n_to), e_to, v_to, c_to};
    __syncthreads();
    const f32x4 sums = lane < PART_WAVES ? sums_of[lane & (PART_WAVES - 1)] : f32x4{};
    auto of_waves = [&](auto v, auto to, auto own, auto &all) {
        using T = decltype(v);
        v += moved<0x111, 15>(v, (T)0), v += moved<0x112, 15>(v, (T)0), v += moved<0x114, 15>(v, (T)0);
        all = of_lane(v, PART_WAVES - 1);
        return (wave ? of_lane(v, wave - 1) : (T)0) + (to - own);
    };
    static_assert(PART_WAVES <= 8, "three steps");
    uint32_t n_all;
    float e_all, v_all, c_all;
    const uint32_t n_before = of_waves(bits_of(sums[0]), n_to, n_sum, n_all);
    const float e_before = of_waves(sums[1], e_to, e_sum, e_all), v_before = of_waves(sums[2], v_to, v_sum, v_all), c_before = of_waves(sums[3], c_to, c_sum, c_all);
    if (how.top_k) {
        // the bins that the cut may lie in: four standard deviations around where it seems to
        const float wanted = (float)how.top_k;
        uint32_t before = n_before;
        float at = e_before, c = c_before;
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) {
            c += b0 + j >= exact ? (VEC - 1) * (float)n[j] : 0.0f;
            if (before < how.top_k && how.top_k <= before + n[j])
                k_mass = at + e[j] * ((wanted - (float)before) / (float)n[j]), k_off = 4.0f * __builtin_sqrtf(c);
            before += n[j], at += e[j];
        }
        __syncthreads();
        const float off = k_off;
        float sum = (float)n_before;
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) {
            const float next = sum + (float)n[j];
            if (sum < wanted - off && wanted - off <= next) k_first = b0 + j;
            if (sum < wanted + off && wanted + off <= next) k_last = b0 + j;
            sum = next;
        }
        if (threadIdx.x == 0 && wanted - off <= 0.0f) k_first = 0;
        e_all = k_mass > 0.0f ? k_mass : e_all;
    }
    if (how.by_mass) {
        // The same.  A share p of the sum of all is passed as early as what lies above is estimated too high and what lies below too low: p^2 and (1 - p)^2 of
        // their variances.  And half a bin's width for the estimate by middles, by far less where many tokens share in it.
        const float p = how.top_p > 1e-6f ? how.top_p : 1e-6f, target = p * e_all;
        if (e_before < target && target <= e_before + e_sum) p_off = v_before + v_sum;
        __syncthreads();
        const float off = 4.0f * __builtin_sqrtf((1.0f - p) * (1.0f - p) * p_off + p * p * (v_all - p_off > 0.0f ? v_all - p_off : 0.0f)), width = target * step;
        float at = e_before;
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) {
            const float next = j + 1 < EACH ? at + e[j] : e_before + e_sum;
            if (at < target + off + width && target + off + width <= next) p_wide = b0 + j;
            if (at < target - off - width / 16 && target - off - width / 16 <= next) p_first = b0 + j;
            if (at < target + off + width / 16 && target + off + width / 16 <= next) p_last = b0 + j;
            at = next;
        }
        if (threadIdx.x == 0 && target - off - width / 16 <= 0.0f) p_first = 0;
    }
    __syncthreads();
    // The listed logits: all down to the cut where those are few; else what lies around the cuts.
    const float INF = __builtin_inff();
    const uint32_t down_to = how.top_k ? k_last : p_wide;
    uint32_t before = n_before;
#pragma unroll
    for (uint32_t j = 0; j < EACH; ++j) {
        before += n[j];
        if (b0 + j == (down_to + 1 < BINS ? down_to + 1 : down_to)) few = before;
    }
    __syncthreads();
    const bool all = few <= LISTED - LISTED / 8;
    auto high_end = [&](uint32_t b) { return b < 2 ? INF : top.grid.end(b - 2, top.width); };
    auto low_end = [&](uint32_t b) { return b + 2 < BINS ? top.grid.end(b + 1, top.width) : -INF; };
    const float k_low = how.top_k ? low_end(k_last) : -INF, k_high = !how.top_k ? -INF : all ? INF : high_end(k_first);
    const float p_low = !how.by_mass ? INF : all ? (how.top_k ? k_low : low_end(p_wide)) : low_end(p_last);
    // (no lower than top_k's, so that all listed logits are below what is weighed)
    const float p_high = all ? INF : how.by_mass ? fmaxf(high_end(p_first), k_high) : k_high;
    // What is over top_p's list is weighed, and so is what lies between it and top_k's; without top_p, what is over top_k's.
    uint64_t low = 0, kept = 0, all_weights = 0;
    uint32_t over = 0, weighed = 0;
    const bool some_kept = how.min_p > 0.0f, by_count = how.top_k != 0;
    auto listed = [&](float v) { return (v >= p_low && v < p_high) || (by_count && v >= k_low && v < k_high); };
    // (what is listed is weighed too, the third launch takes it off again)
    auto weigh = [&](float v, uint32_t i) {
        const double x = by_count && !(v >= k_low) ? 0.0 : w.value(v), first = v >= p_high ? x : 0.0;
        all_weights += w.raised(x), low += w.raised(first);
        if (some_kept) kept += w.raised(least.keeps(first, i) ? first : 0.0);
        if (by_count) over += v >= k_high;
    };
    run.pieces([&](const float (&v)[VEC], uint32_t first) {
        if (by_count) {
            bool any = false;
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) any |= v[j] >= k_low;
            if (!__any(any)) return;                        // (a wave of tokens behind top_k's cut)
        }
        uint64_t in[VEC], some = 0;                         // lanes whose j-th logit is listed
        weighed += VEC;
        if (by_count || some_kept) {
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                in[j] = __ballot(listed(v[j])), some |= in[j];
                weigh(v[j], first + j);
            }
        } else {
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                in[j] = __ballot(v[j] >= p_low && v[j] < p_high), some |= in[j];
                const double x = w.value(v[j]);
                u32x2 over = __builtin_bit_cast(u32x2, x);
                over[1] = v[j] >= p_high ? over[1] : 0;     // (what is left of it is nothing)
                all_weights += w.raised(x), low += w.raised(__builtin_bit_cast(double, over));
            }
        }
        if (some) {
            // one addition a wave, and a lane's place by the lanes before it
            uint32_t sum = 0, at = 0;
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) sum += (uint32_t)__builtin_popcountll(in[j]);
            const uint32_t leader = (uint32_t)__builtin_ctzll(__ballot(1));
            if (lane == leader) at = atomicAdd(&n_listed, sum);
            at = __builtin_amdgcn_readlane(at, leader);
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                if (in[j] == 0) continue;
                const uint32_t to = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(in[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in[j], 0));
                if (in[j] >> lane & 1 && to < PART_LISTED) list[to] = Listed{key_of(v[j]), first + j};
                at += (uint32_t)__builtin_popcountll(in[j]);
            }
        }
    });
    if (run.has_rest) {
        if (listed(run.rest_value)) {
            const uint32_t at = atomicAdd(&n_listed, 1u);
            if (at < PART_LISTED) list[at] = Listed{key_of(run.rest_value), run.rest};
        }
        weigh(run.rest_value, run.rest), ++weighed;
    }
    low -= weighed * magic, all_weights -= weighed * magic, kept -= weighed * magic;
    kept = wave_sum(some_kept ? kept : low);
    if (lane == 0) mine.kept[wave] = kept;
    low = wave_sum(low), all_weights = wave_sum(all_weights), over = wave_sum(over);
    if (lane == 0) low_of[wave] = low, all_of[wave] = all_weights, over_of[wave] = over;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (uint32_t i = 1; i < PART_WAVES; ++i) low += low_of[i], all_weights += all_of[i], over += over_of[i];
        mine.low = low, mine.all = all_weights, mine.over = over, mine.listed = n_listed;
        if (part == 0) a.rows[row] = Row{p_high, p_low, k_high, k_low};
    }
    const uint32_t many = n_listed < PART_LISTED ? n_listed : PART_LISTED;
    Listed *to = a.list + (size_t)blockIdx.x * PART_LISTED;
    for (uint32_t i = threadIdx.x; i < many; i += PART_THREADS) to[i] = list[i];
}

// ---- 3 ------------------------------------------------------------------------------

constexpr uint32_t FEW = 64;                            // a wave's
constexpr uint32_t TOGETHER = 4;                        // listed tokens that a thread asks for at once
struct Shared {
    uint64_t mass[DIGITS];
    uint32_t count[DIGITS];
    uint64_t wave_mass[16], wave_most[DRAW_WAVES], wave_least[DRAW_WAVES];
    uint32_t wave_count[16];
    uint64_t run_mass[MAX_PARTS * PART_WAVES];      // kept weights of each wave's run
    uint64_t few[FEW], few_weight[FEW];
    uint64_t place[LISTED], weight[LISTED];         // the listed tokens'; in the weights' top bits whether min_p keeps them
    uint64_t found_before, found_place;
    uint32_t found, found_count, n_few;
};

// The index of the `nth` (from 1) token with this key, in ascending order; all of them: the last index.
template <int DT> __device__ __forceinline__ uint32_t index_of_tie(const Rows &a, size_t row, uint32_t key, uint32_t nth, Shared &s)
{
    for (uint32_t c = 0; c < a.vocab; c += CHUNK) {
        float v[VEC];
        uint32_t k[VEC], n = 0, total;
        const uint32_t there = load_chunk<DT>(a, row, c + threadIdx.x * VEC, a.vocab, v);
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) k[j] = j < there ? key_of(v[j]) : 0;
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) n += k[j] == key;
        const uint32_t before = block_before<DRAW_WAVES>(n, s.wave_count, total);
        if (before < nth && nth <= before + n) {
            uint32_t seen = before;
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                seen += k[j] == key;
                if (k[j] == key && seen == nth) s.found = c + threadIdx.x * VEC + j;
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
template <int DT, bool MASS> __device__ __forceinline__ Cut select(const Rows &a, size_t row, const Weights &w, const Cut &within, uint64_t target, Shared &s)
{
    uint32_t prefix = 0;
#pragma unroll 1
    for (int shift = 21; shift >= -1; shift -= 11) {
        const int low = shift < 0 ? 0 : shift, bits = shift < 0 ? 10 : 11;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < DIGITS; i += DRAW_THREADS) s.count[i] = 0, s.mass[i] = 0;
        __syncthreads();
#pragma unroll 1
        for (uint32_t c = 0; c < a.vocab; c += CHUNK) {
            float v[VEC];
            const uint32_t there = load_chunk<DT>(a, row, c + threadIdx.x * VEC, a.vocab, v);
#pragma unroll
            for (uint32_t j = 0; j < VEC; ++j) {
                const uint32_t k = key_of(v[j]);
                if (j >= there || (shift != 21 && (k ^ prefix) >> (low + bits) != 0)) continue;
                const uint32_t digit = k >> low & ((1u << bits) - 1);
                if constexpr (MASS) {
                    if (!within.keeps(k, c + threadIdx.x * VEC + j)) continue;
                    add(s.mass[digit], w.whole(w.value(v[j])));
                }
                atomicAdd(&s.count[digit], 1u);
            }
        }
        __syncthreads();
        // some digits a thread, in descending order
        constexpr uint32_t EACH = DIGITS / DRAW_THREADS;
        uint64_t m[EACH], sum = 0, total;
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) {
            const uint32_t digit = DIGITS - 1 - (EACH * threadIdx.x + j);
            sum += m[j] = MASS ? s.mass[digit] : s.count[digit];
        }
        uint64_t before = block_before<DRAW_WAVES>(sum, s.wave_mass, total);
#pragma unroll
        for (uint32_t j = 0; j < EACH; ++j) {
            const uint32_t digit = DIGITS - 1 - (EACH * threadIdx.x + j);
            if (before < target && target <= before + m[j]) s.found = digit, s.found_before = before, s.found_count = s.count[digit];
            before += m[j];
        }
        __syncthreads();
        prefix |= s.found << low;
        target -= s.found_before;
    }
    const uint64_t each = MASS ? w.whole(w.value(value_of(prefix))) : 1, nth = (target + each - 1) / each;
    const uint32_t ties = s.found_count;
    __syncthreads();
    return {prefix, nth >= ties ? within.key == prefix ? within.last : a.vocab - 1 : index_of_tie<DT>(a, row, prefix, (uint32_t)nth, s)};
}

// A token's place in the order as one number, the first of the order having the largest.
__device__ __forceinline__ uint64_t place_of(uint32_t key, uint32_t index) { return (uint64_t)key << 32 | (0xFFFFFFFFu - index); }

// The same among the listed tokens whose places are from `low` to `high`, of which `target` is at most the sum of the weights (each token's is one if not MASS): bins
// between these places, then between those of the bin that the cut lies in, until few are left, which are compared with one another.  The loops are not unrolled, and
// the list stands in shared memory for that: with one workgroup for a row, most of this kernel's time went into the fetching of its instructions.
constexpr uint64_t KEPT = (uint64_t)1 << 63;
__device__ __forceinline__ Cut select_listed(uint32_t listed, uint64_t low, uint64_t high, bool mass, uint64_t target, Shared &s)
{
    int shift;
#pragma unroll 1
    do {
        const uint64_t spread = high - low;
        shift = spread < DRAW_THREADS ? 0 : 64 - __builtin_ctz(DRAW_THREADS) - __builtin_clzll(spread);         // spread >> shift is below DRAW_THREADS
        s.mass[threadIdx.x] = 0, s.count[threadIdx.x] = 0;
        if (threadIdx.x == 0) s.n_few = 0;
        __syncthreads();
#pragma unroll 1
        for (uint32_t j = threadIdx.x; j < listed; j += TOGETHER * DRAW_THREADS) {
            uint64_t place[TOGETHER], m[TOGETHER];
#pragma unroll
            for (uint32_t i = 0; i < TOGETHER; ++i) {
                const uint32_t at = j + i * DRAW_THREADS < listed ? j + i * DRAW_THREADS : j;
                place[i] = s.place[at], m[i] = s.weight[at];
            }
#pragma unroll
            for (uint32_t i = 0; i < TOGETHER; ++i) {
                if (j + i * DRAW_THREADS >= listed || place[i] < low || place[i] > high) continue;
                const uint32_t bin = (uint32_t)((high - place[i]) >> shift);
                add(s.mass[bin], mass ? m[i] & ~KEPT : 1);
                atomicAdd(&s.count[bin], 1u);
            }
        }
        __syncthreads();
        uint64_t total;
        const uint64_t m = s.mass[threadIdx.x], before = block_before<DRAW_WAVES>(m, s.wave_mass, total);
        if (before < target && target <= before + m) s.found = threadIdx.x, s.found_before = before, s.found_count = s.count[threadIdx.x];
        __syncthreads();
        target -= s.found_before, high -= (uint64_t)s.found << shift;
        const uint64_t rest = ((uint64_t)1 << shift) - 1;
        low = high - low > rest ? high - rest : low;
    } while (s.found_count > FEW);
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < listed; i += DRAW_THREADS) {
        const uint64_t place = s.place[i];
        if (place < low || place > high) continue;
        const uint32_t at = atomicAdd(&s.n_few, 1u);
        s.few[at] = place, s.few_weight[at] = mass ? s.weight[i] & ~KEPT : 1;
    }
    __syncthreads();
    if (threadIdx.x < 64) {                             // (a lane each)
        const uint32_t n = __builtin_amdgcn_readfirstlane(s.n_few);
        const uint64_t mine = threadIdx.x < n ? s.few[threadIdx.x] : 0, own = threadIdx.x < n ? s.few_weight[threadIdx.x] : 0;
        uint64_t sum = 0;
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i) sum += of_lane(mine, i) > mine ? of_lane(own, i) : 0;
        if (sum < target && target <= sum + own) s.found_place = mine;
    }
    __syncthreads();
    return {(uint32_t)(s.found_place >> 32), 0xFFFFFFFFu - (uint32_t)s.found_place};
}

template <int DT> __global__ void __launch_bounds__(DRAW_THREADS) draw_kernel(Rows a)
{
    __shared__ Shared s;
    const size_t row = blockIdx.x;
    const uint32_t runs = a.parts * PART_WAVES;
    const Top top(a, row);
    const uint64_t kept = threadIdx.x < runs ? a.part[row * a.parts + threadIdx.x / PART_WAVES].kept[threadIdx.x % PART_WAVES] : 0;
    const Part &part = a.part[row * a.parts + ((threadIdx.x & 63) < a.parts ? threadIdx.x & 63 : 0)];
    const bool a_part = (threadIdx.x & 63) < a.parts;         // (lanes behind the parts add nothing)
    uint64_t low = a_part ? part.low : 0, weights = a_part ? part.all : 0;
    uint32_t over = a_part ? part.over : 0, listed = a_part ? part.listed : 0;
    const Row r = a.rows[row];
    const How how(a, row);
    const bool good = how.good && top.good();
    if (!good || how.greedy()) {
        if (threadIdx.x == 0) {
            a.tokens[row] = good ? (int32_t)top.first : -1;
            if (a.log_probs) a.log_probs[row] = good ? 0.0f : __builtin_nanf("");
        }
        return;
    }
    const Weights w(a, how, top.key);
    const Least least{(double)how.min_p, how.min_p > 1.0f ? top.first : 0xFFFFFFFFu};
    if (threadIdx.x < runs) s.run_mass[threadIdx.x] = kept;
    __syncthreads();
    Cut cut{0, a.vocab - 1};
    if (how.cuts()) {
        // where each part's list begins among all
        const bool whole = wave_max(listed, 0u) <= PART_LISTED;
        const uint32_t lists = wave_up_to(listed), all_listed = of_lane(lists, 63);
        bool done = whole && all_listed <= LISTED;
        if (done) {
            // top_k's part of the list, from its border to below the upper one (a plus infinity is no less than any border: it is over the list, and was counted there)
            uint64_t k_low = (uint64_t)key_of(r.k_low) << 32, k_high = ((uint64_t)key_of(r.k_high) << 32) - 1, most = 0, least_place = ~(uint64_t)0;
            uint32_t in_k = 0, all_k;
#pragma unroll 1
            for (uint32_t j = threadIdx.x; j < all_listed; j += TOGETHER * DRAW_THREADS) {
                Listed l[TOGETHER];
                uint32_t p[TOGETHER] = {}, begin[TOGETHER] = {};
#pragma unroll 1
                for (uint32_t q = 0; q + 1 < a.parts; ++q) {
                    const uint32_t end = of_lane(lists, q);
#pragma unroll
                    for (uint32_t i = 0; i < TOGETHER; ++i)
                        if (j + i * DRAW_THREADS >= end) p[i] = q + 1, begin[i] = end;
                }
#pragma unroll
                for (uint32_t i = 0; i < TOGETHER; ++i)                     // (loads that do not wait for one another)
                    l[i] = j + i * DRAW_THREADS < all_listed ? a.list[(row * a.parts + p[i]) * PART_LISTED + (j + i * DRAW_THREADS - begin[i])] : Listed{};
#pragma unroll
                for (uint32_t i = 0; i < TOGETHER; ++i) {
                    if (j + i * DRAW_THREADS >= all_listed) break;
                    const uint64_t place = place_of(l[i].key, l[i].index);
                    const double x = w.value(value_of(l[i].key));
                    s.place[j + i * DRAW_THREADS] = place, s.weight[j + i * DRAW_THREADS] = w.whole(x) | (least.keeps(x, l[i].index) ? KEPT : 0);
                    most = place > most ? place : most, least_place = place < least_place ? place : least_place;
                    in_k += place >= k_low && place <= k_high;
                }
            }
            most = wave_max(most, (uint64_t)0), least_place = wave_min(least_place, ~(uint64_t)0);
            low = wave_sum(low), weights = wave_sum(weights), over = wave_sum(over);
            if ((threadIdx.x & 63) == 0) s.wave_most[threadIdx.x >> 6] = most, s.wave_least[threadIdx.x >> 6] = least_place;
            block_before<DRAW_WAVES>(in_k, s.wave_count, all_k);
            most = wave_max(s.wave_most[threadIdx.x % DRAW_WAVES], (uint64_t)0), least_place = wave_min(s.wave_least[threadIdx.x % DRAW_WAVES], ~(uint64_t)0);
            if (how.top_k) {
                done = over < how.top_k && how.top_k - over <= all_k;
                if (done) cut = select_listed(all_listed, k_low > least_place ? k_low : least_place, k_high < most ? k_high : most, false, how.top_k - over, s);
            }
            const uint64_t cut_place = place_of(cut.key, cut.last);
            if (how.by_mass && done) {
                // (of all weights down to the end of top_k's list those are not kept that its cut leaves out; listed ones below that end, which top_p's borders reach, are not among them)
                const uint64_t counted = how.top_k ? k_low : 0;
                uint64_t p_low = (uint64_t)key_of(r.p_low) << 32, p_high = ((uint64_t)key_of(r.p_high) << 32) - 1, in = 0, out = 0, sum, left_out;
                p_low = p_low > cut_place ? p_low : cut_place, p_low = p_low > least_place ? p_low : least_place, p_high = p_high < most ? p_high : most;
#pragma unroll 4
                for (uint32_t i = threadIdx.x; i < all_listed; i += DRAW_THREADS) {
                    const uint64_t place = s.place[i], m = s.weight[i] & ~KEPT;
                    in += place >= p_low && place <= p_high ? m : 0, out += place < cut_place && place >= counted ? m : 0;
                }
                block_before<DRAW_WAVES>(in, s.wave_mass, sum);
                block_before<DRAW_WAVES>(out, s.wave_mass, left_out);
                const double wanted = __builtin_ceil((double)how.top_p * (double)(weights - left_out));
                const uint64_t target = wanted < 1.0 ? 1 : (uint64_t)wanted;
                done = target > low && target <= low + sum;
                if (done) cut = select_listed(all_listed, p_low, p_high, true, target - low, s);
            }
            if (done) {
                const uint64_t end = place_of(cut.key, cut.last);
#pragma unroll 1
                for (uint32_t i = threadIdx.x; i < all_listed; i += DRAW_THREADS) {
                    const uint64_t place = s.place[i], m = s.weight[i];
                    if (place >= end && m > KEPT) add(s.run_mass[(0xFFFFFFFFu - (uint32_t)place) / a.run], m & ~KEPT);
                }
            }
        }
        if (__builtin_expect(!done, 0)) {
            cut = Cut{0, a.vocab - 1};
            if (how.top_k) cut = select<DT, false>(a, row, w, cut, how.top_k, s);
            // the kept weights, twice if the second cut needs the first one's
#pragma unroll 1
            for (int round = how.by_mass ? 0 : 1; round < 2; ++round) {
                uint64_t all = 0, total;
                __syncthreads();
                if (threadIdx.x < runs) s.run_mass[threadIdx.x] = 0;
                __syncthreads();
#pragma unroll 1
                for (uint32_t c = 0; c < a.vocab; c += CHUNK) {
                    float v[VEC];
                    uint64_t sum = 0;
                    const uint32_t first = c + threadIdx.x * VEC;       // (a wave's 512 logits are of one run)
                    const uint32_t there = load_chunk<DT>(a, row, first, a.vocab, v);
#pragma unroll
                    for (uint32_t j = 0; j < VEC; ++j) {
                        const double x = w.value(v[j]);
                        sum += j < there && cut.keeps(key_of(v[j]), first + j) && (round == 0 || least.keeps(x, first + j)) ? w.whole(x) : 0;
                    }
                    all += sum;
                    if (round == 1 && sum) add(s.run_mass[first / a.run], sum);
                }
                if (round == 0) {
                    block_before<DRAW_WAVES>(all, s.wave_mass, total);
                    const double wanted = __builtin_ceil((double)how.top_p * (double)total);
                    cut = select<DT, true>(a, row, w, cut, wanted < 1.0 ? 1 : (uint64_t)wanted, s);
                }
            }
        }
    }
    __syncthreads();
    uint64_t total, all;
    const uint64_t run_mass = threadIdx.x < runs ? s.run_mass[threadIdx.x] : 0, run_before = block_before<DRAW_WAVES>(run_mass, s.wave_mass, total);
    uint64_t left = (uint64_t)((double)how.uniform * (double)total);
    left = left < total ? left : total - 1;
    if (run_before <= left && left < run_before + run_mass) s.found = threadIdx.x, s.found_before = run_before;
    __syncthreads();
    left -= s.found_before;
    const uint32_t begin = s.found * a.run, end = begin + a.run < a.vocab ? begin + a.run : a.vocab;
#pragma unroll 1
    for (uint32_t c = begin; c < end; c += CHUNK) {
        float v[VEC];
        uint64_t sum = 0;
        const uint32_t first = c + threadIdx.x * VEC;
        const uint32_t there = load_chunk<DT>(a, row, first, end, v);
        // of the chunk's j-th token, which then goes to the end of the eight
        auto next = [&](uint32_t j) {
            const float l = v[0];
            const double x = w.value(l);
#pragma unroll
            for (uint32_t i = 0; i + 1 < VEC; ++i) v[i] = v[i + 1];
            v[VEC - 1] = l;
            return j < there && cut.keeps(key_of(l), first + j) && least.keeps(x, first + j) ? w.whole(x) : 0;
        };
#pragma unroll 4
        for (uint32_t j = 0; j < VEC; ++j) sum += next(j);
        uint64_t before = block_before<DRAW_WAVES>(sum, s.wave_mass, all);
        if (all <= left) {
            left -= all;
            continue;
        }
        if (left < before || left >= before + sum) return;
        uint64_t mine = 0;
        uint32_t token = 0;
#pragma unroll 1
        for (uint32_t j = 0; j < VEC && left >= before; ++j) mine = next(j), token = first + j, before += mine;
        if (mine) {
            a.tokens[row] = (int32_t)token;
            if (a.log_probs) a.log_probs[row] = (float)-log1p((double)(total - mine) / (double)mine);
        }
        return;
    }
}

}  // namespace sampling
}  // namespace enec

using namespace enec::sampling;

namespace {

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// Parts of a row, whole pieces for each wave: as long as there are fewer workgroups than compute units, of 4096 logits, and as long as there are fewer than four for each, of 16384; of no
// more than 65536 (where 16 parts allow that).  64 rows of 32000 with top_p took 40 us in four parts and 44 in eight, 64 of 8000 38 in two and 50 in one; 256 of 131072 116 in four
// and 121 in two, 128 of 50000 50 in four and 53 in seven; 512 of 131072 302 in two and 534 in one.
constexpr size_t UNITS = 256;
inline size_t least_parts(size_t vocab)
{
    const size_t parts = (vocab + MOST_PART - 1) / MOST_PART;
    return parts < MAX_PARTS ? parts : MAX_PARTS;
}
inline uint32_t part_of(size_t rows, size_t vocab)
{
    const auto up_to = [&](size_t each, size_t workgroups) {
        const size_t by_length = (vocab + each - 1) / each, by_rows = workgroups / rows;
        return by_length < by_rows ? by_length : by_rows;
    };
    const size_t few = up_to(4096, UNITS), many = up_to(16384, 4 * UNITS);
    size_t parts = few > many ? few : many;
    parts = parts < MAX_PARTS ? parts : MAX_PARTS, parts = parts > least_parts(vocab) ? parts : least_parts(vocab);
    const size_t pieces = (vocab + parts * PART_WAVES * PIECE - 1) / (parts * PART_WAVES * PIECE);
    return (uint32_t)(pieces * PART_WAVES * PIECE);
}
// of all rows together, however few they are
inline size_t most_parts(size_t rows, size_t vocab)
{
    const size_t all = rows * MAX_PARTS < 4 * UNITS ? rows * MAX_PARTS : 4 * UNITS, long_ones = rows * least_parts(vocab);
    return all > long_ones ? all : long_ones;
}
inline bool sizes_ok(size_t rows, size_t vocab)         // (threads of a launch have 32 bits)
{
    return vocab != 0 && vocab <= MAX_VOCAB && rows <= (1u << 22) && rows * least_parts(vocab) <= (1u << 22);
}
constexpr size_t PART_BYTES = sizeof(Part) + BINS * 4 + PART_LISTED * sizeof(Listed), ROW_BYTES = sizeof(Row);
static_assert(sizeof(Part) % 16 == 0 && sizeof(Row) % 16 == 0, "what follows is aligned");

}  // namespace

extern "C" {

size_t enec_sample_workspace(size_t rows, size_t vocab)
{
    if (!sizes_ok(rows, vocab) || rows == 0) return 0;
    return most_parts(rows, vocab) * PART_BYTES + rows * ROW_BYTES;
}

int enec_sample(const void *logits, size_t rows, size_t vocab, size_t row_stride, int dtype, const enec_sampling *how, int32_t *tokens, float *log_probs,
                void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (!sizes_ok(rows, vocab) || !how) return ENEC_E_ARG;
    if (rows == 0) return ENEC_OK;
    if (!logits || !aligned(logits, dtype == ENEC_FP32 ? 4 : 2) || row_stride < vocab || !tokens || !how->uniform) return ENEC_E_ARG;
    for (const void *p : {(const void *)tokens, (const void *)log_probs, (const void *)how->temperature, (const void *)how->top_k, (const void *)how->top_p,
                          (const void *)how->min_p, (const void *)how->uniform})
        if (!aligned(p, 4)) return ENEC_E_ARG;
    const size_t need = enec_sample_workspace(rows, vocab);
    if (workspace_bytes < need || !workspace) return ENEC_E_CAPACITY;
    if (!aligned(workspace, 16)) return ENEC_E_ARG;
    uint32_t log_vocab = 0;
    while (((size_t)1 << log_vocab) < vocab) ++log_vocab;
    const uint32_t part = part_of(rows, vocab), parts = (uint32_t)((vocab + part - 1) / part);
    Part *part_at = static_cast<Part *>(workspace);
    uint32_t *bins = reinterpret_cast<uint32_t *>(part_at + rows * parts);
    Row *rows_at = reinterpret_cast<Row *>(bins + rows * parts * BINS);
    const auto there = [&](const void *p) { return p ? p : how->uniform; };
    const Rows a{logits, row_stride, (uint32_t)vocab, log_vocab > 16 ? 62 - log_vocab : 46, parts, part / PART_WAVES, static_cast<const float *>(there(how->temperature)),
                 static_cast<const float *>(there(how->top_p)), static_cast<const float *>(there(how->min_p)), how->uniform,
                 static_cast<const int32_t *>(there(how->top_k)),
                 (how->temperature ? HAS_TEMPERATURE : 0u) | (how->top_k ? HAS_TOP_K : 0u) | (how->top_p ? HAS_TOP_P : 0u) | (how->min_p ? HAS_MIN_P : 0u), tokens, log_probs,
                 part_at, rows_at, reinterpret_cast<Listed *>(rows_at + rows), bins};
    const dim3 all((unsigned)(rows * parts));
    hipStream_t s = (hipStream_t)stream;
    auto survey = dtype == ENEC_BF16 ? survey_kernel<BF16> : dtype == ENEC_FP16 ? survey_kernel<FP16> : survey_kernel<FP32>;
    auto weigh = dtype == ENEC_BF16 ? weigh_kernel<BF16> : dtype == ENEC_FP16 ? weigh_kernel<FP16> : weigh_kernel<FP32>;
    auto draw = dtype == ENEC_BF16 ? draw_kernel<BF16> : dtype == ENEC_FP16 ? draw_kernel<FP16> : draw_kernel<FP32>;
    survey<<<all, PART_THREADS, 0, s>>>(a);
    weigh<<<all, PART_THREADS, 0, s>>>(a);
    draw<<<dim3((unsigned)rows), DRAW_THREADS, 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
