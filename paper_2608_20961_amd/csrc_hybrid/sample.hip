// treewy_sample: temperature, top-k, top-p and min-p from given random numbers.
//
// Likelihoods are held relative to the row's largest as whole multiples of
// 2^-40, so that sums of them are exact in any order: histograms by atomics,
// partial sums of waves and a walk in the order of the vocabulary all agree.
//
// The tokens that the filters keep are a prefix of the order (logit down,
// index up).  It is never sorted: one pass counts tokens and likelihoods by
// bins of 1/12 octave below the largest, which shows the bin that the prefix
// ends in, and passes over the digits of that bin's logits narrow it to one
// logit `cut` and a number of its ties.  A last pass sums what is kept by
// segments of the vocabulary, and the segment that holds the drawn point is
// walked by one wave.
#include "hybrid_launch.h"
#include "device.h"

namespace treewy {

namespace {

typedef unsigned long long u64;

constexpr int ROW_THREADS = 1024, WAVES = ROW_THREADS / 64;
constexpr int EACH = 8;                                  // elements of a thread in one step
constexpr int SEGMENT = 64 * EACH;                       // ... of a wave: one segment of the last pass
constexpr int MAX_V = 1 << 20;
constexpr int BINS = 512;                                // 1/12 octave each; 2^-40 is in bin 480
constexpr float BINS_PER_OCTAVE = 12.0f;

// An unsigned key in the order of the floats (-inf lowest; no NaN, and -0 is +0).
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// floor(W f / 2^31), f a whole number of at most 2^31, W below 2^61
__device__ __forceinline__ u64 share(u64 W, u64 f) { return (W >> 31) * f + (((W & 0x7fffffffull) * f) >> 31); }

// The row's scale of likelihoods.
struct Scale {
    float top, slope;
    __device__ __forceinline__ float octaves(float x) const { return __fmul_rn(x == top ? 0.0f : __fsub_rn(x, top), slope); }
    __device__ __forceinline__ static u64 weight(float y) { return (u64)(__builtin_amdgcn_exp2f(y) * 0x1p40f); }
    // (a logit of -inf has none, also where the slope is zero)
    __device__ __forceinline__ u64 of(float x) const { return x == -INFINITY ? 0ull : weight(octaves(x)); }
};

__device__ __forceinline__ u64 wave_sum(u64 x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
template <typename T> __device__ __forceinline__ T wave_before(T x, int lane) {        // sum over lower lanes
    T s = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    return s - x;
}

template <typename T> __device__ __forceinline__ float logit(const T *row, int i) {
    const float x = to_f32(row[i]);
    return x != x ? -INFINITY : x;
}

// f(logit, index) of every element, in steps that the whole workgroup takes together
template <typename T, typename F> __device__ __forceinline__ void each(const T *row, int V, F &&f) {
    for (int base = threadIdx.x * EACH; base < V; base += ROW_THREADS * EACH)
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            if (base + j < V) f(logit(row, base + j), base + j);
}

struct Shared {
    u64 weight[BINS];
    uint32_t count[BINS];
    u64 segment[MAX_V / SEGMENT];
    uint32_t ties[MAX_V / SEGMENT];
    u64 wave64[WAVES];
    uint32_t wave32[WAVES];
    float wavef[WAVES];
    u64 before64;
    uint32_t before32;
    int at;
};

// Where the running sum over `bins` bins (count or likelihood, from bin 0) reaches `need`: the bin, and both sums before it.
// need is reached in some bin.
__device__ void find(Shared &s, int bins, bool by_weight, u64 need, int &bin, u64 &weight_before, uint32_t &count_before) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x, per = bins / 64;
        u64 w = 0;
        uint32_t c = 0;
        for (int i = 0; i < per; ++i) w += s.weight[lane * per + i], c += s.count[lane * per + i];
        u64 wb = wave_before(w, lane);
        uint32_t cb = wave_before(c, lane);
        const bool here = by_weight ? wb < need && wb + w >= need : cb < need && (u64)cb + c >= need;
        if (here) {
            int i = lane * per;
            while (by_weight ? wb + s.weight[i] < need : (u64)cb + s.count[i] < need) wb += s.weight[i], cb += s.count[i], ++i;
            s.at = i;
            s.before64 = wb;
            s.before32 = cb;
        }
    }
    __syncthreads();
    bin = s.at;
    weight_before = s.before64;
    count_before = s.before32;
}

__device__ void clear(Shared &s, int bins) {
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += ROW_THREADS) s.weight[i] = 0, s.count[i] = 0;
    __syncthreads();
}

template <typename T> __global__ __launch_bounds__(ROW_THREADS) void sample_kernel(SampleArgs a) {
    __shared__ Shared s;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *row = (const T *)a.logits + (int64_t)r * a.row_stride;
    const int V = a.V;

    float top = -INFINITY;
    each(row, V, [&](float x, int) { top = fmaxf(top, x); });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) s.wavef[wave] = top;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s.wavef[w]);
    if (top == -INFINITY) {
        if (tid == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = -INFINITY;
            flag_error(a.err, r, TREEWY_FLAG_NO_TOKEN);
        }
        return;
    }
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if (!(temperature > 0.0f)) {                         // the first of the largest
        uint32_t first = 0xffffffffu;
        each(row, V, [&](float x, int i) { first = x == top ? min(first, (uint32_t)i) : first; });
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) first = min(first, (uint32_t)__shfl_xor((int)first, d));
        if (lane == 0) s.wave32[wave] = first;
        __syncthreads();
        if (tid == 0) {
            for (int w = 0; w < WAVES; ++w) first = min(first, s.wave32[w]);
            a.token[r] = (int)first;
            if (a.logprob) a.logprob[r] = 0.0f;
        }
        return;
    }
    const Scale scale{top, __fdiv_rn(1.44269504088896340736f, temperature)};
    const float min_p = a.min_p ? a.min_p[r] : 0.0f, top_p = a.top_p ? a.top_p[r] : 1.0f;
    const u64 least = min_p > 0.0f ? max((u64)(fminf(min_p, 1.0f) * 0x1p40f), 1ull) : 1ull;
    const int top_k = a.top_k ? a.top_k[r] : 0;
    const bool by_count = top_k > 0 && top_k < V, by_weight = top_p < 1.0f;

    // Kept: keys above `cut`, and the first `ties` of those equal to it.
    uint32_t cut = 0, ties = 0xffffffffu;
    auto bin_of = [&](float y) { return min((int)(-y * BINS_PER_OCTAVE), BINS - 1); };
    if (by_count || by_weight) {
        clear(s, BINS);
        u64 all = 0;
        uint32_t n = 0;
        each(row, V, [&](float x, int) {
            const u64 w = scale.of(x);
            if (w < least) return;
            const int i = bin_of(scale.octaves(x));
            atomicAdd(&s.weight[i], w);
            atomicAdd(&s.count[i], 1u);
            all += w;
            ++n;
        });
        all = wave_sum(all);
        n = (uint32_t)wave_sum((u64)n);
        if (lane == 0) s.wave64[wave] = all, s.wave32[wave] = n;
        __syncthreads();
        all = 0;
        n = 0;
        for (int w = 0; w < WAVES; ++w) all += s.wave64[w], n += s.wave32[w];

        // Inside bin `bin`: the key where the running sum reaches `need` (past what lies before the bin), and its ties.
        auto narrow = [&](int bin, bool weighs, u64 need, u64 &weight_before, uint32_t &count_before) {
            uint32_t prefix = 0, mask = 0;
            for (int shift = 24; shift >= (sizeof(T) == 2 ? 16 : 0); shift -= 8) {
                clear(s, 256);
                each(row, V, [&](float x, int) {
                    const u64 w = scale.of(x);
                    const uint32_t k = key_of(x);
                    if (w < least || bin_of(scale.octaves(x)) != bin || (k & mask) != prefix) return;
                    const int digit = 255 - (int)((k >> shift) & 255u);
                    atomicAdd(&s.weight[digit], w);
                    atomicAdd(&s.count[digit], 1u);
                });
                int digit;
                u64 wb;
                uint32_t cb;
                find(s, 256, weighs, need, digit, wb, cb);
                need -= weighs ? wb : (u64)cb;
                weight_before += wb;
                count_before += cb;
                prefix |= (uint32_t)(255 - digit) << shift;
                mask |= 255u << shift;
            }
            // (a bf16's low half: zeros above zero, ones below)
            cut = sizeof(T) == 2 && !(prefix & 0x80000000u) ? prefix | 0xffffu : prefix;
            const u64 w = scale.of(of_key(cut));
            ties = (uint32_t)(weighs ? (need + w - 1) / w : need);
        };
        u64 kept = all;
        if (by_count && (uint32_t)top_k < n) {
            int bin;
            u64 wb;
            uint32_t cb;
            find(s, BINS, false, top_k, bin, wb, cb);
            narrow(bin, false, (u64)top_k - cb, wb, cb);
            kept = wb + ties * scale.of(of_key(cut));
        }
        if (by_weight) {
            const u64 need = max(share(kept, (u64)(fmaxf(top_p, 0.0f) * 0x1p31f)), 1ull);
            clear(s, BINS);
            each(row, V, [&](float x, int) {
                const u64 w = scale.of(x);
                if (w >= least) atomicAdd(&s.weight[bin_of(scale.octaves(x))], w);
            });
            int bin;
            u64 wb;
            uint32_t cb;
            find(s, BINS, true, need, bin, wb, cb);
            narrow(bin, true, need - wb, wb, cb);
        }
    }

    // Sums of what is kept, by segments of 512 tokens: above the cut, and how many ties.
    const int segments = (V + SEGMENT - 1) / SEGMENT;
    const u64 tie_weight = cut ? scale.of(of_key(cut)) : 0;
    __syncthreads();
    for (int g = wave; g < segments; g += WAVES) {
        u64 w = 0;
        uint32_t t = 0;
        for (int j = 0; j < EACH; ++j) {
            const int i = g * SEGMENT + lane * EACH + j;
            if (i >= V) break;
            const float x = logit(row, i);
            const u64 wx = scale.of(x);
            const uint32_t k = key_of(x);
            if (wx < least || k < cut) continue;
            if (k == cut) ++t;
            else w += wx;
        }
        w = wave_sum(w);
        t = (uint32_t)wave_sum((u64)t);
        if (lane == 0) s.segment[g] = w, s.ties[g] = t;
    }
    __syncthreads();
    if (wave != 0) return;

    // The first wave: the segment that the drawn point lies in, then its tokens.
    auto tied = [&](uint32_t before, uint32_t here) { return tie_weight * (min(ties, before + here) - min(ties, before)); };
    const int per = (segments + 63) / 64;
    uint32_t t = 0;
    for (int i = 0; i < per; ++i) t += lane * per + i < segments ? s.ties[lane * per + i] : 0;
    uint32_t tb = wave_before(t, lane);
    u64 w = tied(tb, t);
    for (int i = 0; i < per; ++i) w += lane * per + i < segments ? s.segment[lane * per + i] : 0;
    u64 wb = wave_before(w, lane);
    const u64 total = wave_sum(w);
    const float u = a.u[r];
    const u64 point = share(total, (u64)(fminf(fmaxf(u, 0.0f), 1.0f - 0x1p-24f) * 0x1p31f));
    const bool mine = wb <= point && point < wb + w;
    int g = lane * per;
    if (mine) {
        for (;; ++g) {
            const u64 here = s.segment[g] + tied(tb, s.ties[g]);
            if (point < wb + here) break;
            wb += here;
            tb += s.ties[g];
        }
    }
    const int from = __builtin_ctzll(__ballot(mine));    // (point is below the total: one lane has it)
    g = __shfl(g, from);
    wb = __shfl(wb, from);
    tb = __shfl(tb, from);
    float x[EACH];
    u64 wx[EACH];
    t = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int i = g * SEGMENT + lane * EACH + j;
        x[j] = i < V ? logit(row, i) : -INFINITY;
        wx[j] = scale.of(x[j]);
        if (wx[j] < least || key_of(x[j]) < cut) wx[j] = 0;
        t += wx[j] && key_of(x[j]) == cut;
    }
    tb += wave_before(t, lane);
    w = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (wx[j] && key_of(x[j]) == cut && tb++ >= ties) wx[j] = 0;
        w += wx[j];
    }
    wb += wave_before(w, lane);
    if (wb <= point && point < wb + w) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (wb <= point && point < wb + wx[j]) {
                a.token[r] = g * SEGMENT + lane * EACH + j;
                if (a.logprob) a.logprob[r] = scale.octaves(x[j]) * 0.69314718055994530942f - logf((float)total * 0x1p-40f);
            }
            wb += wx[j];
        }
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, bool f32, hipStream_t stream) {
    if (f32) hipLaunchKernelGGL((sample_kernel<float>), dim3(a.R), dim3(ROW_THREADS), 0, stream, a);
    else hipLaunchKernelGGL((sample_kernel<__bf16>), dim3(a.R), dim3(ROW_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace treewy
