// Log-probabilities of labels under rows of logits, the paired preference loss on them, and the gradient of the logits.
//
//   lse_t = log sum_v exp(x_tv),  logp_t = x_t,label - lse_t;  a token whose label is outside [0, V) does not count: logp = lse = 0
//   r_i = beta sum_{t of sequence i} (logp_t - ref_t),  z_p = r_p - r_{P+p}
//   loss = mean_p (1 - eps) softplus(-z_p) + eps softplus(z_p);   d loss / d logp_t = -+ beta / P ((1 - eps) sigma(-z) - eps sigma(z))
//   dx_tv = d_t ([v = label] - exp(x_tv - lse_t)),  0 for tokens that do not count
//
// lse is a maximum plus a logarithm, and one fp32 number loses of the logarithm what is below the maximum's last place: all of it where a row
// holds nothing but the type's lowest value.  So logp is formed of the two apart, (x_label - max) - log(sum), lse can be left with its low part
// (lse + low = max + log(sum) to twice the bits), and where a backward call is given no low part, rows whose lse has a last place that matters
// form maximum and sum anew.
//
// A row is read once forward (running maximum and sum) and once backward; rows that do not count are not read at all.  Vocabularies may
// be odd, so a row may begin anywhere: the elements up to the first 16-byte boundary and behind the last one are taken one by one.
// Bound by bytes; the exponentials take about a third of the vector units' time beside them.  In bf16, a third of the tokens not counted:
// 4096 x 32000 forward 36 us (4.85 TB/s), 8192 x 32000 backward 170 to 174 us (5.0 to 5.15 TB/s).
#include "logprob.h"
#include "mx_common.h"

namespace falqon {
namespace {

constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
// what exponents are taken against: the maximum, or 0 where there is nothing above -infinity
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }

template <typename T> __device__ __forceinline__ float element(const T* p);
template <> __device__ __forceinline__ float element(const float* p) { return *p; }
template <> __device__ __forceinline__ float element(const uint16_t* p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = static_cast<uint16_t>(pack_bf16x2(v, v)); }

// A row: `head` elements up to the first whole 16 bytes, `pieces` of those, the rest behind them.
template <typename T>
struct Row {
    static constexpr int E = kPiece<T>;
    const T* p;
    int head, pieces, V;
    __device__ __forceinline__ Row(const T* row, int width) : p(row), V(width)
    {
        head = static_cast<int>((16u - (reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / static_cast<int>(sizeof(T));
        if (head > V) head = V;
        pieces = (V - head) / E;
    }
    __device__ __forceinline__ int tail() const { return head + pieces * E; }
};

struct Running { float m, s; };                                       // maximum, sum of exp(x - maximum)

template <int N>
__device__ __forceinline__ void take(Running& r, const float (&f)[N])
{
    float m = r.m;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, f[i]);
    const float ref = reference(m);
    float s = r.s * exp_of(r.m - ref);
#pragma unroll
    for (int i = 0; i < N; ++i) s += exp_of(f[i] - ref);
    r.m = m;
    r.s = s;
}

// over the workgroup, the same in all threads: over waves, then over the waves' values in every row of 16 lanes
__device__ __forceinline__ float row16_max(float v)
{
    v = fmaxf(v, dpp_move(v, std::integral_constant<int, 0xB1>{}));
    v = fmaxf(v, dpp_move(v, std::integral_constant<int, 0x4E>{}));
    v = fmaxf(v, dpp_move(v, std::integral_constant<int, 0x141>{}));
    return fmaxf(v, dpp_move(v, std::integral_constant<int, 0x140>{}));
}
__device__ __forceinline__ Running join(Running r, float2* s_part)
{
    const float m = wave_max(r.m);
    const float s = wave_sum(r.s * exp_of(r.m - reference(m)));
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = make_float2(m, s);
    barrier_lds_written();
    const float2 v = (threadIdx.x & 15) < (blockDim.x >> 6) ? s_part[threadIdx.x & 15] : make_float2(-INFINITY, 0.0f);
    const float all = row16_max(v.x);
    return {all, row16_sum(v.y * exp_of(v.x - reference(all)))};
}

// lse, and with LOW its low part.  (Kernels of their own, as an argument more costs the calls without it up to 0.6 us: it is read from another line of
// the arguments' memory.)
template <bool LOW, typename F> struct Lse {
    F* hi;
    __device__ __forceinline__ void put(int64_t t, float l, float) const { hi[t] = l; }
    __device__ __forceinline__ float low(int64_t) const { return 0.0f; }
};
template <typename F> struct Lse<true, F> {
    F *hi, *lo;
    __device__ __forceinline__ void put(int64_t t, float l, float low) const { hi[t] = l; lo[t] = low; }
    __device__ __forceinline__ float low(int64_t t) const { return lo[t]; }
};
template <bool LOW, typename F>
Lse<LOW, F> lse_of(F* hi, F* lo)
{
    if constexpr (LOW) return {hi, lo};
    else return {hi};
}

template <bool LOW>
__device__ __forceinline__ void finish(const Running& r, float x_label, int64_t t, float* logp, Lse<LOW, float> lse)
{
    const float m = reference(r.m), log_s = logf(r.s), l = m + log_s;
    const float added = l - m;                                        // what rounding took from m + log_s, exactly
    const float low = (m - (l - added)) + (log_s - added);
    lse.put(t, l, fabsf(l) < INFINITY ? low : 0.0f);
    logp[t] = x_label == -INFINITY && l == l ? -INFINITY : (x_label - m) - log_s;
}

template <typename T, bool LOW>
__global__ void __launch_bounds__(1024)
token_logprob_kernel(const T* __restrict__ logits, int64_t ld, int V, const int64_t* __restrict__ labels, float* __restrict__ logp, Lse<LOW, float> lse,
                     float2* __restrict__ partial)
{
    constexpr int E = kPiece<T>;
    __shared__ float2 s_part[16];
    const int64_t t = blockIdx.x;
    const int64_t label = labels[t];
    const int split = blockIdx.y, splits = gridDim.y;
    if (label < 0 || label >= V) {
        if (split == 0 && threadIdx.x == 0) {
            logp[t] = 0.0f;
            lse.put(t, 0.0f, 0.0f);
        }
        return;
    }
    const Row<T> row(logits + t * ld, V);
    const int from = static_cast<int>(static_cast<int64_t>(row.pieces) * split / splits), to = static_cast<int>(static_cast<int64_t>(row.pieces) * (split + 1) / splits);
    Running r{-INFINITY, 0.0f};
    if (split == 0 && static_cast<int>(threadIdx.x) < row.head) {
        const float f[1] = {element(row.p + threadIdx.x)};
        take(r, f);
    }
    if (split == splits - 1 && static_cast<int>(threadIdx.x) < V - row.tail()) {
        const float f[1] = {element(row.p + row.tail() + threadIdx.x)};
        take(r, f);
    }
    const T* const body = row.p + row.head;
    int i = from + static_cast<int>(threadIdx.x);
    const int step = static_cast<int>(blockDim.x);
    constexpr int AT_ONCE = 32 / E;                                   // pieces: 32 elements share a maximum
    for (; i + (AT_ONCE - 1) * step < to; i += AT_ONCE * step) {
        float f[AT_ONCE][E], all[32];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) load_piece(body + static_cast<int64_t>(i + j * step) * E, f[j]);
#pragma unroll
        for (int j = 0; j < 32; ++j) all[j] = f[j / E][j % E];
        take(r, all);
    }
    for (; i < to; i += step) {
        float f[E];
        load_piece(body + static_cast<int64_t>(i) * E, f);
        take(r, f);
    }
    r = join(r, s_part);
    if (threadIdx.x != 0) return;
    if (splits == 1) finish(r, element(row.p + label), t, logp, lse);
    else partial[t * splits + split] = make_float2(r.m, r.s);
}

// one wave a row: the parts of its splits
template <typename T, bool LOW>
__global__ void __launch_bounds__(256)
token_join_kernel(const T* __restrict__ logits, int64_t ld, int64_t rows, int V, const int64_t* __restrict__ labels, const float2* __restrict__ partial, int splits,
                  float* __restrict__ logp, Lse<LOW, float> lse)
{
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (t >= rows) return;
    const int64_t label = labels[t];
    if (label < 0 || label >= V) return;
    const float2 v = lane < splits ? partial[t * splits + lane] : make_float2(-INFINITY, 0.0f);
    const float m = wave_max(v.x);
    const float s = wave_sum(v.y * exp_of(v.x - reference(m)));
    if (lane == 0) finish(Running{m, s}, element(logits + t * ld + label), t, logp, lse);
}

// Sizes of lse from which half of its last place, 2^-18 of a probability and more, is more than the rest of the arithmetic loses.  4096 x 32000 in bf16 whose rows
// are all beyond: 146 us without the low part, 107 with it, which is what rows within take.
constexpr float kCoarse = 64.0f;
constexpr int kChunk = 1024;                                          // pieces of a row that a workgroup writes

template <typename T, bool PAST, bool LOW>
__global__ void __launch_bounds__(256)
token_logprob_bwd_kernel(const float* __restrict__ d_logp, const T* logits, int64_t ld, int V, const int64_t* __restrict__ labels, Lse<LOW, const float> lse,
                         T* out, int64_t ld_out)
{
    constexpr int E = kPiece<T>;
    __shared__ float2 s_part[16];
    const int64_t t = blockIdx.x;
    const int64_t label = labels[t];
    const bool counts = label >= 0 && label < V;
    float l = counts ? lse.hi[t] : 0.0f, low = counts ? lse.low(t) : 0.0f;
    const float d = counts ? d_logp[t] : 0.0f;
    const bool nothing = !counts || l == -INFINITY;                   // no gradient: written without a look at the logits
    const Row<T> row(logits + t * ld, V), dst(out + t * ld_out, V);
    const int tid = static_cast<int>(threadIdx.x);
    int from = static_cast<int>(blockIdx.y) * kChunk, to_piece = min(dst.pieces, from + kChunk);
    if (!LOW && __builtin_expect(!nothing && fabsf(l) >= kCoarse && fabsf(l) < INFINITY, 0)) {
        // The workgroup takes the whole row, as its results may lie over what the sum reads.
        if (blockIdx.y != 0) return;
        to_piece = dst.pieces;
        Running r{-INFINITY, 0.0f};
        for (int i = tid; i < row.pieces; i += 256) {
            float f[E];
            load_piece(row.p + row.head + static_cast<int64_t>(i) * E, f);
            take(r, f);
        }
        if (tid < row.head) {
            const float f[1] = {element(row.p + tid)};
            take(r, f);
        }
        if (tid < V - row.tail()) {
            const float f[1] = {element(row.p + row.tail() + tid)};
            take(r, f);
        }
        r = join(r, s_part);                                          // its barrier stands between the reads and the writes below
        l = reference(r.m);
        low = logf(r.s);
    }
    const float low2 = low * kLog2e;
    auto probability = [&](float x) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x - l, kLog2e, -low2)); };
    // pieces of the row that is written; what is read may lie otherwise
    const bool alike = dst.head == row.head;
    T* const to = out + t * ld_out;
    auto value = [&](int v) {
        if (nothing) return 0.0f;
        const float p = probability(element(row.p + v));
        return v == static_cast<int>(label) ? d * (1.0f - p) : -d * p;
    };
    if (blockIdx.y == 0) {
        if (tid < dst.head) put(to + tid, value(tid));
        if (tid < V - dst.tail()) put(to + dst.tail() + tid, value(dst.tail() + tid));
    }
    for (int i = from + tid; i < to_piece; i += 256) {
        const int v = dst.head + i * E;
        float f[E] = {};
        if (!nothing) {
            if (alike) {
                load_piece(row.p + v, f);
            } else {
#pragma unroll
                for (int k = 0; k < E; ++k) f[k] = element(row.p + v + k);
            }
            const int at = static_cast<int>(label) - v;
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float p = probability(f[k]);
                f[k] = k == at ? d * (1.0f - p) : -d * p;
            }
        }
        store_piece<PAST>(to + v, pack_piece(f));
    }
}

// The sum over a wave, in a fixed tree, in all lanes.
__device__ __forceinline__ double wave_sum(double v)
{
    auto moved = [](double x, auto ctrl) {
        constexpr int C = decltype(ctrl)::value;
        return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(x), C, 0xf, 0xf, true), __builtin_amdgcn_mov_dpp(__double2loint(x), C, 0xf, 0xf, true));
    };
    v += moved(v, std::integral_constant<int, 0xB1>{});
    v += moved(v, std::integral_constant<int, 0x4E>{});
    v += moved(v, std::integral_constant<int, 0x141>{});
    v += moved(v, std::integral_constant<int, 0x140>{});
    auto both = [](auto lo, auto hi) {
        return __hiloint2double(static_cast<int>(hi[0]), static_cast<int>(lo[0])) + __hiloint2double(static_cast<int>(hi[1]), static_cast<int>(lo[1]));
    };
    unsigned lo = static_cast<unsigned>(__double2loint(v)), hi = static_cast<unsigned>(__double2hiint(v));
    v = both(__builtin_amdgcn_permlane16_swap(lo, lo, false, false), __builtin_amdgcn_permlane16_swap(hi, hi, false, false));
    lo = static_cast<unsigned>(__double2loint(v));
    hi = static_cast<unsigned>(__double2hiint(v));
    return both(__builtin_amdgcn_permlane32_swap(lo, lo, false, false), __builtin_amdgcn_permlane32_swap(hi, hi, false, false));
}
// over a workgroup of W waves, in all threads
template <int W>
__device__ __forceinline__ double block_sum(double v, double* s_part)
{
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < W; ++k) sum += s_part[k];
    __syncthreads();
    return sum;
}

// softplus(-z), softplus(z) and the logistic function at +-z, none of which overflows
__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v))); }
__device__ __forceinline__ float logistic(float v)
{
    const float e = expf(-fabsf(v));
    return (v >= 0.0f ? 1.0f : e) / (1.0f + e);
}

struct Preference {
    const float *logp, *ref;
    const int64_t* offsets;
    int64_t T;
    int P;
    float beta, smoothing;
    float *loss, *rewards, *d_logp;
    __device__ __forceinline__ int64_t bound(int i) const
    {
        const int64_t o = offsets[i];
        return o < 0 ? 0 : o > T ? T : o;
    }
    // of one pair's loss, and of the loss by its chosen reward's sum of log-probabilities
    // (z is infinite where a label was masked: without smoothing the second part is then 0, not 0 times infinity)
    __device__ __forceinline__ float term(float z) const { return (1.0f - smoothing) * softplus(-z) + (smoothing > 0.0f ? smoothing * softplus(z) : 0.0f); }
    __device__ __forceinline__ float slope(float z) const { return beta / static_cast<float>(P) * (smoothing * logistic(z) - (1.0f - smoothing) * logistic(-z)); }
};

// a thread's share of sum (logp - ref) over [from, to), `step` threads side by side
__device__ __forceinline__ double ratio_share(const Preference& a, int64_t from, int64_t to, int thread, int step)
{
    double sum = 0.0;
    int64_t t = from + thread;
    for (; t + 7 * step < to; t += 8 * step) {
        float p[8], r[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) { p[k] = a.logp[t + k * step]; r[k] = a.ref[t + k * step]; }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += static_cast<double>(p[k]) - static_cast<double>(r[k]);
    }
    for (; t < to; t += step) sum += static_cast<double>(a.logp[t]) - static_cast<double>(a.ref[t]);
    return sum;
}

// All of it in one workgroup, a wave a sequence: few pairs of few tokens, where a second launch would cost more.  us in one workgroup and in one a pair
// (those 7.1 to 8.1 throughout): 4 pairs of 16384 tokens in all 5.0, of 32768 6.7, of 65536 10.1 (8.3); 32 pairs of 16384 7.1, of 24000 8.2 (7.8);
// 48 of 4096 to 16384 7.6 to 8.4, 256 25, 1024 93; one pair of 12000 8.0, of 16384 9.1 (8.1).
constexpr int kOnePairs = 32, kOneTokens = 16384;
__global__ void __launch_bounds__(1024)
preference_one_kernel(const Preference a)
{
    __shared__ float s_reward[2 * kOnePairs];                         // rewards, then slopes in the first half
    __shared__ double s_part[16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int i = wave; i < 2 * a.P; i += 16) {
        const float reward = static_cast<float>(static_cast<double>(a.beta) * wave_sum(ratio_share(a, a.bound(i), a.bound(i + 1), lane, 64)));
        if (lane == 0) {
            s_reward[i] = reward;
            a.rewards[i] = reward;
        }
    }
    __syncthreads();
    double sum = 0.0;
    if (static_cast<int>(threadIdx.x) < a.P) {
        const float z = s_reward[threadIdx.x] - s_reward[a.P + threadIdx.x];
        sum = static_cast<double>(a.term(z));
        s_reward[threadIdx.x] = a.slope(z);                           // read by nobody else before the barrier
    }
    sum = block_sum<16>(sum, s_part);
    if (threadIdx.x == 0) *a.loss = static_cast<float>(sum / a.P);
    for (int i = wave; i < 2 * a.P; i += 16) {
        const float d = i < a.P ? s_reward[i] : -s_reward[i - a.P];
        for (int64_t t = a.bound(i) + lane, end = a.bound(i + 1); t < end; t += 64) a.d_logp[t] = d;
    }
    for (int64_t t = threadIdx.x, end = a.bound(0); t < end; t += 1024) a.d_logp[t] = 0.0f;                 // tokens of no sequence
    for (int64_t t = a.bound(2 * a.P) + threadIdx.x; t < a.T; t += 1024) a.d_logp[t] = 0.0f;
}

// One workgroup a pair, and one for the mean.
__global__ void __launch_bounds__(256)
preference_pair_kernel(const Preference a, float* __restrict__ pair_loss)
{
    __shared__ double s_part[4];
    const int pair = blockIdx.x;
    const int64_t from[2] = {a.bound(pair), a.bound(a.P + pair)}, to[2] = {a.bound(pair + 1), a.bound(a.P + pair + 1)};
    float reward[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        reward[k] = static_cast<float>(static_cast<double>(a.beta) * block_sum<4>(ratio_share(a, from[k], to[k], threadIdx.x, 256), s_part));
    const float z = reward[0] - reward[1], dz = a.slope(z);
    if (threadIdx.x == 0) {
        a.rewards[pair] = reward[0];
        a.rewards[a.P + pair] = reward[1];
        pair_loss[pair] = a.term(z);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        for (int64_t t = from[k] + threadIdx.x; t < to[k]; t += 256) a.d_logp[t] = k == 0 ? dz : -dz;
    if (pair == 0) {                                                  // tokens of no sequence
        for (int64_t t = threadIdx.x; t < from[0]; t += 256) a.d_logp[t] = 0.0f;
        for (int64_t t = a.bound(2 * a.P) + threadIdx.x; t < a.T; t += 256) a.d_logp[t] = 0.0f;
    }
}

__global__ void __launch_bounds__(256)
preference_mean_kernel(const float* __restrict__ pair_loss, int P, float* __restrict__ loss)
{
    __shared__ double s_part[4];
    double sum = 0.0;
    for (int p = threadIdx.x; p < P; p += 256) sum += static_cast<double>(pair_loss[p]);
    sum = block_sum<4>(sum, s_part);
    if (threadIdx.x == 0) *loss = static_cast<float>(sum / P);
}

template <typename T, bool LOW>
void fwd(const TokenLogprob& a, int splits, hipStream_t stream)
{
    const T* const logits = static_cast<const T*>(a.logits);
    const int V = static_cast<int>(a.V);
    const dim3 grid(static_cast<unsigned>(a.T), static_cast<unsigned>(splits));
    const auto lse = lse_of<LOW>(a.lse, a.lse_low);
    // Long rows of which there are two a CU at most: 16 waves share one.  us with 256 and with 1024 threads: fp32 512 x 16000 9.3, 7.8, 640 x 16000 10.4, 10.2,
    // 640 x 32000 15.3, 17.2; bf16 256 x 24000 6.2, 4.9, 512 x 12000 5.0, 5.1, 640 x 12000 5.9, 6.5; 301 x 8192 3.9, 4.5 (bf16) and 3.9, 4.8 (fp32).
    const int threads = a.T <= 512 && a.V >= 12000 ? 1024 : 256;
    token_logprob_kernel<T, LOW><<<grid, threads, 0, stream>>>(logits, a.ld, V, a.labels, a.logp, lse, a.partial);
    if (splits > 1)
        token_join_kernel<T, LOW><<<static_cast<unsigned>((a.T + 3) / 4), 256, 0, stream>>>(logits, a.ld, a.T, V, a.labels, a.partial, splits, a.logp, lse);
}

template <typename T, bool LOW>
void bwd(const TokenLogprobBwd& a, hipStream_t stream)
{
    const int pieces = static_cast<int>((a.V + kPiece<T> - 1) / kPiece<T>);
    const dim3 grid(static_cast<unsigned>(a.T), static_cast<unsigned>((pieces + kChunk - 1) / kChunk));
    const bool past = a.T * a.V * static_cast<int64_t>(sizeof(T)) > kPastCaches;       // 8192 x 32000 in bf16: 178 to 172 us
    const auto kernel = past ? &token_logprob_bwd_kernel<T, true, LOW> : &token_logprob_bwd_kernel<T, false, LOW>;
    kernel<<<grid, 256, 0, stream>>>(a.d_logp, static_cast<const T*>(a.logits), a.ld, static_cast<int>(a.V), a.labels, lse_of<LOW>(a.lse, a.lse_low),
                                     static_cast<T*>(a.out), a.ld_out);
}

}  // namespace

// Very few rows are split over workgroups, down to 8192 elements each.
int token_splits(int64_t T, int64_t V)
{
    int s = 1;
    while (s < 64 && T * s < 256 && V / (2 * s) >= 8192) s *= 2;
    return s;
}

hipError_t launch_token_logprob(const TokenLogprob& a, bool f32, hipStream_t stream)
{
    const int splits = token_splits(a.T, a.V);
    if (a.lse_low) f32 ? fwd<float, true>(a, splits, stream) : fwd<uint16_t, true>(a, splits, stream);
    else f32 ? fwd<float, false>(a, splits, stream) : fwd<uint16_t, false>(a, splits, stream);
    return hipGetLastError();
}

hipError_t launch_token_logprob_bwd(const TokenLogprobBwd& a, bool f32, hipStream_t stream)
{
    if (a.lse_low) f32 ? bwd<float, true>(a, stream) : bwd<uint16_t, true>(a, stream);
    else f32 ? bwd<float, false>(a, stream) : bwd<uint16_t, false>(a, stream);
    return hipGetLastError();
}

hipError_t launch_preference_loss(const float* logp, const float* ref, const int64_t* offsets, int64_t T, int64_t P, float beta, float smoothing, float* pair_loss,
                                  float* loss, float* rewards, float* d_logp, hipStream_t stream)
{
    const Preference a{logp, ref, offsets, T, static_cast<int>(P), beta, smoothing, loss, rewards, d_logp};
    if (T <= kOneTokens && P <= kOnePairs) {
        preference_one_kernel<<<1, 1024, 0, stream>>>(a);
    } else {
        preference_pair_kernel<<<static_cast<unsigned>(P), 256, 0, stream>>>(a, pair_loss);
        preference_mean_kernel<<<1, 256, 0, stream>>>(pair_loss, static_cast<int>(P), loss);
    }
    return hipGetLastError();
}

}  // namespace falqon
