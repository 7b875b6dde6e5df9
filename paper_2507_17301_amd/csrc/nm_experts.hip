// Routing of tokens to experts, and the weighted sum of what the experts answer.
#include "nm_mx4_device.h"

#include <type_traits>

namespace nm {
namespace {

// ---------------------------------------------------------------- routing
// Tokens go by in chunks, one a workgroup, a chunk in batches of 64.  A token belongs to L lanes, of V adjacent experts each.  A logit and its
// expert are one number (a rank): its upper bits sort like the logits, 10 below them fall with the expert, so that a maximum finds the largest
// logit and of equal ones the lowest expert.  Of bf16 it has 32 bits; of fp32 it is a double in [1, 2), with 42 bits of the fraction.
// The choices are taken one after another.
// The order by expert comes of one 64-bit mask an expert and batch, with a bit for each token that chose it: an expert's count is the number of
// its bits, a token's place among the batch's the number of bits below its own.  So no order of atomics shows in a result.
// Bound by the launches and the chain of steps for few tokens (16 x 64 logits 5.0 us), for many by the vector instructions of the choices (16384
// x 256, 8 choices: 10.2 us in bf16, 11.9 in fp32; with key and expert compared apart 14.2) and by what the second kernel adds up.
constexpr int kThreads = 1024, kBatch = NM_ROUTE_ONE_LAUNCH, kChunks = 256;
static_assert(kBatch == 64, "a bit for each token");

template <int CTRL> __device__ inline unsigned dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }

template <int CTRL> __device__ inline double dpp(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)dpp<CTRL>((unsigned)(u >> 32)) << 32 | dpp<CTRL>((unsigned)u));
}

template <int L> __device__ inline float sum_of(float v)
{
    for (int m = 1; m < L; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// 32 bits that sort like the values.  0 and -0 are the same, a NaN is more than infinity.
__device__ inline unsigned key_of(float f)
{
    if (f != f) return 0xffffffffu;
    const unsigned u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float logit_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
constexpr unsigned kClosed = 0x007fffffu;   // the key of minus infinity; no open expert has one as small
constexpr int kLast = NM_ROUTE_MAX_EXPERTS - 1;

template <bool BF16> struct Rank;
template <> struct Rank<true> {   // (a key's lower 16 bits are those of its sign)
    using Type = unsigned;
    static __device__ inline Type make(float f, int expert) { return (key_of(f) >> 16) << 10 | (unsigned)(kLast - expert); }
    static __device__ inline bool open(Type r) { return r >> 10 > kClosed >> 16; }
    static __device__ inline float logit(Type r) { return logit_of((r >> 10) << 16 | (r >> 25 & 1 ? 0u : 0xffffu)); }
    static __device__ inline int expert(Type r) { return kLast - (int)(r & kLast); }
    static __device__ inline Type larger(Type a, Type b) { return max(a, b); }
    template <int CTRL> static __device__ inline Type with(Type r) { return max(r, dpp<CTRL>(r)); }
    static __device__ inline Type without(Type r, Type taken) { return r == taken ? 0u : r; }
};
template <> struct Rank<false> {
    using Type = double;
    static __device__ inline unsigned low(Type r) { return (unsigned)__builtin_bit_cast(uint64_t, r); }   // (tells experts apart)
    static __device__ inline unsigned key(Type r) { return (unsigned)(__builtin_bit_cast(uint64_t, r) >> 10); }
    static __device__ inline Type make(float f, int expert)
    {
        return __builtin_bit_cast(double, 0x3ff0000000000000ull | (uint64_t)key_of(f) << 10 | (unsigned)(kLast - expert));
    }
    static __device__ inline bool open(Type r) { return key(r) > kClosed; }
    static __device__ inline float logit(Type r) { return logit_of(key(r)); }
    static __device__ inline int expert(Type r) { return kLast - (int)(low(r) & kLast); }
    // fmax of doubles that are no NaN (the compiler makes its own of two instructions each)
    static __device__ inline Type larger(Type a, Type b)
    {
        Type r;
        asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
        return r;
    }
    template <int CTRL> static __device__ inline Type with(Type r) { return fmax(r, dpp<CTRL>(r)); }
    static __device__ inline Type without(Type r, Type taken)   // (leaves a key below 2^22: closed)
    {
        return low(r) == low(taken) ? __builtin_bit_cast(double, 0x3ff0000000000000ull | low(r)) : r;
    }
};

template <int L, bool BF16> __device__ inline typename Rank<BF16>::Type best_of(typename Rank<BF16>::Type b)
{
    using R = Rank<BF16>;
    b = R::template with<0xb1>(b);    // lane ^ 1
    b = R::template with<0x4e>(b);    // lane ^ 2
    b = R::template with<0x141>(b);   // mirrored in eight
    b = R::template with<0x140>(b);   // mirrored in sixteen
    if constexpr (L == 64) {
        b = max(b, __shfl_xor(b, 16));
        b = max(b, __shfl_xor(b, 32));
    }
    return b;
}

// The ranks of V adjacent experts of a token.
template <int V, bool BF16> __device__ inline void ranks_of(const Route& r, int64_t token, int first, typename Rank<BF16>::Type (&rank)[V])
{
    constexpr int ES = Elem<BF16>::kBytes;
    float f[V];
    const char* row = (const char*)r.logits + (token * r.ld + first) * ES;
    if (first + V <= r.experts) {   // (through memcpy: rows start anywhere)
        if constexpr (BF16) {
            unsigned w[V / 2];
            __builtin_memcpy(w, row, V * 2);
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = __uint_as_float(v & 1 ? w[v / 2] & 0xffff0000u : w[v / 2] << 16);
        } else {
            __builtin_memcpy(f, row, V * 4);
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = first + v < r.experts ? Elem<BF16>::load1(row + v * ES) : -__builtin_inff();
    }
#pragma unroll
    for (int v = 0; v < V; ++v) rank[v] = Rank<BF16>::make(f[v], first + v);
}

// Chooses for the tokens of one batch; their bits go into mask.
template <int L, int V, bool BF16>
__device__ inline void choose(const Route& r, int64_t first, int count, unsigned long long* mask)
{
    constexpr int PER = kThreads / L, SLOTS = NM_ROUTE_MAX_CHOICES / L;   // tokens at a time; choices a lane keeps
    const int l = threadIdx.x % L;
    for (int t = threadIdx.x / L; t < count; t += PER) {
        const int64_t token = first + t;
        using R = Rank<BF16>;
        typename R::Type rank[V];
        ranks_of<V, BF16>(r, token, l * V, rank);
        float top = 0.0f, sum = 0.0f, p[SLOTS];
        int id[SLOTS];
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) { p[s] = 0.0f; id[s] = -1; }
        for (int j = 0; j < r.choices; ++j) {
            typename R::Type half = rank[V / 2], b = rank[0];
#pragma unroll
            for (int v = 1; v < V / 2; ++v) {
                b = R::larger(b, rank[v]);
                half = R::larger(half, rank[V / 2 + v]);
            }
            b = best_of<L, BF16>(max(b, half));
            if (!R::open(b)) break;   // (the same for all lanes of a token)
            const float logit = R::logit(b);
            if (j == 0) {
                top = logit;
                if (!r.normalise) {
                    float part = 0.0f;
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (R::open(rank[v])) part += expf(R::logit(rank[v]) - top);
                    sum = sum_of<L>(part);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) rank[v] = R::without(rank[v], b);
            const float e = expf(logit - top);
            if (r.normalise) sum += e;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s)
                if (j == s * L + l) { p[s] = e; id[s] = R::expert(b); }
        }
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const int j = s * L + l;
            if (j < r.choices) {
                const int64_t at = token * r.choices + j;
                r.ids[at] = id[s];
                r.weights[at] = id[s] < 0 ? 0.0f : p[s] / sum;
                if (id[s] >= 0) atomicOr(&mask[id[s]], 1ull << t);
            }
        }
    }
}

// Gives a batch's choices their entries; base: an expert's first entry for this batch.
__device__ inline void place(const Route& r, int64_t first, int count, const unsigned long long* mask, const int* base)
{
    for (int i = threadIdx.x; i < count * r.choices; i += kThreads) {
        const int t = i / r.choices;
        const int64_t at = first * r.choices + i;
        const int e = r.ids[at];
        int slot = -1;
        if (e >= 0) {
            slot = base[e] + __popcll(mask[e] & ((1ull << t) - 1));
            r.rows[slot] = (int)(first + t);
        }
        r.slots[at] = slot;
    }
}

// Entries past the last one, by all workgroups together.
__device__ inline void clear_rows(const Route& r, int from)
{
    for (int64_t i = from + (int64_t)blockIdx.x * kThreads + threadIdx.x; i < r.tokens * r.choices; i += (int64_t)gridDim.x * kThreads) r.rows[i] = -1;
}

struct Shared {
    unsigned long long mask[NM_ROUTE_MAX_EXPERTS];
    int base[NM_ROUTE_MAX_EXPERTS + 1];
    int part[2][kThreads];
    int waves[kThreads / 64];
};

// base[e] becomes the sum of base[0 .. e - 1]; returns the sum of all.
__device__ inline int scan(Shared& s, int experts)
{
    const int t = threadIdx.x, lane = t & 63;
    const int mine = t < experts ? s.base[t] : 0;
    int v = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(v, d);
        if (lane >= d) v += up;
    }
    if (lane == 63) s.waves[t >> 6] = v;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
        before += w < (t >> 6) ? s.waves[w] : 0;
        all += s.waves[w];
    }
    if (t < experts) s.base[t] = before + v - mine;
    __syncthreads();
    return all;
}

// A chunk's counts: bytes where it is one batch, in rows of whole words, otherwise ints.
__host__ __device__ inline int count_stride(int experts) { return (experts + 3) & ~3; }

// All that there is to do where the tokens are one batch; otherwise the choices and each chunk's counts.
template <int L, int V, bool BF16>
__global__ __launch_bounds__(kThreads) void route_choose_kernel(Route r, int chunk, void* counts)
{
    __shared__ Shared s;
    const int64_t first = (int64_t)blockIdx.x * chunk;
    const int64_t end = first + chunk < r.tokens ? first + chunk : r.tokens;
    const int e = threadIdx.x;
    int total = 0;
    for (int64_t at = first; at < end || at == first; at += kBatch) {
        if (e < r.experts) s.mask[e] = 0;
        __syncthreads();
        const int count = (int)(end - at < kBatch ? (end > at ? end - at : 0) : kBatch);
        choose<L, V, BF16>(r, at, count, s.mask);
        __syncthreads();
        if (e < r.experts) total += __popcll(s.mask[e]);
    }
    if (counts) {
        const int64_t row = (int64_t)blockIdx.x * count_stride(r.experts);
        if (e < r.experts) {
            if (chunk == kBatch) ((uint8_t*)counts)[row + e] = (uint8_t)total;
            else ((int*)counts)[row + e] = total;
        }
        return;
    }
    if (e < r.experts) s.base[e] = total;
    __syncthreads();
    const int all = scan(s, r.experts);
    if (e < r.experts) r.offsets[e] = s.base[e];
    if (e == 0) r.offsets[r.experts] = all;
    place(r, 0, (int)r.tokens, s.mask, s.base);
    clear_rows(r, all);
}

// The entries of one chunk: its first for each expert come after those of the experts and the chunks before.
// Every workgroup adds up all chunks' counts.  BYTES (chunks of one batch, 256 at most): a word has those of four experts, which are added as
// two pairs of 16 bits.  (16384 tokens of 256 experts: 6.4 us, with ints throughout 8.4; of 1024 experts the whole routing 45 and 55.)
template <bool BYTES>
__global__ __launch_bounds__(kThreads) void route_place_kernel(Route r, int chunk, const void* counts)
{
    __shared__ Shared s;
    constexpr int PER = BYTES ? 4 : 1, SUMS = BYTES ? 2 : 1;   // experts of a word; sums that a thread has
    const int t = threadIdx.x, chunks = gridDim.x, mine = blockIdx.x, words = count_stride(r.experts) / PER;
    int pad = 64;
    while (pad < words) pad <<= 1;   // threads of a part: the chunks are dealt to kThreads / pad of them
    const int parts = kThreads / pad, part = t / pad, w = t % pad;
    int all[SUMS] = {}, before[SUMS] = {};
    if (w < words) {
#pragma unroll 16
        for (int c = part; c < chunks; c += parts) {
            const int n = ((const int*)counts)[(int64_t)c * words + w];
            if constexpr (BYTES) {
                const int low = n & 0x00ff00ff, high = (n >> 8) & 0x00ff00ff;
                all[0] += low;
                all[1] += high;
                before[0] += c < mine ? low : 0;
                before[1] += c < mine ? high : 0;
            } else {
                all[0] += n;
                before[0] += c < mine ? n : 0;
            }
        }
    }
    auto put = [&](const int (&v)[SUMS]) {
#pragma unroll
        for (int i = 0; i < SUMS; ++i) s.part[i][t] = v[i];
    };
    auto sum = [&] {   // over the parts, of expert t
        int n = 0;
        for (int i = 0; i < parts; ++i) {
            if constexpr (BYTES) n += (s.part[t & 1][i * pad + (t >> 2)] >> (t & 2 ? 16 : 0)) & 0xffff;
            else n += s.part[0][i * pad + t];
        }
        return n;
    };
    put(all);
    __syncthreads();
    if (t < r.experts) s.base[t] = sum();
    __syncthreads();
    put(before);
    const int entries = scan(s, r.experts);
    if (mine == 0) {
        if (t < r.experts) r.offsets[t] = s.base[t];
        if (t == 0) r.offsets[r.experts] = entries;
    }
    if (t < r.experts) {   // (after scan's last barrier, which s.part's writes precede)
        s.base[t] += sum();
    }
    const int64_t first = (int64_t)mine * chunk;
    const int64_t end = first + chunk < r.tokens ? first + chunk : r.tokens;
    for (int64_t at = first; at < end; at += kBatch) {
        const int count = (int)(end - at < kBatch ? end - at : kBatch);
        if (t < r.experts) s.mask[t] = 0;
        __syncthreads();
        for (int i = t; i < count * r.choices; i += kThreads) {
            const int id = r.ids[at * r.choices + i];
            if (id >= 0) atomicOr(&s.mask[id], 1ull << (i / r.choices));
        }
        __syncthreads();
        place(r, at, count, s.mask, s.base);
        __syncthreads();
        if (t < r.experts) s.base[t] += __popcll(s.mask[t]);
    }
    clear_rows(r, entries);
}

inline int chunk_of(int64_t tokens)
{
    const int64_t each = (tokens + kChunks - 1) / kChunks;
    return (int)((each + kBatch - 1) / kBatch * kBatch);
}

// ---------------------------------------------------------------- combination
// Eight adjacent values of a row a thread.  Bound by HBM: the experts' rows are read once (4096 x 8 choices x 2048: of fp32
// 58 us, of bf16 31, 5.2 and 5.4 TB/s).
template <bool YBF16, bool BF16>
__global__ __launch_bounds__(256) void combine_kernel(Combine p, int units)
{
    constexpr int YS = Elem<YBF16>::kBytes, ES = Elem<BF16>::kBytes;
    const int64_t total = p.tokens * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = total <= 0xffffffffll ? (int64_t)((unsigned)i / (unsigned)units) : i / units;
        const int c = (int)(i - row * units) * 8;
        const bool whole = c + 8 <= p.width;
        float sum[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
        const int* slots = p.slots + row * p.choices;
        const float* weights = p.weights + row * p.choices;
#pragma unroll 4
        for (int j = 0; j < p.choices; ++j) {
            const int slot = slots[j];
            if (slot == -1) continue;
            const bool there = slot >= 0 && slot < p.entries;
            const float w = there ? weights[j] : __uint_as_float(0x7fc00000u);
            const char* py = (const char*)p.y + (there ? slot : 0) * p.ldy * YS + (size_t)c * YS;
            float v[8];
            if (whole && there) {
                Elem<YBF16>::load8(py, v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = there && c + e < p.width ? Elem<YBF16>::load1(py + e * YS) : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = fmaf(w, v[e], sum[e]);
        }
        char* po = (char*)p.out + (row * p.ldo + c) * ES;
        const char* pr = p.res ? (const char*)p.res + (row * p.ldr + c) * ES : nullptr;
        if (whole) {
            if (pr) {
                float r[8];
                Elem<BF16>::load8(pr, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += r[e];
            }
            Elem<BF16>::store8(po, sum);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < p.width) Elem<BF16>::store1(po + e * ES, pr ? sum[e] + Elem<BF16>::load1(pr + e * ES) : sum[e]);
        }
    }
}

}  // namespace

size_t route_workspace(int64_t tokens, int experts)
{
    if (tokens <= kBatch) return 0;
    const int chunk = chunk_of(tokens);
    return (size_t)((tokens + chunk - 1) / chunk) * count_stride(experts) * sizeof(int);
}

int run_route(const Route& r, void* workspace, hipStream_t s)
{
    const bool one = r.tokens <= kBatch;
    const int chunk = one ? kBatch : chunk_of(r.tokens);
    const dim3 grid(one ? 1u : (unsigned)((r.tokens + chunk - 1) / chunk));
    void* counts = one ? nullptr : workspace;
    auto choose = [&](auto bf16) {
        constexpr bool BF16 = decltype(bf16)::value;
        if (r.experts <= 64) hipLaunchKernelGGL((route_choose_kernel<16, 4, BF16>), grid, dim3(kThreads), 0, s, r, chunk, counts);
        else if (r.experts <= 256) hipLaunchKernelGGL((route_choose_kernel<16, 16, BF16>), grid, dim3(kThreads), 0, s, r, chunk, counts);
        else hipLaunchKernelGGL((route_choose_kernel<64, 16, BF16>), grid, dim3(kThreads), 0, s, r, chunk, counts);
    };
    if (r.bf16) choose(std::true_type{});
    else choose(std::false_type{});
    NM_HIP_CHECK(hipGetLastError());
    if (one) return NM_OK;
    if (chunk == kBatch) hipLaunchKernelGGL((route_place_kernel<true>), grid, dim3(kThreads), 0, s, r, chunk, (const void*)counts);
    else hipLaunchKernelGGL((route_place_kernel<false>), grid, dim3(kThreads), 0, s, r, chunk, (const void*)counts);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

int run_combine(const Combine& c, hipStream_t s)
{
    const int units = (c.width + 7) / 8;
    const int64_t blocks = (c.tokens * units + 255) / 256;
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
    if (c.y_bf16 && c.bf16) hipLaunchKernelGGL((combine_kernel<true, true>), grid, dim3(256), 0, s, c, units);
    else if (c.y_bf16) hipLaunchKernelGGL((combine_kernel<true, false>), grid, dim3(256), 0, s, c, units);
    else if (c.bf16) hipLaunchKernelGGL((combine_kernel<false, true>), grid, dim3(256), 0, s, c, units);
    else hipLaunchKernelGGL((combine_kernel<false, false>), grid, dim3(256), 0, s, c, units);
    NM_HIP_CHECK(hipGetLastError());
    return NM_OK;
}

}  // namespace nm
