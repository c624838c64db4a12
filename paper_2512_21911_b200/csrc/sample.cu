// sv_sample: temperature, top-k, top-p and min-p on rows of logits, the kept entries' distribution and a token drawn from it.
//
// Mathematics: e(x) = 2^((x - max) log2 e / temperature).  The entries in descending order are never sorted: the k-th largest and the last
// one of the nucleus are found digit by digit of an order-preserving 32-bit key, by the number and the mass of the entries that share the
// digits so far.  Masses are whole multiples of 2^-40 (e <= 1, at most 2^20 entries: 60 bits), so that every sum is exact and no order
// of adding changes a result.  Simple form: a CTA per row, the logits read again by every pass.
#include <cuda_bf16.h>

#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxVocab = 1 << 20;

struct Params {
    const void *logits;
    long long stride;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *tokens;
    float *probs;
    int V, rows_per_param;
};

// Ascending in the logit; -0 equals +0.  Entries that are not there (NaN, -infinity) are 0.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x) == 0x80000000u ? 0u : __float_as_uint(x);
    return !(x > -INFINITY) ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

struct Row {
    const void *p;
    bool half;
    __device__ float operator[](int i) const
    {
        return half ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]) : static_cast<const float *>(p)[i];
    }
};

template <class T, class Op>
__device__ __forceinline__ T over_block(T v, T *shared, Op op)
{
    __syncthreads();
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[threadIdx.x & 31];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

using Mass = unsigned long long;

template <bool kHalf>
__global__ void __launch_bounds__(kThreads) sample_kernel(const Params p)
{
    __shared__ Mass scratch[kWarps];
    __shared__ uint32_t scratch32[kWarps];
    __shared__ Mass mass_of[256];
    __shared__ uint32_t count_of[256];
    __shared__ int chosen, token;
    __shared__ Mass ahead;
    svk::grid_dependency_wait();
    svk::grid_launch_dependents();
    const int r = blockIdx.x, tid = threadIdx.x, g = r / p.rows_per_param, V = p.V;
    const Row x{static_cast<const char *>(p.logits) + r * p.stride * (kHalf ? 2 : 4), kHalf};
    const auto add = [](Mass a, Mass b) { return a + b; };
    const auto most = [](uint32_t a, uint32_t b) { return max(a, b); };

    uint32_t top = 0;
    for (int i = tid; i < V; i += kThreads) top = max(top, key_of(x[i]));
    top = over_block(top, scratch32, most);
    const float T = p.temperature ? p.temperature[g] : 1.f;
    const bool greedy = !(T > 0.f);
    const float peak = logit_of(top), rate = 1.4426950408889634f / T;
    const auto e_of = [&](uint32_t key) { return key == top ? 1.f : key == 0 ? 0.f : svk::fast_exp2((logit_of(key) - peak) * rate); };
    const auto q_of = [&](uint32_t key) { return (Mass)__float2ull_rn(e_of(key) * 1099511627776.f); };

    // The entries that stay: those above `least`, and the first `ties` of those that equal it.
    uint32_t least = 1, ties = (uint32_t)V;
    const int k = greedy ? 1 : p.top_k ? p.top_k[g] : 0;
    const float top_p = p.top_p && !greedy ? p.top_p[g] : 1.f;
    const bool by_count = k > 0 && k < V, by_mass = top_p < 1.f;
    for (int step = 0; step < 2; ++step) {
        if (!(step ? by_mass : by_count)) continue;
        Mass goal = (Mass)k;   // what the entries up to the last one reach
        if (step) {
            Mass all = 0;
            for (int i = tid; i < V; i += kThreads) {
                const uint32_t key = key_of(x[i]);
                if (key > least || (key == least && ties == (uint32_t)V)) all += q_of(key);
            }
            all = over_block(all, scratch, add);
            if (ties != (uint32_t)V) all += ties * q_of(least);
            goal = max((Mass)1, (Mass)ceil((double)fmaxf(top_p, 0.f) * (double)all));
        }
        uint32_t prefix = 0, known = 0;
        Mass passed = 0;
        bool found = true;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) mass_of[tid] = 0, count_of[tid] = 0;
            __syncthreads();
            for (int i = tid; i < V; i += kThreads) {
                const uint32_t key = key_of(x[i]);
                if (key < least || key == 0 || (key & known) != prefix) continue;
                if (step && key == least && ties != (uint32_t)V) continue;
                atomicAdd(&count_of[key >> shift & 255], 1u);
                if (step) atomicAdd(&mass_of[key >> shift & 255], q_of(key));
            }
            __syncthreads();
            if (tid == 0) {
                if (step && ties != (uint32_t)V && (least & known) == prefix) {
                    mass_of[least >> shift & 255] += ties * q_of(least);
                    count_of[least >> shift & 255] += ties;
                }
                Mass sum = passed;
                int d = 255;
                for (; d >= 0; --d) {
                    const Mass here = step ? mass_of[d] : count_of[d];
                    if (count_of[d] && sum + here >= goal) break;
                    sum += here;
                }
                chosen = d, ahead = sum;
            }
            __syncthreads();
            if (chosen < 0) {   // fewer entries than that: all of them stay
                found = false;
                break;
            }
            prefix |= (uint32_t)chosen << shift, known |= 255u << shift;
            passed = ahead;
        }
        if (!found) continue;
        const Mass each = step ? q_of(prefix) : 1;
        const Mass need = goal - passed;
        Mass n = each ? (need + each - 1) / each : 0;
        if (prefix == least) n = min(n, (Mass)ties);
        least = prefix, ties = (uint32_t)max((Mass)1, min(n, (Mass)V));
    }
    float min_e = p.min_p && !greedy ? p.min_p[g] : 0.f;
    if (!(min_e > 0.f)) min_e = 0.f;

    // Entries in the order of the vocabulary, kThreads at a time: those that equal `least` are counted, the masses summed.
    Mass total = 0;
    for (int pass = 0; pass < 2; ++pass) {
        Mass before = 0;
        uint32_t equal_before = 0;
        const float u = pass && p.tokens ? fminf(fmaxf(p.u[r], 0.f), 1.f) : 0.f;
        const Mass target = pass ? max((Mass)1, min(total, (Mass)ceil((double)u * (double)total))) : 0;
        const float inv = pass ? 1099511627776.f / (float)total : 0.f;
        if (pass && tid == 0) token = -1;
        for (int base = 0; base < V; base += kThreads) {
            const int i = base + tid;
            const uint32_t key = i < V ? key_of(x[i]) : 0;
            const bool equal = key == least && key > 0;
            const uint32_t lower = (1u << (tid & 31)) - 1u, ballot = __ballot_sync(0xffffffffu, equal);
            __syncthreads();
            if ((tid & 31) == 0) scratch32[tid >> 5] = __popc(ballot);
            __syncthreads();
            uint32_t rank = equal_before + __popc(ballot & lower);
            for (int w = 0; w < kWarps; ++w) {
                if (w < tid >> 5) rank += scratch32[w];
                equal_before += scratch32[w];
            }
            const float e = e_of(key);
            const bool keep = key > 0 && (key > least || (equal && rank < ties)) && (e >= min_e || key == top);
            const Mass mine = keep ? q_of(key) : 0;
            Mass upto = mine;
            for (int d = 1; d < 32; d <<= 1) {
                const Mass o = __shfl_up_sync(0xffffffffu, upto, d);
                if ((tid & 31) >= d) upto += o;
            }
            if ((tid & 31) == 31) scratch[tid >> 5] = upto;
            __syncthreads();
            Mass chunk = 0;
            for (int w = 0; w < kWarps; ++w) {
                if (w < tid >> 5) upto += scratch[w];
                chunk += scratch[w];
            }
            if (pass && mine && before + upto >= target && before + upto - mine < target) token = i;
            if (pass && p.probs && i < V) p.probs[(size_t)r * V + i] = keep ? e * inv : 0.f;
            before += chunk;
        }
        __syncthreads();
        total = pass ? total : before;
    }
    if (tid == 0 && p.tokens) p.tokens[r] = token;
}

}  // namespace

extern "C" sv_status sv_sample(int32_t n_rows, int32_t vocab, const void *logits, int32_t logits_bf16, int64_t row_stride,
                               int32_t rows_per_param, const float *temperature, const int32_t *top_k, const float *top_p,
                               const float *min_p, const float *u, int32_t *tokens, float *probs, void *stream)
{
    if (n_rows < 0 || vocab < 1 || rows_per_param < 1 || n_rows % rows_per_param || row_stride < vocab) return SV_ERR_SHAPE;
    if (vocab > kMaxVocab) return SV_ERR_UNSUPPORTED;
    if ((!tokens && !probs) || (n_rows > 0 && (!logits || (tokens && !u)))) return SV_ERR_NULL;
    if (!svh::aligned(logits, logits_bf16 ? 2 : 4) || !svh::aligned(probs, 4)) return SV_ERR_ALIGN;
    if (n_rows == 0) return SV_OK;
    const Params p = {logits, row_stride, temperature, top_p, min_p, u, top_k, tokens, probs, vocab, rows_per_param};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n_rows);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    svh::pdl_attribute(attr);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, logits_bf16 ? sample_kernel<true> : sample_kernel<false>, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}
