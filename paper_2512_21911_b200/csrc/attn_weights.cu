// sv_attn_weights: what attention weight the rows of a step give every cached token, added to what earlier steps gave it.
//
// Mathematics: w_t += sum over the rows r of a KV head of exp(scale * q_r . k_t - lse_r); the denominators lse are the attention's, which
// knows them only when it is through, so that the weights take a pass over the keys of their own.  Bound by HBM: 256 bytes of keys and 8 of
// weights a token.  A chain of eight over 32 K tokens (8 KV heads, 69 MB): 17.8 us, 60 % of a copy's rate, the rest being the beginning and the end
// of the launch; 16 sequences over 48 kept blocks (112 MB): 28.4.
//
// S^T[128 keys x N rows] = K . Q^T on the tensor cores, the keys as operand A as TMA brings them (M128 N K16, N = 16, 32 or 64 rows): a thread
// has a key's scores against all rows in its lane of tensor memory, and its weight is a sum within the thread.  A worker is a warpgroup
// with a ring of key tiles, queries and tensor memory of its own and takes an equal share of the batch's keys (q4_shares.h); the next unit's
// product runs under the exponentials of this one.
#include <cuda.h>
#include <cuda_bf16.h>

#include "attn_common.cuh"
#include "shares.cuh"
#include "sv_host.h"
#include "sv_ptx.cuh"

namespace {

using namespace svk;
using svq::kUnit;

struct Params {
    const int32_t *block_table, *seq_lens, *sel_idx, *sel_cnt, *path, *n_path;
    const __nv_bfloat16 *q;
    const float *lse, *before;
    float *after;
    int32_t *status;
    int S, Hq, Hkv, G, T, B, NBmax, n_pages, max_sel;
    float scale_log2;
};

template <int N>
struct Form {
    static constexpr int kWorkers = 2, kThreads = kWorkers * 128, kStages = 3;
    static constexpr int kHalf = 16384, kUnitBytes = 2 * kHalf;   // [2 halves of the dims][128 keys][128 bytes]
    static constexpr int kQBytes = N * 256;
    static constexpr int kOffQ = kWorkers * kStages * kUnitBytes;
    static constexpr int kOffMisc = kOffQ + kWorkers * kQBytes;
    // per worker: minus the denominators, barriers (stages, two products), of a stage's slabs their tokens and first one
    static constexpr int kNeg = 0, kBars = N * 4, kSlabs = kBars + (kStages + 2) * 8 + 8, kMiscBytes = (kSlabs + kStages * 16 + 127) / 128 * 128;
    static constexpr int kOffShared = kOffMisc + kWorkers * kMiscBytes;
    static constexpr int kSmem = 1024 + kOffShared + 256;
    static constexpr int kColumns = 2 * N;
    static_assert(kSmem <= 232448 && kSlabs % 16 == 0, "");
};

struct Place {
    int s, h, len, slabs, cnt;
    long long cost;
};
__device__ __forceinline__ Place place(const Params &p, int e)
{
    Place r;
    r.s = e / p.Hkv, r.h = e - r.s * p.Hkv;
    r.len = min(max(__ldg(p.seq_lens + r.s), 0), (int)min((long long)p.NBmax * p.B, 0x7fffffffll));
    r.cnt = p.sel_idx ? min(max(__ldg(p.sel_cnt + e), 0), min(p.max_sel, svq::kMostBlocks)) : 0;
    r.slabs = p.sel_idx ? r.cnt * (p.B / 64) : (r.len + 63) / 64;
    r.cost = svq::kItemCost + (long long)kUnit * ((r.slabs + 1) / 2);
    return r;
}

template <int N>
struct Worker {
    using F = Form<N>;
    const Params &p;
    const CUtensorMap &tm_k;
    uint32_t q_tile, ring, misc, shared, tmem;
    int wg, tid, lane, warp;
    uint32_t of_s = 0;              // parities of the two products
    int taken = 0, asked = 0;       // units of the ring
    int issued = 0;

    __device__ uint32_t bar_full(int i) const { return misc + F::kBars + i * 8; }
    __device__ uint32_t bar_s(int i) const { return bar_full(F::kStages + i); }
    __device__ void sync() const { named_bar_sync(1 + wg, 128); }
    __device__ bool aborted() const
    {
        uint32_t v;
        asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(v) : "r"(shared + 4) : "memory");
        return v != 0;
    }
    // Bounded.  Where it gives up it says so, later waits of the CTA look once, and everybody goes on to the end with what there is.
    __device__ void wait(uint32_t bar, uint32_t parity, int bit) const
    {
#pragma unroll 1
        for (int n = 0; n < 1 << 13; ++n) {
#pragma unroll 1
            for (int i = 0; i < 64; ++i)
                if (mbar_try_wait(bar, parity)) return;
            if (aborted()) return;
        }
        sts32(shared + 4, 1);
        if (p.status) atomicOr(p.status, bit);
    }
    // copies and products that nobody waited for, when a wait gave up
    __device__ void drain() const
    {
        if (!aborted()) return;
#pragma unroll 1
        for (int i = 0; i < F::kStages; ++i) {
            const int n = asked > i ? (asked - i + F::kStages - 1) / F::kStages : 0;
            if (n > 0) (void)mbar_wait_bounded(bar_full(i), (n - 1) & 1);
        }
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            const int n = (issued + 1 - i) / 2;
            if (n > 0) (void)mbar_wait_bounded(bar_s(i), (n - 1) & 1);
        }
    }

    int list_base = -1, known_row = 0, known_first = 0, known_valid = 0;   // (warp 0) a slab a lane: its first row of the pool, its first token, its tokens
    __device__ void look_up(const Place &pl, int from)
    {
        list_base = from;
        const int j = from + lane, per = p.B / 64;
        known_row = known_first = known_valid = 0;
        if (j >= pl.slabs) return;
        int b = j / per;
        const int sub = j - b * per;
        bool bad = false;
        if (p.sel_idx) {
            b = __ldg(p.sel_idx + ((size_t)pl.s * p.Hkv + pl.h) * p.max_sel + b);
            bad = (unsigned)b >= (unsigned)p.NBmax;
            b = min(max(b, 0), p.NBmax - 1);
        }
        int page = __ldg(p.block_table + (size_t)pl.s * p.NBmax + b);
        known_first = b * p.B + sub * 64;
        known_valid = (int)min(max((long long)pl.len - known_first, 0ll), 64ll);
        if (known_valid > 0) bad = bad || (unsigned)page >= (unsigned)p.n_pages;
        page = min(max(page, 0), p.n_pages - 1);
        if (bad && p.status) atomicOr(p.status, kStatusIndex);
        known_row = (page * p.Hkv + pl.h) * p.B + sub * 64;
    }
    __device__ void ask(const Place &pl, int u)
    {
        if (list_base < 0 || 2 * u >= list_base + 32) look_up(pl, 2 * u);
        const int i = 2 * u - list_base, stage = asked % F::kStages;
        const int ra = __shfl_sync(0xffffffffu, known_row, i), rb = __shfl_sync(0xffffffffu, known_row, (i + 1) & 31);
        const int fa = __shfl_sync(0xffffffffu, known_first, i), fb = __shfl_sync(0xffffffffu, known_first, (i + 1) & 31);
        const int va = __shfl_sync(0xffffffffu, known_valid, i), vb = __shfl_sync(0xffffffffu, known_valid, (i + 1) & 31);
        if (elect_one()) {
            const uint32_t full = bar_full(stage), dst = ring + stage * F::kUnitBytes;
            sts128(misc + F::kSlabs + stage * 16, make_uint4(va, vb, fa, fb));
            const bool second = 2 * u + 1 < pl.slabs;
            mbar_arrive_expect_tx(full, second ? F::kUnitBytes : F::kHalf);
            const uint64_t policy = policy_evict_first();
            tma_load_3d(dst, &tm_k, 0, ra, 0, full, policy);
            tma_load_3d(dst + F::kHalf, &tm_k, 0, ra, 1, full, policy);
            if (second) {
                tma_load_3d(dst + F::kHalf / 2, &tm_k, 0, rb, 0, full, policy);
                tma_load_3d(dst + F::kHalf + F::kHalf / 2, &tm_k, 0, rb, 1, full, policy);
            }
        }
        __syncwarp();
        ++asked;
    }
    // S^T of the next unit, into the place of its turn
    __device__ void issue()
    {
        constexpr uint32_t idesc = umma_idesc_bf16(128, N, false);
        const int stage = issued % F::kStages;
        wait(bar_full(stage), (issued / F::kStages) & 1, 1);
        if (elect_one()) {
            tc_fence_after_sync();
            const uint64_t dk = umma_desc_sw128(ring + stage * F::kUnitBytes, 16, 1024), dq = umma_desc_sw128(q_tile, 16, 1024);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                tc_mma_bf16(tmem + (issued & 1) * N, dk + (uint64_t)((ks & 3) * 2 + (ks >> 2) * (F::kHalf >> 4)),
                            dq + (uint64_t)((ks & 3) * 2 + (ks >> 2) * (N * 128 >> 4)), idesc, ks > 0);
            tc_commit(bar_s(issued & 1));
        }
        __syncwarp();
    }
    // What the tokens between this part's blocks had, and those behind the last block, where the sums go to another buffer.  A warp a gap:
    // their loads overlap those of the keys, and one another.  (The warpgroup gap by gap, a float a thread, ahead of the first keys: 36.6 us instead
    // of 28.1 where 16 sequences of up to 16 K tokens keep 48 blocks.)
    __device__ void keep(const Place &pl, const svq::Part &part, int units, size_t base) const
    {
        const int32_t *list = p.sel_idx + ((size_t)pl.s * p.Hkv + pl.h) * p.max_sel;
        const int per = p.B / 64, e0 = (2 * part.u0 + per - 1) / per;
        const int e1 = part.u1 == units ? pl.cnt + 1 : min((2 * part.u1 + per - 1) / per, pl.cnt);   // (the gap in front of block e, or of the end)
#pragma unroll 1
        for (int e = e0 + warp; e < e1; e += 4) {
            // (a list that may be bad: inside the sequence whatever it says)
            const long long from = e ? max((__ldg(list + e - 1) + 1ll) * p.B, 0ll) : 0ll, to = e < pl.cnt ? min((long long)__ldg(list + e) * p.B, (long long)pl.len) : pl.len;
            const float4 *src = reinterpret_cast<const float4 *>(p.before + base);
            float4 *dst = reinterpret_cast<float4 *>(p.after + base);
#pragma unroll 1
            for (long long t = from / 4 + lane; t < to / 4; t += 256) {
                float4 x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (t + 32 * i < to / 4) x[i] = __ldg(src + t + 32 * i);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (t + 32 * i < to / 4) dst[t + 32 * i] = x[i];
            }
            const long long t = to / 4 * 4 + lane;   // (the sequence ends where it likes)
            if (t >= from && t < to) p.after[base + t] = __ldg(p.before + base + t);
        }
    }

    __device__ void run(const Place &pl, const svq::Part &part)
    {
        const int units = (pl.slabs + 1) / 2, n_units = part.u1 - part.u0;
        const size_t base = ((size_t)pl.s * p.Hkv + pl.h) * p.NBmax * p.B;
        const int kept = p.path ? min(max(__ldg(p.n_path + pl.s), 0), p.T) : p.T, rows = kept * p.G;
#pragma unroll 1
        for (int row0 = 0; row0 < max(rows, 1); row0 += N) {
            sync();   // (the last queries have been used)
            if (warp == 0) {
                list_base = -1;
                for (int u = 0; u < min(n_units, F::kStages); ++u) ask(pl, part.u0 + u);
            }
            const auto token_of = [&](int row) {
                int i = row / p.G;
                if (p.path) {
                    i = __ldg(p.path + (size_t)pl.s * p.T + i);
                    if ((unsigned)i >= (unsigned)p.T) {
                        if (p.status) atomicOr(p.status, kStatusIndex);
                        i = min(max(i, 0), p.T - 1);
                    }
                }
                return ((size_t)pl.s * p.T + i) * p.Hq + pl.h * p.G + row % p.G;
            };
#pragma unroll
            for (int i = 0; i < N / 8; ++i) {
                const int c = i * 128 + tid, r = c >> 4, ch = c & 15;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (row0 + r < rows) v = __ldg(reinterpret_cast<const uint4 *>(p.q + token_of(row0 + r) * 128) + ch);
                sts128(q_tile + (ch >> 3) * (N * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4), v);
            }
            if (const int r = tid - (128 - N); r >= 0) {   // (not by the warp that has just waited for the lists)
                // (a row without a denominator gives nothing, as do rows that there are not)
                float neg = -INFINITY;
                if (row0 + r < rows) {
                    const float lse = __ldg(p.lse + token_of(row0 + r));
                    if (lse != -INFINITY) neg = -1.4426950408889634f * lse;
                }
                stsf(misc + F::kNeg + r * 4, neg);
            }
            fence_proxy_async();
            sync();
            if (warp == 0 && n_units > 0) issue();
            if (n_units > 0) ++issued;
            if (row0 == 0 && p.sel_idx && p.before != p.after) keep(pl, part, units, base);
            const unsigned long long scale2 = f2_pack(p.scale_log2, p.scale_log2);
#pragma unroll 1
            for (int k = 0; k < n_units; ++k) {
                const int stage = taken % F::kStages, place = taken & 1;
                wait(bar_full(stage), (taken / F::kStages) & 1, 1);
                const uint4 slabs = lds128(misc + F::kSlabs + stage * 16);
                const int slab = tid >> 6, valid = slab ? slabs.y : slabs.x, first = slab ? slabs.w : slabs.z;
                const size_t at = base + first + (tid & 63);
                const bool there = (tid & 63) < valid;
                float had = 0.f;
                if (there) had = row0 ? p.after[at] : p.before[at];
                sync();   // (everybody has read the scores of the unit before)
                if (k + 1 < n_units) {
                    if (warp == 0) issue();
                    ++issued;
                }
                wait(bar_s(place), of_s >> place & 1, 2);
                of_s ^= 1u << place;
                tc_fence_after_sync();
                ++taken;
                if (warp == 0 && k + F::kStages < n_units) ask(pl, part.u0 + k + F::kStages);
                unsigned long long sum2[2] = {0ull, 0ull};
                uint32_t s[N];
#pragma unroll
                for (int c = 0; c < N; c += 16) tmem_ld_x16(tmem + ((uint32_t)(warp * 32) << 16) + place * N + c, s + c);
                tmem_ld_wait();
#pragma unroll
                for (int r = 0; r < N; r += 4) {
                    const uint4 neg = lds128(misc + F::kNeg + r * 4);
                    float a, b, c, d;
                    f2_unpack(f2_fma(f2_pack(__uint_as_float(s[r]), __uint_as_float(s[r + 1])), scale2, f2_pack(__uint_as_float(neg.x), __uint_as_float(neg.y))), a, b);
                    f2_unpack(f2_fma(f2_pack(__uint_as_float(s[r + 2]), __uint_as_float(s[r + 3])), scale2, f2_pack(__uint_as_float(neg.z), __uint_as_float(neg.w))), c, d);
                    sum2[0] = f2_add(sum2[0], f2_pack(fast_exp2(a), fast_exp2(b)));
                    sum2[1] = f2_add(sum2[1], f2_pack(fast_exp2(c), fast_exp2(d)));
                }
                float a, b;
                f2_unpack(f2_add(sum2[0], sum2[1]), a, b);
                float sum = a + b;
                if (sum != sum) {   // a key that is not finite: rows that do not count give nothing all the same
                    sum = 0.f;
#pragma unroll
                    for (int r = 0; r < N; ++r) {
                        const float neg = __uint_as_float(lds32(misc + F::kNeg + r * 4));
                        if (neg != -INFINITY) sum += fast_exp2(fmaf(__uint_as_float(s[r]), p.scale_log2, neg));
                    }
                }
                if (there) p.after[at] = had + sum;
                tc_fence_before_sync();
            }
        }
    }
};

template <int N>
__global__ void __launch_bounds__(Form<N>::kThreads, 1) attn_weights_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ Params p)
{
    using F = Form<N>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u, shared = smem0 + F::kOffShared;
    const int tid = threadIdx.x, wg = tid >> 7, warp = tid >> 5;
    if (tid == 0) {
#pragma unroll 1
        for (int w = 0; w < F::kWorkers; ++w)
#pragma unroll 1
            for (int i = 0; i < F::kStages + 2; ++i) mbar_init(smem0 + F::kOffMisc + w * F::kMiscBytes + F::kBars + i * 8, 1);
        mbar_fence_init();
        sts32(shared + 4, 0);
        tma_prefetch_desc(&tm_k);
    }
    if (warp == 0) tmem_alloc(shared, 256);
    grid_dependency_wait();
    const int entries = p.S * p.Hkv;
    int per_cta;
    bool no_list = false;
    tc_fence_before_sync();
    const svq::Line line = find_shares<F::kThreads, F::kWorkers>(entries, 1, shared + 64, shared + 192, per_cta, [&](int e) {
        if (p.sel_idx) no_list |= __ldg(p.sel_cnt + e) < 0;
        return place(p, e).cost;
    });
    tc_fence_after_sync();
    if (no_list && blockIdx.x == 0 && p.status) atomicOr(p.status, kStatusNoList);
    const uint32_t tmem = lds32(shared);
    const int share = blockIdx.x * per_cta + wg;
    if (wg < per_cta && share < line.shares) {
        Worker<N> w{p, tm_k};
        w.wg = wg, w.tid = tid & 127, w.lane = tid & 31, w.warp = warp & 3;
        w.q_tile = smem0 + F::kOffQ + wg * F::kQBytes;
        w.ring = smem0 + wg * F::kStages * F::kUnitBytes;
        w.misc = smem0 + F::kOffMisc + wg * F::kMiscBytes;
        w.shared = shared;
        w.tmem = tmem + wg * F::kColumns;
        int e = (int)lds_ll(shared + 192 + wg * 16);
        long long at = lds_ll(shared + 192 + wg * 16 + 8);
        const long long hi = line.bound(share + 1);
#pragma unroll 1
        for (; e < entries && at < hi; ++e) {
            const Place pl = place(p, e);
            const svq::Part part = svq::part_of(line, share, at, pl.cost, (pl.slabs + 1) / 2, 1);
            if (part.mine) w.run(pl, part);
            at += pl.cost;
        }
        w.drain();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 0) tmem_dealloc(tmem, 256);
    grid_launch_dependents();
}

template <int N>
sv_status launch(const CUtensorMap &tm_k, const Params &p, void *stream)
{
    using F = Form<N>;
    static svh::OncePerDevice once;
    if (once.run([] { return cudaFuncSetAttribute(attn_weights_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmem); }) != cudaSuccess) {
        (void)cudaGetLastError();
        return SV_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(svh::sm_count());
    cfg.blockDim = dim3(F::kThreads);
    cfg.dynamicSmemBytes = F::kSmem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    svh::pdl_attribute(attr);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attn_weights_kernel<N>, tm_k, p) == cudaSuccess ? svh::launch_status() : SV_ERR_CUDA;
}

}  // namespace

extern "C" sv_status sv_attn_weights(const sv_geom *geom, const void *q, const sv_kv *kv, const float *lse, const int32_t *sel_idx,
                                     const int32_t *sel_cnt, int32_t max_sel, const int32_t *path, const int32_t *n_path, float softmax_scale,
                                     const float *weights, float *weights_out, int32_t *status_word, void *stream)
{
    sv_status st = svh::check_geom(geom);
    if (st != SV_OK) return st;
    st = svh::check_ragged(geom, 0);
    if (st != SV_OK) return st;
    st = svh::check_kv(geom, kv, false);
    if (st != SV_OK) return st;
    if (!q || !lse || !weights || !weights_out || (sel_idx && !sel_cnt) || (!path) != (!n_path)) return SV_ERR_NULL;
    if ((sel_idx && max_sel < 1) || !(softmax_scale >= 0.f && softmax_scale < INFINITY)) return SV_ERR_SHAPE;
    if ((int64_t)geom->n_seq * geom->n_kv_heads >= (int64_t)1 << 31) return SV_ERR_SHAPE;
    if (!svh::aligned(q, 16) || !svh::aligned(weights, 16) || !svh::aligned(weights_out, 16)) return SV_ERR_ALIGN;
    Params p = {};
    p.block_table = kv->block_table, p.seq_lens = kv->seq_lens, p.n_pages = kv->n_pages;
    p.sel_idx = sel_idx, p.sel_cnt = sel_cnt, p.max_sel = max_sel, p.path = path, p.n_path = n_path;
    p.q = static_cast<const __nv_bfloat16 *>(q), p.lse = lse, p.before = weights, p.after = weights_out, p.status = status_word;
    p.S = geom->n_seq, p.Hq = geom->n_q_heads, p.Hkv = geom->n_kv_heads, p.G = p.Hq / p.Hkv, p.T = geom->n_draft, p.B = geom->block_size,
    p.NBmax = geom->max_blocks;
    p.scale_log2 = (softmax_scale == 0.f ? 0.08838834764831845f : softmax_scale) * 1.4426950408889634f;
    CUtensorMap tm_k;
    if (!half_rows_tensor_map(kv->k_pool, (int64_t)p.n_pages * p.Hkv * p.B, 1, &tm_k)) return SV_ERR_CUDA;
    const int rows = p.G * p.T;
    return rows <= 16 ? launch<16>(tm_k, p, stream) : rows <= 32 ? launch<32>(tm_k, p, stream) : launch<64>(tm_k, p, stream);
}
