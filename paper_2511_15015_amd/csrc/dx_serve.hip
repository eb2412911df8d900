// Serving steps around the expert layers: the host side of the calls on the
// paged key/value cache, the plan of a step's pages and slots, the writes into
// the cache, and the verification of drafted tokens.  Attention is in
// dx_attention.hip.
#include "dx_internal.h"
#include "dx_route_core.h"

#include <cmath>

namespace {

// ---- the plan of a step --------------------------------------------------------------
// One block: prefix sums over the requests of pages returned, pages taken and new tokens, in LDS.  Then a thread deals with a
// request's pages and tokens if they are few (decoding), and lists it otherwise; the listed ones are dealt out to the wavefronts by
// 512 items, eight loads of a lane on their way together.  Bound by the latency of its dependent rounds of loads and
// barriers: 1001 requests, 15 thousand pages returned and 8000 new tokens 20 us a pass, 32 requests 8.  (A bisection of the prefix sums for
// every item 44 and 9, eight of them side by side 40 and 17: that is bound by LDS.)
constexpr int kPlanThreads = 1024, kMost = 1 << 22; // most pages, and new tokens, of a request (sums of a wavefront's in 32 bits)

struct request {
    int base, count, held, want; // tokens kept, new tokens, pages held, pages wanted
    bool bad;
};

__device__ request read_request(const dx_plan_args &a, int b)
{
    const long l = a.lens_in[b], d = a.drops ? a.drops[b] : 0, n = a.new_lens[b];
    const long most = (long)a.stride << a.page_shift, pm = (1L << a.page_shift) - 1;
    request r{};
    r.bad = l < 0 || d < 0 || d > l || n < -1 || l > most || (n > 0 && l - d + n > most) || n > kMost || l >> a.page_shift > kMost;
    if (r.bad) return r;
    r.base = n < 0 ? 0 : (int)(l - d);
    r.count = n < 0 ? 0 : (int)n;
    r.held = (int)((l + pm) >> a.page_shift);
    r.want = (int)((r.base + r.count + pm) >> a.page_shift);
    return r;
}

// For the items 0 .. pre[b + 1] - pre[b] - 1 of every request b: x = load(b, item), then use(b, item, x).  All threads of the block
// call it; s_list, s_listed (0 on entry): LDS.
template <class L, class U> __device__ __forceinline__ void for_items(const int *pre, int B, int *s_list, int *s_listed, L load, U use)
{
    constexpr int FEW = 8, PART = 512;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int b = threadIdx.x; b < B; b += kPlanThreads) {
        const int n = pre[b + 1] - pre[b];
        if (n > FEW) {
            s_list[atomicAdd(s_listed, 1)] = b; // (in any order)
        } else if (n > 0) {
            int x[FEW];
#pragma unroll
            for (int j = 0; j < FEW; ++j)
                if (j < n) x[j] = load(b, j);
#pragma unroll
            for (int j = 0; j < FEW; ++j)
                if (j < n) use(b, j, x[j]);
        }
    }
    __syncthreads();
    const int listed = *s_listed;
    for (int e0 = 0; e0 < listed; e0 += 64) {
        const int e = e0 + lane, own_b = e < listed ? s_list[e] : 0, own_n = e < listed ? pre[own_b + 1] - pre[own_b] : 0;
        const int own_at = ((wave - e) & (kPlanThreads / 64 - 1)) * PART; // this wavefront's first part
        for (unsigned long long m = __ballot(own_at < own_n); m; m &= m - 1) {
            const int k = __ffsll(m) - 1, b = __shfl(own_b, k), n = __shfl(own_n, k);
            for (int at = __shfl(own_at, k); at < n; at += kPlanThreads / 64 * PART) {
                int x[PART / 64];
#pragma unroll
                for (int j = 0; j < PART / 64; ++j)
                    if (at + 64 * j + lane < n) x[j] = load(b, at + 64 * j + lane);
#pragma unroll
                for (int j = 0; j < PART / 64; ++j)
                    if (at + 64 * j + lane < n) use(b, at + 64 * j + lane, x[j]);
            }
        }
    }
}

__global__ __launch_bounds__(kPlanThreads) void k_plan(dx_plan_args a)
{
    constexpr int MOST = DX_SERVE_MAX_REQUESTS;
    __shared__ int s_ret[MOST + 1], s_take[MOST + 1], s_q[MOST + 1]; // pages returned, pages taken, new tokens before a request
    __shared__ int s_fewer[MOST], s_base[MOST];                      // the smaller of the pages held and wanted; tokens kept
    __shared__ long s_wave[kPlanThreads / 64][3];
    __shared__ int s_list[MOST], s_listed[4];
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long free_in = a.free_in[0];
    if (tid == 0) s_bad = 0;
    if (tid < 4) s_listed[tid] = 0;
    const int per = (a.B + kPlanThreads - 1) / kPlanThreads;
    uint32_t sum[3] = {0, 0, 0};
    int bad = 0;
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b >= a.B) break;
        const request r = read_request(a, b);
        bad += r.bad;
        s_fewer[b] = min(r.held, r.want);
        s_base[b] = r.base;
        // (this request's own numbers for now)
        s_ret[b] = max(r.held - r.want, 0);
        s_take[b] = max(r.want - r.held, 0);
        s_q[b] = r.count;
        sum[0] += s_ret[b];
        sum[1] += s_take[b];
        sum[2] += s_q[b];
    }
    uint32_t inc[3];
    for (int k = 0; k < 3; ++k) {
        inc[k] = (uint32_t)dx_route_core::wave_scan_inclusive((int)sum[k]);
        if (lane == 63) s_wave[wave][k] = inc[k];
    }
    __syncthreads();
    if (bad) atomicAdd(&s_bad, bad);
    long before[3] = {0, 0, 0}, total[3] = {0, 0, 0};
    for (int w = 0; w < kPlanThreads / 64; ++w)
        for (int k = 0; k < 3; ++k) {
            if (w < wave) before[k] += s_wave[w][k];
            total[k] += s_wave[w][k];
        }
    for (int k = 0; k < 3; ++k) before[k] += (long)(inc[k] - sum[k]);
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b >= a.B) break;
        int *const pre[3] = {s_ret, s_take, s_q};
        for (int k = 0; k < 3; ++k) {
            const int own = pre[k][b];
            pre[k][b] = (int)before[k];
            before[k] += own;
        }
    }
    // (totals beyond 31 bits need more pages or tokens than there can be: refused below)
    const long n_ret = total[0], n_take = total[1], n_new = total[2];
    if (tid == 0) {
        s_ret[a.B] = (int)n_ret;
        s_take[a.B] = (int)n_take;
        s_q[a.B] = (int)n_new;
        if (n_new > a.T || free_in < 0 || n_ret > a.n_pages || free_in + n_ret > a.n_pages) atomicAdd(&s_bad, 1);
    }
    __syncthreads();
    const bool sane = s_bad == 0;
    auto entry = [&](int b, int i) -> int32_t & { return a.table[(long)b * a.stride + s_fewer[b] + i]; };
    __syncthreads();
    if (sane) {
        int none = 0;
        for_items(s_ret, a.B, s_list, s_listed, entry, [&](int, int, int page) { none += (uint32_t)page >= (uint32_t)a.n_pages; });
        if (none) atomicAdd(&s_bad, none);
    }
    __syncthreads();
    const int n_bad = s_bad;
    const long top = free_in + n_ret, missing = n_bad ? 0 : max(n_take - top, 0L);
    const bool fine = n_bad == 0 && missing == 0;
    if (fine) {
        for_items(s_ret, a.B, s_list, s_listed + 1, entry, [&](int b, int i, int page) { a.free_list[free_in + s_ret[b] + i] = page; });
        __threadfence_block();
        __syncthreads();
        for_items(s_take, a.B, s_list, s_listed + 2, [&](int b, int i) { return a.free_list[top - 1 - (s_take[b] + i)]; },
                  [&](int b, int i, int page) { entry(b, i) = page; });
    }
    for (int i = 0; i < per; ++i) { // (lens_out may be lens_in, of which the block has read everything)
        const int b = tid * per + i;
        if (b >= a.B) break;
        a.lens_out[b] = fine ? s_base[b] + s_q[b + 1] - s_q[b] : a.lens_in[b];
        if (a.spent && fine) a.spent[b] = 0; // (read by the same thread)
    }
    for (int b = tid; b <= a.B; b += kPlanThreads) a.q_offsets[b] = fine ? s_q[b] : 0;
    if (tid == 0) {
        a.free_out[0] = (int)(fine ? top - n_take : free_in);
        a.status[0] = fine ? (int)n_take : 0;
        a.status[1] = fine ? (int)n_ret : 0;
        a.status[2] = (int)min(missing, 0x7FFFFFFFL);
        a.status[3] = n_bad;
    }
    __threadfence_block();
    __syncthreads();
    const int n_real = fine ? (int)n_new : 0;
    if (fine)
        for_items(
            s_q, a.B, s_list, s_listed + 3, [&](int b, int i) { return a.table[(long)b * a.stride + ((s_base[b] + i) >> a.page_shift)]; },
            [&](int b, int i, int page) {
                const int pos = s_base[b] + i, t = s_q[b] + i;
                a.positions[t] = pos;
                a.slots[t] = (uint32_t)page < (uint32_t)a.n_pages ? (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
            });
    for (int t = n_real + tid; t < a.T; t += kPlanThreads) a.slots[t] = a.positions[t] = -1;
}

// ---- writes into the cache ------------------------------------------------------
struct write_args {
    dx_kv_cache c;
    const dx_bf16 *k, *v;
    long k_stride, v_stride;
    const int32_t *slots;
    int T, page_shift;
};

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

__device__ float widen(uint32_t x) { return __uint_as_float(x << 16); }

// Division by the scale of a head, cut to the largest e4m3 value (NaN passes).  With the correctly rounded reciprocal r,
// q = x r is off by an ulp at most, and q + r (x - q s), both steps fused, is the correctly rounded quotient (Markstein);
// infinities and what is cut anyway stay as they are.  A scale whose reciprocal leaves the range is divided by as it is.
struct divide {
    float s, r;
    __device__ divide(float scale) : s(scale), r(__fdiv_rn(1.f, scale)) {}
    __device__ float operator()(float x) const
    {
        float q;
        if (s > 1e-30f && s < 1e30f) {
            q = x * r;
            const float off = __builtin_fmaf(-q, s, x), better = __builtin_fmaf(off, r, q);
            q = fabsf(q) < 1000.f && off != 0.f ? better : q; // (off = 0: also -0 as it is)
        } else {
            q = __fdiv_rn(x, s);
        }
        return q > 448.f ? 448.f : q < -448.f ? -448.f : q;
    }
};
// four bf16 (two words) as four e4m3, nearest even
__device__ uint32_t to_e4m3(uint32_t lo, uint32_t hi, const divide &by)
{
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(by(widen(lo & 0xFFFF)), by(widen(lo >> 16)), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(by(widen(hi & 0xFFFF)), by(widen(hi >> 16)), w, true);
}

// WAVES wavefronts per token.  Keys: 16 bytes of the cache are X channels of one token.  Values: 16 bytes are X tokens of one channel, so where
// X tokens in a row go to one such group of slots (prompts), each of them writes an X-th of the channels for all; other tokens
// (decoding) write single elements.  Bound by memory for prompts, by latency for few tokens: 7001 tokens of 2 heads of 256 channels, us a
// pass, in e4m3 (22 MB) 10.3 and in bf16 (29 MB) 8.9; every token to a slot of its own somewhere 17.5 and 18.5 (a line of 16
// or 8 channels is written for an element of each); one token 6, of which 5 are any launch.  Of a group's channels two to a thread for four
// tokens: for all X of them 13.3 and 9.3.
template <bool FP8, int WAVES> __global__ __launch_bounds__(256) void k_kv_write(write_args a)
{
    constexpr int X = FP8 ? 16 : 8, THREADS = 64 * WAVES;
    const int D = a.c.head_dim, per = a.c.kv_heads * D, lane = threadIdx.x & 63, P = 1 << a.page_shift;
    const int t = blockIdx.x * (256 / THREADS) + __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS), tid = threadIdx.x % THREADS;
    if (t >= a.T) return;
    // lane i: the slot of token t - X + 1 + i
    const int near = t - X + 1 + lane;
    const int32_t mine = lane < 2 * X - 1 && near >= 0 && near < a.T ? a.slots[near] : -1;
    const int slot = __shfl(mine, X - 1);
    const int page = slot >> a.page_shift, off = slot & (P - 1);
    if (slot < 0 || page >= a.c.n_pages) return;
    // the X tokens of the slot's group, if they are in a row: lanes X - 1 - off % X and on
    const int lead = X - 1 - off % X;
    const unsigned long long in_row = __ballot(mine == slot + lane - (X - 1)) >> lead;
    const bool together = (in_row & ((1ull << X) - 1)) == (1ull << X) - 1;
    const long head_size = (long)D * P, base = (long)page * a.c.kv_heads * head_size;
    const char *k = reinterpret_cast<const char *>(a.k + t * a.k_stride), *v = reinterpret_cast<const char *>(a.v + t * a.v_stride);
#pragma unroll 2
    for (int i = tid; i < per / X; i += THREADS) {
        const int h = i * X / D, d = i * X % D;
        const long at = base + h * head_size + (long)(d * P + off * X);
        if constexpr (FP8) {
            const u32x4 x = reinterpret_cast<const u32x4 *>(k)[2 * i], y = reinterpret_cast<const u32x4 *>(k)[2 * i + 1];
            const divide s(a.c.k_scale[h]);
            *reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(a.c.k) + at) =
                u32x4{to_e4m3(x[0], x[1], s), to_e4m3(x[2], x[3], s), to_e4m3(y[0], y[1], s), to_e4m3(y[2], y[3], s)};
        } else {
            *reinterpret_cast<u32x4 *>(static_cast<dx_bf16 *>(a.c.k) + at) = reinterpret_cast<const u32x4 *>(k)[i];
        }
    }
    // two channels to a thread
    const int pairs = per / 2;
    auto to_v = [&](int i, int first) { // 16 bytes of the first of channels 2 i and 2 i + 1 (those of the second follow), from token `first` of X on
        return static_cast<char *>(a.c.v) + (base + 2 * i / D * head_size + ((long)(off / X) * D + 2 * i % D) * X + first) * (16 / X);
    };
    if (together) { // each of the tokens writes its part of the channels for all, a thread those of four
        const int first = pairs / X * (off % X), four = tid % (X / 4) * 4;
        v += 2 * (four - off % X) * a.v_stride;
#pragma unroll 4
        for (int i = first + tid / (X / 4); i < first + pairs / X; i += THREADS / (X / 4)) {
            uint32_t w[4]; // two channels of a token
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = reinterpret_cast<const uint32_t *>(v + 2 * j * a.v_stride)[i];
            const uint32_t lo[2] = {(w[0] & 0xFFFF) | w[1] << 16, (w[2] & 0xFFFF) | w[3] << 16};
            const uint32_t hi[2] = {w[0] >> 16 | (w[1] & 0xFFFF0000), w[2] >> 16 | (w[3] & 0xFFFF0000)};
            char *to = to_v(i, four);
            if constexpr (FP8) {
                const divide s(a.c.v_scale[2 * i / D]);
                *reinterpret_cast<uint32_t *>(to) = to_e4m3(lo[0], lo[1], s);
                *reinterpret_cast<uint32_t *>(to + 16) = to_e4m3(hi[0], hi[1], s);
            } else {
                *reinterpret_cast<u32x2 *>(to) = u32x2{lo[0], lo[1]};
                *reinterpret_cast<u32x2 *>(to + 16) = u32x2{hi[0], hi[1]};
            }
        }
        return;
    }
#pragma unroll 4
    for (int i = tid; i < pairs; i += THREADS) {
        const uint32_t w = reinterpret_cast<const uint32_t *>(v)[i];
        char *to = to_v(i, off % X);
        if constexpr (FP8) {
            const uint32_t e = to_e4m3(w, 0, divide(a.c.v_scale[2 * i / D]));
            to[0] = (char)e;
            to[16] = (char)(e >> 8);
        } else {
            *reinterpret_cast<dx_bf16 *>(to) = (dx_bf16)w;
            *reinterpret_cast<dx_bf16 *>(to + 16) = (dx_bf16)(w >> 16);
        }
    }
}

// ---- verification of drafts -------------------------------------------------------
// Every block judges its request's drafts (a lane to a draft) and adds up the weights of one chunk of the vocabulary; the last block of a request
// to do so finds the chunk, then the token, that the mark falls into.  Sums of whole numbers, so that neither the chunks nor their
// order matter.  Bound by one row of p and one of q per request, by latency for few requests.
constexpr int kChunk = 4096, kVerifyThreads = 256; // tokens of a chunk, 16 to a thread
// In a sum that has been stored (a sum is below 2^51).  The last block looks for it in every one, so that nothing hangs on the order in which the
// others' sums and counts become visible: a fence in every block, which would settle that order, took 61 requests from 15 to 82 us.
constexpr unsigned long long kStored = 1ull << 63;
constexpr int kCount = (1 << 20) / kChunk, kSums = kCount + 32; // (counts of several requests in one line: 26 us)

struct verify_args {
    const float *p, *q;
    const int32_t *draft, *offsets;
    const float *u_accept, *u_sample;
    int32_t *tokens, *accepted, *drops; // drops may be null
    int B, n_drafts, max_n, V;
    unsigned long long *sums; // [B, kSums], 0 between calls: of a request's chunks (and kStored), from kCount on how many there are
    const int32_t *status;    // of the step's plan, or null
};

struct verdict {
    int first, n, a; // first draft of the request, drafts that are judged, accepted ones
    int more;        // drafts behind those
};

// (offsets outside the arrays are cut to them)
__device__ verdict drafts_of(const verify_args &a, int b)
{
    verdict r;
    const int lo = min(max(a.offsets[b], 0), a.n_drafts), hi = min(max(a.offsets[b + 1], lo), a.n_drafts);
    r.first = lo;
    r.n = min(hi - lo, a.max_n);
    r.a = r.n;
    r.more = hi - lo - r.n;
    return r;
}

// the accepted drafts of request b, the same in every wavefront
__device__ verdict judge(const verify_args &a, int b)
{
    verdict r = drafts_of(a, b);
    const int lane = threadIdx.x & 63;
    for (int i0 = 0; i0 < r.n; i0 += 64) {
        const int i = i0 + lane;
        bool refused = false;
        if (i < r.n) {
            const int x = a.draft[r.first + i];
            refused = true;
            if (x >= 0 && x < a.V) {
                const double px = a.p[(long)(r.first + b + i) * a.V + x], qx = a.q ? a.q[(long)(r.first + i) * a.V + x] : 1.f;
                refused = !((double)a.u_accept[r.first + i] * qx < px);
            }
        }
        const unsigned long long m = __ballot(refused);
        if (m) {
            r.a = i0 + __ffsll(m) - 1;
            break;
        }
    }
    return r;
}

// a weight, as the whole number that it is: a power of two times a float, truncated
__device__ float weight(float p, float q) { return truncf(fminf(fmaxf(p - q, 0.f), 1.f) * 549755813888.f); } // 2^39; (fmaxf drops a NaN)

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef f32x4 f32x4_any __attribute__((aligned(4))); // rows start at any multiple of 4 bytes

// What is drawn from at r.a: p - q of the refused draft, or p alone.  q null in the call: q is 1 at the draft.
struct rest {
    const float *p, *q;
    int taken; // token of which q is all, or -1
    __device__ rest(const verify_args &a, int b, const verdict &r)
    {
        p = a.p + (long)(r.first + b + r.a) * a.V;
        q = r.a < r.n && a.q ? a.q + (long)(r.first + r.a) * a.V : nullptr;
        taken = r.a < r.n && !a.q ? a.draft[r.first + r.a] : -1;
    }
    // 4 weights from v on (0 past the end)
    __device__ void read(int v, int V, float *w) const
    {
        f32x4 pv = {0.f, 0.f, 0.f, 0.f}, qv = pv;
        if (v + 4 <= V) {
            pv = *reinterpret_cast<const f32x4_any *>(p + v);
            if (q) qv = *reinterpret_cast<const f32x4_any *>(q + v);
        } else {
            for (int i = 0; i < 4; ++i)
                if (v + i < V) {
                    pv[i] = p[v + i];
                    if (q) qv[i] = q[v + i];
                }
        }
        if (taken >= 0)
            for (int i = 0; i < 4; ++i) qv[i] = v + i == taken ? 1.f : 0.f;
        for (int i = 0; i < 4; ++i) w[i] = weight(pv[i], qv[i]);
    }
};

// inclusive prefix sum over the block; total: of all
__device__ unsigned long long block_scan(unsigned long long x, unsigned long long *s_wave, unsigned long long &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long up = __shfl_up(x, o);
        if (lane >= o) x += up;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = x;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kVerifyThreads / 64; ++w) {
        if (w < wave) x += s_wave[w];
        total += s_wave[w];
    }
    return x;
}

// PLANNED: of a step whose plan's status there is (a branch on the pointer instead cost the calls without one 0.5 to 1 us)
template <bool PLANNED> __global__ __launch_bounds__(kVerifyThreads) void k_verify(verify_args a)
{
    static_assert((1 << 20) / kChunk <= kVerifyThreads, "a chunk's sum to a thread");
    __shared__ double s_sum[kVerifyThreads / 64];
    __shared__ unsigned long long s_wave[kVerifyThreads / 64], s_best[kVerifyThreads / 64], s_before;
    __shared__ int s_found, s_last;
    const int b = blockIdx.y, chunks = gridDim.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long *const sums = a.sums + (long)b * kSums;
    if (PLANNED && (a.status[2] | a.status[3])) { // there was no step: p is of no tokens
        if (blockIdx.x == 0) {
            for (int i = tid; i <= a.max_n; i += kVerifyThreads) a.tokens[(long)b * (a.max_n + 1) + i] = -1;
            if (tid == 0) a.accepted[b] = 0;
        }
        return;
    }
    const verdict r = judge(a, b);
    const rest s(a, b, r);
    double sum = 0.; // exact: 4096 whole numbers of up to 2^39
#pragma unroll
    for (int i = 0; i < kChunk / (4 * kVerifyThreads); ++i) {
        float w[4];
        s.read(blockIdx.x * kChunk + 4 * (i * kVerifyThreads + tid), a.V, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += w[e];
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kVerifyThreads / 64; ++w) sum += s_sum[w];
        __hip_atomic_store(&sums[blockIdx.x], (unsigned long long)sum | kStored, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = __hip_atomic_fetch_add(&sums[kCount], 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned long long)chunks - 1;
        if (s_last) __hip_atomic_store(&sums[kCount], 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
    unsigned long long own = 0;
    if (tid < chunks) {
        unsigned long long *const at = &sums[tid];
        do own = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); // (all have been sent: this ends)
        while (!(own & kStored));
        own &= ~kStored;
        __hip_atomic_store(at, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    const float us = fminf(fmaxf(a.u_sample[b], 0.f), 1.f);
    const unsigned long long u = min((unsigned long long)(us * 16777216.f), 16777215ull);
    unsigned long long W;
    const unsigned long long upto = block_scan(own, s_wave, W), mark = (W >> 24) * u + (((W & 0xFFFFFF) * u) >> 24);
    int token;
    if (W) {
        if (upto > mark && upto - own <= mark) { // (mark < W: one thread's)
            s_found = tid;
            s_before = upto - own;
        }
        __syncthreads();
        const int v0 = s_found * kChunk + 16 * tid;
        unsigned long long before = s_before, mine = 0, all;
        float w[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) s.read(v0 + 4 * i, a.V, w + 4 * i);
#pragma unroll
        for (int i = 0; i < 16; ++i) mine += (unsigned long long)w[i];
        before += block_scan(mine, s_wave, all) - mine;
        if (mark >= before && mark < before + mine) {
            int at = v0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                before += (unsigned long long)w[i];
                at += before <= mark;
            }
            s_found = at;
        }
        __syncthreads();
        token = s_found;
    } else { // nothing to draw from: the largest p, the first of its kind
        unsigned long long best = 0;
        for (int v = tid; v < a.V; v += kVerifyThreads)
            if (s.p[v] > 0.f) best = max(best, (unsigned long long)__float_as_uint(s.p[v]) << 32 | (uint32_t)~v);
        for (int o = 32; o; o >>= 1) best = max(best, __shfl_xor(best, o));
        if (lane == 0) s_best[tid >> 6] = best;
        __syncthreads();
        best = max(max(s_best[0], s_best[1]), max(s_best[2], s_best[3]));
        token = best ? (int)~(uint32_t)best : 0;
    }
    for (int i = tid; i <= a.max_n; i += kVerifyThreads)
        a.tokens[(long)b * (a.max_n + 1) + i] = i < r.a ? a.draft[r.first + i] : i == r.a ? token : -1;
    if (tid == 0) {
        a.accepted[b] = r.a;
        if (a.drops) a.drops[b] = r.n - r.a + (PLANNED ? r.more : 0);
    }
}

// ---- checks -------------------------------------------------------------------------
int page_shift(int page_size)
{
    for (int s = 4; s <= 8; ++s)
        if (page_size == 1 << s) return s;
    return -1;
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

dx_status reserved(dx_ctx *c, const char *who, int B)
{
    if (!c->serve_requests) DX_FAIL(c, DX_ERR_INVALID, "%s: dx_serve_reserve has not been called", who);
    if (B < 0 || B > c->serve_requests) DX_FAIL(c, DX_ERR_INVALID, "%s: B=%d outside [0,%d]", who, B, c->serve_requests);
    return DX_OK;
}

dx_status check_cache(dx_ctx *c, const char *who, const dx_kv_cache *k)
{
    if (!k || !k->k || !k->v) DX_FAIL(c, DX_ERR_INVALID, "%s: null cache", who);
    if (k->fmt != DX_KV_BF16 && k->fmt != DX_KV_E4M3) DX_FAIL(c, DX_ERR_INVALID, "%s: cache format %d", who, k->fmt);
    if (k->head_dim != 64 && k->head_dim != 128 && k->head_dim != 256)
        DX_FAIL(c, DX_ERR_INVALID, "%s: head_dim=%d is not 64, 128 or 256", who, k->head_dim);
    if (k->kv_heads < 1 || k->kv_heads > 1024) DX_FAIL(c, DX_ERR_INVALID, "%s: kv_heads=%d outside [1,1024]", who, k->kv_heads);
    if (page_shift(k->page_size) < 0)
        DX_FAIL(c, DX_ERR_INVALID, "%s: page_size=%d is not 16, 32, 64, 128 or 256", who, k->page_size);
    if (k->n_pages < 1 || (int64_t)k->n_pages * k->page_size > 0x7FFFFFFFLL)
        DX_FAIL(c, DX_ERR_INVALID, "%s: n_pages=%d (of %d tokens) outside the range of 31-bit slots", who, k->n_pages, k->page_size);
    if (!aligned(k->k, 16) || !aligned(k->v, 16)) DX_FAIL(c, DX_ERR_INVALID, "%s: cache not aligned to 16 bytes", who);
    if (k->fmt == DX_KV_E4M3 && (!k->k_scale || !k->v_scale)) DX_FAIL(c, DX_ERR_INVALID, "%s: an e4m3 cache needs scales", who);
    return DX_OK;
}

dx_status plan(dx_ctx *c, const char *who, int page_size, dx_plan_args a)
{
    if (const dx_status s = reserved(c, who, a.B)) return s;
    if (a.T < 0 || a.T > c->cfg.max_tokens) DX_FAIL(c, DX_ERR_INVALID, "%s: T=%d outside [0,%d]", who, a.T, c->cfg.max_tokens);
    a.page_shift = page_shift(page_size);
    if (a.page_shift < 0) DX_FAIL(c, DX_ERR_INVALID, "%s: page_size=%d is not 16, 32, 64, 128 or 256", who, page_size);
    if (a.n_pages < 1 || (int64_t)a.n_pages * page_size > 0x7FFFFFFFLL)
        DX_FAIL(c, DX_ERR_INVALID, "%s: n_pages=%d (of %d tokens) outside the range of 31-bit slots", who, a.n_pages, page_size);
    if (a.stride < 1 || (int64_t)a.stride * page_size > 0x7FFFFFFFLL)
        DX_FAIL(c, DX_ERR_INVALID, "%s: table_stride=%d (pages of %d tokens) outside the range", who, a.stride, page_size);
    if (!a.free_in || !a.free_list || !a.free_out || !a.q_offsets || !a.status || (a.T > 0 && (!a.slots || !a.positions)) ||
        (a.B > 0 && (!a.new_lens || !a.lens_in || !a.table || !a.lens_out)))
        DX_FAIL(c, DX_ERR_INVALID, "%s: null pointer", who);
    hipLaunchKernelGGL(k_plan, dim3(1), dim3(kPlanThreads), 0, c->compute, a);
    DX_HIP(c, hipGetLastError());
    return DX_OK;
}

dx_status verify(dx_ctx *c, const char *who, verify_args a)
{
    if (const dx_status s = reserved(c, who, a.B)) return s;
    if (a.V < 1 || a.V > 1 << 20) DX_FAIL(c, DX_ERR_INVALID, "%s: V=%d outside [1,2^20]", who, a.V);
    if (a.max_n < 0 || a.max_n > 255) DX_FAIL(c, DX_ERR_INVALID, "%s: max_n=%d outside [0,255]", who, a.max_n);
    if (a.n_drafts < 0 || (int64_t)a.n_drafts > (int64_t)a.B * a.max_n)
        DX_FAIL(c, DX_ERR_INVALID, "%s: n_drafts=%d outside [0, B * max_n]", who, a.n_drafts);
    if (a.B == 0) return DX_OK;
    if (!a.p || !a.offsets || !a.u_sample || !a.tokens || !a.accepted || (a.n_drafts > 0 && (!a.draft || !a.u_accept)))
        DX_FAIL(c, DX_ERR_INVALID, "%s: null pointer", who);
    a.sums = reinterpret_cast<unsigned long long *>(c->serve_scratch + c->verify_scratch);
    const dim3 grid((a.V + kChunk - 1) / kChunk, a.B), threads(kVerifyThreads);
    if (a.status) hipLaunchKernelGGL((k_verify<true>), grid, threads, 0, c->compute, a);
    else hipLaunchKernelGGL((k_verify<false>), grid, threads, 0, c->compute, a);
    DX_HIP(c, hipGetLastError());
    return DX_OK;
}

} // namespace

extern "C" dx_status dx_serve_reserve(dx_ctx *c, int max_requests, int max_head_dim)
{
    if (!c) return DX_ERR_INVALID;
    if (c->serve_requests) DX_FAIL(c, DX_ERR_BUSY, "dx_serve_reserve: already reserved");
    if (max_requests < 1 || max_requests > DX_SERVE_MAX_REQUESTS)
        DX_FAIL(c, DX_ERR_INVALID, "dx_serve_reserve: max_requests=%d outside [1,%d]", max_requests, DX_SERVE_MAX_REQUESTS);
    if (max_head_dim != 64 && max_head_dim != 128 && max_head_dim != 256)
        DX_FAIL(c, DX_ERR_INVALID, "dx_serve_reserve: max_head_dim=%d is not 64, 128 or 256", max_head_dim);
    DX_HIP(c, hipStreamSynchronize(c->compute));
    const size_t of_attention = dxk_attention_scratch(c->n_cu, nullptr, nullptr);
    const size_t of_verify = (size_t)max_requests * kSums * sizeof(unsigned long long);
    char *scratch = nullptr;
    hipError_t e = hipMalloc(&scratch, of_attention + of_verify);
    if (e != hipSuccess)
        DX_FAIL(c, e == hipErrorOutOfMemory ? DX_ERR_NOMEM : DX_ERR_HIP, "dx_serve_reserve: scratch: %s", hipGetErrorString(e));
    e = hipMemsetAsync(scratch + of_attention, 0, of_verify, c->compute); // (k_verify leaves it at 0)
    if (e == hipSuccess) e = hipStreamSynchronize(c->compute);
    if (e != hipSuccess) {
        (void)hipFree(scratch);
        DX_FAIL(c, DX_ERR_HIP, "dx_serve_reserve: scratch: %s", hipGetErrorString(e));
    }
    c->serve_scratch = scratch;
    c->verify_scratch = of_attention;
    c->serve_requests = max_requests;
    c->serve_dim = max_head_dim;
    return DX_OK;
}

extern "C" dx_status dx_pages_plan(dx_ctx *c, int B, int T, int page_size, int n_pages, int table_stride,
                                   const int32_t *new_lens, const int32_t *lens_in, const int32_t *drops,
                                   const int32_t *free_in, int32_t *free_list, int32_t *table, int32_t *lens_out,
                                   int32_t *free_out, int32_t *q_offsets, int32_t *slots, int32_t *positions, int32_t *status)
{
    if (!c) return DX_ERR_INVALID;
    return plan(c, "dx_pages_plan", page_size,
                dx_plan_args{new_lens, lens_in, drops, free_in, nullptr, free_list, table, lens_out, free_out, q_offsets, slots, positions,
                             status, B, T, 0, n_pages, table_stride});
}

extern "C" dx_status dx_pages_plan_in_place(dx_ctx *c, int B, int T, int page_size, int n_pages, int table_stride,
                                            const int32_t *new_lens, int32_t *lens, int32_t *drops, int32_t *free_pages,
                                            int32_t *free_list, int32_t *table, int32_t *q_offsets, int32_t *slots,
                                            int32_t *positions, int32_t *status)
{
    if (!c) return DX_ERR_INVALID;
    return plan(c, "dx_pages_plan_in_place", page_size,
                dx_plan_args{new_lens, lens, drops, free_pages, drops, free_list, table, lens, free_pages, q_offsets, slots, positions,
                             status, B, T, 0, n_pages, table_stride});
}

extern "C" dx_status dx_kv_write(dx_ctx *c, const dx_kv_cache *cache, const void *k, int64_t k_stride, const void *v,
                                 int64_t v_stride, const int32_t *slots, int T)
{
    if (!c) return DX_ERR_INVALID;
    if (const dx_status s = check_cache(c, "dx_kv_write", cache)) return s;
    if (T < 0 || T > c->cfg.max_tokens) DX_FAIL(c, DX_ERR_INVALID, "dx_kv_write: T=%d outside [0,%d]", T, c->cfg.max_tokens);
    if (T == 0) return DX_OK;
    if (!k || !v || !slots) DX_FAIL(c, DX_ERR_INVALID, "dx_kv_write: null pointer");
    const int64_t row = (int64_t)cache->kv_heads * cache->head_dim;
    if (!aligned(k, 16) || !aligned(v, 16) || k_stride % 8 || v_stride % 8 || k_stride < row || v_stride < row)
        DX_FAIL(c, DX_ERR_INVALID, "dx_kv_write: k and v need starts at 16 bytes and strides of a multiple of 8 that hold a row");
    write_args a{*cache, static_cast<const dx_bf16 *>(k), static_cast<const dx_bf16 *>(v), (long)k_stride, (long)v_stride, slots, T,
                 page_shift(cache->page_size)};
    // a block per token while that leaves compute units over, else a wavefront
    const bool few = T <= 2 * c->n_cu;
    const dim3 grid(few ? T : (T + 3) / 4);
    if (cache->fmt == DX_KV_E4M3) {
        if (few) hipLaunchKernelGGL((k_kv_write<true, 4>), grid, dim3(256), 0, c->compute, a);
        else hipLaunchKernelGGL((k_kv_write<true, 1>), grid, dim3(256), 0, c->compute, a);
    } else {
        if (few) hipLaunchKernelGGL((k_kv_write<false, 4>), grid, dim3(256), 0, c->compute, a);
        else hipLaunchKernelGGL((k_kv_write<false, 1>), grid, dim3(256), 0, c->compute, a);
    }
    DX_HIP(c, hipGetLastError());
    return DX_OK;
}

extern "C" dx_status dx_paged_attention(dx_ctx *c, const dx_kv_cache *cache, const void *q, int64_t q_stride, int q_heads,
                                        const int32_t *q_offsets, const int32_t *lens, const int32_t *table, int table_stride,
                                        int B, int T, int max_q, float scale, int window, void *out, int64_t out_stride, float *lse)
{
    if (!c) return DX_ERR_INVALID;
    if (const dx_status s = reserved(c, "dx_paged_attention", B)) return s;
    if (const dx_status s = check_cache(c, "dx_paged_attention", cache)) return s;
    if (cache->head_dim > c->serve_dim)
        DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: head_dim=%d above the %d of dx_serve_reserve", cache->head_dim, c->serve_dim);
    if (T < 0 || T > c->cfg.max_tokens) DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: T=%d outside [0,%d]", T, c->cfg.max_tokens);
    if (q_heads < 1 || q_heads > 1024 || q_heads % cache->kv_heads)
        DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: q_heads=%d is no multiple of kv_heads=%d, or above 1024", q_heads, cache->kv_heads);
    // (keys are counted in 32 bits, some units past the end)
    if (table_stride < 1 || (int64_t)table_stride * cache->page_size > 1LL << 30)
        DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: table_stride=%d (pages of %d tokens) outside the range", table_stride, cache->page_size);
    if ((int64_t)T * q_heads > 1LL << 30) DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: T=%d of %d heads", T, q_heads);
    if (max_q < 0 || window < 0) DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: max_q=%d or window=%d is negative", max_q, window);
    if (!std::isfinite(scale)) DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: scale is not finite");
    if (B == 0 || T == 0) return DX_OK;
    if (!q || !q_offsets || !lens || !table || !out) DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: null pointer");
    const int64_t row = (int64_t)q_heads * cache->head_dim;
    if (!aligned(q, 16) || !aligned(out, 16) || q_stride % 8 || out_stride % 8 || q_stride < row || out_stride < row)
        DX_FAIL(c, DX_ERR_INVALID, "dx_paged_attention: q and out need starts at 16 bytes and strides of a multiple of 8 that hold a row");
    dx_attn_args a{};
    a.cache = *cache;
    a.q = static_cast<const dx_bf16 *>(q);
    a.out = static_cast<dx_bf16 *>(out);
    a.lse = lse;
    a.q_offsets = q_offsets;
    a.lens = lens;
    a.table = table;
    a.q_stride = (long)q_stride;
    a.out_stride = (long)out_stride;
    a.B = B;
    a.T = T;
    a.q_heads = q_heads;
    a.group = q_heads / cache->kv_heads;
    a.table_stride = table_stride;
    a.page_shift = page_shift(cache->page_size);
    a.window = window;
    a.max_q = max_q;
    a.scale = scale;
    (void)dxk_attention_scratch(c->n_cu, c->serve_scratch, &a);
    DX_HIP(c, dxk_paged_attention(a, c->compute));
    return DX_OK;
}

extern "C" dx_status dx_draft_verify(dx_ctx *c, const float *p, const float *q, const int32_t *draft, const int32_t *offsets,
                                     int B, int n_drafts, int max_n, int V, const float *u_accept, const float *u_sample,
                                     int32_t *tokens, int32_t *accepted, int32_t *drops)
{
    if (!c) return DX_ERR_INVALID;
    return verify(c, "dx_draft_verify", verify_args{p, q, draft, offsets, u_accept, u_sample, tokens, accepted, drops, B, n_drafts, max_n, V, nullptr, nullptr});
}

extern "C" dx_status dx_draft_verify_planned(dx_ctx *c, const int32_t *status, const float *p, const float *q, const int32_t *draft,
                                             const int32_t *offsets, int B, int n_drafts, int max_n, int V, const float *u_accept,
                                             const float *u_sample, int32_t *tokens, int32_t *accepted, int32_t *drops)
{
    if (!c) return DX_ERR_INVALID;
    if (!status) DX_FAIL(c, DX_ERR_INVALID, "dx_draft_verify_planned: null status");
    return verify(c, "dx_draft_verify_planned",
                  verify_args{p, q, draft, offsets, u_accept, u_sample, tokens, accepted, drops, B, n_drafts, max_n, V, nullptr, status});
}
