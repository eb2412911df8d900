// Attention of the new tokens of a step over the paged key/value cache.
//
// A row is a (new token, query head); the rows of a request that read one kv head, token by token, are cut into tiles.
// Scores are computed transposed, S^T = K Q^T (keys the first operand of the matrix instructions, rows the second), so
// that a lane holds scores of ONE row: its maximum and its factor are the lane's own numbers, and the
// probabilities, in the order in which the accumulators hold them, are the second operand of O^T = V^T P^T without a
// move.  v_mfma_f32_16x16x32_bf16: accumulator element i of lane l is row 4 * (l / 16) + i, column l % 16; its operands hold
// elements 8 * (l / 16) .. + 7 of the summed index for row or column l % 16.  A unit of keys is 4 X (X: elements in 16
// bytes); lane group l / 16 owns X consecutive ones: row r of key tile a is the key X * (r / 4) + 4 a + r % 4 of the unit, so
// that its accumulators are the keys X * (l / 16) + 4 a + i, which are also the 16 bytes of a value channel that the lane
// reads.  The cache is laid out for that: both operands come from memory as they are.
//
// Softmax in base 2 with a running maximum per row that is only raised when a score exceeds it by more than 8: a
// probability is at most 2^8, and most units need neither a reduction across lanes nor a change of the sums.
#include "dx_internal.h"
#include "dx_route_core.h"

#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
#define DX_GLOBAL __attribute__((address_space(1)))

constexpr float kNothing = -3.402823466e38f; // maximum of a row that has seen no key yet: the lowest number
constexpr float kRise = 8.f;
constexpr float kFar = 16777216.f; // 2^24 (raise_maximum)
constexpr float kLn2 = 0.69314718055994531f, kLog2e = 1.4426950408889634f;

__device__ uint32_t pack_bf16(float a, float b) // nearest even
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// largest (sum) over the four lanes l % 16 + 16 n of a wavefront
__device__ float max_over_groups(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ float sum_over_groups(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// half h of 16 bytes of fp8 as an operand of bf16
__device__ u32x4 widen_half(const u32x4 &c, int h)
{
    u32x4 to;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const uint32_t x = c[2 * h + w];
        to[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
        to[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true));
    }
    return to;
}
__device__ void widen_fp8(const u32x4 &c, u32x4 &lo, u32x4 &hi)
{
    lo = widen_half(c, 0);
    hi = widen_half(c, 1);
}

__device__ f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// ---- which part of the step a block computes ----------------------------------------
// The work of a launch is a line: for every kv head, request and tile of its rows, a length of about as many units of keys as the
// tile's rows see (kFine parts of a unit; within a request it grows evenly from the first tile to the last, as under a
// causal mask).  Every block takes an equal stretch of it, so that all end together whatever the lengths are; it derives its
// stretch from the lengths (the host does not know them), and of a tile that it has a part of the line of, the same part of the units.
// A tile that lies in one stretch is written out by its block.  The others are joined: a stretch has at most two
// unfinished tiles, one that it found begun (slot 2 * block) and one that it leaves (slot 2 * block + 1); for each there is an entry
// in what the block leaves to k_join (a.left).  Joining costs as much as some units, so a cut that close to either end of a tile is moved there.
constexpr int kFine = 16;
// In units (k_keys: 32 or 64 keys) and stages (k_rows: 64): what a tile costs beside its units, the shortest stretch, and how far cuts
// are moved.  Measured as each was set, in bf16 (the same numbers for e4m3 and other heads), us a pass, 2000 new tokens (32 heads on 4 of 128 channels: tiles of 1 to 32 stages): tiles at their units alone 108, with
// 2, 3, 4 stages more 77, 75, 74; cuts moved over 4, 8, 12 stages without that 108, 95, 85, but 512 tokens after 8000 105, 110, 119.
// Stretches of at least 6 and 4 stages: 300 new tokens 25.9 and 21.7, 100 after 1500 30.3 and 29.6, 9 requests with prompts of 9 to 300 27.8 and 26.8.
constexpr int kKeysOver = 6, kKeysMin = 8, kKeysNear = 4, kRowsOver = 4, kRowsMin = 4, kRowsNear = 3;

// memory (16 bytes from a lane's address) to LDS (at + 16 * lane); completion is awaited with vmcnt
__device__ __forceinline__ void load_to_lds(uint32_t at, uint64_t from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from) : "memory");
}
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ uint32_t lds_of(char *p) { return (uint32_t)(uintptr_t)(lds_char *)p; }

// What a kernel's line is made of: tiles of ROWS rows, units of UNIT keys; in units, what a tile costs beside its own, the
// shortest stretch, how far cuts are moved, and how much longer stretches may be (even_units, even_tiles; whole_tiles).  A launch takes the requests of at most
// a.few rows (FEW), or those of more.
template <int ROWS_, int UNIT_, int OVER_, int MIN_, int NEAR_, bool FEW_, int MORE_, int WHOLE_> struct kind {
    static constexpr int ROWS = ROWS_, UNIT = UNIT_, OVER = OVER_, MIN = MIN_, NEAR = NEAR_, MORE = MORE_, WHOLE = WHOLE_;
    static constexpr bool FEW = FEW_;
    static constexpr int LEAST = FEW_ ? 4 : 2, GROUP = ROWS_, TWO = 4, FOUR = 4;
};

struct request {
    int tiles;      // of rows
    int first, add; // length of the first tile on the line, and how much longer each next one is
    __device__ long start(int tile) const { return (long)tile * first + (long)tile * (tile - 1) / 2 * add; }
    __device__ int length(int tile) const { return first + tile * add; }
};

// Tokens of a request: first new one, how many, length in the cache.  Those of up to 64 requests are kept in the lanes of
// every wavefront (a call of 3 short requests 14 us; read where they are needed 15).
struct tokens {
    int first, n, len;
};
struct batch {
    bool in_lanes;
    tokens mine;
    __device__ static tokens read(const dx_attn_args &a, int b)
    {
        const int first = min(max(a.q_offsets[b], 0), a.T);
        return tokens{first, min(max(a.q_offsets[b + 1], 0), a.T) - first, a.lens[b]};
    }
    __device__ batch(const dx_attn_args &a) : in_lanes(a.B <= 64), mine{0, 0, 0}
    {
        const int lane = threadIdx.x & 63;
        if (in_lanes && lane < a.B) mine = read(a, lane);
    }
    __device__ tokens get(const dx_attn_args &a, int b) const // b is uniform
    {
        if (!in_lanes) return read(a, b);
        return tokens{__builtin_amdgcn_readlane(mine.first, b), __builtin_amdgcn_readlane(mine.n, b), __builtin_amdgcn_readlane(mine.len, b)};
    }
};

__device__ int capacity(const dx_attn_args &a) { return a.table_stride << a.page_shift; }
// x / a.group for 0 <= x < 2^31 (dxk_paged_attention)
__device__ int by_group(const dx_attn_args &a, int x) { return a.group == 1 ? x : (int)(__umulhi((uint32_t)x, a.group_mul) >> a.group_shift); }

// first key of a window's that a row at pos sees (a position below 0, of a row that sees nothing, less a window that is as long as the type allows
// would leave it)
__device__ int window_from(const dx_attn_args &a, int pos) { return max(max(pos, 0) - a.window + 1, 0); }

// The rows of a tile and the keys that they see.
struct tile_rows {
    int token, first, rows; // first token of the request, first row of the tile in it, rows of the tile
    int pos;                // position of the request's first new token
    int lo, hi;             // keys that some row of the tile sees
    int all_lo, all_hi;     // keys that all of them see
    template <int UNIT> __device__ int first_unit() const { return lo / UNIT; }
    template <int UNIT> __device__ int units() const { return hi > lo ? (hi - 1) / UNIT - lo / UNIT + 1 : 0; }
};

// rows `first` .. of a request, `rows` of them at most
__device__ tile_rows see(const dx_attn_args &a, const tokens &of, int first, int rows)
{
    tile_rows t;
    t.token = of.first;
    t.first = first;
    t.rows = min(of.n * a.group - first, rows);
    t.pos = of.len - of.n;
    const int p0 = t.pos + by_group(a, first), p1 = t.pos + by_group(a, first + t.rows - 1);
    t.hi = max(min(min(p1 + 1, of.len), capacity(a)), 0);
    t.all_hi = min(p0 + 1, t.hi);
    t.lo = a.window ? min(window_from(a, p0), t.hi) : 0;
    t.all_lo = a.window ? window_from(a, p1) : 0;
    return t;
}

// units of a tile by what they cost: those of more than K::GROUP (2 K::GROUP) rows K::TWO (K::FOUR) quarters of the others
template <class K> __device__ int weighed(const tile_rows &t)
{
    const int units = t.template units<K::UNIT>();
    if (K::ROWS == K::GROUP || t.rows <= K::GROUP) return units;
    return (int)((long)units * (t.rows <= 2 * K::GROUP ? K::TWO : K::FOUR) / 4);
}
// even > 0: every tile is cut into parts of up to so many units, which are equally long on the line, a stretch each; even < 0: a stretch is so
// many whole tiles (whole_tiles)
template <class K> __device__ request make_request(const dx_attn_args &a, const tokens &of, int even)
{
    const int rows = of.n * a.group;
    request r{0, kFine, 0};
    if (of.n <= 0 || (rows <= a.few) != K::FEW) return r;
    r.tiles = (rows + K::ROWS - 1) / K::ROWS;
    if (even < 0) return r;
    if (even) {
        const int units = weighed<K>(see(a, of, (r.tiles - 1) * K::ROWS, K::ROWS));
        r.first = kFine * even * max((units + even - 1) / even, 1);
        return r;
    }
    r.first = kFine * (max(weighed<K>(see(a, of, 0, K::ROWS)), 1) + K::OVER);
    if (r.tiles > 1)
        r.add = max(kFine * (weighed<K>(see(a, of, (r.tiles - 1) * K::ROWS, K::ROWS)) + K::OVER) - r.first, 0) / (r.tiles - 1);
    return r;
}

// Prefix sums of a line's lengths over the requests of one kv head: this thread's requests (b = lane of every wavefront, or B / 256 each in
// the block) are `work` long, behind `before`, of `total`.
struct line_part {
    long before, work, total;
    int even; // (make_request)
};
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(dx_route_core::wave_scan_inclusive(x), 63); }

// The units of a stretch if every tile is cut on its own, so that no block has parts of two, each of which costs it as much as several
// units: the shortest for which `blocks` are enough, if it is no more than K::MORE (many rows, whose blocks end with others': 2 and an eighth) above
// an equal share of all units, and that is short enough for it to matter.  Measured, us a pass, without and with: 3 short requests 13.7 and 11.0, one of
// 4000 tokens 16.9 and 12.9, 33 with drafts in fp8 69 and 64, but MORE = 5 70; one of 150 thousand tokens, 256 channels, MORE = 8 61 against 58; where
// there is none it costs 0.5 to 1.  Many rows beside few: a chunk of 512 and 32 decoding 87 and 78, of 401 and 2, 256 channels, 65 and 55, of
// 201 and 1, 64 channels, 19.5 and 18.6; but of 200 and 11 50.2 and 51.9, of 451 and 9 58.2 and 59.2; at 1 and an eighth 301 and 4 64 (59.5), at
// 6 more 451 and 9 64.
template <class K> __device__ int even_units(const dx_attn_args &a, const batch &n, int blocks)
{
    if (!n.in_lanes || blocks < 1) return 0;
    const request r = make_request<K>(a, n.mine, 1);
    const int units = r.first / kFine; // (of the request's longest tile)
    const int equal = (int)((float)wave_sum((int)min((long)r.tiles * units, 1L << 24)) * a.cache.kv_heads / blocks);
    if (equal > 5 * K::MORE) return 0;
    const int more = K::FEW ? K::MORE : 2 + equal / 8;
    for (int s = max(equal, K::LEAST); s <= max(equal, K::LEAST) + more; ++s)
        if (wave_sum(min(r.tiles * ((units + s - 1) / s), 1 << 16)) * a.cache.kv_heads <= blocks) return s;
    return 0;
}

// Tiles of a single request are not cut where so many whole ones to a block, the longest and the shortest in pairs, take no more than K::WHOLE units
// above an equal share of all: a cut is two parts of 128 rows written and read again.  The pairs are as long as each other, and stay
// together from head to head if every other head's order is turned round.  Returns minus that number, or 0.  Measured, us a pass, cut and whole,
// 32 heads on 4 of 128 channels, a call of one request (of eight places, seven of them idle, 4096 after 4001 418): 512 new tokens 31.9 and 26.8, 4001 162 and 140, 4096 after 4001 404 and 379, 8192 547 and 519; where
// they are cut anyway the look costs 0.4.  At WHOLE = 16 also 1024 tokens 37.8 and 41.2.
template <class K> __device__ int whole_tiles(const dx_attn_args &a, const request &r, int blocks)
{
    const int tiles = r.tiles * a.cache.kv_heads, each = (tiles + blocks - 1) / blocks, longest = r.length(r.tiles - 1);
    const long all = max(r.start(r.tiles) * a.cache.kv_heads, (long)blocks * K::MIN * kFine);
    const long most = (each >> 1) * (long)(r.length(0) + longest) + (each & 1) * longest;
    return uniform(most * blocks <= all + (long)blocks * K::WHOLE * kFine ? -each : 0);
}
// even (make_request) for a single request, of which r is the line: as many parts of a tile as the blocks allow, unless that leaves them longer than an
// equal share, what a tile costs beside its units included, by more than K::MORE.  (All lanes get here; lane 0 has the request.)  Measured, us a
// pass, without and with: 100 tokens after 3000, 32 heads on 4 of 128 channels, 31 and 26.4, 201 after 16000 86 and 78, 512 after 8000 90 and 82,
// 501 after 200, 256 channels, 47 and 32; at MORE = 3 301 after 9000 68 and 66; where it is not taken it costs 0.3 (measured while the join still went
// by the place on the line: 501 tokens now 28.6).
template <class K> __device__ int even_tiles(const dx_attn_args &a, const batch &n, const request &r, int blocks)
{
    const int units = make_request<K>(a, n.mine, 1).first / kFine; // of the longest tile
    const int tiles = max(r.tiles * a.cache.kv_heads, 1), each = blocks / tiles;
    const int s = max((units + each - 1) / max(each, 1), K::LEAST);
    const bool fits = each > 0 && r.tiles > 0 && (long)s * kFine * blocks <= r.start(r.tiles) * a.cache.kv_heads + (long)blocks * kFine * K::MORE;
    return uniform(fits ? s : 0);
}
__device__ int paired(int i, int tiles, int head) // tile in place i
{
    if (head & 1) i = tiles - 1 - i;
    return i & 1 ? i >> 1 : tiles - 1 - (i >> 1);
}

template <class K> __device__ line_part measure(const dx_attn_args &a, const batch &n, int even, long *s_sum)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    line_part l{0, 0, 0, even};
    if (n.in_lanes) {
        request r = make_request<K>(a, n.mine, even);
        if (K::WHOLE && a.B == 1) {
            l.even = whole_tiles<K>(a, r, gridDim.x);
            if (l.even) {
                r = request{r.tiles, kFine, 0};
            } else {
                l.even = even_tiles<K>(a, n, r, gridDim.x);
                if (l.even) r = make_request<K>(a, n.mine, l.even);
            }
        }
        l.work = r.start(r.tiles);
    } else {
        const int per = (a.B + 255) / 256;
        for (int b = tid * per; b < min((tid + 1) * per, a.B); ++b) {
            const request r = make_request<K>(a, batch::read(a, b), 0);
            l.work += r.start(r.tiles);
        }
    }
    // (in two parts of 24 and 32 bits)
    const uint32_t lo = dx_route_core::wave_scan_inclusive((uint32_t)(l.work & 0xFFFFFF)), hi = dx_route_core::wave_scan_inclusive((uint32_t)(l.work >> 24));
    const long inc = ((long)hi << 24) + lo;
    l.before = inc - l.work;
    const long of_wave = ((long)(uint32_t)__builtin_amdgcn_readlane((int)hi, 63) << 24) + (uint32_t)__builtin_amdgcn_readlane((int)lo, 63);
    l.total = of_wave;
    if (!n.in_lanes) {
        if (lane == 63) s_sum[wave] = of_wave;
        __syncthreads();
        l.total = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) l.before += s_sum[w];
            l.total += s_sum[w];
        }
    }
    return l;
}

struct stretch {
    long share, near;  // length of the stretches before cuts are moved; how near to the end of a tile they are
    int even;          // (make_request)
    int block, blocks; // among the blocks of this line, the first of which is block `base` of the launch
    int base;
    int head, b, tile; // a tile of it, and where that starts on the line
    long start;
    long end; // this block has none of the tiles that start behind it
    request r;
    // the blocks that have a part of the tile
    __device__ int first_block() const { return (int)min((start + near + share - 1) / share - 1, (long)blocks - 1); }
    __device__ int last_block() const { return (int)max((start + r.length(tile) - near) / share, 0L); }
};

// Puts p at the first tile of its block, or at one in front of it: stretches of at least MIN units, cuts moved over up to NEAR.  All threads of
// the block call it; s_found: 3 words of LDS.  False: there is none.
template <class K> __device__ bool locate(const dx_attn_args &a, const batch &n, const line_part &l, stretch &p, int *s_found)
{
    const long line = l.total * a.cache.kv_heads;
    p.even = l.even;
    p.share = l.even ? abs(l.even) * kFine : max((line + p.blocks - 1) / p.blocks, (long)K::MIN * kFine);
    p.near = l.even ? 1 : K::NEAR * kFine;
    const long at = max(p.block * p.share - p.near, 0L);
    if (at >= line) return false;
    p.end = min((p.block + 1) * p.share - p.near, line - 1); // (first_block)
    p.head = uniform((int)(at / l.total));
    long in = at - p.head * l.total; // of the head's requests, then of one, then of a tile
    if (n.in_lanes) {
        const unsigned long long behind = __ballot(in < l.before + l.work);
        p.b = __ffsll(behind) - 1;
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)l.before, p.b), hi = (uint32_t)__builtin_amdgcn_readlane((int)(l.before >> 32), p.b);
        in -= (long)((unsigned long long)hi << 32 | lo);
    } else {
        if (in >= l.before && in < l.before + l.work) {
            const int per = (a.B + 255) / 256;
            long before = l.before;
            for (int b = threadIdx.x * per;; ++b) { // (one of the thread's requests ends it)
                const request r = make_request<K>(a, batch::read(a, b), 0);
                if (in < before + r.start(r.tiles)) {
                    s_found[0] = b;
                    s_found[1] = (int)(uint32_t)(in - before);
                    s_found[2] = (int)((in - before) >> 32);
                    break;
                }
                before += r.start(r.tiles);
            }
        }
        __syncthreads();
        p.b = uniform(s_found[0]);
        in = (long)((unsigned long long)(uint32_t)uniform(s_found[2]) << 32 | (uint32_t)uniform(s_found[1]));
    }
    p.r = make_request<K>(a, n.get(a, p.b), p.even);
    int lo = 0, hi = p.r.tiles; // the tile that starts at or before it
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.r.start(mid) <= in) lo = mid;
        else hi = mid;
    }
    p.tile = uniform(lo);
    p.start = at - (in - p.r.start(lo));
    return true;
}

// the tile behind; false: there is none, or it is another block's
template <class K> __device__ bool advance(const dx_attn_args &a, const batch &n, stretch &p)
{
    p.start += p.r.length(p.tile);
    if (p.start > p.end) return false;
    if (++p.tile < p.r.tiles) return true;
    p.tile = 0;
    // The next request that has some, 64 looked at at once.  Looked at one after another, us a pass, and so: 3 live requests of 1024 254 and 21 (of 3:
    // 11), a chunk of 512 tokens beside 999 decoding 387 and 168.  (They are not all without tiles: then there is no line.)
    const int lane = threadIdx.x & 63;
    for (int from = p.b + 1;;) {
        const int at = n.in_lanes ? lane : from + lane;
        const tokens of = n.in_lanes ? n.mine : at < a.B ? batch::read(a, at) : tokens{0, 0, 0};
        const unsigned long long some = __ballot(at >= from && of.n > 0 && (of.n * a.group <= a.few) == K::FEW);
        if (some) {
            const int in = __ffsll(some) - 1;
            p.b = n.in_lanes ? in : from + in;
            p.r = make_request<K>(a, tokens{__builtin_amdgcn_readlane(of.first, in), __builtin_amdgcn_readlane(of.n, in), __builtin_amdgcn_readlane(of.len, in)}, p.even);
            return true;
        }
        from += 64;
        if (n.in_lanes || from >= a.B) {
            from = 0;
            if (++p.head == a.cache.kv_heads) return false;
        }
    }
}

// What a block does next: a tile, some units of it, and where its rows go.
struct task {
    tile_rows t;
    tokens of;
    int begin, end; // units
    long slot;      // of unfinished rows, or -1
};

// The block's part of the tile that p is at, or of a later one; false: it has no more.
template <class K> __device__ bool next_task(const dx_attn_args &a, const batch &n, stretch &p, task &k)
{
    int first, last;
    for (;;) {
        first = p.first_block();
        last = max(p.last_block(), first);
        if (p.block < first) return false;
        if (p.block <= last) break;
        if (!advance<K>(a, n, p)) return false;
    }
    k.of = n.get(a, p.b);
    k.of = tokens{uniform(k.of.first), uniform(k.of.n), uniform(k.of.len)};
    p.tile = uniform(p.tile);
    p.head = uniform(p.head);
    p.b = uniform(p.b);
    k.t = see(a, k.of, (!K::FEW && p.even < 0 ? paired(p.tile, p.r.tiles, p.head) : p.tile) * K::ROWS, K::ROWS);
    const int length = p.r.length(p.tile);
    const long from = p.block == first ? 0 : p.block * p.share - p.start, to = p.block == last ? length : (p.block + 1) * p.share - p.start;
    const long units = k.t.template units<K::UNIT>();
    k.begin = uniform(k.t.template first_unit<K::UNIT>() + (int)(units * from / length));
    k.end = uniform(k.t.template first_unit<K::UNIT>() + (int)(units * to / length));
    k.slot = -1;
    if (first < last) {
        k.slot = 2L * (p.base + p.block) + (p.block > first ? 0 : 1);
        if (threadIdx.x == 0)
            a.left[blockIdx.x].joint[p.block > first ? 0 : 1] =
                dx_attn_joint{p.base + first, last - first + 1, k.t.token, k.t.first, k.t.rows, p.head, !K::FEW, p.block - first};
    }
    return true;
}

// a finished row of a tile: 4 channels from d on, and its lse
struct row_at {
    dx_bf16 *out;
    float *lse; // or null
    __device__ row_at(const dx_attn_args &a, int token0, int head, int row)
    {
        const int i = by_group(a, row), token = token0 + i, h = head * a.group + row - i * a.group;
        out = a.out + token * a.out_stride + (long)h * a.cache.head_dim;
        lse = a.lse ? a.lse + (long)token * a.q_heads + h : nullptr;
    }
    __device__ void store(int d, const f32x4 &o) const { *reinterpret_cast<u32x2 *>(out + d) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])}; }
    __device__ void store_lse(float top, float all) const
    {
        if (lse) *lse = all == 0.f ? -INFINITY : (top + log2_fast(all)) * kLn2;
    }
};
__device__ float inverse(float all, float v_scale) { return all == 0.f ? 0.f : v_scale / all; }

// Unfinished rows: pieces of 4 channels in the order that the kernel has them in, which is not that of the rows for k_rows (there
// a lane's accumulators are a piece: item (16-row tile, channel tile, lane)).
template <int D> struct piece_of {
    int row, d;
    __device__ piece_of(int item, bool by_lanes)
    {
        if (by_lanes) {
            const int lane = item & 63, dt = item / 64 % (D / 16);
            row = item / (4 * D) * 16 + (lane & 15);
            d = 16 * dt + 4 * (lane >> 4);
        } else {
            row = item / (D / 4);
            d = item % (D / 4) * 4;
        }
    }
};

// ---- what both kernels do with scores --------------------------------------------------
// Queries of 16 NT rows from `first` on as operands of the score product (rows past the last: that one again, they are not
// stored), and the last and first key that each sees.  The factor of the scores is folded in as far as it is not positive, so that
// the largest score is the largest product.
template <int D, bool FP8, int NT> struct queries {
    u32x4 q[NT][D / 32];
    int k_max[NT], k_min[NT];
    float c; // scores in base 2 per product, > 0
    __device__ void load(const dx_attn_args &a, const tile_rows &t, int head, int first, int lane)
    {
        const int col = lane & 15, grp = lane >> 4;
        c = a.scale * kLog2e * (FP8 ? a.cache.k_scale[head] : 1.f);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = t.first + min(first + 16 * n + col, t.rows - 1);
            const int i = by_group(a, row), g = row - i * a.group;
            const DX_GLOBAL dx_bf16 *at = (const DX_GLOBAL dx_bf16 *)a.q + (long)(t.token + i) * a.q_stride + (long)(head * a.group + g) * D;
            k_max[n] = min(t.pos + i, t.hi - 1);
            k_min[n] = a.window ? window_from(a, t.pos + i) : 0;
#pragma unroll
            for (int s = 0; s < D / 32; ++s)
                q[n][s] = *reinterpret_cast<const DX_GLOBAL u32x4 *>(at + (FP8 ? 64 * (s / 2) + 16 * grp + 8 * (s % 2) : 32 * s + 8 * grp));
        }
        if (c <= 0.f) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int s = 0; s < D / 32; ++s) q[n][s] = c < 0.f ? q[n][s] ^ 0x80008000u : u32x4{0, 0, 0, 0};
            c = c < 0.f ? -c : 1.f;
        }
    }
};

// Scores of X consecutive keys from `key` on (KT key tiles), of which row n sees k_min[n] .. k_max[n]; page_ok: the keys' page is one.
template <int X, int NT> __device__ void mask(f32x4 (*s)[NT], int key, bool page_ok, const int *k_min, const int *k_max)
{
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        // the row sees the keys from `lo` on, `more` of them behind it
        const int hi = page_ok ? k_max[n] - key : -1, lo = max(k_min[n] - key, 0);
        const int from = hi < lo ? X : lo;
        const uint32_t more = hi < lo ? 0u : (uint32_t)(hi - lo);
#pragma unroll
        for (int b = 0; b < X / 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((uint32_t)(4 * b + i - from) > more) s[b][n][i] = -INFINITY;
    }
}

// What no row sees may be anything in memory, and 0 * NaN is NaN: 16-byte pieces of the values of X keys from `key` on without the
// keys outside lo .. hi - 1.
template <int X, int N> __device__ void blank(u32x4 (&v)[N], int key, bool page_ok, int lo, int hi)
{
    const int seen_lo = min(max(lo - key, 0), X), seen_hi = page_ok ? min(max(hi - key, 0), X) : 0;
    const uint32_t seen = ((1u << seen_hi) - 1) & ~((1u << seen_lo) - 1); // a bit for each key
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t keep = 0;
#pragma unroll
        for (int e = 0; e < X / 4; ++e) keep |= (0u - (seen >> (X / 4 * i + e) & 1u) & (X == 16 ? 0xFFu : 0xFFFFu)) << (X == 16 ? 8 : 16) * e;
#pragma unroll
        for (int d = 0; d < N; ++d) v[d][i] &= keep;
    }
}

// (passes a NaN on; fmaxf would need its operands quieted first, as many instructions again)
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

// Products of KT key tiles: the running maximum m of every row, to which its sums l (this lane's part) and o are brought if it rises.
// Then c is the factor that takes the products to scores less the maximum, fused.  A maximum is a product rounded after the factor, and the fused
// s c - m leaves what that rounding took: nothing to speak of near 0, but from 2^31 on more than the exponents there are, so that a row's own
// largest key would get 0 or infinity.  So once a maximum is beyond kFar (far: a bit for each lane), the products are rounded as it was and c is 1.
template <int KT, int NT, int DT>
__device__ __forceinline__ void raise_maximum(f32x4 (&s)[KT][NT], float scale, float &c, unsigned long long &far, float (&m)[NT], float (&l)[NT], f32x4 (&o)[DT][NT])
{
    float top[NT];
    bool rise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = max3(s[0][n][0], s[0][n][0], s[0][n][1]);
        top[n] = max3(top[n], s[0][n][2], s[0][n][3]);
#pragma unroll
        for (int b = 1; b < KT; ++b) top[n] = max3(max3(top[n], s[b][n][0], s[b][n][1]), s[b][n][2], s[b][n][3]);
        top[n] *= scale;
        rise |= top[n] > m[n] + kRise;
    }
    if (__ballot(rise) | far) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float next = fmaxf(m[n], max_over_groups(top[n])), f = exp2_fast(m[n] - next);
            m[n] = next;
            l[n] *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d][n] *= f;
            far |= __ballot(fabsf(next) > kFar && next != kNothing);
        }
        if (far) {
            c = 1.f;
#pragma unroll
            for (int b = 0; b < KT; ++b)
#pragma unroll
                for (int n = 0; n < NT; ++n) s[b][n] *= scale;
        }
    }
}
// Products of two key tiles to probabilities, an operand of the product with the values; adds them to l.  They are rounded to bf16, the type that the
// values of a bf16 cache have in that product (2^-8 of a probability at most; the results are 0.0023 from 64 bits, 0.0017 with probabilities in
// 32 bits); l takes them as they were.  Values in e4m3 would fit f16 probabilities, too, at the same number of instructions.
template <int NT> __device__ __forceinline__ void probabilities(const f32x4 (*s)[NT], float c, const float (&m)[NT], float (&l)[NT], u32x4 (&pr)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[i] = exp2_fast(__builtin_fmaf(s[b][n][i], c, -m[n]));
                l[n] += e[i];
            }
            pr[n][2 * b] = pack_bf16(e[0], e[1]);
            pr[n][2 * b + 1] = pack_bf16(e[2], e[3]);
        }
}
// nothing is moved over this point
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// Where the keys and values of one request and kv head are.
template <int D, bool FP8> struct pages {
    static constexpr int X = FP8 ? 16 : 8, UNIT = 4 * X, KT = X / 4;
    const DX_GLOBAL char *k, *v;
    const DX_GLOBAL int32_t *table;
    long page_bytes;
    int n_pages, shift, hi;
    __device__ pages(const dx_attn_args &a, int b, int head, int key_end)
    {
        shift = a.page_shift;
        const long head_bytes = (long)D * (16 / X) << shift;
        page_bytes = head_bytes * a.cache.kv_heads;
        k = (const DX_GLOBAL char *)a.cache.k + head * head_bytes;
        v = (const DX_GLOBAL char *)a.cache.v + head * head_bytes;
        table = (const DX_GLOBAL int32_t *)a.table + (long)b * a.table_stride;
        n_pages = a.cache.n_pages;
        hi = key_end;
    }
    // page of key group g of a unit, -1 past the last key
    __device__ int page_of(int u, int g) const
    {
        const int key = u * UNIT + X * g;
        return key < hi ? table[key >> shift] : -1;
    }
    __device__ bool real(int page) const { return (uint32_t)page < (uint32_t)n_pages; }
    // (what is loaded for a page that is none is not used)
    __device__ const DX_GLOBAL char *keys(int u, int page, int col, int grp) const
    {
        const int off = ((u * UNIT + X * (col >> 2)) & ((1 << shift) - 1)) + (col & 3);
        return k + (real(page) ? page : 0) * page_bytes + (((long)grp << shift) + off) * 16;
    }
    template <bool ONCE> __device__ static u32x4 read(const DX_GLOBAL char *at)
    {
        if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const DX_GLOBAL u32x4 *>(at));
        else return *reinterpret_cast<const DX_GLOBAL u32x4 *>(at);
    }
    // ONCE: nobody else reads it soon
    template <bool ONCE = false> __device__ u32x4 key_piece(const DX_GLOBAL char *at, int i, int b) const { return read<ONCE>(at + ((long)(i * 64) << shift) + 64 * b); }
    __device__ const DX_GLOBAL char *values(int u, int page, int col, int grp) const
    {
        const int off = (u * UNIT + X * grp) & ((1 << shift) - 1);
        return v + (real(page) ? page : 0) * page_bytes + ((long)(off / X) * D + col) * 16;
    }
    template <bool ONCE = false> __device__ static u32x4 value_piece(const DX_GLOBAL char *at, int d) { return read<ONCE>(at + 256 * d); }
};

// ---- values that are no numbers --------------------------------------------------------
// The rows of a tile do not all see the same keys, and 0 times a value that is no number is NaN: what a later token brought (or one that has left a row's
// window) reaches rows of its tile that do not see it.  The loops over the keys do not look for that.  A result that is NaN is looked into once it has been
// stored, and computed again from the keys that its row sees, alone, where a hidden value can have been the cause: among the keys that some rows
// see and others do not, and none that the row does see is NaN anyway.  k_join does that, for tiles that a block stored whole, too (dx_attn_odd): as a part of
// few_rows and many_rows it takes registers from their loops (a chunk of 512 tokens beside 32 decoding 79 us a pass, 84 with; drafts in e4m3 60 and 63).
// It need not be fast: 4096 tokens after 4001, one of them NaN, 102 ms, all of them 13 ms (whoever sees one is NaN rightly).
__device__ float bf16_at(uint32_t two, int i) { return __uint_as_float(i ? two & 0xFFFF0000u : two << 16); }
// NaN if it has been, or an element of v is
__device__ __forceinline__ float nan_of(float x, const f32x4 &v) { return max3(max3(x, v[0], v[1]), v[2], v[3]); }

// Attention of one row, the same in all lanes, over keys lo .. hi - 1: channel 64 i + lane in o[i].  c: scores in base 2 per product.  A lane to a key for the
// scores, to a channel for the sums.
template <int D, bool FP8>
__device__ void one_row(const pages<D, FP8> &kv, const dx_bf16 *q, float c, float v_scale, int lo, int hi, float (&o)[D / 64])
{
    constexpr int X = FP8 ? 16 : 8;
    const int lane = threadIdx.x & 63, in_page = (1 << kv.shift) - 1;
    float m = kNothing, l = 0.f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] = 0.f;
    for (int base = lo & ~63; base < hi; base += 64) {
        const int key = base + lane, page = key < hi ? kv.table[key >> kv.shift] : -1;
        const bool ok = key >= lo && kv.real(page);
        float s = 0.f;
        if (ok) {
            const DX_GLOBAL char *at = kv.k + page * kv.page_bytes + (key & in_page) * 16;
#pragma unroll 1
            for (int x = 0; x < D / X; ++x) {
                const u32x4 k = *reinterpret_cast<const DX_GLOBAL u32x4 *>(at + ((long)x << kv.shift) * 16);
#pragma unroll
                for (int h = 0; h < X / 8; ++h) {
                    const u32x4 wide = FP8 ? widen_half(k, h) : k, by = reinterpret_cast<const u32x4 *>(q)[x * (X / 8) + h];
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = __builtin_fmaf(bf16_at(wide[e / 2], e % 2), bf16_at(by[e / 2], e % 2), s);
                }
            }
        }
        s = ok ? s * c : -INFINITY;
        float top = s;
        for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float next = fmaxf(m, top), f = exp2_fast(m - next), p = exp2_fast(s - next);
        float sum = p;
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        m = next;
        l = l * f + sum;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) o[i] *= f;
        const unsigned long long seen = __ballot(ok);
#pragma unroll 1
        for (int g = 0; g < 64; g += X) {
            const uint32_t see = (uint32_t)(seen >> g) & ((1u << X) - 1);
            if (!see) continue;
            const DX_GLOBAL char *at = kv.v + __builtin_amdgcn_readlane(page, g) * kv.page_bytes + ((long)(((base + g) & in_page) / X) * D + lane) * 16;
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const u32x4 v = *reinterpret_cast<const DX_GLOBAL u32x4 *>(at + 1024 * i);
#pragma unroll
                for (int h = 0; h < X / 8; ++h) {
                    const u32x4 wide = FP8 ? widen_half(v, h) : v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float by = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), g + 8 * h + e));
                        if (see >> (8 * h + e) & 1) o[i] = __builtin_fmaf(by, bf16_at(wide[e / 2], e % 2), o[i]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] *= inverse(l, v_scale);
}

// The stored results of row `row` of a tile at 4 channels from d on.  All lanes of a wavefront call it, live: with a row.
template <int D, bool FP8>
__device__ void look_into(const dx_attn_args &a, const tile_rows &t, int b, int head, int row, int d, bool live)
{
    constexpr int X = FP8 ? 16 : 8, SIZE = 16 / X;
    const pages<D, FP8> kv(a, b, head, t.hi);
    // the keys of row r: from first_key on, up to in front of end_key
    auto first_key = [&](int r) { return a.window ? window_from(a, t.pos + by_group(a, t.first + r)) : 0; };
    auto end_key = [&](int r) { return min(t.pos + by_group(a, t.first + r) + 1, t.hi); };
    dx_bf16 *const out = row_at(a, t.token, head, t.first + row).out;
    uint32_t nan = 0, redo = 0; // a bit for each channel
    if (live) {
        const u32x2 is = *reinterpret_cast<const u32x2 *>(out + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) nan |= (uint32_t)((is[e / 2] >> 16 * (e % 2) & 0x7FFF) > 0x7F80) << e;
    }
    if (nan) {
        const int lo = first_key(row), hi = end_key(row);
#pragma unroll 1
        for (int key = t.lo; key < t.hi; ++key) {
            if (key >= t.all_lo && key < t.all_hi) { // every row sees it
                key = t.all_hi - 1;
                continue;
            }
            const int page = kv.table[key >> kv.shift], off = key & ((1 << kv.shift) - 1);
            if (!kv.real(page)) continue;
            const DX_GLOBAL char *at = kv.v + page * kv.page_bytes + ((long)(off / X) * D + d) * 16 + off % X * SIZE;
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
                const int x = FP8 ? (at[16 * e] & 0x7F) : (*reinterpret_cast<const DX_GLOBAL dx_bf16 *>(at + 16 * e) & 0x7FFF);
                if (key < lo || key >= hi) redo |= (uint32_t)(x >= (FP8 ? 0x7F : 0x7F80)) << e;
                else if (x > (FP8 ? 0x7E : 0x7F80)) nan &= ~(1u << e);
            }
        }
        redo &= nan;
    }
    for (unsigned long long m; (m = __ballot(redo != 0));) {
        const int r = __builtin_amdgcn_readlane(row, __ffsll(m) - 1), i = by_group(a, t.first + r);
        const dx_bf16 *q = a.q + (long)(t.token + i) * a.q_stride + (long)(head * a.group + t.first + r - i * a.group) * D;
        float o[D / 64];
        one_row<D, FP8>(kv, q, a.scale * kLog2e * (FP8 ? a.cache.k_scale[head] : 1.f), FP8 ? a.cache.v_scale[head] : 1.f, first_key(r), end_key(r), o);
        const bool mine = row == r;
#pragma unroll 1
        for (int x = 0; x < 4; ++x) {
            const int channel = d + x;
            float value = 0.f;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                const float of = __shfl(o[j], channel & 63);
                if (channel >> 6 == j) value = of;
            }
            if (mine && redo >> x & 1) out[channel] = (dx_bf16)pack_bf16(value, 0.f);
        }
        if (mine) redo = 0;
    }
}
// (with one token, or with as many that see the same, there is nothing to look for)
__device__ bool may_differ(const tile_rows &t) { return t.lo < t.all_lo || t.all_hi < t.hi; }
// A wavefront has stored a result that is NaN, of the tile that p is at and has all of.
template <class K> __device__ __forceinline__ void note_odd(const dx_attn_args &a, const stretch &p)
{
    if (threadIdx.x & 63) return;
    dx_attn_odd &odd = a.left[blockIdx.x].odd[threadIdx.x >> 6];
    const dx_attn_place at{p.head, p.b, p.tile};
    if (!odd.rows) odd.first = at; // (cleared by this wavefront: take_place)
    odd.last = at;
    odd.paired = p.even < 0;
    odd.rows = K::FEW ? -K::ROWS : K::ROWS;
}
// k_join: those tiles, from the first of them to the last on the line (all between are the block's own)
template <int D> __device__ void look_into_odd(const dx_attn_args &a, const dx_attn_odd &odd)
{
    const int lane = threadIdx.x & 63, rows = abs(odd.rows);
    for (dx_attn_place at = odd.first;;) {
        const tokens of = batch::read(a, at.b);
        const int all = of.n * a.group, tiles = of.n > 0 && (all <= a.few) == (odd.rows < 0) ? (all + rows - 1) / rows : 0;
        if (at.tile < tiles) {
            const tile_rows t = see(a, of, (odd.paired ? paired(at.tile, tiles, at.head) : at.tile) * rows, rows);
#pragma unroll 1
            for (int e = lane; may_differ(t) && e - lane < t.rows * (D / 4); e += 64) {
                const bool live = e < t.rows * (D / 4);
                const int row = min(e / (D / 4), t.rows - 1), d = e % (D / 4) * 4;
                if (a.cache.fmt == DX_KV_E4M3) look_into<D, true>(a, t, at.b, at.head, row, d, live);
                else look_into<D, false>(a, t, at.b, at.head, row, d, live);
            }
            if (at.head == odd.last.head && at.b == odd.last.b && at.tile == odd.last.tile) return;
            ++at.tile;
        } else { // the next request, of the next head
            at.tile = 0;
            if (++at.b == a.B) {
                at.b = 0;
                if (++at.head == a.cache.kv_heads) return;
            }
        }
    }
}

// ---- few rows: the wavefronts of a block share the keys --------------------------------
// Decoding and drafts: up to 16 NT RG rows for a request and kv head (more: several tiles).  Bound by reading the cache once: 64 requests of 500
// to 8000 tokens, 4 heads of 128 channels, 550 MB, 92 us = 6.0 TB/s; one of 150 thousand, 2 of 256, 307 MB, 53 us = 5.8 TB/s; in e4m3 with 1 to 6
// new tokens also by the vector instructions (47 % of the time, the products 20 %): 33 requests, 227 MB, 51 us = 4.5 TB/s.
// The four wavefronts are as many groups of 16 NT rows as the tile needs, 1 to RG, times takers of units in turn.  Keys and values of a wavefront's next
// unit are loaded into the registers that the scores, and the sums, have just been taken from: two wavefronts to a SIMD
// keep the memory busy in each other's computation.  At the end of a tile the takers join their sums through LDS.
template <int D, bool FP8, int NT, int RG> struct few {
    static constexpr int X = FP8 ? 16 : 8, UNIT = 4 * X, WROWS = 16 * NT, PITCH = D + 4;
    struct K : kind<WROWS * RG, UNIT, kKeysOver, kKeysMin, kKeysNear, true, D == 256 ? 4 : 8, 0> {
        // Measured, us a pass, 1 to 6 new tokens a request, at equal weights, these, and a quarter more: 20 requests, 256 channels, bf16 134, 88, 91, fp8 71,
        // 59, 62; 33 of 128 channels, fp8 64.7, 60.4, 61.5, bf16 (where a unit takes as long as its memory) 98.1 at both, 99.4.
        static constexpr int GROUP = WROWS, TWO = NT == 1 ? 6 : FP8 ? 5 : 4, FOUR = 10;
    };
    static constexpr int LDS = 4 * WROWS * (PITCH + 2) * 4;
};
template <int D, bool FP8, int NT, int RG> __device__ __forceinline__ void few_rows(const dx_attn_args &a, const batch &n_of, stretch &p, char *lds)
{
    using S = few<D, FP8, NT, RG>;
    using K = typename S::K;
    constexpr int X = S::X, UNIT = S::UNIT, KT = X / 4, WROWS = S::WROWS, PITCH = S::PITCH; // KT: key tiles of 16 in a unit
    constexpr int LOADS = D / UNIT; // 16-byte pieces of a key per lane
    float *s_o = reinterpret_cast<float *>(lds), *s_m = s_o + 4 * WROWS * PITCH, *s_l = s_m + 4 * WROWS;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    task job;
    while (next_task<K>(a, n_of, p, job)) {
        const tile_rows t = job.t;
        const int groups = RG == 1 || t.rows <= WROWS ? 1 : RG == 2 || t.rows <= 2 * WROWS ? 2 : 4, takers = 4 / groups;
        const int rg = wave % groups, kg = wave / groups;
        queries<D, FP8, NT> q;
        q.load(a, t, p.head, WROWS * rg, lane);
        f32x4 o[D / 16][NT];
        float m[NT], l[NT];
        float c = q.c;
        unsigned long long far = 0;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = kNothing;
            l[n] = 0.f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const pages<D, FP8> kv(a, p.b, p.head, t.hi);
        u32x4 k[D / 16], v[D / 16];
        // Non-temporal (ONCE) where one wavefront reads a unit (64 requests decoding 95 us a pass, 107 without); groups of rows find
        // what the others have brought (33 requests of up to 48 rows, fp8, 73 us, 89 with).  The code is there for each, because a
        // branch around the loads alone is merged into one kind of load.
        auto units = [&](auto once) {
            constexpr bool ONCE = RG == 1 || decltype(once)::value;
            auto load_k = [&](const DX_GLOBAL char *at, int h) { // key tiles 2 h and 2 h + 1
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
#pragma unroll
                    for (int b = 2 * h; b < 2 * h + 2; ++b) k[i * KT + b] = kv.template key_piece<ONCE>(at, i, b);
            };
            auto load_v = [&](int u, int page) {
                const DX_GLOBAL char *at = kv.values(u, page, col, grp);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) v[i] = kv.template value_piece<ONCE>(at, i);
            };

            int u = job.begin + kg;
            if (u >= job.end) return;
            int page_v = kv.page_of(u, grp), next_k = kv.page_of(u + takers, col >> 2), next_v = kv.page_of(u + takers, grp);
            const DX_GLOBAL char *at = kv.keys(u, kv.page_of(u, col >> 2), col, grp);
#pragma unroll
            for (int h = 0; h < KT / 2; ++h) load_k(at, h);
            load_v(u, page_v);
            for (;;) {
                const bool again = u + takers < job.end;
                const int key = u * UNIT + X * grp; // of element 0 of key tile 0
                const bool page_ok = kv.real(page_v), partly = u * UNIT < t.all_lo || (u + 1) * UNIT > t.all_hi || !__all(page_ok);
                at = kv.keys(u + takers, next_k, col, grp);
                if (partly) blank<X>(v, key, page_ok, t.lo, t.hi);
#pragma unroll
                for (int h = 0; h < KT / 2; ++h) { // 32 keys at a time
                    f32x4 s[2][NT];
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int n = 0; n < NT; ++n) s[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < LOADS; ++i)
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            const u32x4 &piece = k[i * KT + 2 * h + b];
                            if constexpr (FP8) {
                                u32x4 lo, hi;
                                widen_fp8(piece, lo, hi);
#pragma unroll
                                for (int n = 0; n < NT; ++n) s[b][n] = mfma(lo, q.q[n][2 * i], s[b][n]);
#pragma unroll
                                for (int n = 0; n < NT; ++n) s[b][n] = mfma(hi, q.q[n][2 * i + 1], s[b][n]);
                            } else {
#pragma unroll
                                for (int n = 0; n < NT; ++n) s[b][n] = mfma(piece, q.q[n][i], s[b][n]);
                            }
                        }
                    if (again) load_k(at, h);
                    if (partly) mask<8, NT>(s, key + 8 * h, page_ok, q.k_min, q.k_max);
                    raise_maximum(s, q.c, c, far, m, l, o);
                    u32x4 pr[NT];
                    probabilities(s, c, m, l, pr);
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        const u32x4 x = FP8 ? widen_half(v[d], h) : v[d];
#pragma unroll
                        for (int n = 0; n < NT; ++n) o[d][n] = mfma(x, pr[n], o[d][n]);
                    }
                }
                if (!again) break;
                u += takers;
                page_v = next_v;
                load_v(u, page_v);
                next_k = kv.page_of(u + takers, col >> 2);
                next_v = kv.page_of(u + takers, grp);
            }
        };
        if (RG == 1 || groups == 1) units(std::true_type{});
        else units(std::false_type{});

        // join the wavefronts of a group of rows
        const float v_scale = FP8 ? a.cache.v_scale[p.head] : 1.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] = sum_over_groups(l[n]);
            if (grp == 0) {
                s_m[wave * WROWS + 16 * n + col] = m[n];
                s_l[wave * WROWS + 16 * n + col] = l[n];
            }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = m[n];
            for (int w = rg; w < 4; w += groups) top = fmaxf(top, s_m[w * WROWS + 16 * n + col]);
            const float f = exp2_fast(m[n] - top);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4 *>(&s_o[(wave * WROWS + 16 * n + col) * PITCH + 16 * d + 4 * grp]) = o[d][n] * f;
        }
        __syncthreads();
        float nan = 0.f;
        for (int e = tid; e < t.rows * (D / 4); e += 256) {
            const int r = e / (D / 4), d = e % (D / 4) * 4, in = r % WROWS;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            float top = kNothing, all = 0.f;
            for (int w = r / WROWS; w < 4; w += groups) {
                sum += *reinterpret_cast<const f32x4 *>(&s_o[(w * WROWS + in) * PITCH + d]);
                top = fmaxf(top, s_m[w * WROWS + in]);
            }
            for (int w = r / WROWS; w < 4; w += groups) all += s_l[w * WROWS + in] * exp2_fast(s_m[w * WROWS + in] - top);
            if (job.slot >= 0) {
                *reinterpret_cast<f32x4 *>(a.part + (job.slot * DX_ATTN_ROWS + r) * D + d) = sum;
                if (d == 0) a.part_ml[job.slot * DX_ATTN_ROWS + r] = float2{top, all};
            } else {
                const row_at to(a, t.token, p.head, t.first + r);
                to.store(d, sum * inverse(all, v_scale));
                if (d == 0) to.store_lse(top, all);
                nan = nan_of(nan, sum);
            }
        }
        if (__builtin_expect(__any(nan != nan), 0)) note_odd<K>(a, p);
        if (!advance<K>(a, n_of, p)) break;
        __syncthreads();
    }
}

// ---- many rows: the wavefronts of a block share keys and values through LDS --------------
// Prompts and chunks of them: 128 rows, 32 to a wavefront.  A stage of keys and values lies in LDS as the wavefronts' operands
// are (1 KB pieces, a lane's 16 bytes at 16 * lane: no bank conflicts), two stages in turn with one barrier each.  The next
// stage is on its way meanwhile: bf16 straight to LDS, fp8 to registers, to be widened before it is stored.  Bound by the instructions of
// the products (1024 cycles of a wavefront's stage) and of the softmax (1040), which two wavefronts to a SIMD run side by side only in part: 4096
// tokens after 4001, 32 heads of 128 channels, 4.06e11 operations, 378 us = 1.07 PFLOP/s (a library's product of 8192^3 1.12 the same day, 1.37 on
// another); 2000 tokens after 1000, 16 heads of 256 channels 134 us = 0.49, in e4m3 146 = 0.45, 32 of 128 in e4m3 104 = 0.63, 4000 after 1000, 16 of 64 90 = 0.55.
template <int D, bool FP8> struct many {
    static constexpr int X = FP8 ? 16 : 8, UNIT = 4 * X, STAGE = 64, NU = STAGE / UNIT; // keys, units of a stage
    static constexpr int PIECES = NU * (D / 8), WIDE = FP8 ? 2 : 1;                     // 16-byte pieces of a stage, operands of a piece
    static constexpr int BYTES = PIECES * WIDE * 1024, LDS = 2 * BYTES + 2 * NU * 4 * 4;
    using K = kind<DX_ATTN_ROWS, STAGE, kRowsOver, kRowsMin, kRowsNear, false, 6, 9>;
};
template <int D, bool FP8> __device__ __forceinline__ void many_rows(const dx_attn_args &a, const batch &n_of, stretch &p, char *s_kv)
{
    using S = many<D, FP8>;
    using K = typename S::K;
    constexpr int NT = 2, X = S::X, UNIT = S::UNIT, KT = X / 4, WROWS = 16 * NT, ROWS = K::ROWS;
    static_assert(ROWS == 4 * WROWS, "four wavefronts");
    constexpr int STAGE = S::STAGE, NU = S::NU, ST = NU * KT; // ST: key tiles of a stage
    constexpr int PW = S::PIECES / 4, WIDE = S::WIDE, BYTES = S::BYTES; // PW: pieces that a wavefront brings
    int(*s_page)[NU][4] = reinterpret_cast<int(*)[NU][4]>(s_kv + 2 * BYTES);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    // a wavefront brings keys or values of one unit of a stage: pieces my_piece ..
    const int my_unit = wave * PW / (D / 8), my_piece = wave * PW % (D / 16);
    const bool my_values = wave * PW % (D / 8) >= D / 16;
    task job;
    while (next_task<K>(a, n_of, p, job)) {
        const tile_rows t = job.t;
        queries<D, FP8, NT> q;
        q.load(a, t, p.head, WROWS * wave, lane);
        // this wavefront's rows
        const bool idle = WROWS * wave >= t.rows;
        const tile_rows mine = see(a, job.of, idle ? t.first : t.first + WROWS * wave, WROWS);
        f32x4 o[D / 16][NT];
        float m[NT], l[NT];
        float c = q.c;
        unsigned long long far = 0;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = kNothing;
            l[n] = 0.f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const pages<D, FP8> kv(a, p.b, p.head, t.hi);
        const int my_group = my_values ? grp : col >> 2;
        auto page_at = [&](int stage) { return kv.page_of(stage * NU + my_unit, my_group); };
        int page = -1, next = -1;
        // keys that no row sees among those of this wavefront's values
        auto at_edge = [&](int stage) {
            const int key = (stage * NU + my_unit) * UNIT;
            return my_values && (key < t.lo || key + UNIT > t.hi || !__all(kv.real(page)));
        };
        u32x4 w[FP8 ? PW : 1]; // fp8: the next stage's pieces, on their way
        auto bring = [&](int stage) {
            const int u = stage * NU + my_unit;
            const DX_GLOBAL char *at = my_values ? kv.values(u, page, col, grp) : kv.keys(u, page, col, grp);
            [[maybe_unused]] const uint32_t to = lds_of(s_kv) + (stage & 1) * BYTES + wave * PW * 1024;
#pragma unroll
            for (int i = 0; i < PW; ++i) {
                const int j = my_piece + i;
                const long off = my_values ? 256 * j : ((long)(j / KT * 64) << kv.shift) + 64 * (j % KT);
                if constexpr (FP8) w[i] = *reinterpret_cast<const DX_GLOBAL u32x4 *>(at + off);
                else load_to_lds((uint32_t)uniform((int)to) + 1024 * i, (uint64_t)(at + off));
            }
        };
        // the stage's pieces of this wavefront are in LDS, once its loads have landed
        auto deliver = [&](int stage) {
            char *at = s_kv + (stage & 1) * BYTES + wave * PW * WIDE * 1024 + lane * 16;
            const bool edge = at_edge(stage);
            const int key = (stage * NU + my_unit) * UNIT + X * grp;
            if constexpr (FP8) {
                if (edge) blank<X>(w, key, kv.real(page), t.lo, t.hi);
#pragma unroll
                for (int i = 0; i < PW; ++i) {
                    u32x4 lo, hi;
                    widen_fp8(w[i], lo, hi);
                    *reinterpret_cast<u32x4 *>(at + 2048 * i) = lo;
                    *reinterpret_cast<u32x4 *>(at + 2048 * i + 1024) = hi;
                }
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                if (edge)
                    for (int i = 0; i < PW; ++i) {
                        w[0] = *reinterpret_cast<const u32x4 *>(at + 1024 * i);
                        blank<X>(w, key, kv.real(page), t.lo, t.hi);
                        *reinterpret_cast<u32x4 *>(at + 1024 * i) = w[0];
                    }
            }
            if (my_values && col == 0) s_page[stage & 1][my_unit][grp] = kv.real(page);
        };
        if (job.begin < job.end) {
            page = page_at(job.begin);
            next = page_at(job.begin + 1);
            bring(job.begin);
        }
        for (int stage = job.begin; stage < job.end; ++stage) {
            deliver(stage);
            __syncthreads();
            if (stage + 1 < job.end) {
                page = next;
                bring(stage + 1);
                next = page_at(stage + 2);
            }
            if (idle || stage * STAGE >= mine.hi || (stage + 1) * STAGE <= mine.lo) continue;
            const char *at = s_kv + (stage & 1) * BYTES + lane * 16;
            auto piece = [&](int i) { return *reinterpret_cast<const u32x4 *>(at + 1024 * i); };
            // scores: operands are read four ahead of their products
            f32x4 s[ST][NT];
#pragma unroll
            for (int b = 0; b < ST; ++b)
#pragma unroll
                for (int n = 0; n < NT; ++n) s[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
            constexpr int QK = ST * (D / 32), AHEAD = 4;
            u32x4 k[QK];
            auto read_key = [&](int j) {
                const int b = j / (D / 32), i = j % (D / 32);
                k[j] = FP8 ? piece(2 * (i / 2 * KT + b) + i % 2) : piece(b / KT * (D / 8) + i * KT + b % KT);
            };
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) read_key(j);
            in_order();
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int j = 0; j < QK; ++j) {
                if (j + AHEAD < QK) read_key(j + AHEAD);
                in_order();
#pragma unroll
                for (int n = 0; n < NT; ++n) s[j / (D / 32)][n] = mfma(k[j], q.q[n][j % (D / 32)], s[j / (D / 32)][n]);
                in_order();
            }
            __builtin_amdgcn_s_setprio(0);
            bool page_ok[NU], all_ok = true;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                page_ok[u] = s_page[stage & 1][u][grp] != 0;
                all_ok &= page_ok[u];
            }
            if (stage * STAGE < mine.all_lo || (stage + 1) * STAGE > mine.all_hi || !__all(all_ok)) {
#pragma unroll
                for (int u = 0; u < NU; ++u) mask<X, NT>(s + u * KT, (stage * NU + u) * UNIT + X * grp, page_ok[u], q.k_min, q.k_max);
            }
            raise_maximum(s, q.c, c, far, m, l, o);
            // the sums in two halves: the second half's probabilities between the first one's products
            constexpr int PV = D / 16, PAIRS = 4 * NT;
            u32x4 v[2 * PV], pr[2][NT];
            auto read_value = [&](int j) {
                const int b = j / PV, d = j % PV;
                v[j] = FP8 ? piece(2 * (D / 16 + d) + b) : piece(b * (D / 8) + D / 16 + d);
            };
            float e[2][2]; // of a pair, and of the one before it, which are added up and packed one step later: exp takes its time
            auto pair = [&](int h, int j) {
                if (j < PAIRS) {
                    const int n = j / 4, b = 2 * h + j / 2 % 2, i = 2 * (j % 2);
                    e[j % 2][0] = exp2_fast(__builtin_fmaf(s[b][n][i], c, -m[n]));
                    e[j % 2][1] = exp2_fast(__builtin_fmaf(s[b][n][i + 1], c, -m[n]));
                }
                if (j > 0) {
                    const int x = j - 1, n = x / 4;
                    l[n] += e[x % 2][0];
                    l[n] += e[x % 2][1];
                    pr[h][n][x % 4] = pack_bf16(e[x % 2][0], e[x % 2][1]);
                }
            };
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) read_value(j);
#pragma unroll
            for (int j = 0; j <= PAIRS; ++j) pair(0, j);
            in_order();
#pragma unroll
            for (int j = 0; j < 2 * PV; ++j) {
                if (j + AHEAD < 2 * PV) read_value(j + AHEAD);
                in_order();
#pragma unroll
                for (int n = 0; n < NT; ++n) o[j % PV][n] = mfma(v[j], pr[j / PV][n], o[j % PV][n]);
                if (j < PV)
#pragma unroll
                    for (int x = j * PAIRS / PV; x < (j + 1) * PAIRS / PV; ++x) pair(1, x);
                if (j == PV - 1) pair(1, PAIRS);
                if (j == PV - 1) __builtin_amdgcn_s_setprio(1);
                in_order();
            }
        }
        __builtin_amdgcn_s_setprio(0);
        const float v_scale = FP8 ? a.cache.v_scale[p.head] : 1.f;
        float nan = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] = sum_over_groups(l[n]);
            const int r = WROWS * wave + 16 * n + col;
            if (job.slot >= 0) {
                f32x4 *to = reinterpret_cast<f32x4 *>(a.part) + job.slot * (ROWS * D / 4) + (NT * wave + n) * (4 * D) + lane;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) to[64 * d] = o[d][n];
                if (grp == 0) a.part_ml[job.slot * ROWS + r] = float2{m[n], l[n]};
            } else if (r < t.rows) {
                const row_at to(a, t.token, p.head, t.first + r);
                const float f = inverse(l[n], v_scale);
#pragma unroll
                for (int d = 0; d < D / 16; ++d) {
                    to.store(16 * d + 4 * grp, o[d][n] * f);
                    nan = nan_of(nan, o[d][n]);
                }
                if (grp == 0) to.store_lse(m[n], l[n]);
            }
        }
        if (__builtin_expect(__any(nan != nan), 0)) note_odd<K>(a, p);
        if (!advance<K>(a, n_of, p)) break;
        __syncthreads();
    }
}

// ---- kernels ------------------------------------------------------------------------
// blocks of a launch to a compute unit, by their registers; what is left of a launch's tiles is joined by as many blocks
template <int D, int NT> constexpr int kBlocks = D == 256 ? 1 : NT == 1 && D == 64 ? 4 : 2;

// The block takes a place on a line (whose first block is place `base` of the launch): what it leaves says nothing yet.
__device__ __forceinline__ void take_place(const dx_attn_args &a, stretch &p, int block, int blocks, int base)
{
    p.block = block;
    p.blocks = blocks;
    p.base = base;
    // (written later, if at all, by the same wavefront)
    if (threadIdx.x < 2) a.left[blockIdx.x].joint[threadIdx.x].n = 0;
    if (threadIdx.x % 64 == 0) a.left[blockIdx.x].odd[threadIdx.x / 64].rows = 0;
}

template <int D, bool FP8, int NT, int RG> __global__ __launch_bounds__(256, (kBlocks<D, NT>)) void k_keys(dx_attn_args a)
{
    using S = few<D, FP8, NT, RG>;
    __shared__ __attribute__((aligned(16))) char lds[S::LDS];
    __shared__ long s_sum[4];
    __shared__ int s_found[3];
    const batch n(a);
    const line_part l = measure<typename S::K>(a, n, even_units<typename S::K>(a, n, gridDim.x), s_sum);
    stretch p;
    take_place(a, p, blockIdx.x, gridDim.x, 0);
    if (locate<typename S::K>(a, n, l, p, s_found)) few_rows<D, FP8, NT, RG>(a, n, p, lds);
}

// Neighbours on the line read the same keys, so each XCD (block index modulo 8) takes a piece of it: the place of block i of n.
__device__ __forceinline__ int by_xcd(int i, int n)
{
    const int x = i & 7;
    return x * (n >> 3) + min(x, n & 7) + (i >> 3);
}

template <int D, bool FP8> __global__ __launch_bounds__(256, (kBlocks<D, 2>)) void k_rows(dx_attn_args a)
{
    using S = many<D, FP8>;
    __shared__ __attribute__((aligned(16))) char lds[S::LDS];
    __shared__ long s_sum[4];
    __shared__ int s_found[3];
    const batch n(a);
    const line_part l = measure<typename S::K>(a, n, 0, s_sum);
    stretch p;
    take_place(a, p, by_xcd(blockIdx.x, gridDim.x), gridDim.x, 0);
    if (locate<typename S::K>(a, n, l, p, s_found)) many_rows<D, FP8>(a, n, p, lds);
}

// Both kinds in one launch (chunks of prompts beside decoding requests): the first blocks take the requests of few rows, which are
// bound by memory, the others those of many, which are not, so that each has the half that the other leaves.  They are as many as
// the lines are long, a stage of many rows taking as long as kStage units of few (set at 32 heads on 4 of 128 channels in bf16).  A chunk of 512 tokens beside 32 decoding requests of 1000
// to 6000, 32 heads on 4 of 128 channels, 78 us; one of 385 beside 8, 64 channels, a window of 1024, 25, of which the launch, the search
// for the block's place and the first loads are more than half.
constexpr int kStage = 2;
template <int D, bool FP8> __global__ __launch_bounds__(256, (kBlocks<D, 2>)) void k_both(dx_attn_args a)
{
    using F = few<D, FP8, 1, 4>;
    using M = many<D, FP8>;
    __shared__ __attribute__((aligned(16))) char lds[F::LDS > M::LDS ? F::LDS : M::LDS];
    __shared__ long s_sum[2][4];
    __shared__ int s_found[3];
    const batch n(a);
    const line_part f = measure<typename F::K>(a, n, 0, s_sum[0]);
    line_part m = measure<typename M::K>(a, n, 0, s_sum[1]);
    const int blocks = gridDim.x;
    int of_few = (int)((float)blocks * (float)f.total / ((float)f.total + kStage * (float)m.total + 1.f) + 0.5f);
    of_few = __builtin_amdgcn_readfirstlane(min(max(of_few, f.total ? 1 : 0), m.total ? blocks - 1 : blocks));
    const int even = even_units<typename M::K>(a, n, blocks - of_few);
    if (even) m = measure<typename M::K>(a, n, even, s_sum[1]);
    stretch p;
    if ((int)blockIdx.x < of_few) {
        take_place(a, p, blockIdx.x, of_few, 0);
        if (locate<typename F::K>(a, n, f, p, s_found)) few_rows<D, FP8, 1, 4>(a, n, p, lds);
    } else {
        take_place(a, p, by_xcd(blockIdx.x - of_few, blocks - of_few), blocks - of_few, of_few);
        if (locate<typename M::K>(a, n, m, p, s_found)) many_rows<D, FP8>(a, n, p, lds);
    }
}

// Tiles whose keys several blocks shared.  As many blocks as shared a tile join it, each a part of its rows' channels, four channels to
// a thread; where that leaves threads over, several take turns on the parts.  A block joins what the block of its index left, because that had the
// same XCD, and with it, in k_rows, the tile's other blocks: their sums are in its L2 (joined by the place on the line: 501 tokens
// after 200, 256 channels, 33 us a pass, 28.6 so; a chunk of 385 beside 8 decoding 27.6, 25.1).  Latency: 2 to 4.8 us if there is nothing to join, 4 to 6 else (one request
// of 150 thousand tokens, all blocks' parts of 16 heads of 256 channels, 4.6).
template <int D> __global__ __launch_bounds__(256) void k_join(dx_attn_args a)
{
    __shared__ __attribute__((aligned(16))) float s_sum[256][4];
    __shared__ float s_top[256], s_all[256];
    const int tid = threadIdx.x;
    const dx_attn_joint joints[2] = {a.left[blockIdx.x].joint[0], a.left[blockIdx.x].joint[1]};
    const dx_attn_odd &odd = a.left[blockIdx.x].odd[uniform(tid >> 6)];
    const int odd_rows = odd.rows;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const dx_attn_joint j = joints[e];
        if (j.n < 2) continue;
        const int me = j.me, all_items = (j.by_lanes ? (j.rows + 15) / 16 * 16 : j.rows) * (D / 4);
        const int first = (int)((long)all_items * me / j.n), items = (int)((long)all_items * (me + 1) / j.n) - first;
        const int lg = items <= 1 ? 0 : items > 128 ? 8 : 32 - __clz(items - 1), wide = 1 << lg, sets = 256 >> lg; // wide: items at a time
        const int set = tid >> lg;
        const float v_scale = a.cache.fmt == DX_KV_E4M3 ? a.cache.v_scale[j.head] : 1.f;
        float nan = 0.f;
        for (int base = 0; base < items; base += wide) {
            const int item = first + min(base + (tid & (wide - 1)), items - 1);
            const piece_of<D> piece(item, j.by_lanes);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            float top = kNothing, all = 0.f;
            auto add = [&](float x, float y, const f32x4 &v) {
                const float next = fmaxf(top, x), f = exp2_fast(top - next), g = exp2_fast(x - next);
                top = next;
                all = all * f + y * g;
                sum = sum * f + v * g;
            };
#pragma unroll 4
            for (int s = set; s < j.n; s += sets) {
                const long at = (2L * (j.block + s) + (s == 0 ? 1 : 0)) * DX_ATTN_ROWS;
                const float2 ml = a.part_ml[at + piece.row];
                add(ml.x, ml.y, reinterpret_cast<const f32x4 *>(a.part)[at * (D / 4) + item]);
            }
            for (int half = sets >> 1; half; half >>= 1) { // the sets in pairs
                *reinterpret_cast<f32x4 *>(s_sum[tid]) = sum;
                s_top[tid] = top;
                s_all[tid] = all;
                __syncthreads();
                const int other = tid + (half << lg);
                if (set < half) add(s_top[other], s_all[other], *reinterpret_cast<const f32x4 *>(s_sum[other]));
                __syncthreads();
            }
            if (set == 0 && base + tid < items && piece.row < j.rows) {
                const row_at to(a, j.token, j.head, j.first + piece.row);
                to.store(piece.d, sum * inverse(all, v_scale));
                if (piece.d == 0) to.store_lse(top, all);
                nan = nan_of(nan, sum);
            }
        }
        if (__builtin_expect(__any(nan != nan), 0)) {
            int b = 0; // whose tile it is
            tokens of = batch::read(a, b);
            while ((of.first != j.token || of.n * a.group < j.first + j.rows) && b + 1 < a.B) of = batch::read(a, ++b);
            const tile_rows t = see(a, of, j.first, j.rows);
            if (may_differ(t))
#pragma unroll 1
                for (int base = 0; base < items; base += wide) {
                    const piece_of<D> piece(first + min(base + (tid & (wide - 1)), items - 1), j.by_lanes);
                    const bool live = set == 0 && base + tid < items && piece.row < j.rows;
                    const int row = min(piece.row, j.rows - 1);
                    if (a.cache.fmt == DX_KV_E4M3) look_into<D, true>(a, t, b, j.head, row, piece.d, live);
                    else look_into<D, false>(a, t, b, j.head, row, piece.d, live);
                }
        }
    }
    if (__builtin_expect(odd_rows != 0, 0)) look_into_odd<D>(a, odd);
}

// Requests of up to so many rows (new tokens * group) for a kv head are few_rows', where the kinds of a call are not known beforehand.
constexpr int kFewRows = 64;

template <int D, bool FP8> void launch(dx_attn_args a, hipStream_t s)
{
    const long rows = (long)a.max_q * a.group;
    const dim3 threads(256);
    int blocks = kBlocks<D, 2> * a.n_cu;
    if (rows <= kFewRows) { // decoding, drafts
        a.few = 0x7FFFFFFF;
        if constexpr (D == 256) {
            hipLaunchKernelGGL((k_keys<D, FP8, 1, 4>), dim3(blocks), threads, 0, s, a);
        } else if (rows <= 16) {
            blocks = kBlocks<D, 1> * a.n_cu;
            hipLaunchKernelGGL((k_keys<D, FP8, 1, 1>), dim3(blocks), threads, 0, s, a);
        } else {
            hipLaunchKernelGGL((k_keys<D, FP8, 2, 2>), dim3(blocks), threads, 0, s, a);
        }
    } else if (a.B == 1) {
        a.few = 0;
        hipLaunchKernelGGL((k_rows<D, FP8>), dim3(blocks), threads, 0, s, a);
    } else {
        a.few = kFewRows;
        hipLaunchKernelGGL((k_both<D, FP8>), dim3(blocks), threads, 0, s, a);
    }
    hipLaunchKernelGGL((k_join<D>), dim3(blocks), threads, 0, s, a);
}

} // namespace

size_t dxk_attention_scratch(int n_cu, char *base, dx_attn_args *a)
{
    // slots of DX_ATTN_ROWS rows, two for each of the most blocks of a launch (kBlocks: as many as 256 channels have heads)
    const size_t slots = 2 * 4 * (size_t)n_cu, channels = 2 * 256 * (size_t)n_cu;
    static_assert(kBlocks<64, 1> * 64 <= 256 && kBlocks<128, 1> * 128 <= 256 && kBlocks<256, 1> * 256 <= 256, "scratch");
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = base + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    char *part = take(channels * DX_ATTN_ROWS * sizeof(float));
    char *ml = take(slots * DX_ATTN_ROWS * sizeof(float2));
    char *left = take(slots / 2 * sizeof(dx_attn_left));
    if (a) {
        a->part = reinterpret_cast<float *>(part);
        a->part_ml = reinterpret_cast<float2 *>(ml);
        a->left = reinterpret_cast<dx_attn_left *>(left);
        a->n_cu = n_cu;
    }
    return at;
}

hipError_t dxk_paged_attention(const dx_attn_args &args, hipStream_t s)
{
    // x / group as a product: 2^(31 + l) / group, l = ceil(log2 group), rounded up (exact for x < 2^31)
    dx_attn_args a = args;
    int l = 0;
    while (1 << l < a.group) ++l;
    a.group_mul = a.group > 1 ? (uint32_t)((1ull << (31 + l)) / a.group + 1) : 0;
    a.group_shift = l - 1;
    const bool fp8 = a.cache.fmt == DX_KV_E4M3;
    switch (a.cache.head_dim) {
    case 64: fp8 ? launch<64, true>(a, s) : launch<64, false>(a, s); break;
    case 128: fp8 ? launch<128, true>(a, s) : launch<128, false>(a, s); break;
    case 256: fp8 ? launch<256, true>(a, s) : launch<256, false>(a, s); break;
    }
    return hipGetLastError();
}
