// dblp_embed and dblp_embed_grad: table lookup with scaling, and the table's gradient by sorted tokens.
//
// The lookup is a gather copy, bound by HBM (latency for a few tokens).
//
// The gradient sums, for every table row, the gradient rows of the tokens that named it.  Sorting the (token, position)
// pairs first makes every sum a run of the sorted list, so that nothing is added by atomics and each sum has one fixed
// order.  The steps, all on the caller's stream:
//   1. sort by (token, position): rank counting up to kRankMax tokens (one launch), else a radix sort by 8-bit digits (two
//      launches a digit); a bitmap of the rows that occur comes with it;
//   2. k_grad_tiles: the sorted list is cut into tiles of 32 positions whatever the runs' lengths, so a token that fills
//      half the batch is spread over as many warps as any other rows are.  Runs inside a tile are finished; a run that
//      crosses a tile's end leaves a partial sum.  Other warps of
//      the launch write zeros to the rows that do not occur, so that reading dout and writing the table overlap;
//   3. k_grad_join: joins the partial sums of crossing runs in tile order.
// The floor is reading dout once and writing the table once.  Measured: 32768 x 1600 fp32 into 50257 rows 113 us (4.7 TB/s over
// all; 101 us when it is added to what the table holds), 8192 x 1024 bf16 into 30522 rows 31 us, where the chain of launches is the
// time; 29 tokens into 30522 x 1600 fp32 30 to 34 us (5.8 to 6.5 TB/s).  The lookup: 8192 x 1600 fp32 14 us (5.3 TB/s), one token
// 1.9 us; 20000 x 769 bf16, rows that no vector access may touch, 17 us and the gradient 50.
#include "types.cuh"

namespace dblp {

constexpr int kEmbedThreads = 256;

template <typename I>
__device__ __forceinline__ int64_t token_at(const I* tokens, uint64_t i) { return (int64_t)tokens[i]; }

// ---- lookup ----------------------------------------------------------------------------------------------------------
// A row is `gpr` groups of 8 elements; consecutive threads take consecutive groups, and kLookUnrollOf groups (64 bytes)
// a thread with all table loads issued before the first store.
template <typename TI> constexpr int kLookUnrollOf = sizeof(TI) == 4 ? 2 : 4;

template <typename I, typename TI, typename TO>
__global__ void __launch_bounds__(kEmbedThreads)
k_embed(const TI* __restrict__ table, int64_t ts, int64_t rows, const I* __restrict__ tokens, uint64_t n, int64_t padding,
        float scale, TO* __restrict__ out, int64_t os, FastDiv gpr, unsigned long long* bad)
{
    constexpr int kLookUnroll = kLookUnrollOf<TI>;
    // n * groups < 2^32 a launch (the host cuts longer lists): the division by the row's groups is a multiply and a shift
    const uint32_t items = (uint32_t)n * gpr.d, base = blockIdx.x * (kEmbedThreads * kLookUnroll) + threadIdx.x;
    uint32_t row[kLookUnroll];
    uint32_t grp[kLookUnroll];
    int64_t tok[kLookUnroll];
#pragma unroll
    for (int u = 0; u < kLookUnroll; ++u) {
        const uint32_t it = base + u * kEmbedThreads;
        row[u] = gpr.div(it);
        grp[u] = it - row[u] * gpr.d;
        tok[u] = it < items ? token_at(tokens, row[u]) : -1;
    }
    Vec8<TI> v[kLookUnroll];
    float x[8];
#pragma unroll
    for (int u = 0; u < kLookUnroll; ++u)
        if (tok[u] >= 0 && tok[u] < rows && tok[u] != padding) v[u].load(table + tok[u] * ts + grp[u] * 8);
#pragma unroll
    for (int u = 0; u < kLookUnroll; ++u) {
        if (base + u * kEmbedThreads >= items) break;
        const bool inside = tok[u] >= 0 && tok[u] < rows, live = inside && tok[u] != padding;
        if (!inside && bad && grp[u] == 0) atomicAdd(bad, 1ull);
        Vec8<TO> o;
        if (live) {
            v[u].get(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __fmul_rn(x[i], scale);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        }
        o.set(x);
        o.store(out + (int64_t)row[u] * os + grp[u] * 8);
    }
}

// Any width, stride and alignment: one warp a row and slab of 256 columns, 8 a lane 32 apart, so that the token and the row's
// place are worked out once (element by element with a division each took twice the time for 20000 x 769 bf16).
constexpr int kAnyCols = 8;

template <typename I, typename TI, typename TO>
__global__ void __launch_bounds__(kEmbedThreads)
k_embed_any(const TI* __restrict__ table, int64_t ts, int64_t rows, const I* __restrict__ tokens, uint32_t n, int64_t padding,
            float scale, TO* __restrict__ out, int64_t os, uint32_t width, FastDiv slabs, unsigned long long* bad)
{
    const uint32_t lane = threadIdx.x & 31, w = blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5), row = slabs.div(w), slab = w - row * slabs.d;
    if (row >= n) return;
    const int64_t tok = token_at(tokens, row);
    const bool inside = tok >= 0 && tok < rows, live = inside && tok != padding;
    if (!inside && bad && slab == 0 && lane == 0) atomicAdd(bad, 1ull);
    const uint32_t c0 = slab * (32 * kAnyCols) + lane;
    const TI* src = table + (live ? tok : 0) * ts + c0;
    TO* dst = out + (int64_t)row * os + c0;
    TI v[kAnyCols];
#pragma unroll
    for (int i = 0; i < kAnyCols; ++i)
        if (live && c0 + 32 * i < width) v[i] = src[32 * i];
#pragma unroll
    for (int i = 0; i < kAnyCols; ++i)
        if (c0 + 32 * i < width) dst[32 * i] = from_f32<TO>(live ? __fmul_rn(to_f32(v[i]), scale) : 0.0f);
}

// ---- sort ------------------------------------------------------------------------------------------------------------
// Sort keys: the token, or `rows` for padding and bad tokens, which so come last and are not summed.
template <typename I>
__device__ __forceinline__ uint32_t key_of(const I* tokens, uint64_t i, int64_t rows, int64_t padding, unsigned long long* bad)
{
    const int64_t t = token_at(tokens, i);
    if (t < 0 || t >= rows) {                                  // before the padding id, which is one only inside the table
        if (bad) atomicAdd(bad, 1ull);
        return (uint32_t)rows;
    }
    return t == padding ? (uint32_t)rows : (uint32_t)t;
}

// Stable rank by counting: a block takes 32 tokens, its 8 warps an eighth of all keys each, and lane l counts for token l
// how many of them sort before it.  n^2 comparisons, but one launch and no dependent passes: about 5 us for 4096 tokens, 26 us
// for 8192, where four launches of the radix sort take 14.
constexpr uint32_t kRankMax = 4096, kSeenWords = 128;

template <typename I>
__global__ void __launch_bounds__(256)
k_rank_sort(const I* __restrict__ tokens, uint32_t n, int64_t rows, int64_t padding, uint32_t* __restrict__ keys,
            uint32_t* __restrict__ pos, uint32_t* __restrict__ seen, uint32_t seen_words, unsigned long long* bad)
{
    after_start();
    extern __shared__ __align__(16) uint32_t s_key[];          // all n keys, padded to a multiple of 32 with all-ones; read 16 bytes at a time
    __shared__ uint32_t s_cnt[8][32], s_seen[kSeenWords];
    const uint32_t n32 = (n + 31) & ~31u, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = blockIdx.x * 32 + lane;
    for (uint32_t i = threadIdx.x; i < n32; i += 256)
        s_key[i] = i < n ? key_of(tokens, i, rows, padding, i / 32 == blockIdx.x ? bad : nullptr) : 0xFFFFFFFFu;
    __syncthreads();
    // The bitmap of the rows that occur: every block has all keys at hand and builds a share of the words.
    for (uint32_t w0 = blockIdx.x * kSeenWords; w0 < seen_words; w0 += gridDim.x * kSeenWords) {
        const uint32_t nw = min(kSeenWords, seen_words - w0);
        for (uint32_t i = threadIdx.x; i < nw; i += 256) s_seen[i] = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n; i += 256) {
            const uint32_t k = s_key[i], w = (k >> 5) - w0;
            if (k < rows && w < nw) atomicOr(&s_seen[w], 1u << (k & 31));
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < nw; i += 256) seen[w0 + i] = s_seen[i];
        __syncthreads();
    }
    if (blockIdx.x * 32 >= n32) return;                        // blocks for the bitmap alone
    const uint32_t key = s_key[mine], groups = n32 / 4, per = (groups + 7) / 8;
    const uint32_t lo = min(groups, warp * per), hi = min(groups, lo + per);
    const uint4* __restrict__ k4 = reinterpret_cast<const uint4*>(s_key);
    uint32_t cnt = 0;
    const uint32_t own = blockIdx.x * 8;                       // the block's own 32 tokens are groups own .. own + 7
    for (uint32_t g = lo; g < min(hi, own); ++g) {             // earlier tokens: equal keys sort before
        const uint4 k = k4[g];
        cnt += (k.x <= key) + (k.y <= key) + (k.z <= key) + (k.w <= key);
    }
    for (uint32_t g = max(lo, own); g < min(hi, own + 8); ++g) {
        const uint4 k = k4[g];
        const uint32_t j = g * 4;
        cnt += (k.x < key || (k.x == key && j < mine)) + (k.y < key || (k.y == key && j + 1 < mine)) +
               (k.z < key || (k.z == key && j + 2 < mine)) + (k.w < key || (k.w == key && j + 3 < mine));
    }
    for (uint32_t g = max(lo, own + 8); g < hi; ++g) {
        const uint4 k = k4[g];
        cnt += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
    }
    s_cnt[warp][lane] = cnt;
    __syncthreads();
    if (warp == 0 && mine < n) {
        uint32_t r = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) r += s_cnt[w][lane];
        keys[r] = key;
        pos[r] = mine;
    }
}

// One digit of the radix sort.  Block b owns the contiguous range of `per` items starting at b * per; table[b * 256 + d]
// is its count of digit d.
constexpr int kRadix = 256;
constexpr uint32_t kRadixBlocks = kSms, kRadixStage = 2048;     // blocks at most; items a block keeps in shared memory

template <typename I, bool FIRST>
__device__ __forceinline__ uint32_t radix_key(const I* tokens, const uint32_t* keys, uint32_t i, int64_t rows, int64_t padding,
                                              unsigned long long* bad)
{
    return FIRST ? key_of(tokens, i, rows, padding, bad) : keys[i];
}

template <typename I, bool FIRST>
__global__ void __launch_bounds__(256)
k_radix_count(const I* __restrict__ tokens, const uint32_t* __restrict__ keys, uint32_t n, uint32_t per, uint32_t shift,
              int64_t rows, int64_t padding, uint32_t* __restrict__ table, uint32_t* __restrict__ seen, uint32_t seen_words,
              unsigned long long* bad)
{
    __shared__ uint32_t s_hist[kRadix];
    after_start();
    wait_before();
    s_hist[threadIdx.x] = 0;
    if (FIRST)
        for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < seen_words; i += gridDim.x * 256) seen[i] = 0;
    __syncthreads();
    const uint32_t lo = blockIdx.x * per, hi = min(n, lo + per);
    for (uint32_t i = lo + threadIdx.x; i < hi; i += 256)
        atomicAdd(&s_hist[radix_key<I, FIRST>(tokens, keys, i, rows, padding, bad) >> shift & (kRadix - 1)], 1u);
    __syncthreads();
    table[blockIdx.x * kRadix + threadIdx.x] = s_hist[threadIdx.x];
}

template <typename I, bool FIRST>
__global__ void __launch_bounds__(256)
k_radix_scatter(const I* __restrict__ tokens, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ pos, uint32_t n,
                uint32_t per, uint32_t shift, int64_t rows, int64_t padding, const uint32_t* __restrict__ table,
                uint32_t* __restrict__ keys_out, uint32_t* __restrict__ pos_out, uint32_t* __restrict__ seen)
{
    __shared__ uint32_t s_key[kRadixStage], s_pos[kRadixStage];
    __shared__ uint32_t s_warp[8][kRadix];                     // counts, then next free place, per warp and digit
    __shared__ uint32_t s_scan[8];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nb = gridDim.x;
    for (uint32_t i = tid; i < 8 * kRadix; i += 256) (&s_warp[0][0])[i] = 0;
    after_start();
    wait_before();
    const uint32_t blo = blockIdx.x * per, bhi = min(n, blo + per);
    const bool staged = per <= kRadixStage;
    if (staged)
        for (uint32_t i = blo + tid; i < bhi; i += 256) {
            s_key[i - blo] = radix_key<I, FIRST>(tokens, keys, i, rows, padding, nullptr);
            s_pos[i - blo] = FIRST ? i : pos[i];
        }
    auto key_at = [&](uint32_t i) { return staged ? s_key[i - blo] : radix_key<I, FIRST>(tokens, keys, i, rows, padding, nullptr); };
    // place of this block's first item of digit `tid`: items of smaller digits, then those of earlier blocks
    uint32_t before = 0, total = 0;
#pragma unroll 32
    for (uint32_t b = 0; b < nb; ++b) {
        const uint32_t c = table[b * kRadix + tid];
        before += b < blockIdx.x ? c : 0;
        total += c;
    }
    uint32_t x = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= (uint32_t)o) x += y;
    }
    if (lane == 31) s_scan[warp] = x;
    __syncthreads();
    uint32_t base = x - total + before;
    for (uint32_t w = 0; w < warp; ++w) base += s_scan[w];
    // a warp's share of the block's items is contiguous and a multiple of 32, so warp order is item order
    const uint32_t wper = per / 8;
    const uint32_t lo = min(bhi, blo + warp * wper), hi = min(bhi, lo + wper);
    for (uint32_t i = lo + lane; i < hi; i += 32)
        atomicAdd(&s_warp[warp][key_at(i) >> shift & (kRadix - 1)], 1u);
    __syncthreads();
    for (uint32_t w = 0; w < 8; ++w) {
        const uint32_t c = s_warp[w][tid];
        s_warp[w][tid] = base;
        base += c;
    }
    __syncthreads();
    for (uint32_t i0 = lo; i0 < hi; i0 += 32) {
        const uint32_t i = i0 + lane;
        const bool in = i < hi;
        const uint32_t active = __ballot_sync(0xFFFFFFFFu, in);
        if (in) {
            const uint32_t key = key_at(i);
            const uint32_t d = key >> shift & (kRadix - 1), same = __match_any_sync(active, d);
            const uint32_t at = s_warp[warp][d] + __popc(same & ((1u << lane) - 1));
            __syncwarp(active);
            if ((same >> lane) == 1u) s_warp[warp][d] = at + 1;  // the highest lane of the digit
            keys_out[at] = key;
            pos_out[at] = staged ? s_pos[i - blo] : FIRST ? i : pos[i];
            if (FIRST && key < rows && !(*(volatile uint32_t*)&seen[key >> 5] >> (key & 31) & 1)) atomicOr(&seen[key >> 5], 1u << (key & 31));
        }
        __syncwarp();
    }
}

// ---- sums ------------------------------------------------------------------------------------------------------------
// One warp sums one tile of 32 sorted positions over one slab of 32 * G columns.  G = 8: a lane's columns lie side by side (vector
// loads); G = 4: they are 32 apart, for any width, stride and alignment.  part: [tiles][2][width]: slot 0 is the tile's share
// of a run that began before the tile, slot 1 of a run that begins here and goes on.
constexpr uint32_t kTile = 32;
constexpr int kGradWarps = 8;

template <int G> __device__ __forceinline__ uint32_t first_column(uint32_t slab, uint32_t lane)
{
    return G == 8 ? (slab * 32 + lane) * 8 : slab * (32 * G) + lane;
}

// A lane's elements as they lie in memory: rows in flight are kept this way, half the registers of their fp32 values.  `left`:
// columns from the first one to the row's end.
template <typename T, int G> struct RawGroup {
    T v[G];
    __device__ __forceinline__ void load(const T* p, uint32_t left)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) v[i] = 32u * i < left ? p[32 * i] : T();
    }
    __device__ __forceinline__ void get(float* x) const
    {
#pragma unroll
        for (int i = 0; i < G; ++i) x[i] = to_f32(v[i]);
    }
    __device__ __forceinline__ void put(const float* x, T* p, uint32_t left) const
    {
#pragma unroll
        for (int i = 0; i < G; ++i)
            if (32u * i < left) p[32 * i] = from_f32<T>(x[i]);
    }
};
template <typename T> struct RawGroup<T, 8> {
    Vec8<T> v;
    __device__ __forceinline__ void load(const T* p, uint32_t) { v.load(p); }
    __device__ __forceinline__ void get(float* x) const { v.get(x); }
    __device__ __forceinline__ void put(const float* x, T* p, uint32_t)
    {
        v.set(x);
        v.store(p);
    }
};

template <typename T, int G>
__device__ __forceinline__ void load_group(const T* p, uint32_t left, float* x)
{
    RawGroup<T, G> v;
    v.load(p, left);
    v.get(x);
}

template <typename T, int G>
__device__ __forceinline__ void store_group(T* p, uint32_t left, const float* x)
{
    RawGroup<T, G> v;
    v.put(x, p, left);
}

template <typename T, int G>
__device__ __forceinline__ void finish_row(T* p, uint32_t left, float* acc, float scale, bool accumulate)
{
    float old[G];
    if (accumulate) load_group<T, G>(p, left, old);
#pragma unroll
    for (int i = 0; i < G; ++i) {
        acc[i] = __fmul_rn(acc[i], scale);
        if (accumulate) acc[i] = __fadd_rn(acc[i], old[i]);
    }
    store_group<T, G>(p, left, acc);
}

// Zeros to row `row` if no token names it; one row a warp (4 rows a warp, with the stores of that time: 9 % slower for 30522 x 1600
// fp32 with 29 tokens, the last blocks run alone for longer).  A warp's store covers 512 bytes in one piece.
template <typename TO, int G>
__device__ __forceinline__ void zero_row(uint32_t row, const uint32_t* __restrict__ seen, uint32_t width, TO* __restrict__ dtable, int64_t ts)
{
    const uint32_t lane = threadIdx.x & 31;
    if (seen[row >> 5] >> (row & 31) & 1) return;
    TO* p = dtable + (int64_t)row * ts;
    if constexpr (G == 8) {
        uint4* v = reinterpret_cast<uint4*>(p);
        for (uint32_t c = lane; c < width * sizeof(TO) / 16; c += 32) v[c] = make_uint4(0, 0, 0, 0);
    } else {
        for (uint32_t c = lane; c < width; c += 32) p[c] = from_f32<TO>(0.0f);
    }
}

template <typename TI, typename TO, int G>
__global__ void __launch_bounds__(kGradWarps * 32)
k_grad_tiles(const TI* __restrict__ dout, int64_t ds, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ pos,
             uint32_t n, uint32_t rows, uint32_t width, uint32_t slabs, float scale, TO* __restrict__ dtable, int64_t ts,
             uint32_t accumulate, float* __restrict__ part, const uint32_t* __restrict__ seen, uint32_t sum_blocks)
{
    constexpr int kAhead = G == 8 && sizeof(TI) == 4 ? 4 : 8;     // rows in flight a lane
    after_start();
    wait_before();
    const uint32_t lane = threadIdx.x & 31;
    // blocks that sum and blocks that write zeros take turns while there are both, so that reading and writing overlap
    const uint32_t both = min(sum_blocks, gridDim.x - sum_blocks);
    const bool sums = blockIdx.x < 2 * both ? blockIdx.x % 2 == 0 : sum_blocks > both;
    const uint64_t w = (uint64_t)(blockIdx.x < 2 * both ? blockIdx.x / 2 : blockIdx.x - both) * kGradWarps + (threadIdx.x >> 5);
    if (!sums) {
        if (w < rows) zero_row<TO, G>((uint32_t)w, seen, width, dtable, ts);
        return;
    }
    const uint32_t tile = (uint32_t)(w / slabs), slab = (uint32_t)(w - (uint64_t)tile * slabs);
    const uint64_t p0 = (uint64_t)tile * kTile;
    if (p0 >= n) return;
    const uint32_t cnt = min(kTile, (uint32_t)(n - p0));
    const uint32_t key = lane < cnt ? keys[p0 + lane] : 0xFFFFFFFFu, at = lane < cnt ? pos[p0 + lane] : 0;
    const uint32_t prev = p0 ? keys[p0 - 1] : 0xFFFFFFFFu, next = p0 + cnt < n ? keys[p0 + cnt] : 0xFFFFFFFFu;
    const uint32_t live = __popc(__ballot_sync(0xFFFFFFFFu, key < rows));      // keys >= rows are at the end
    if (live == 0) return;

    const uint32_t c0 = first_column<G>(slab, lane), left = c0 < width ? width - c0 : 0;
    const bool in = left > 0;
    float acc[G];
#pragma unroll
    for (int i = 0; i < G; ++i) acc[i] = 0.0f;
    uint32_t cur = __shfl_sync(0xFFFFFFFFu, key, 0);
    bool began = cur != prev;                                           // the current run begins inside this tile
    RawGroup<TI, G> x[kAhead];
    for (uint32_t r0 = 0; r0 < live; r0 += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t a = __shfl_sync(0xFFFFFFFFu, at, (r0 + u) & 31);
            if (in && r0 + u < live) x[u].load(dout + (int64_t)a * ds + c0, left);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t r = r0 + u;
            if (r < live) {                                             // uniform over the warp
                const uint32_t k = __shfl_sync(0xFFFFFFFFu, key, r & 31);
                if (k != cur) {                                         // the run of `cur` ended with the row before
                    if (in) {
                        if (began) {
                            finish_row<TO, G>(dtable + (int64_t)cur * ts + c0, left, acc, scale, accumulate);
                        } else {
                            store_group<float, G>(part + ((uint64_t)tile * 2) * width + c0, left, acc);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < G; ++i) acc[i] = 0.0f;
                    cur = k;
                    began = true;
                }
                if (in) {
                    float y[G];
                    x[u].get(y);
#pragma unroll
                    for (int i = 0; i < G; ++i) acc[i] = __fadd_rn(acc[i], y[i]);
                }
            }
        }
    }
    if (!in) return;
    const bool goes_on = live == cnt && next == cur;
    if (began && !goes_on) {
        finish_row<TO, G>(dtable + (int64_t)cur * ts + c0, left, acc, scale, accumulate);
    } else {
        store_group<float, G>(part + ((uint64_t)tile * 2 + (began ? 1 : 0)) * width + c0, left, acc);
    }
}

// Joining a run that crosses tiles: slot 1 of the tile in which it begins, then slot 0 of each tile that continues it, in
// tile order.  A tile continues a run when its first key is the key before it.
// Short runs (up to kLongRun - 1 partial sums): one warp a (tile, slab), which ends at once unless a run begins in its tile
// and goes on.  Longer ones: a run of kLongRun or more sums continues over at least one tile whose number is a multiple of 16;
// the first such tile names the run, and a block adds it in 8 contiguous parts by 8 warps, joined in order.
constexpr uint32_t kLongRun = 17;

__device__ __forceinline__ bool continues(const uint32_t* __restrict__ keys, uint32_t tile, uint32_t tiles, uint32_t key)
{
    return tile > 0 && tile < tiles && keys[(uint64_t)tile * kTile] == key && keys[(uint64_t)tile * kTile - 1] == key;
}

// Tiles from `from` on, one after the other, that continue key's run.
__device__ __forceinline__ uint32_t continued(const uint32_t* __restrict__ keys, uint32_t from, uint32_t tiles, uint32_t key)
{
    uint32_t more = 0;
    for (uint32_t t = from;; t += 32) {
        const uint32_t b = __ballot_sync(0xFFFFFFFFu, continues(keys, t + (threadIdx.x & 31), tiles, key));
        more += b == 0xFFFFFFFFu ? 32 : __ffs(~b) - 1;
        if (b != 0xFFFFFFFFu) return more;
    }
}

// Terms lo .. hi - 1 of the run that begins in `tile`, columns c0 ..
template <int G>
__device__ __forceinline__ void add_terms(const float* __restrict__ part, uint32_t tile, uint32_t lo, uint32_t hi, uint32_t width, uint32_t c0, float* acc)
{
#pragma unroll 8
    for (uint32_t m = lo; m < hi; ++m) {
        float x[G];
        load_group<float, G>(part + ((uint64_t)(tile + m) * 2 + (m == 0 ? 1 : 0)) * width + c0, width - c0, x);
#pragma unroll
        for (int i = 0; i < G; ++i) acc[i] = __fadd_rn(acc[i], x[i]);
    }
}

template <typename TO, int G>
__global__ void __launch_bounds__(kGradWarps * 32)
k_grad_join(const uint32_t* __restrict__ keys, uint32_t n, uint32_t rows, uint32_t width, uint32_t slabs, float scale,
            TO* __restrict__ dtable, int64_t ts, uint32_t accumulate, const float* __restrict__ part, uint32_t short_blocks)
{
    __shared__ float s_part[kGradWarps][32 * G];
    wait_before();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tiles = (n + kTile - 1) / kTile;
    float acc[G];
#pragma unroll
    for (int i = 0; i < G; ++i) acc[i] = 0.0f;
    if (blockIdx.x < short_blocks) {
        const uint64_t w = (uint64_t)blockIdx.x * kGradWarps + warp;
        const uint32_t tile = (uint32_t)(w / slabs), slab = (uint32_t)(w - (uint64_t)tile * slabs), c0 = first_column<G>(slab, lane);
        if (tile + 1 >= tiles) return;                                  // nothing goes on from the last tile
        const uint64_t end = (uint64_t)(tile + 1) * kTile;
        const uint32_t key = keys[end - 1];
        if (key >= rows || keys[end] != key || continues(keys, tile, tiles, key)) return;
        const uint32_t terms = 1 + continued(keys, tile + 1, tiles, key);
        if (terms >= kLongRun || c0 >= width) return;
        add_terms<G>(part, tile, 0, terms, width, c0, acc);
        finish_row<TO, G>(dtable + (int64_t)key * ts + c0, width - c0, acc, scale, accumulate);
        return;
    }
    const uint32_t at = blockIdx.x - short_blocks, u = (at / slabs + 1) * 16, slab = at % slabs, c0 = first_column<G>(slab, lane);
    const uint32_t key = keys[(uint64_t)u * kTile];
    if (key >= rows || !continues(keys, u, tiles, key) || continues(keys, u - 16, tiles, key)) return;
    // u - 16 does not continue the run, so it begins in one of the 16 tiles before u
    const uint32_t back = __ffs(~__ballot_sync(0xFFFFFFFFu, lane < 16 && continues(keys, u - 1 - lane, tiles, key))) - 1;
    const uint32_t tile = u - back - 1, terms = 1 + back + continued(keys, u, tiles, key);
    if (terms < kLongRun) return;
    const uint32_t per = (terms + kGradWarps - 1) / kGradWarps, lo = min(terms, warp * per), hi = min(terms, lo + per);
    if (c0 < width) add_terms<G>(part, tile, lo, hi, width, c0, acc);
#pragma unroll
    for (int i = 0; i < G; ++i) s_part[warp][lane * G + i] = acc[i];
    __syncthreads();
    if (warp || c0 >= width) return;
    for (int p = 1; p < kGradWarps; ++p)
#pragma unroll
        for (int i = 0; i < G; ++i) acc[i] = __fadd_rn(acc[i], s_part[p][lane * G + i]);
    finish_row<TO, G>(dtable + (int64_t)key * ts + c0, width - c0, acc, scale, accumulate);
}

// Places in the workspace, each on a 256-byte boundary.
struct GradSpace {
    uint64_t keys[2], pos[2], table, seen, part, bytes;
    GradSpace(uint64_t n, uint64_t rows, uint32_t width)
    {
        uint64_t at = 0;
        auto take = [&](uint64_t b) { const uint64_t p = at; at += (b + 255) & ~255ull; return p; };
        for (int i = 0; i < 2; ++i) { keys[i] = take(n * 4); pos[i] = take(n * 4); }
        table = take(4ull * kRadix * kRadixBlocks);
        seen = take((rows + 31) / 32 * 4);
        const uint64_t w8 = (width + 7ull) / 8 * 8;
        part = take((n + kTile - 1) / kTile * 2 * w8 * 4);
        bytes = at;
    }
};

template <typename I>
static int sort_tokens(const I* tokens, uint32_t n, uint32_t rows, int64_t padding, uint8_t* ws, const GradSpace& sp,
                       unsigned long long* bad, const uint32_t** keys, const uint32_t** pos, cudaStream_t s)
{
    uint32_t* k[2] = {(uint32_t*)(ws + sp.keys[0]), (uint32_t*)(ws + sp.keys[1])};
    uint32_t* p[2] = {(uint32_t*)(ws + sp.pos[0]), (uint32_t*)(ws + sp.pos[1])};
    uint32_t *table = (uint32_t*)(ws + sp.table), *seen = (uint32_t*)(ws + sp.seen);
    const uint32_t seen_words = (rows + 31) / 32;
    if (n <= kRankMax) {
        const uint32_t n32 = (n + 31) & ~31u;
        const uint32_t for_seen = (seen_words + kSeenWords - 1) / kSeenWords;
        const uint32_t grid = n32 / 32 > for_seen ? n32 / 32 : for_seen < kSms ? for_seen : kSms;
        k_rank_sort<I><<<grid, 256, n32 * 4, s>>>(tokens, n, rows, padding, k[0], p[0], seen, seen_words, bad);
        DBLP_LAUNCHED();
        *keys = k[0]; *pos = p[0];
        return DBLP_OK;
    }
    // Every block reads all blocks' counts: up to 64 of them while a block's items fit in its shared memory, then more.
    uint32_t per = (n + 63) / 64;
    if (per > kRadixStage) per = (n + kRadixBlocks - 1) / kRadixBlocks > kRadixStage ? (n + kRadixBlocks - 1) / kRadixBlocks : kRadixStage;
    per = (per + 255) / 256 * 256;
    const uint32_t nb = (n + per - 1) / per;
    int from = 1;
    for (uint32_t shift = 0; shift == 0 || (shift < 32 && (rows >> shift) != 0); shift += 8) {      // keys go up to `rows`
        const int to = from ^ 1;
        if (shift == 0) {
            k_radix_count<I, true><<<nb, 256, 0, s>>>(tokens, nullptr, n, per, shift, rows, padding, table, seen, seen_words, bad);
            DBLP_LAUNCHED();
            DBLP_NEXT(launch_next(k_radix_scatter<I, true>, nb, 256, 0, s, tokens, nullptr, nullptr, n, per, shift, rows, padding, table, k[to], p[to], seen));
        } else {
            DBLP_NEXT(launch_next(k_radix_count<I, false>, nb, 256, 0, s, tokens, k[from], n, per, shift, rows, padding, table, nullptr, 0, nullptr));
            DBLP_NEXT(launch_next(k_radix_scatter<I, false>, nb, 256, 0, s, tokens, k[from], p[from], n, per, shift, rows, padding, table, k[to], p[to], seen));
        }
        from = to;
    }
    *keys = k[from]; *pos = p[from];
    return DBLP_OK;
}

template <typename TI, typename TO, int G>
static int launch_sums(const TI* dout, int64_t ds, const uint32_t* keys, const uint32_t* pos, uint32_t n, uint32_t rows, uint32_t width,
                       float scale, TO* dtable, int64_t ts, uint32_t accumulate, float* part, const uint32_t* seen, cudaStream_t s)
{
    const uint32_t slabs = (width + 32 * G - 1) / (32 * G), tiles = (n + kTile - 1) / kTile;
    const uint64_t sums = (uint64_t)tiles * slabs, zeros = accumulate ? 0 : rows;
    const uint64_t sum_blocks = (sums + kGradWarps - 1) / kGradWarps, grid = sum_blocks + (zeros + kGradWarps - 1) / kGradWarps;
    DBLP_REQUIRE(grid < (1ull << 31), DBLP_ECAPACITY, "embed_grad: too many tokens times columns");
    DBLP_NEXT(launch_next(k_grad_tiles<TI, TO, G>, (unsigned)grid, kGradWarps * 32, 0, s, dout, ds, keys, pos, n, rows, width, slabs, scale, dtable,
                          ts, accumulate, part, seen, (uint32_t)sum_blocks));
    if (tiles > 1) {                                                   // a run can cross tiles
        const uint64_t brief = ((tiles - 1ull) * slabs + kGradWarps - 1) / kGradWarps, lengthy = (uint64_t)((tiles - 1) / 16) * slabs;
        DBLP_REQUIRE(brief + lengthy < (1ull << 31), DBLP_ECAPACITY, "embed_grad: too many tokens times columns");
        DBLP_NEXT(launch_next(k_grad_join<TO, G>, (unsigned)(brief + lengthy), kGradWarps * 32, 0, s, keys, n, rows, width, slabs, scale, dtable, ts,
                              accumulate, part, (uint32_t)brief));
    }
    return DBLP_OK;
}

static bool vector_rows(const void* p, int64_t stride, uint64_t nrows, int es)
{
    return aligned16(p) && (nrows <= 1 || stride * es % 16 == 0);
}

}  // namespace dblp

using namespace dblp;

static int check_tokens(const char* who, const void* tokens, uint32_t token_bytes, const void* bad, uint64_t rows, uint32_t width, int ta, int tb)
{
    DBLP_REQUIRE(known_dtype(ta) && known_dtype(tb), DBLP_EINVAL, "%s: unknown dtype %d or %d", who, ta, tb);
    DBLP_REQUIRE(token_bytes == 4 || token_bytes == 8, DBLP_EINVAL, "%s: tokens of %u bytes (4 or 8)", who, token_bytes);
    DBLP_REQUIRE((uintptr_t)tokens % token_bytes == 0, DBLP_EALIGN, "%s: tokens are not aligned to their type", who);
    DBLP_REQUIRE((uintptr_t)bad % 8 == 0, DBLP_EALIGN, "%s: bad_tokens is not aligned to its type", who);
    DBLP_REQUIRE(rows < (1ull << 31) && width < (1u << 30), DBLP_ECAPACITY, "%s: 2^31 rows or 2^30 columns or more", who);
    return DBLP_OK;
}

extern "C" int dblp_embed(const void* table, int64_t table_stride, uint64_t rows, uint32_t width, int table_dtype,
                          const void* tokens, uint32_t token_bytes, uint64_t n, int64_t padding, float scale, void* out,
                          int64_t out_stride, int out_dtype, uint64_t* bad_tokens, void* stream)
{
    const int rc = check_tokens("embed", tokens, token_bytes, bad_tokens, rows, width, table_dtype, out_dtype);
    if (rc != DBLP_OK) return rc;
    if (n == 0 || width == 0) return DBLP_OK;
    DBLP_REQUIRE(tokens && out && (table || rows == 0), DBLP_EINVAL, "embed: null pointer");
    DBLP_REQUIRE(n < (1ull << 40), DBLP_ECAPACITY, "embed: 2^40 tokens or more");
    DBLP_REQUIRE(n == 1 || out_stride >= (int64_t)width || out_stride <= -(int64_t)width, DBLP_EINVAL,
                 "embed: rows of the output overlap (stride %lld, width %u)", (long long)out_stride, width);
    const int tb = element_bytes(table_dtype), ob = element_bytes(out_dtype);
    DBLP_REQUIRE((uintptr_t)table % tb == 0 && (uintptr_t)out % ob == 0, DBLP_EALIGN, "embed: a pointer is not aligned to its type");
    const bool vec = width % 8 == 0 && vector_rows(table, table_stride, rows, tb) && vector_rows(out, out_stride, n, ob);
    // groups of 8 columns, a thread each, or slabs, a warp each; tokens a launch: their items fit in 32 bits
    const uint32_t per_row = vec ? width / 8 : (width + 32 * kAnyCols - 1) / (32 * kAnyCols);
    const uint64_t most = 0xFFFF0000u / per_row;
    return with_type(table_dtype, [&](auto ti) -> int {
        return with_type(out_dtype, [&](auto to) -> int {
            using TI = decltype(ti);
            using TO = decltype(to);
            auto launch = [&](auto id) -> int {
                using I = decltype(id);
                const uint32_t per_block = vec ? kEmbedThreads * kLookUnrollOf<TI> : kEmbedThreads / 32;
                for (uint64_t first = 0; first < n; first += most) {
                    const uint64_t m = n - first < most ? n - first : most;
                    const unsigned grid = (unsigned)((m * per_row + per_block - 1) / per_block);
                    const I* tk = (const I*)tokens + first;
                    TO* o = (TO*)out + (int64_t)first * out_stride;
                    if (vec) k_embed<I, TI, TO><<<grid, kEmbedThreads, 0, (cudaStream_t)stream>>>(
                        (const TI*)table, table_stride, (int64_t)rows, tk, m, padding, scale, o, out_stride, FastDiv(per_row), (unsigned long long*)bad_tokens);
                    else k_embed_any<I, TI, TO><<<grid, kEmbedThreads, 0, (cudaStream_t)stream>>>(
                        (const TI*)table, table_stride, (int64_t)rows, tk, (uint32_t)m, padding, scale, o, out_stride, width, FastDiv(per_row),
                        (unsigned long long*)bad_tokens);
                    DBLP_LAUNCHED();
                }
                return DBLP_OK;
            };
            return token_bytes == 4 ? launch(int32_t()) : launch(int64_t());
        });
    });
}

extern "C" int dblp_embed_grad_workspace_bytes(uint64_t n, uint64_t rows, uint32_t width, size_t* bytes)
{
    DBLP_REQUIRE(bytes, DBLP_EINVAL, "embed_grad_workspace_bytes: null output");
    DBLP_REQUIRE(n < (1ull << 31) && rows < (1ull << 31) && width < (1u << 30), DBLP_ECAPACITY,
                 "embed_grad: 2^31 tokens or rows, or 2^30 columns, or more");
    *bytes = GradSpace(n, rows, width).bytes;
    return DBLP_OK;
}

extern "C" int dblp_embed_grad(const void* dout, int64_t dout_stride, int dout_dtype, const void* tokens, uint32_t token_bytes,
                               uint64_t n, int64_t padding, float scale, void* dtable, int64_t dtable_stride, uint64_t rows,
                               uint32_t width, int dtable_dtype, uint32_t flags, uint64_t* bad_tokens, void* ws, size_t ws_bytes,
                               void* stream)
{
    const int rc = check_tokens("embed_grad", tokens, token_bytes, bad_tokens, rows, width, dout_dtype, dtable_dtype);
    if (rc != DBLP_OK) return rc;
    DBLP_REQUIRE((flags & ~(uint32_t)DBLP_ACCUMULATE) == 0, DBLP_EINVAL, "embed_grad: unknown flags %u", flags);
    DBLP_REQUIRE(n < (1ull << 31), DBLP_ECAPACITY, "embed_grad: 2^31 tokens or more");
    if (rows == 0 || width == 0 || (n == 0 && (flags & DBLP_ACCUMULATE))) return DBLP_OK;
    DBLP_REQUIRE(dtable && (n == 0 || (dout && tokens)), DBLP_EINVAL, "embed_grad: null pointer");
    DBLP_REQUIRE(rows == 1 || dtable_stride >= (int64_t)width || dtable_stride <= -(int64_t)width, DBLP_EINVAL,
                 "embed_grad: rows of the gradient overlap (stride %lld, width %u)", (long long)dtable_stride, width);
    const int db = element_bytes(dout_dtype), tb = element_bytes(dtable_dtype);
    DBLP_REQUIRE((uintptr_t)dout % db == 0 && (uintptr_t)dtable % tb == 0, DBLP_EALIGN, "embed_grad: a pointer is not aligned to its type");
    const GradSpace sp(n, rows, width);
    DBLP_REQUIRE(ws && ((uintptr_t)ws & 255) == 0, ws ? DBLP_EALIGN : DBLP_EINVAL, "embed_grad: the workspace is null or not 256-byte aligned");
    DBLP_REQUIRE(ws_bytes >= sp.bytes, DBLP_ECAPACITY, "embed_grad: workspace of %zu bytes, needs %llu", ws_bytes, (unsigned long long)sp.bytes);
    uint8_t* w = (uint8_t*)ws;
    cudaStream_t s = (cudaStream_t)stream;
    const uint32_t *keys = (const uint32_t*)(w + sp.keys[0]), *pos = (const uint32_t*)(w + sp.pos[0]);
    uint32_t* seen = (uint32_t*)(w + sp.seen);
    if (n == 0) {
        DBLP_CUDA(cudaMemsetAsync(seen, 0, (rows + 31) / 32 * 4, s));
    } else {
        const int rs = token_bytes == 4
            ? sort_tokens((const int32_t*)tokens, (uint32_t)n, (uint32_t)rows, padding, w, sp, (unsigned long long*)bad_tokens, &keys, &pos, s)
            : sort_tokens((const int64_t*)tokens, (uint32_t)n, (uint32_t)rows, padding, w, sp, (unsigned long long*)bad_tokens, &keys, &pos, s);
        if (rs != DBLP_OK) return rs;
    }
    const bool vec = width % 8 == 0 && vector_rows(dout, dout_stride, n, db) && vector_rows(dtable, dtable_stride, rows, tb);
    return with_type(dout_dtype, [&](auto ti) {
        return with_type(dtable_dtype, [&](auto to) {
            using TI = decltype(ti);
            using TO = decltype(to);
            return vec ? launch_sums<TI, TO, 8>((const TI*)dout, dout_stride, keys, pos, (uint32_t)n, (uint32_t)rows, width, scale, (TO*)dtable,
                                                dtable_stride, flags & DBLP_ACCUMULATE, (float*)(w + sp.part), seen, s)
                       : launch_sums<TI, TO, 4>((const TI*)dout, dout_stride, keys, pos, (uint32_t)n, (uint32_t)rows, width, scale, (TO*)dtable,
                                                dtable_stride, flags & DBLP_ACCUMULATE, (float*)(w + sp.part), seen, s);
        });
    });
}
