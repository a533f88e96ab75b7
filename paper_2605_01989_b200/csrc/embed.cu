// dblp_embed and dblp_embed_grad: table lookup with scaling, and the table's gradient by sorted tokens.
//
// The lookup is a gather copy, bound by HBM (latency for a few tokens).
//
// The gradient sums, for every table row, the gradient rows of the tokens that named it.  Sorting the (token, position)
// pairs first makes every sum a run of the sorted list, so that nothing is added by atomics and each sum has one fixed
// order.  The steps, all on the caller's stream:
//   1. sort by (token, position): rank counting up to kRankMax tokens (one launch), else a radix sort by 8-bit digits (two
//      launches a digit);
//   2. k_grad_tiles: the sorted list is cut into tiles of 32 positions whatever the runs' lengths, so a token that fills
//      half the batch is spread over as many warps as any other rows are.  Runs inside a tile are finished; a run that
//      crosses a tile's end leaves a partial sum.  Marks the rows that occur in a bitmap;
//   3. k_grad_finish: joins the partial sums of crossing runs in tile order, and writes zeros to the rows that do not occur.
// The floor is reading dout once and writing the table once.
#include "types.cuh"

namespace dblp {

constexpr int kEmbedThreads = 256;

template <typename I>
__device__ __forceinline__ int64_t token_at(const I* tokens, uint64_t i) { return (int64_t)tokens[i]; }

// ---- lookup ----------------------------------------------------------------------------------------------------------
// A row is `gpr` groups of G elements; consecutive threads take consecutive groups, and kLookUnroll groups a thread with
// all table loads issued before the first store.
constexpr int kLookUnroll = 4;

template <typename I, typename TI, typename TO, int G>
__global__ void __launch_bounds__(kEmbedThreads)
k_embed(const TI* __restrict__ table, int64_t ts, int64_t rows, const I* __restrict__ tokens, uint64_t n, int64_t padding,
        float scale, TO* __restrict__ out, int64_t os, uint32_t gpr, unsigned long long* bad)
{
    const uint64_t items = n * gpr, base = (uint64_t)blockIdx.x * (kEmbedThreads * kLookUnroll) + threadIdx.x;
    uint64_t row[kLookUnroll];
    uint32_t grp[kLookUnroll];
    int64_t tok[kLookUnroll];
#pragma unroll
    for (int u = 0; u < kLookUnroll; ++u) {
        const uint64_t it = base + (uint64_t)u * kEmbedThreads;
        row[u] = it / gpr;
        grp[u] = (uint32_t)(it - row[u] * gpr);
        tok[u] = it < items ? token_at(tokens, row[u]) : -1;
    }
    if constexpr (G == 8) {
        Vec8<TI> v[kLookUnroll];
        float x[8];
#pragma unroll
        for (int u = 0; u < kLookUnroll; ++u)
            if (tok[u] >= 0 && tok[u] < rows && tok[u] != padding) v[u].load(table + tok[u] * ts + grp[u] * 8);
#pragma unroll
        for (int u = 0; u < kLookUnroll; ++u) {
            if (base + (uint64_t)u * kEmbedThreads >= items) break;
            const bool live = tok[u] >= 0 && tok[u] < rows && tok[u] != padding;
            if (!live && bad && tok[u] != padding && grp[u] == 0) atomicAdd(bad, 1ull);
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
    } else {
        TI v[kLookUnroll];
#pragma unroll
        for (int u = 0; u < kLookUnroll; ++u)
            if (tok[u] >= 0 && tok[u] < rows && tok[u] != padding) v[u] = table[tok[u] * ts + grp[u]];
#pragma unroll
        for (int u = 0; u < kLookUnroll; ++u) {
            if (base + (uint64_t)u * kEmbedThreads >= items) break;
            const bool live = tok[u] >= 0 && tok[u] < rows && tok[u] != padding;
            if (!live && bad && tok[u] != padding && grp[u] == 0) atomicAdd(bad, 1ull);
            out[(int64_t)row[u] * os + grp[u]] = from_f32<TO>(live ? __fmul_rn(to_f32(v[u]), scale) : 0.0f);
        }
    }
}

// ---- sort ------------------------------------------------------------------------------------------------------------
// Sort keys: the token, or `rows` for padding and bad tokens, which so come last and are not summed.
template <typename I>
__device__ __forceinline__ uint32_t key_of(const I* tokens, uint64_t i, int64_t rows, int64_t padding, unsigned long long* bad)
{
    const int64_t t = token_at(tokens, i);
    if (t == padding) return (uint32_t)rows;
    if (t < 0 || t >= rows) {
        if (bad) atomicAdd(bad, 1ull);
        return (uint32_t)rows;
    }
    return (uint32_t)t;
}

__device__ __forceinline__ void clear_words(uint32_t* p, uint32_t words)
{
    for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < words; i += gridDim.x * blockDim.x) p[i] = 0;
}

// Stable rank by counting: a block takes 32 tokens, its 8 warps an eighth of all keys each, and lane l counts for token l
// how many of them sort before it.  n^2 comparisons, but one launch and no dependent passes.
constexpr uint32_t kRankMax = 8192;

template <typename I>
__global__ void __launch_bounds__(256)
k_rank_sort(const I* __restrict__ tokens, uint32_t n, int64_t rows, int64_t padding, uint32_t* __restrict__ keys,
            uint32_t* __restrict__ pos, uint32_t* __restrict__ seen, uint32_t seen_words, unsigned long long* bad)
{
    extern __shared__ uint32_t s_key[];                        // all n keys, padded to a multiple of 32 with all-ones
    __shared__ uint32_t s_cnt[8][32];
    clear_words(seen, seen_words);
    const uint32_t n32 = (n + 31) & ~31u, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = blockIdx.x * 32 + lane;
    for (uint32_t i = threadIdx.x; i < n32; i += 256)
        s_key[i] = i < n ? key_of(tokens, i, rows, padding, i / 32 == blockIdx.x ? bad : nullptr) : 0xFFFFFFFFu;
    __syncthreads();
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

// One digit of the radix sort.  Block b owns the contiguous range of `per` items starting at b * per; table[d * blocks + b]
// is its count of digit d.
constexpr int kRadix = 256;
constexpr uint32_t kRadixBlocks = 148;

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
    s_hist[threadIdx.x] = 0;
    if (FIRST) clear_words(seen, seen_words);
    __syncthreads();
    const uint32_t lo = blockIdx.x * per, hi = min(n, lo + per);
    for (uint32_t i = lo + threadIdx.x; i < hi; i += 256)
        atomicAdd(&s_hist[radix_key<I, FIRST>(tokens, keys, i, rows, padding, bad) >> shift & (kRadix - 1)], 1u);
    __syncthreads();
    table[threadIdx.x * gridDim.x + blockIdx.x] = s_hist[threadIdx.x];
}

template <typename I, bool FIRST>
__global__ void __launch_bounds__(256)
k_radix_scatter(const I* __restrict__ tokens, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ pos, uint32_t n,
                uint32_t per, uint32_t shift, int64_t rows, int64_t padding, const uint32_t* __restrict__ table,
                uint32_t* __restrict__ keys_out, uint32_t* __restrict__ pos_out)
{
    __shared__ uint32_t s_warp[8][kRadix];                     // counts, then next free place, per warp and digit
    __shared__ uint32_t s_scan[8];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nb = gridDim.x;
    for (uint32_t i = tid; i < 8 * kRadix; i += 256) (&s_warp[0][0])[i] = 0;
    // place of this block's first item of digit `tid`: items of smaller digits, then those of earlier blocks
    uint32_t before = 0, total = 0;
    for (uint32_t b = 0; b < nb; ++b) {
        const uint32_t c = table[tid * nb + b];
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
    const uint32_t blo = blockIdx.x * per, bhi = min(n, blo + per), wper = per / 8;
    const uint32_t lo = min(bhi, blo + warp * wper), hi = min(bhi, lo + wper);
    for (uint32_t i = lo + lane; i < hi; i += 32)
        atomicAdd(&s_warp[warp][radix_key<I, FIRST>(tokens, keys, i, rows, padding, nullptr) >> shift & (kRadix - 1)], 1u);
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
            const uint32_t key = radix_key<I, FIRST>(tokens, keys, i, rows, padding, nullptr);
            const uint32_t d = key >> shift & (kRadix - 1), same = __match_any_sync(active, d);
            const uint32_t at = s_warp[warp][d] + __popc(same & ((1u << lane) - 1));
            __syncwarp(active);
            if ((same >> lane) == 1u) s_warp[warp][d] = at + 1;  // the highest lane of the digit
            keys_out[at] = key;
            pos_out[at] = FIRST ? i : pos[i];
        }
        __syncwarp();
    }
}

// ---- sums ------------------------------------------------------------------------------------------------------------
// One warp sums one tile of 32 sorted positions over one slab of 32 * G columns.  G = 8 elements a lane (vector loads) or 1
// (any width, stride and alignment).  part: [tiles][2][width]: slot 0 is the tile's share of a run that began before the
// tile, slot 1 of a run that begins here and goes on.
constexpr uint32_t kTile = 32;
constexpr int kGradWarps = 8;

template <typename T, int G>
__device__ __forceinline__ void load_group(const T* p, float* x)
{
    if constexpr (G == 8) {
        Vec8<T> v;
        v.load(p);
        v.get(x);
    } else {
        x[0] = to_f32(*p);
    }
}

template <typename T, int G>
__device__ __forceinline__ void store_group(T* p, const float* x)
{
    if constexpr (G == 8) {
        Vec8<T> v;
        v.set(x);
        v.store(p);
    } else {
        *p = from_f32<T>(x[0]);
    }
}

template <typename T, int G>
__device__ __forceinline__ void finish_row(T* p, float* acc, float scale, bool accumulate)
{
    float old[G];
    if (accumulate) load_group<T, G>(p, old);
#pragma unroll
    for (int i = 0; i < G; ++i) {
        acc[i] = __fmul_rn(acc[i], scale);
        if (accumulate) acc[i] = __fadd_rn(acc[i], old[i]);
    }
    store_group<T, G>(p, acc);
}

template <typename TI, typename TO, int G>
__global__ void __launch_bounds__(kGradWarps * 32)
k_grad_tiles(const TI* __restrict__ dout, int64_t ds, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ pos,
             uint32_t n, uint32_t rows, uint32_t width, uint32_t slabs, float scale, TO* __restrict__ dtable, int64_t ts,
             uint32_t accumulate, float* __restrict__ part, uint32_t* __restrict__ seen)
{
    constexpr int kAhead = G == 8 ? (sizeof(TI) == 2 ? 8 : 4) : 16;     // rows in flight a lane
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t w = (uint64_t)blockIdx.x * kGradWarps + (threadIdx.x >> 5);
    const uint32_t tile = (uint32_t)(w / slabs), slab = (uint32_t)(w - (uint64_t)tile * slabs);
    const uint64_t p0 = (uint64_t)tile * kTile;
    if (p0 >= n) return;
    const uint32_t cnt = min(kTile, (uint32_t)(n - p0));
    const uint32_t key = lane < cnt ? keys[p0 + lane] : 0xFFFFFFFFu, at = lane < cnt ? pos[p0 + lane] : 0;
    const uint32_t prev = p0 ? keys[p0 - 1] : 0xFFFFFFFFu, next = p0 + cnt < n ? keys[p0 + cnt] : 0xFFFFFFFFu;
    const uint32_t live = __popc(__ballot_sync(0xFFFFFFFFu, key < rows));      // keys >= rows are at the end
    if (live == 0) return;
    const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, key, 1);
    if (slab == 0 && lane < live && key != (lane ? up : prev)) atomicOr(&seen[key >> 5], 1u << (key & 31));

    const uint32_t c0 = (slab * 32 + lane) * G;
    const bool in = c0 < width;
    float acc[G];
#pragma unroll
    for (int i = 0; i < G; ++i) acc[i] = 0.0f;
    uint32_t cur = __shfl_sync(0xFFFFFFFFu, key, 0);
    bool began = cur != prev;                                           // the current run begins inside this tile
    float x[kAhead][G];
    for (uint32_t r0 = 0; r0 < live; r0 += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t a = __shfl_sync(0xFFFFFFFFu, at, (r0 + u) & 31);
            if (in && r0 + u < live) load_group<TI, G>(dout + (int64_t)a * ds + c0, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t r = r0 + u;
            if (r < live) {                                             // uniform over the warp
                const uint32_t k = __shfl_sync(0xFFFFFFFFu, key, r & 31);
                if (k != cur) {                                         // the run of `cur` ended with the row before
                    if (in) {
                        if (began) {
                            finish_row<TO, G>(dtable + (int64_t)cur * ts + c0, acc, scale, accumulate);
                        } else {
#pragma unroll
                            for (int i = 0; i < G; ++i) part[((uint64_t)tile * 2) * width + c0 + i] = acc[i];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < G; ++i) acc[i] = 0.0f;
                    cur = k;
                    began = true;
                }
#pragma unroll
                for (int i = 0; i < G; ++i) acc[i] = __fadd_rn(acc[i], x[u][i]);
            }
        }
    }
    if (!in) return;
    const bool goes_on = live == cnt && next == cur;
    if (began && !goes_on) {
        finish_row<TO, G>(dtable + (int64_t)cur * ts + c0, acc, scale, accumulate);
    } else {
        float* q = part + ((uint64_t)tile * 2 + (began ? 1 : 0)) * width + c0;
#pragma unroll
        for (int i = 0; i < G; ++i) q[i] = acc[i];
    }
}

// Blocks below `join_blocks` take one (tile, slab) each: if a run begins in the tile and goes on, they add its partial
// sums, slot 1 of this tile and slot 0 of the following ones, in 8 contiguous parts by 8 warps that are then joined in
// order (runs over fewer than 8 tiles: by the first warp alone).  The other blocks write zeros to the rows whose bit is
// not set, kZeroRows rows each.
constexpr uint32_t kZeroRows = 32;

template <typename TO, int G>
__global__ void __launch_bounds__(kGradWarps * 32)
k_grad_finish(const uint32_t* __restrict__ keys, uint32_t n, uint32_t rows, uint32_t width, uint32_t slabs, float scale,
              TO* __restrict__ dtable, int64_t ts, uint32_t accumulate, const float* __restrict__ part,
              const uint32_t* __restrict__ seen, uint32_t join_blocks)
{
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x >= join_blocks) {
        const uint32_t r0 = (blockIdx.x - join_blocks) * kZeroRows;
        uint32_t absent = ~seen[r0 >> 5];
        if (rows - r0 < 32) absent &= (1u << (rows - r0)) - 1;
        float z[G];
#pragma unroll
        for (int i = 0; i < G; ++i) z[i] = 0.0f;
        for (uint32_t m = absent; m; m &= m - 1) {
            TO* row = dtable + (int64_t)(r0 + __ffs(m) - 1) * ts;
            for (uint32_t c = threadIdx.x * G; c < width; c += kGradWarps * 32 * G) store_group<TO, G>(row + c, z);
        }
        return;
    }
    __shared__ float s_part[kGradWarps][32 * G];
    const uint32_t tile = blockIdx.x / slabs, slab = blockIdx.x - tile * slabs, tiles = (n + kTile - 1) / kTile;
    const uint64_t p0 = (uint64_t)tile * kTile;
    if (p0 + kTile >= n) return;                                        // the last tile: nothing goes on
    const uint32_t key = keys[p0 + kTile - 1];
    if (key >= rows || keys[p0 + kTile] != key) return;
    if (p0 && keys[p0 - 1] == key) return;                              // began in an earlier tile
    // tiles after this one whose first key is still `key`
    uint32_t more = 0;
    for (uint32_t t = tile + 1; ; t += 32) {
        const bool same = t + lane < tiles && keys[(uint64_t)(t + lane) * kTile] == key;
        const uint32_t b = __ballot_sync(0xFFFFFFFFu, same);
        more += b == 0xFFFFFFFFu ? 32 : __ffs(~b) - 1;
        if (b != 0xFFFFFFFFu) break;
    }
    const uint32_t c0 = (slab * 32 + lane) * G, terms = more + 1;
    const bool in = c0 < width;
    const uint32_t parts = terms < 8 ? 1 : 8, per = (terms + parts - 1) / parts;
    const uint32_t lo = min(terms, warp * per), hi = warp < parts ? min(terms, lo + per) : lo;
    float acc[G];
#pragma unroll
    for (int i = 0; i < G; ++i) acc[i] = 0.0f;
    if (in) {
#pragma unroll 4
        for (uint32_t m = lo; m < hi; ++m) {
            const float* q = part + ((uint64_t)(tile + m) * 2 + (m == 0 ? 1 : 0)) * width + c0;
            float x[G];
            load_group<float, G>(q, x);
#pragma unroll
            for (int i = 0; i < G; ++i) acc[i] = __fadd_rn(acc[i], x[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < G; ++i) s_part[warp][lane * G + i] = acc[i];
    __syncthreads();
    if (warp || !in) return;
    for (uint32_t p = 1; p < parts; ++p)
#pragma unroll
        for (int i = 0; i < G; ++i) acc[i] = __fadd_rn(acc[i], s_part[p][lane * G + i]);
    finish_row<TO, G>(dtable + (int64_t)key * ts + c0, acc, scale, accumulate);
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
        k_rank_sort<I><<<n32 / 32, 256, n32 * 4, s>>>(tokens, n, rows, padding, k[0], p[0], seen, seen_words, bad);
        DBLP_LAUNCHED();
        *keys = k[0]; *pos = p[0];
        return DBLP_OK;
    }
    uint32_t per = (n + kRadixBlocks - 1) / kRadixBlocks;
    per = (per + 255) / 256 * 256;
    const uint32_t nb = (n + per - 1) / per;
    int from = 1;
    for (uint32_t shift = 0; shift == 0 || (shift < 32 && (rows >> shift) != 0); shift += 8) {      // keys go up to `rows`
        const int to = from ^ 1;
        if (shift == 0) {
            k_radix_count<I, true><<<nb, 256, 0, s>>>(tokens, nullptr, n, per, shift, rows, padding, table, seen, seen_words, bad);
            DBLP_LAUNCHED();
            k_radix_scatter<I, true><<<nb, 256, 0, s>>>(tokens, nullptr, nullptr, n, per, shift, rows, padding, table, k[to], p[to]);
        } else {
            k_radix_count<I, false><<<nb, 256, 0, s>>>(tokens, k[from], n, per, shift, rows, padding, table, seen, seen_words, nullptr);
            DBLP_LAUNCHED();
            k_radix_scatter<I, false><<<nb, 256, 0, s>>>(tokens, k[from], p[from], n, per, shift, rows, padding, table, k[to], p[to]);
        }
        DBLP_LAUNCHED();
        from = to;
    }
    *keys = k[from]; *pos = p[from];
    return DBLP_OK;
}

template <typename TI, typename TO, int G>
static int launch_sums(const TI* dout, int64_t ds, const uint32_t* keys, const uint32_t* pos, uint32_t n, uint32_t rows, uint32_t width,
                       float scale, TO* dtable, int64_t ts, uint32_t accumulate, float* part, uint32_t* seen, cudaStream_t s)
{
    const uint32_t slabs = (width + 32 * G - 1) / (32 * G), tiles = (n + kTile - 1) / kTile;
    const uint64_t warps = (uint64_t)tiles * slabs, grid = (warps + kGradWarps - 1) / kGradWarps;
    // join blocks exist where a run can cross tiles; zero blocks unless the rows are accumulated into
    const uint64_t join = tiles > 1 ? warps : 0, zero = accumulate ? 0 : (rows + kZeroRows - 1) / kZeroRows;
    DBLP_REQUIRE(grid < (1ull << 31) && join + zero < (1ull << 31), DBLP_ECAPACITY, "embed_grad: too many tokens times columns");
    if (tiles) {
        k_grad_tiles<TI, TO, G><<<(unsigned)grid, kGradWarps * 32, 0, s>>>(dout, ds, keys, pos, n, rows, width, slabs, scale, dtable, ts,
                                                                         accumulate, part, seen);
        DBLP_LAUNCHED();
    }
    if (join + zero) {
        k_grad_finish<TO, G><<<(unsigned)(join + zero), kGradWarps * 32, 0, s>>>(keys, n, rows, width, slabs, scale, dtable, ts,
                                                                               accumulate, part, seen, (uint32_t)join);
        DBLP_LAUNCHED();
    }
    return DBLP_OK;
}

static bool vector_rows(const void* p, int64_t stride, uint64_t nrows, int es)
{
    return aligned16(p) && (nrows <= 1 || stride * es % 16 == 0);
}

}  // namespace dblp

using namespace dblp;

static int check_tokens(const char* who, const void* tokens, uint32_t token_bytes, uint64_t rows, uint32_t width, int ta, int tb)
{
    DBLP_REQUIRE(known_dtype(ta) && known_dtype(tb), DBLP_EINVAL, "%s: unknown dtype %d or %d", who, ta, tb);
    DBLP_REQUIRE(token_bytes == 4 || token_bytes == 8, DBLP_EINVAL, "%s: tokens of %u bytes (4 or 8)", who, token_bytes);
    DBLP_REQUIRE((uintptr_t)tokens % token_bytes == 0, DBLP_EALIGN, "%s: tokens are not aligned to their type", who);
    DBLP_REQUIRE(rows < (1ull << 31) && width < (1u << 30), DBLP_ECAPACITY, "%s: 2^31 rows or 2^30 columns or more", who);
    return DBLP_OK;
}

extern "C" int dblp_embed(const void* table, int64_t table_stride, uint64_t rows, uint32_t width, int table_dtype,
                          const void* tokens, uint32_t token_bytes, uint64_t n, int64_t padding, float scale, void* out,
                          int64_t out_stride, int out_dtype, uint64_t* bad_tokens, void* stream)
{
    const int rc = check_tokens("embed", tokens, token_bytes, rows, width, table_dtype, out_dtype);
    if (rc != DBLP_OK) return rc;
    if (n == 0 || width == 0) return DBLP_OK;
    DBLP_REQUIRE(tokens && out && (table || rows == 0), DBLP_EINVAL, "embed: null pointer");
    DBLP_REQUIRE(n < (1ull << 40), DBLP_ECAPACITY, "embed: 2^40 tokens or more");
    DBLP_REQUIRE(n == 1 || out_stride >= (int64_t)width || out_stride <= -(int64_t)width, DBLP_EINVAL,
                 "embed: rows of the output overlap (stride %lld, width %u)", (long long)out_stride, width);
    const int tb = element_bytes(table_dtype), ob = element_bytes(out_dtype);
    DBLP_REQUIRE((uintptr_t)table % tb == 0 && (uintptr_t)out % ob == 0, DBLP_EALIGN, "embed: a pointer is not aligned to its type");
    const bool vec = width % 8 == 0 && vector_rows(table, table_stride, rows, tb) && vector_rows(out, out_stride, n, ob);
    const uint32_t gpr = vec ? width / 8 : width;
    const uint64_t grid = (n * gpr + kEmbedThreads * kLookUnroll - 1) / (kEmbedThreads * kLookUnroll);
    DBLP_REQUIRE(grid < (1ull << 31), DBLP_ECAPACITY, "embed: too many elements in one call");
    return with_type(table_dtype, [&](auto ti) {
        return with_type(out_dtype, [&](auto to) {
            using TI = decltype(ti);
            using TO = decltype(to);
            auto launch = [&](auto id) -> int {
                using I = decltype(id);
                if (vec) k_embed<I, TI, TO, 8><<<(unsigned)grid, kEmbedThreads, 0, (cudaStream_t)stream>>>(
                    (const TI*)table, table_stride, (int64_t)rows, (const I*)tokens, n, padding, scale, (TO*)out, out_stride, gpr, (unsigned long long*)bad_tokens);
                else k_embed<I, TI, TO, 1><<<(unsigned)grid, kEmbedThreads, 0, (cudaStream_t)stream>>>(
                    (const TI*)table, table_stride, (int64_t)rows, (const I*)tokens, n, padding, scale, (TO*)out, out_stride, gpr, (unsigned long long*)bad_tokens);
                DBLP_LAUNCHED();
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
    const int rc = check_tokens("embed_grad", tokens, token_bytes, rows, width, dout_dtype, dtable_dtype);
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
    uint32_t* seen = (uint32_t*)(w + sp.seen);
    const uint32_t *keys = (const uint32_t*)(w + sp.keys[0]), *pos = (const uint32_t*)(w + sp.pos[0]);
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
                       : launch_sums<TI, TO, 1>((const TI*)dout, dout_stride, keys, pos, (uint32_t)n, (uint32_t)rows, width, scale, (TO*)dtable,
                                                dtable_stride, flags & DBLP_ACCUMULATE, (float*)(w + sp.part), seen, s);
        });
    });
}
