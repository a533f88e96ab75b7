// dblp_norm_rotate, dblp_norm_rotate_grad: root-mean-square norm of every head of q and k, and the rotation by position.
//
// A lane holds sixteen elements of a head's row as two groups of eight, chosen so that both members of a rotated pair are its own:
// columns u .. u + 7 and R / 2 + u .. (interleaved, and behind the rotated part: sixteen in a row).  L lanes, a power of two, make
// a row; the norm is a shuffle reduction, the rotation needs none.  (One group a lane, the other member by shuffles: 39 us for
// 8 x 1024 tokens, 25 + 25 heads of 64, bf16, bound by instructions.)
// Cosines and sines of a step's tokens are computed once per block into shared memory: the angle, pos * freq / 2 pi, in 64 bits,
// less its nearest integer, then one fp32 sincospi.
// The backward pass recomputes r from x instead of reading a stored one: x is needed anyway.
#include <math.h>

#include "tc.cuh"

namespace dblp {

constexpr int kRotThreads = 256;
constexpr int kRotRows = 2;                      // rows in flight per lane group

struct RotHeads {
    const void* p;
    int64_t sb, st, sh;
};

// q or k: rows number token * heads + head
struct RotSide {
    RotHeads x, d;                               // input; gradient of the output
    RotHeads y;                                  // output; gradient of the input
    const void* weight;
    uint32_t heads, rows, blocks;
    FastDiv by_heads;
    float* partial;                              // [blocks][D] sums of the weight's gradient, or null
};

struct RotArgs {
    RotSide side[2];
    uint32_t tokens, D, R, L, weight_dtype, table_tokens;
    FastDiv by_tokens;
    float eps, inv_d;
    const int32_t* positions;
    int64_t position_stride;
    const double* freqs;
};

// Columns of a lane's two groups: a .. a + 7 and b .. b + 7; from D on a group is empty.
struct RotPlace {
    uint32_t a, b;
    bool turns;                                  // part of the rotated columns (interleaved: a may be, b need not)
};
template <bool INTER> __device__ __forceinline__ RotPlace place_of(uint32_t unit, uint32_t R)
{
    if (INTER) return {unit * 16, unit * 16 + 8, unit * 16 < R};
    const uint32_t turning = R / 16;
    if (unit < turning) return {unit * 8, R / 2 + unit * 8, true};
    return {R + (unit - turning) * 16, R + (unit - turning) * 16 + 8, false};
}

// (cos, sin) of the angles of tokens first .. first + n - 1 (of batch * tokens in all): R / 2 cosines, then R / 2 sines a token.
__device__ __forceinline__ void fill_angles(const RotArgs& a, float* table, uint32_t first, uint32_t n)
{
    const uint32_t half = a.R / 2;
    for (uint32_t i = threadIdx.x; i < n * half; i += kRotThreads) {
        const uint32_t j = i / half, f = i - j * half, t = first + j, b = a.by_tokens.div(t);
        const double turns = (double)a.positions[(int64_t)b * a.position_stride + (t - b * a.tokens)] * a.freqs[f] * 0.15915494309189533577;
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        table[j * a.R + f] = c;
        table[j * a.R + half + f] = s;
    }
}

__device__ __forceinline__ float2 neg2(float2 x) { return make_float2(-x.x, -x.y); }

// A lane's sixteen values (a in the first four pairs, b in the last) turned by +t, BACK by -t; angles of its token.
template <bool INTER, bool BACK> __device__ __forceinline__ void turn(float2* v, const float* angles, const RotPlace& p, uint32_t R)
{
    const uint32_t half = R / 2;
    if (INTER) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t at = p.a / 2 + i;
            if (at >= half) break;
            const float c = angles[at], s = BACK ? -angles[half + at] : angles[half + at];
            v[i] = make_float2(v[i].x * c - v[i].y * s, v[i].x * s + v[i].y * c);
        }
    } else if (p.turns) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float4 c = *reinterpret_cast<const float4*>(angles + p.a + 4 * q), s = *reinterpret_cast<const float4*>(angles + half + p.a + 4 * q);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float2 cc = h ? make_float2(c.z, c.w) : make_float2(c.x, c.y), ss = h ? make_float2(s.z, s.w) : make_float2(s.x, s.y);
                const float2 x = v[2 * q + h], y = v[4 + 2 * q + h], up = BACK ? neg2(ss) : ss;
                v[2 * q + h] = fma2(y, neg2(up), mul2(x, cc));
                v[4 + 2 * q + h] = fma2(x, up, mul2(y, cc));
            }
        }
    }
}

struct RotRow {
    bool live;
    uint32_t token, b, t, h;
};
__device__ __forceinline__ RotRow row_of(const RotArgs& a, const RotSide& s, uint32_t row)
{
    RotRow r;
    r.live = row < s.rows;
    const uint32_t x = r.live ? row : 0;
    r.token = s.by_heads.div(x);
    r.h = x - r.token * s.heads;
    r.b = a.by_tokens.div(r.token);
    r.t = r.token - r.b * a.tokens;
    return r;
}
__device__ __forceinline__ int64_t offset(const RotHeads& h, const RotRow& r) { return (int64_t)r.b * h.sb + (int64_t)r.t * h.st + (int64_t)r.h * h.sh; }

// A lane's part of a row; zeros where there is none.
template <typename T> struct RotData {
    Vec8<T> a, b;
    __device__ __forceinline__ void load(const T* p, const RotPlace& at, bool has_a, bool has_b)
    {
        const float zero[8] = {};
        if (has_a) a.load(p + at.a);
        else a.set(zero);
        if (has_b) b.load(p + at.b);
        else b.set(zero);
    }
    __device__ __forceinline__ void get(float2* v) const
    {
        a.get(reinterpret_cast<float*>(v));
        b.get(reinterpret_cast<float*>(v + 4));
    }
    __device__ __forceinline__ static void put(T* p, const RotPlace& at, bool has_a, bool has_b, const float2* v)
    {
        Vec8<T> w;
        if (has_a) {
            w.set(reinterpret_cast<const float*>(v));
            w.store(p + at.a);
        }
        if (has_b) {
            w.set(reinterpret_cast<const float*>(v + 4));
            w.store(p + at.b);
        }
    }
};

__device__ __forceinline__ void load_weight(const RotArgs& a, const void* w, const RotPlace& at, float2* out)
{
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) {
        const uint32_t c = i < 8 ? at.a + i : at.b + i - 8;
        float v = 1.0f;
        if (w && c < a.D)
            v = a.weight_dtype == DBLP_F32 ? ((const float*)w)[c]
                                           : (a.weight_dtype == DBLP_BF16 ? to_f32(((const __nv_bfloat16*)w)[c]) : to_f32(((const __half*)w)[c]));
        if (i & 1) out[i / 2].y = v;
        else out[i / 2].x = v;
    }
}

// A block walks over rows of one side, a stride of the side's blocks apart.  The rows of the next step are on their way while this
// step's are worked on; one barrier a step, since the angles of two steps alternate between two tables.  GRAD keeps the block's
// share of the weight's gradient in registers.
template <typename T, bool INTER, bool GRAD> __global__ void __launch_bounds__(kRotThreads, GRAD ? 2 : 3) k_norm_rotate(const __grid_constant__ RotArgs a)
{
    constexpr int U = GRAD ? 1 : kRotRows;
    extern __shared__ __align__(16) float tables[];
    if (GRAD) after_start();
    const bool second = blockIdx.x >= a.side[0].blocks;
    const RotSide& s = a.side[second];
    const uint32_t block = blockIdx.x - (second ? a.side[0].blocks : 0), L = a.L, per = kRotThreads / L, group = threadIdx.x / L;
    const RotPlace at = place_of<INTER>(threadIdx.x & (L - 1), a.R);
    const bool has_a = at.a < a.D, has_b = at.b < a.D;
    RotData<T> x[U], g[U];
    auto bring = [&](uint64_t r0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const RotRow row = row_of(a, s, r0 < s.rows ? (uint32_t)r0 + u * per + group : s.rows);
            x[u].load((const T*)s.x.p + offset(s.x, row), at, row.live && has_a, row.live && has_b);
            if (GRAD) g[u].load((const T*)s.d.p + offset(s.d, row), at, row.live && has_a, row.live && has_b);
        }
    };
    const uint64_t stride = (uint64_t)s.blocks * per * U;
    bring((uint64_t)block * per * U);
    float2 w[8], dw[8] = {};
    load_weight(a, s.weight, at, w);
    uint32_t step = 0;
    for (uint64_t r0 = (uint64_t)block * per * U; r0 < s.rows; r0 += stride, ++step) {
        float* table = tables + (step & 1) * a.table_tokens * a.R;
        const uint32_t first = s.by_heads.div((uint32_t)r0), last = s.by_heads.div(min((uint32_t)r0 + per * U, s.rows) - 1);
        if (a.R) {
            fill_angles(a, table, first, last - first + 1);
            __syncthreads();
        }
        float2 vs[U][8], ds[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u].get(vs[u]);
            if (GRAD) g[u].get(ds[u]);
        }
        bring(r0 + stride);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const RotRow row = row_of(a, s, (uint32_t)r0 + u * per + group);
            const float* angles = table + (row.live ? row.token - first : 0) * a.R;
            float2 *v = vs[u], *d = ds[u], sum = make_float2(0.0f, 0.0f), along = sum;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fma2(v[i], v[i], sum);
            if (GRAD) {
                if (a.R) turn<INTER, true>(d, angles, at, a.R);
#pragma unroll
                for (int i = 0; i < 8; ++i) along = fma2(mul2(w[i], d[i]), v[i], along);
            }
            float ss = sum.x + sum.y, dot = along.x + along.y;
            for (uint32_t m = L / 2; m; m >>= 1) {
                ss += __shfl_xor_sync(0xFFFFFFFFu, ss, m);
                if (GRAD) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, m);
            }
            const float r = rsqrtf(ss * a.inv_d + a.eps);
            const float2 rr = make_float2(r, r);
            if (GRAD) {
                const float q = -dot * a.inv_d * r * r * r;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (row.live) dw[i] = fma2(mul2(d[i], v[i]), rr, dw[i]);
                    v[i] = fma2(v[i], make_float2(q, q), mul2(mul2(w[i], d[i]), rr));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = mul2(v[i], mul2(w[i], rr));
                if (a.R) turn<INTER, false>(v, angles, at, a.R);
            }
            RotData<T>::put((T*)s.y.p + offset(s.y, row), at, row.live && has_a, row.live && has_b, v);
        }
    }
    if (!GRAD || !s.partial) return;
    // the block's sum of its lane groups, in their order: a row of sixteen places a unit
    __syncthreads();
    float* sum = tables;                                                // kRotThreads * 16 floats
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<float2*>(sum + threadIdx.x * 16 + 2 * i) = dw[i];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < L * 16; i += kRotThreads) {
        const RotPlace p = place_of<INTER>(i / 16, a.R);
        const uint32_t c = (i & 8) ? p.b + (i & 7) : p.a + (i & 7);
        if (c >= a.D) continue;
        float t = 0.0f;
        for (uint32_t k = 0; k < per; ++k) t += sum[k * L * 16 + i];
        s.partial[(size_t)block * a.D + c] = t;
    }
}

// The weights' gradients from the blocks' sums: 32 threads a column take every 32nd block, all their loads at once, then add up in
// order.  (8 threads, a load after the other: 11 us of 49 for 296 blocks.)
struct RotJoin {
    const float* partial[2];
    void* dw[2];
    uint32_t blocks[2], D, dtype, accumulate;
};
__global__ void __launch_bounds__(1024) k_rotate_join(RotJoin j)
{
    __shared__ float part[32][32];
    const int side = blockIdx.y;
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float t = 0.0f;
    wait_before();
    after_start();
    if (!j.dw[side]) return;
    if (c < j.D)
#pragma unroll 16
        for (uint32_t b = y; b < j.blocks[side]; b += 32) t += j.partial[side][(size_t)b * j.D + c];
    part[y][x] = t;
    __syncthreads();
    if (y || c >= j.D) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) t += part[i][x];
    if (j.dtype == DBLP_F32) {
        float* p = (float*)j.dw[side] + c;
        *p = j.accumulate ? *p + t : t;
    } else if (j.dtype == DBLP_BF16) {
        __nv_bfloat16* p = (__nv_bfloat16*)j.dw[side] + c;
        *p = from_f32<__nv_bfloat16>(j.accumulate ? to_f32(*p) + t : t);
    } else {
        __half* p = (__half*)j.dw[side] + c;
        *p = from_f32<__half>(j.accumulate ? to_f32(*p) + t : t);
    }
}

static int check_rotate(const char* who, const dblp_norm_rotate_t* a, bool grad)
{
    DBLP_REQUIRE(a, DBLP_EINVAL, "%s: null argument", who);
    DBLP_REQUIRE(known_dtype(a->dtype) && known_dtype(a->weight_dtype), DBLP_EINVAL, "%s: unknown dtype %d or %d", who, a->dtype, a->weight_dtype);
    DBLP_REQUIRE(a->head_dim >= 8 && a->head_dim <= 256 && a->head_dim % 8 == 0, DBLP_EINVAL,
                 "%s: head_dim %u is not a multiple of 8 up to 256", who, a->head_dim);
    const uint32_t known = DBLP_ROTATE_INTERLEAVED | (grad ? DBLP_ACCUMULATE : 0);
    DBLP_REQUIRE((a->flags & ~known) == 0, DBLP_EINVAL, "%s: unknown flags %u", who, a->flags);
    const uint32_t unit = a->flags & DBLP_ROTATE_INTERLEAVED ? 2 : 16;
    DBLP_REQUIRE(a->rotary_dim <= a->head_dim && a->rotary_dim % unit == 0, DBLP_EINVAL, "%s: rotary_dim %u is not a multiple of %u up to head_dim %u",
                 who, a->rotary_dim, unit, a->head_dim);
    DBLP_REQUIRE(a->eps > 0.0f && a->eps < INFINITY, DBLP_EINVAL, "%s: eps %g is not finite and positive", who, a->eps);
    const uint64_t heads = a->q_heads > a->k_heads ? a->q_heads : a->k_heads, tokens = (uint64_t)a->batch * a->tokens;
    DBLP_REQUIRE(tokens < (1ull << 31) && heads < (1ull << 31) && tokens * heads < (1ull << 31), DBLP_ECAPACITY, "%s: 2^31 heads or more", who);
    return DBLP_OK;
}

static int check_positions(const char* who, const dblp_norm_rotate_t* a)
{
    if (a->rotary_dim == 0) return DBLP_OK;
    DBLP_REQUIRE(a->positions && a->freqs, DBLP_EINVAL, "%s: positions or freqs are null", who);
    DBLP_REQUIRE(((uintptr_t)a->positions & 3) == 0 && ((uintptr_t)a->freqs & 7) == 0, DBLP_EALIGN, "%s: positions or freqs are not aligned to their type", who);
    return DBLP_OK;
}

static int check_side(const char* who, const char* name, const dblp_norm_rotate_t* a, const dblp_heads_t* h, uint32_t nheads, bool output)
{
    DBLP_REQUIRE(h && h->data, DBLP_EINVAL, "%s: %s is null", who, name);
    const int64_t unit = 16 / element_bytes(a->dtype);
    const struct { int64_t stride; uint64_t extent; } dim[3] = {{h->batch_stride, a->batch}, {h->token_stride, a->tokens}, {h->head_stride, nheads}};
    bool aligned = aligned16(h->data);
    for (auto& d : dim) {
        if (d.extent <= 1) continue;
        aligned = aligned && d.stride % unit == 0;
        DBLP_REQUIRE(d.stride >= 0 && d.stride < (1ll << 39), DBLP_EINVAL, "%s: %s has a stride of %lld", who, name, (long long)d.stride);
    }
    DBLP_REQUIRE(aligned, DBLP_EALIGN, "%s: %s has data or a stride that is not a multiple of 16 bytes", who, name);
    if (output) {                                   // sorted by stride, each dimension must clear the ones below it
        uint64_t reach = a->head_dim;
        bool used[3] = {false, false, false};
        for (int r = 0; r < 3; ++r) {
            int best = -1;
            for (int i = 0; i < 3; ++i)
                if (!used[i] && dim[i].extent > 1 && (best < 0 || dim[i].stride < dim[best].stride)) best = i;
            if (best < 0) break;
            used[best] = true;
            DBLP_REQUIRE((uint64_t)dim[best].stride >= reach, DBLP_EINVAL, "%s: sections of %s overlap", who, name);
            reach = (uint64_t)dim[best].stride * (dim[best].extent - 1) + reach;
        }
    }
    return DBLP_OK;
}

// Blocks of one side write while blocks of the other still read and write: what begins in one place would mix.
static int check_sides(const char* who, const char* x, const void* a, const char* y, const void* b)
{
    DBLP_REQUIRE(a != b, DBLP_EINVAL, "%s: %s lies over %s", who, x, y);
    return DBLP_OK;
}

static uint32_t lanes_of(uint32_t head_dim)
{
    uint32_t l = 1;
    while (l * 16 < head_dim) l *= 2;
    return l;
}

// Blocks that walk over the rows of one side: as many as the device holds for both sides together, by their share of the rows.
static uint32_t blocks_of(const dblp_norm_rotate_t* a, uint32_t heads, bool grad)
{
    const uint64_t rows = (uint64_t)a->batch * a->tokens * heads, per = kRotThreads / lanes_of(a->head_dim) * (grad ? 1 : kRotRows);
    const uint64_t steps = (rows + per - 1) / per, all = a->q_heads + (uint64_t)a->k_heads;
    uint64_t share = all ? (grad ? 2 : 3) * (uint64_t)kSms * heads / all : 1;
    if (share < 1) share = 1;
    return (uint32_t)(steps < share ? steps : share);
}

static size_t partial_bytes(const dblp_norm_rotate_t* a, uint32_t heads)
{
    return ((size_t)blocks_of(a, heads, true) * a->head_dim * 4 + 255) & ~(size_t)255;
}

static RotHeads rot_heads(const dblp_heads_t* h) { return RotHeads{h->data, h->batch_stride, h->token_stride, h->head_stride}; }

static RotArgs rot_args(const dblp_norm_rotate_t* a)
{
    RotArgs r{};
    r.tokens = a->tokens;
    r.by_tokens = FastDiv(a->tokens ? a->tokens : 1);           // without tokens only the weights' gradients are written
    r.D = a->head_dim;
    r.R = a->rotary_dim;
    r.L = lanes_of(a->head_dim);
    r.weight_dtype = a->weight_dtype;
    r.eps = a->eps;
    r.inv_d = 1.0f / a->head_dim;
    r.positions = a->positions;
    r.position_stride = a->position_stride;
    r.freqs = a->freqs;
    return r;
}

static RotSide rot_side(const dblp_norm_rotate_t* a, const dblp_heads_t* x, const void* weight, const dblp_heads_t* y, uint32_t heads)
{
    RotSide s{};
    s.heads = heads;
    s.by_heads = FastDiv(heads ? heads : 1);
    s.rows = a->batch * a->tokens * heads;
    if (heads) {
        s.x = rot_heads(x);
        s.y = rot_heads(y);
        s.weight = weight;
    }
    return s;
}

// Two tables of angles take up to 64 KB (a single head of a full rotation), 3.5 KB with 25 heads of 64; the gradient's sums, in the same
// place, 16 KB.
template <typename T, bool INTER, bool GRAD> static int launch_rotate(const RotArgs& r, size_t smem, cudaStream_t s)
{
    constexpr auto kernel = k_norm_rotate<T, INTER, GRAD>;
    DBLP_CUDA(allow_shared<kernel>(65536));
    kernel<<<r.side[0].blocks + r.side[1].blocks, kRotThreads, smem, s>>>(r);
    DBLP_LAUNCHED();
    return DBLP_OK;
}

// Tokens that `rows` consecutive rows of a side can touch.
static uint32_t tokens_of(uint32_t rows, uint32_t heads) { return heads ? (heads == 1 ? rows : rows / heads + 2) : 0; }

static int check_weight(const char* who, const char* name, const void* w, int dtype)
{
    DBLP_REQUIRE((uintptr_t)w % element_bytes(dtype) == 0, DBLP_EALIGN, "%s: %s is not aligned to its type", who, name);
    return DBLP_OK;
}

}  // namespace dblp

using namespace dblp;

#define DBLP_TRY(call)                      \
    do {                                    \
        const int rc_ = (call);             \
        if (rc_ != DBLP_OK) return rc_;     \
    } while (0)

extern "C" int dblp_norm_rotate(const dblp_norm_rotate_t* a, const dblp_heads_t* q, const void* q_weight, const dblp_heads_t* q_out,
                                const dblp_heads_t* k, const void* k_weight, const dblp_heads_t* k_out, void* stream)
{
    DBLP_TRY(check_rotate("norm_rotate", a, false));
    if (a->batch == 0 || a->tokens == 0 || a->q_heads + a->k_heads == 0) return DBLP_OK;
    DBLP_TRY(check_positions("norm_rotate", a));
    if (a->q_heads) {
        DBLP_TRY(check_side("norm_rotate", "q", a, q, a->q_heads, false));
        DBLP_TRY(check_side("norm_rotate", "q_out", a, q_out, a->q_heads, true));
        DBLP_TRY(check_weight("norm_rotate", "q_weight", q_weight, a->weight_dtype));
    }
    if (a->k_heads) {
        DBLP_TRY(check_side("norm_rotate", "k", a, k, a->k_heads, false));
        DBLP_TRY(check_side("norm_rotate", "k_out", a, k_out, a->k_heads, true));
        DBLP_TRY(check_weight("norm_rotate", "k_weight", k_weight, a->weight_dtype));
    }
    if (a->q_heads && a->k_heads) {
        DBLP_TRY(check_sides("norm_rotate", "q_out", q_out->data, "k", k->data));
        DBLP_TRY(check_sides("norm_rotate", "k_out", k_out->data, "q", q->data));
        DBLP_TRY(check_sides("norm_rotate", "q_out", q_out->data, "k_out", k_out->data));
    }
    RotArgs r = rot_args(a);
    r.side[0] = rot_side(a, q, q_weight, q_out, a->q_heads);
    r.side[1] = rot_side(a, k, k_weight, k_out, a->k_heads);
    const uint32_t per = kRotThreads / r.L * kRotRows;
    for (RotSide& s : r.side) {
        s.blocks = s.rows ? blocks_of(a, s.heads, false) : 0;
        r.table_tokens = max(r.table_tokens, tokens_of(per, s.heads));
    }
    const size_t smem = (size_t)r.table_tokens * r.R * 2 * sizeof(float);
    return with_type(a->dtype, [&](auto tag) -> int {
        using T = decltype(tag);
        return a->flags & DBLP_ROTATE_INTERLEAVED ? launch_rotate<T, true, false>(r, smem, (cudaStream_t)stream)
                                                  : launch_rotate<T, false, false>(r, smem, (cudaStream_t)stream);
    });
}

extern "C" int dblp_norm_rotate_grad_workspace_bytes(const dblp_norm_rotate_t* a, size_t* bytes)
{
    DBLP_TRY(check_rotate("norm_rotate_grad_workspace_bytes", a, true));
    DBLP_REQUIRE(bytes, DBLP_EINVAL, "norm_rotate_grad_workspace_bytes: null output");
    *bytes = partial_bytes(a, a->q_heads) + partial_bytes(a, a->k_heads);
    return DBLP_OK;
}

extern "C" int dblp_norm_rotate_grad(const dblp_norm_rotate_t* a, const dblp_heads_t* q, const void* q_weight, const dblp_heads_t* dq_out,
                                     const dblp_heads_t* dq, void* dq_weight, const dblp_heads_t* k, const void* k_weight,
                                     const dblp_heads_t* dk_out, const dblp_heads_t* dk, void* dk_weight, void* ws, size_t ws_bytes,
                                     void* stream)
{
    const char* who = "norm_rotate_grad";
    DBLP_TRY(check_rotate(who, a, true));
    if (a->q_heads + a->k_heads == 0) return DBLP_OK;
    const bool empty = a->batch == 0 || a->tokens == 0;
    if (!empty) DBLP_TRY(check_positions(who, a));
    if (!empty && a->q_heads) {
        DBLP_TRY(check_side(who, "q", a, q, a->q_heads, false));
        DBLP_TRY(check_side(who, "dq_out", a, dq_out, a->q_heads, false));
        DBLP_TRY(check_side(who, "dq", a, dq, a->q_heads, true));
        DBLP_TRY(check_weight(who, "q_weight", q_weight, a->weight_dtype));
    }
    if (!empty && a->k_heads) {
        DBLP_TRY(check_side(who, "k", a, k, a->k_heads, false));
        DBLP_TRY(check_side(who, "dk_out", a, dk_out, a->k_heads, false));
        DBLP_TRY(check_side(who, "dk", a, dk, a->k_heads, true));
        DBLP_TRY(check_weight(who, "k_weight", k_weight, a->weight_dtype));
    }
    if (a->q_heads == 0) dq_weight = nullptr;
    if (a->k_heads == 0) dk_weight = nullptr;
    DBLP_TRY(check_weight(who, "dq_weight", dq_weight, a->weight_dtype));
    DBLP_TRY(check_weight(who, "dk_weight", dk_weight, a->weight_dtype));
    const bool join = dq_weight || dk_weight;
    if (empty && !join) return DBLP_OK;
    const size_t q_bytes = partial_bytes(a, a->q_heads), need = join ? q_bytes + partial_bytes(a, a->k_heads) : 0;
    if (need) {
        DBLP_REQUIRE(ws, DBLP_EINVAL, "%s: the workspace is null", who);
        DBLP_REQUIRE(((uintptr_t)ws & 255) == 0, DBLP_EALIGN, "%s: the workspace is not 256-byte aligned", who);
        DBLP_REQUIRE(ws_bytes >= need, DBLP_ECAPACITY, "%s: workspace of %zu bytes, needs %zu", who, ws_bytes, need);
    }
    if (!empty && a->q_heads && a->k_heads) {
        DBLP_TRY(check_sides(who, "dq", dq->data, "k", k->data));
        DBLP_TRY(check_sides(who, "dq", dq->data, "dk_out", dk_out->data));
        DBLP_TRY(check_sides(who, "dk", dk->data, "q", q->data));
        DBLP_TRY(check_sides(who, "dk", dk->data, "dq_out", dq_out->data));
        DBLP_TRY(check_sides(who, "dq", dq->data, "dk", dk->data));
    }
    if (dq_weight && dk_weight) {                               // each is a sum of its own: one place would hold either of them
        const uintptr_t p = (uintptr_t)dq_weight, q0 = (uintptr_t)dk_weight, bytes = (uintptr_t)a->head_dim * element_bytes(a->weight_dtype);
        DBLP_REQUIRE(p + bytes <= q0 || q0 + bytes <= p, DBLP_EINVAL, "%s: dq_weight lies over dk_weight", who);
    }
    float* const partial[2] = {(float*)ws, (float*)((char*)ws + q_bytes)};
    RotArgs r = rot_args(a);
    if (!empty) {
        r.side[0] = rot_side(a, q, q_weight, dq, a->q_heads);
        r.side[1] = rot_side(a, k, k_weight, dk, a->k_heads);
        if (a->q_heads) r.side[0].d = rot_heads(dq_out);
        if (a->k_heads) r.side[1].d = rot_heads(dk_out);
        const uint32_t per = kRotThreads / r.L;
        for (int i = 0; i < 2; ++i) {
            RotSide& s = r.side[i];
            s.blocks = s.rows ? blocks_of(a, s.heads, true) : 0;
            s.partial = (i ? dk_weight : dq_weight) ? partial[i] : nullptr;
            r.table_tokens = max(r.table_tokens, tokens_of(per, s.heads));
        }
        const size_t smem = max((size_t)r.table_tokens * r.R * 2 * sizeof(float), (size_t)kRotThreads * 16 * sizeof(float));
        DBLP_TRY(with_type(a->dtype, [&](auto tag) -> int {
            using T = decltype(tag);
            return a->flags & DBLP_ROTATE_INTERLEAVED ? launch_rotate<T, true, true>(r, smem, (cudaStream_t)stream)
                                                      : launch_rotate<T, false, true>(r, smem, (cudaStream_t)stream);
        }));
    }
    if (!join) return DBLP_OK;
    RotJoin j{{partial[0], partial[1]}, {dq_weight, dk_weight}, {r.side[0].blocks, r.side[1].blocks}, a->head_dim, (uint32_t)a->weight_dtype,
              a->flags & (uint32_t)DBLP_ACCUMULATE};
    DBLP_NEXT(launch_next(k_rotate_join, dim3((a->head_dim + 31) / 32, 2), 1024, 0, (cudaStream_t)stream, j));
    return DBLP_OK;
}
