// The 4-bit K/V cache: append (quantise), read (decode) and eviction. The format is described in cache4.cuh.
// 8266 rows of 2048: append 24 us (86 MB; its instructions fill 80 % of the issue slots), read 17 us (86 MB). Eviction of 8 images of up to 2237
// rows of 1920 to 1216: 10 us to choose, 10 to move; of 32 images of 10521 rows of 2048 to 4096, read back included, 362 us (1.98 GB).
#include "cache4.cuh"

namespace {

using namespace c4;

constexpr int kPer = 2;                // words of a row, keys and values, per thread of append and read: all loads before the first store

// ---- append ------------------------------------------------------------------------------------------------
// Per word of a row, eight channels of keys and values: 16 bytes of each in, a word of codes of each out, the four threads of
// a group agree on its scale by two shuffles. Magnitudes are compared as integers, which orders NaN above everything.
struct AppendParams {
    const uint4 *k, *v;
    int64_t ld;                        // row stride of k and v in 16-byte pieces
    const int32_t* cu;
    int32_t* kv_len;
    uint32_t *k_codes, *v_codes;
    uint16_t *k_scales, *v_scales;
    int B, M, C, Lmax;
    int advance;
    unsigned int *status, *ticket;
};

__device__ __forceinline__ uint32_t quantise8(const uint4& x, uint16_t& scale)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
    top = max(top & 0xffffu, top >> 16);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if (top >= 0x7b80u) {              // 2^120 and above, infinities, NaN
        scale = 0x7fc0u;
        return 0x88888888u;
    }
    const float raw = __fdiv_rn(__uint_as_float(top << 16), 7.f);
    float s = __uint_as_float((__float_as_uint(raw) + 0x7ffffu) & ~0x7ffffu);
    s = top ? fmaxf(s, 7.52316385e-37f) : 0.f;          // 2^-120
    scale = (uint16_t)(__float_as_uint(s) >> 16);
    if (top == 0) return 0x88888888u;
    // x / s without a division: x times the rounded reciprocal is off by at most 2^-20, while x / s is a whole number of halves
    // or at least 2^-10 from one. Rounded to a multiple of 2^-11 (the multiply-add's sum has no finer bits), a half comes out as
    // exactly that, and everything else stays on its side of it; the second sum rounds to a whole number, ties to even, in the low bits.
    const float inv = __frcp_rn(s);
    uint64_t inv2, grid2, back2, whole2;
    asm("mov.b64 %0, {%1, %1};" : "=l"(inv2) : "f"(inv));
    asm("mov.b64 %0, {%1, %1};" : "=l"(grid2) : "f"(6144.f));
    asm("mov.b64 %0, {%1, %1};" : "=l"(back2) : "f"(-6144.f));
    asm("mov.b64 %0, {%1, %1};" : "=l"(whole2) : "f"(12582920.f));          // 1.5 2^23 + 8
    uint32_t even[4], odd[4];          // codes plus 8 in the low byte
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint64_t x;
        asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "r"(w[i] << 16), "r"(w[i] & 0xffff0000u));
        asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(x) : "l"(inv2), "l"(grid2));
        asm("add.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(back2));
        asm("add.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(whole2));
        asm("mov.b64 {%0, %1}, %2;" : "=r"(even[i]), "=r"(odd[i]) : "l"(x));
    }
    // four bytes of codes to four nibbles, in bytes 0 and 2
    auto nibbles = [](const uint32_t (&u)[4]) {
        const uint32_t b = __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
        return b | b >> 4;
    };
    return __byte_perm(nibbles(even), nibbles(odd), 0x6420);
}

__global__ void __launch_bounds__(256)
cache4_append_kernel(const AppendParams p)
{
    pdl_wait();
    pdl_launch_dependents();
    const unsigned vec = p.C >> 3;                       // a multiple of 8: the four threads of a group are in one warp
    const int rows = min(p.M, p.cu[p.B]);
    uint4 k[kPer], v[kPer];
    long dst[kPer];
    unsigned c[kPer];
    int b = 0, c0 = 0, c1 = 0, len = -1;                 // the image of the last row looked up
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const unsigned i = blockIdx.x * (256u * kPer) + j * 256u + threadIdx.x, r = i / vec;
        c[j] = i - r * vec;
        dst[j] = -1;
        k[j] = v[j] = make_uint4(0, 0, 0, 0);
        if (r < (unsigned)rows) {
            k[j] = p.k[r * p.ld + c[j]];
            v[j] = p.v[r * p.ld + c[j]];
            if (j == 0 || (int)r >= c1) {
                b = image_of(p.cu, p.B, (int)r);
                c0 = p.cu[b];
                c1 = p.cu[b + 1];
                len = p.kv_len[b];
            }
            if ((int)r >= c0 && rows_fit(len, min(c1, p.M) - c0, p.Lmax)) dst[j] = (long)b * p.Lmax + len + ((int)r - c0);
            else atomicOr(p.status, NOVA_DEV_SHAPE);
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        uint16_t ks, vs;
        const uint32_t kc = quantise8(k[j], ks), vc = quantise8(v[j], vs);
        if (dst[j] >= 0) {
            p.k_codes[dst[j] * vec + c[j]] = kc;
            p.v_codes[dst[j] * vec + c[j]] = vc;
            if ((c[j] & 3) == 0) {
                const long g = dst[j] * (vec >> 2) + (c[j] >> 2);
                p.k_scales[g] = ks;
                p.v_scales[g] = vs;
                if (ks == 0x7fc0u || vs == 0x7fc0u) atomicOr(p.status, NOVA_DEV_NONFINITE);
            }
        }
    }
    if (p.advance) {
        // The block that draws the last ticket finds every other one past its read of the lengths.
        __shared__ bool last;
        __syncthreads();
        if (threadIdx.x == 0) last = atomicInc(p.ticket, gridDim.x - 1) == gridDim.x - 1;
        __syncthreads();
        if (last)
            for (int b = threadIdx.x; b < p.B; b += 256) {
                const int len = p.kv_len[b], n = min(p.cu[b + 1], p.M) - p.cu[b];
                if (n > 0 && rows_fit(len, n, p.Lmax)) p.kv_len[b] = len + n;
            }
    }
}

// ---- read ---------------------------------------------------------------------------------------------------
// Per word of a row, keys and values: 4 bytes of codes in, 16 bytes out. Bound by the bytes written.
struct ReadParams {
    const uint32_t *k_codes, *v_codes;
    const uint16_t *k_scales, *v_scales;
    const int32_t *cu, *first;
    uint4 *k, *v;
    int64_t ld;                        // row stride of k and v in 16-byte pieces
    int B, M, C, Lmax;
    unsigned int* status;
};

__global__ void __launch_bounds__(256)
cache4_read_kernel(const ReadParams p)
{
    pdl_wait();
    pdl_launch_dependents();
    const unsigned vec = p.C >> 3;
    const int rows = min(p.M, p.cu[p.B]);
    uint32_t kw[kPer], vw[kPer];
    uint16_t ks[kPer], vs[kPer];
    long to[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const unsigned i = blockIdx.x * (256u * kPer) + j * 256u + threadIdx.x, r = i / vec, c = i - r * vec;
        to[j] = -1;
        if (r < (unsigned)rows) {
            const int b = image_of(p.cu, p.B, (int)r);
            const long row = (long)(p.first ? p.first[b] : 0) + ((int)r - p.cu[b]);
            if (row >= 0 && row < p.Lmax) {
                const long src = (long)b * p.Lmax + row, g = src * (vec >> 2) + (c >> 2);
                to[j] = r * p.ld + c;
                kw[j] = p.k_codes[src * vec + c];
                vw[j] = p.v_codes[src * vec + c];
                ks[j] = p.k_scales[g];
                vs[j] = p.v_scales[g];
            } else {
                atomicOr(p.status, NOVA_DEV_SHAPE);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (to[j] >= 0) {
            uint32_t x[4];
            decode8(kw[j], Scale2(both(ks[j])), x);
            __stcs(p.k + to[j], make_uint4(x[0], x[1], x[2], x[3]));
            decode8(vw[j], Scale2(both(vs[j])), x);
            __stcs(p.v + to[j], make_uint4(x[0], x[1], x[2], x[3]));
        }
}

// ---- eviction: which rows stay ---------------------------------------------------------------------------------
// One CTA per image with the rows' weights in registers as order-preserving integers (of more than 32768 rows they are read
// anew in every pass). The weight T of the last row that stays, and
// how many rows equal to it do, come from a most-significant-digit radix select on 11-bit digits. Then an ordered pass by warp
// ballots writes the numbers of the rows that stay in ascending order.
// Many equal weights (rows that received nothing) would serialise the histogram's shared-memory atomics: the lanes of a warp with
// the same digit as the first of them count once.
constexpr int kEvThreads = 1024;
constexpr int kEvBins = 2048;
constexpr uint32_t kWholeBin = 0xffffffffu;

struct EvictParams {
    const float* weight;               // [B, Lmax]
    const int32_t* kv_len;
    int32_t* src_row;                  // [B, budget]
    int32_t* dst_len;
    int Lmax, budget, recent;
};

__device__ __forceinline__ uint32_t order_key(float f)
{
    uint32_t u = __float_as_uint(f);
    if (u == 0x80000000u) u = 0;                       // -0 and +0 are the same weight
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// KEYS: weights per thread, 0: as many as it takes
template <int KEYS>
__global__ void __launch_bounds__(kEvThreads)
cache4_evict_select(const EvictParams p)
{
    const int keys = KEYS ? KEYS : (p.Lmax + kEvThreads - 1) / kEvThreads;
    __shared__ uint32_t hist[kEvBins], warp_a[32], warp_b[32];
    __shared__ uint32_t sh_digit, sh_need, sh_count;
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x;
    const int len = min(max(p.kv_len[b], 0), p.Lmax);
    const int old = max(len - p.recent, 0);            // rows that may go
    const int kept = min(len, p.budget);
    const int take = len <= p.budget ? old : kept - (len - old);   // of which this many stay
    const int i0 = warp * 32 * keys + lane;            // lane-interleaved
    const float* w = p.weight + (long)b * p.Lmax;
    uint32_t held[KEYS ? KEYS : 1] = {};
    auto load = [&](int j) { return i0 + j * 32 < old ? order_key(w[i0 + j * 32]) : 0u; };
    auto key = [&](int j) { return KEYS ? held[KEYS ? j : 0] : load(j); };
#pragma unroll
    for (int j = 0; j < KEYS; ++j) held[j] = load(j);

    uint32_t T = 0, need = (uint32_t)max(take, 0);
    const bool every = take >= old, digits = take > 0 && !every;
    if (digits) {
        int bits = 32;
        while (bits > 0) {
            const int shift = max(bits - 11, 0);
            const uint32_t mask = (1u << (bits - shift)) - 1u;
            for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < keys; ++j) {
                const uint32_t k = key(j), d = (k >> shift) & mask;
                const bool in = i0 + j * 32 < old && (bits >= 32 || ((k ^ T) >> bits) == 0);
                const uint32_t who = __ballot_sync(0xffffffffu, in);
                if (who == 0) continue;
                const int head = __ffs((int)who) - 1;
                const uint32_t d0 = __shfl_sync(0xffffffffu, d, head);
                const uint32_t same = __ballot_sync(0xffffffffu, in && d == d0);
                if (lane == head) atomicAdd(&hist[d0], (uint32_t)__popc(same));
                else if (in && d != d0) atomicAdd(&hist[d], 1u);
            }
            __syncthreads();
            // thread t owns the bins 2047 - 2t and 2046 - 2t
            const uint32_t c0 = hist[kEvBins - 1 - 2 * tid], c1 = hist[kEvBins - 2 - 2 * tid], tot = c0 + c1;
            uint32_t incl = tot;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            if (lane == 31) warp_a[warp] = incl;
            __syncthreads();
            const uint32_t above = __reduce_add_sync(0xffffffffu, lane < warp ? warp_a[lane] : 0u) + incl - tot;
            if (above < need && need <= above + tot) {
                const bool first = need <= above + c0;
                sh_digit = (uint32_t)(first ? kEvBins - 1 - 2 * tid : kEvBins - 2 - 2 * tid);
                sh_need = need - above - (first ? 0u : c0);
                sh_count = first ? c0 : c1;
            }
            __syncthreads();
            T |= sh_digit << shift;
            need = sh_need;
            bits = shift;
            if (sh_count == need) {                     // the whole bin stays: T is its lowest possible key
                need = kWholeBin;
                break;
            }
        }
    }

    // ---- ordered emit: rows above T, the first `need` of those equal to it, the recent ones
    auto is_top = [&](int j) {
        const int i = i0 + j * 32;
        return i < len && (i >= old || every || (digits && (key(j) > T || (need == kWholeBin && key(j) == T))));
    };
    auto is_eq = [&](int j) { return i0 + j * 32 < old && digits && need != kWholeBin && key(j) == T; };
    uint32_t n_top = 0, n_eq = 0;
#pragma unroll
    for (int j = 0; j < keys; ++j) {
        n_top += __popc(__ballot_sync(0xffffffffu, is_top(j)));
        n_eq += __popc(__ballot_sync(0xffffffffu, is_eq(j)));
    }
    __syncthreads();
    if (lane == 0) { warp_a[warp] = n_top; warp_b[warp] = n_eq; }
    __syncthreads();
    uint32_t top_before = __reduce_add_sync(0xffffffffu, lane < warp ? warp_a[lane] : 0u);
    uint32_t eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? warp_b[lane] : 0u);
    int32_t* out = p.src_row + (long)b * p.budget;
    const uint32_t lt = (1u << lane) - 1u;
#pragma unroll
    for (int j = 0; j < keys; ++j) {
        const bool top = is_top(j), eq = is_eq(j);
        const uint32_t bt = __ballot_sync(0xffffffffu, top), be = __ballot_sync(0xffffffffu, eq);
        const uint32_t e = eq_before + __popc(be & lt);
        const uint32_t at = top_before + __popc(bt & lt) + min(e, need);      // equal rows before this one that stay
        if ((top || (eq && e < need)) && at < (uint32_t)kept) out[at] = i0 + j * 32;
        top_before += __popc(bt);
        eq_before += __popc(be);
    }
    for (int i = kept + tid; i < p.budget; i += kEvThreads) out[i] = -1;
    if (tid == 0) p.dst_len[b] = kept;
}

// ---- eviction: the rows move --------------------------------------------------------------------------------------
// One warp for two rows of the new cache: codes in 16-byte pieces, scales in 4-byte pieces, the weight. Bound by the bytes.
constexpr int kMoveRows = 2;
struct MoveParams {
    const uint4 *k_codes, *v_codes;
    const uint32_t *k_scales, *v_scales;
    uint4 *k_codes_out, *v_codes_out;
    uint32_t *k_scales_out, *v_scales_out;
    const float* weight;
    float* weight_out;                 // [B, Lmax_out] or NULL
    const int32_t* src_row;
    int Lmax, Lmax_out, budget, C;
    long rows;                         // B * (weight_out ? Lmax_out : budget)
};

__global__ void __launch_bounds__(256)
cache4_move_kernel(const MoveParams p)
{
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, per = p.weight_out ? p.Lmax_out : p.budget;
    const long r0 = ((long)blockIdx.x * 8 + (threadIdx.x >> 5)) * kMoveRows;
    const int pieces = p.C >> 5, words = p.C >> 6;
    long src[kMoveRows], dst[kMoveRows];
#pragma unroll
    for (int j = 0; j < kMoveRows; ++j) {
        src[j] = -1;
        const long r = r0 + j;
        if (r >= p.rows) continue;
        const int b = (int)(r / per), i = (int)(r - (long)b * per);
        const int s = i < p.budget ? p.src_row[(long)b * p.budget + i] : -1;
        dst[j] = (long)b * p.Lmax_out + i;
        if ((unsigned)s < (unsigned)p.Lmax) src[j] = (long)b * p.Lmax + s;
        if (lane == 0 && p.weight_out) p.weight_out[dst[j]] = src[j] >= 0 ? p.weight[src[j]] : 0.f;
    }
    for (int c = lane; c < pieces; c += 32) {
        uint4 k[kMoveRows], v[kMoveRows];
#pragma unroll
        for (int j = 0; j < kMoveRows; ++j)
            if (src[j] >= 0) { k[j] = p.k_codes[src[j] * pieces + c]; v[j] = p.v_codes[src[j] * pieces + c]; }
#pragma unroll
        for (int j = 0; j < kMoveRows; ++j)
            if (src[j] >= 0) { p.k_codes_out[dst[j] * pieces + c] = k[j]; p.v_codes_out[dst[j] * pieces + c] = v[j]; }
    }
    for (int c = lane; c < words; c += 32) {
        uint32_t k[kMoveRows], v[kMoveRows];
#pragma unroll
        for (int j = 0; j < kMoveRows; ++j)
            if (src[j] >= 0) { k[j] = p.k_scales[src[j] * words + c]; v[j] = p.v_scales[src[j] * words + c]; }
#pragma unroll
        for (int j = 0; j < kMoveRows; ++j)
            if (src[j] >= 0) { p.k_scales_out[dst[j] * words + c] = k[j]; p.v_scales_out[dst[j] * words + c] = v[j]; }
    }
}

bool aligned4(const void* p) { return (((uintptr_t)p) & 3u) == 0; }

}  // namespace

nova_status nova_cache4_check(nova_ctx* ctx, const char* who, const nova_cache4* c)
{
    auto fail = [&](nova_status s, const char* what) {
        snprintf(ctx->err, sizeof(ctx->err), "%s: %s", who, what);
        return s;
    };
    if (!c) return fail(NOVA_ERR_INVALID_ARG, "null cache");
    if (c->B < 0 || c->Lmax < 0) return fail(NOVA_ERR_INVALID_ARG, "negative size");
    if (c->C < 64 || c->C % 64 || c->C > (1 << 20) || c->n_heads < 1 || c->C % c->n_heads) return fail(NOVA_ERR_SHAPE, "C must be a multiple of 64 and of the heads");
    const int dh = c->C / c->n_heads;
    if (dh != 64 && dh != 128) return fail(NOVA_ERR_SHAPE, "head dimension must be 64 or 128");
    if (c->B > 0 && c->Lmax > 0) {
        if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return fail(NOVA_ERR_INVALID_ARG, "null cache tensor");
        if (!nova_aligned16(c->k_codes) || !nova_aligned16(c->v_codes) || !nova_aligned16(c->k_scales) || !nova_aligned16(c->v_scales))
            return fail(NOVA_ERR_ALIGNMENT, "cache tensors must be 16-byte aligned");
    }
    if (c->B > 0 && (!c->kv_len || !aligned4(c->kv_len))) return fail(NOVA_ERR_INVALID_ARG, "null or misaligned kv_len");
    return NOVA_OK;
}

nova_status nova_cache4_check_rows(nova_ctx* ctx, const char* who, const nova_cache4* c, const void* a, const void* b,
                                   const int32_t* cu_rows, int M, int64_t ld)
{
    auto fail = [&](nova_status s, const char* what) {
        snprintf(ctx->err, sizeof(ctx->err), "%s: %s", who, what);
        return s;
    };
    if (M < 0) return fail(NOVA_ERR_INVALID_ARG, "negative row count");
    if (M == 0 || c->B == 0) return NOVA_OK;
    if (!a || !b || !cu_rows) return fail(NOVA_ERR_INVALID_ARG, "null tensor");
    if (ld < c->C) return fail(NOVA_ERR_INVALID_ARG, "row stride smaller than C");
    if (!nova_aligned16(a) || !nova_aligned16(b) || ld % 8) return fail(NOVA_ERR_ALIGNMENT, "rows must be 16-byte aligned");
    return NOVA_OK;
}

nova_status nova_launch_cache4_append(nova_ctx* ctx, const nova_cache4* c, const void* k, const void* v, int64_t ld, const int32_t* cu,
                                      int M, int advance, cudaStream_t st)
{
    if (M == 0 || c->B == 0) return NOVA_OK;
    const long blocks = ((long)M * (c->C / 8) + 256 * kPer - 1) / (256 * kPer);
    if (blocks * 256 * kPer > 0xffffffffL) return nova_fail(ctx, NOVA_ERR_SHAPE, "nova_cache4_append: too many rows");
    AppendParams p;
    p.k = (const uint4*)k; p.v = (const uint4*)v; p.ld = ld / 8; p.cu = cu; p.kv_len = c->kv_len;
    p.k_codes = (uint32_t*)c->k_codes; p.v_codes = (uint32_t*)c->v_codes;
    p.k_scales = (uint16_t*)c->k_scales; p.v_scales = (uint16_t*)c->v_scales;
    p.B = c->B; p.M = M; p.C = c->C; p.Lmax = c->Lmax; p.advance = advance != 0;
    p.status = ctx->dev_status; p.ticket = ctx->dev_status + NOVA_APPEND_TICKET_WORD;
    nova_launch_scope scope(ctx, NOVA_K_CACHE4, st);
    NOVA_CUDA_CHECK(ctx, nova_launch_pdl(cache4_append_kernel, dim3((unsigned)blocks), dim3(256), 0, st, 0, p));
    return NOVA_OK;
}

extern "C" {

nova_status nova_cache4_append(nova_ctx* ctx, const nova_cache4* c, const void* k, const void* v, int64_t ld,
                               const int32_t* cu_rows, int M, int advance, void* stream)
{
    if (!ctx) return NOVA_ERR_INVALID_ARG;
    nova_status rc = nova_cache4_check(ctx, "nova_cache4_append", c);
    if (rc == NOVA_OK) rc = nova_cache4_check_rows(ctx, "nova_cache4_append", c, k, v, cu_rows, M, ld);
    if (rc != NOVA_OK) return rc;
    if (M == 0 || c->B == 0) return NOVA_OK;
    NOVA_DEVICE_GUARD(ctx, "nova_cache4_append");
    cudaStream_t st = (cudaStream_t)stream;
    rc = nova_debug_check_lists(ctx, "nova_cache4_append", nullptr, nullptr, cu_rows, c->B, M, M, false, st);
    if (rc != NOVA_OK) return rc;
    return nova_launch_cache4_append(ctx, c, k, v, ld, cu_rows, M, advance, st);
}

nova_status nova_cache4_read(nova_ctx* ctx, const nova_cache4* c, const int32_t* first, const int32_t* cu_rows, int M,
                             void* k_out, void* v_out, int64_t ld, void* stream)
{
    if (!ctx) return NOVA_ERR_INVALID_ARG;
    nova_status rc = nova_cache4_check(ctx, "nova_cache4_read", c);
    if (rc == NOVA_OK) rc = nova_cache4_check_rows(ctx, "nova_cache4_read", c, k_out, v_out, cu_rows, M, ld);
    if (rc != NOVA_OK) return rc;
    if (M == 0 || c->B == 0) return NOVA_OK;
    const long blocks = ((long)M * (c->C / 8) + 256 * kPer - 1) / (256 * kPer);
    if (blocks * 256 * kPer > 0xffffffffL) return nova_fail(ctx, NOVA_ERR_SHAPE, "nova_cache4_read: too many rows");
    NOVA_DEVICE_GUARD(ctx, "nova_cache4_read");
    cudaStream_t st = (cudaStream_t)stream;
    rc = nova_debug_check_lists(ctx, "nova_cache4_read", nullptr, nullptr, cu_rows, c->B, M, M, false, st);
    if (rc != NOVA_OK) return rc;
    ReadParams p;
    p.k_codes = (const uint32_t*)c->k_codes; p.v_codes = (const uint32_t*)c->v_codes;
    p.k_scales = (const uint16_t*)c->k_scales; p.v_scales = (const uint16_t*)c->v_scales;
    p.cu = cu_rows; p.first = first; p.k = (uint4*)k_out; p.v = (uint4*)v_out; p.ld = ld / 8;
    p.B = c->B; p.M = M; p.C = c->C; p.Lmax = c->Lmax; p.status = ctx->dev_status;
    {
        nova_launch_scope scope(ctx, NOVA_K_CACHE4, st);
        NOVA_CUDA_CHECK(ctx, nova_launch_pdl(cache4_read_kernel, dim3((unsigned)blocks), dim3(256), 0, st, 0, p));
    }
    return NOVA_OK;
}

nova_status nova_cache4_evict(nova_ctx* ctx, const nova_cache4* c, const float* weight, int budget, int recent,
                              const nova_cache4* dst, float* weight_out, int32_t* src_row, void* stream)
{
    if (!ctx) return NOVA_ERR_INVALID_ARG;
    nova_status rc = nova_cache4_check(ctx, "nova_cache4_evict", c);
    if (rc == NOVA_OK) rc = nova_cache4_check(ctx, "nova_cache4_evict", dst);
    if (rc != NOVA_OK) return rc;
    if (dst->B != c->B || dst->C != c->C || dst->n_heads != c->n_heads)
        return nova_fail(ctx, NOVA_ERR_INVALID_ARG, "nova_cache4_evict: the two caches differ in images, width or heads");
    if (budget < 0 || recent < 0 || recent > budget) return nova_fail(ctx, NOVA_ERR_INVALID_ARG, "nova_cache4_evict: need 0 <= recent <= budget");
    if (budget > dst->Lmax) return nova_fail(ctx, NOVA_ERR_SHAPE, "nova_cache4_evict: budget larger than the new cache");
    if (c->Lmax > (1 << 30)) return nova_fail(ctx, NOVA_ERR_SHAPE, "nova_cache4_evict: too many rows");
    if (c->B == 0) return NOVA_OK;
    // what is written must not overlap anything that is read, or what else is written
    const size_t rows_in = (size_t)c->B * c->Lmax, rows_out = (size_t)c->B * dst->Lmax;
    struct { const void* p; size_t bytes; bool written; } mem[] = {
        {c->k_codes, rows_in * (c->C / 2), false}, {c->v_codes, rows_in * (c->C / 2), false}, {c->k_scales, rows_in * (c->C / 16), false},
        {c->v_scales, rows_in * (c->C / 16), false}, {c->kv_len, (size_t)c->B * 4, false}, {weight, rows_in * 4, false},
        {dst->k_codes, rows_out * (c->C / 2), true}, {dst->v_codes, rows_out * (c->C / 2), true}, {dst->k_scales, rows_out * (c->C / 16), true},
        {dst->v_scales, rows_out * (c->C / 16), true}, {dst->kv_len, (size_t)c->B * 4, true}, {weight_out, rows_out * 4, true},
        {src_row, (size_t)c->B * budget * 4, true}};
    const int n_mem = (int)(sizeof(mem) / sizeof(mem[0]));
    for (int i = 0; i < n_mem; ++i)
        for (int j = 0; j < i; ++j)
            if (mem[i].written && mem[i].p && mem[j].p && mem[i].bytes && mem[j].bytes &&
                (uintptr_t)mem[i].p < (uintptr_t)mem[j].p + mem[j].bytes && (uintptr_t)mem[j].p < (uintptr_t)mem[i].p + mem[i].bytes)
                return nova_fail(ctx, NOVA_ERR_INVALID_ARG, "nova_cache4_evict: the new cache, its weights or the list overlap other memory of the call");
    if (c->Lmax > 0 && !weight) return nova_fail(ctx, NOVA_ERR_INVALID_ARG, "nova_cache4_evict: null weights");
    if (!aligned4(weight) || !aligned4(weight_out) || !aligned4(src_row))
        return nova_fail(ctx, NOVA_ERR_ALIGNMENT, "nova_cache4_evict: misaligned tensor");
    int32_t* list = src_row;
    if (!list) budget = budget < c->Lmax ? budget : c->Lmax;      // (the same rows: nobody has more than Lmax; the list is ours)
    if (!list && budget > 0) {
        if (!ctx->workspace || ctx->workspace_bytes < (size_t)c->B * budget * sizeof(int32_t))
            return nova_fail(ctx, NOVA_ERR_WORKSPACE, "nova_cache4_evict: workspace missing or too small for the list of rows");
        list = (int32_t*)ctx->workspace;
    }
    MoveParams m;
    m.k_codes = (const uint4*)c->k_codes; m.v_codes = (const uint4*)c->v_codes;
    m.k_scales = (const uint32_t*)c->k_scales; m.v_scales = (const uint32_t*)c->v_scales;
    m.k_codes_out = (uint4*)dst->k_codes; m.v_codes_out = (uint4*)dst->v_codes;
    m.k_scales_out = (uint32_t*)dst->k_scales; m.v_scales_out = (uint32_t*)dst->v_scales;
    m.weight = weight; m.weight_out = weight_out; m.src_row = list;
    m.Lmax = c->Lmax; m.Lmax_out = dst->Lmax; m.budget = budget; m.C = c->C;
    m.rows = (long)c->B * (weight_out ? dst->Lmax : budget);
    const long blocks = (m.rows + 8 * kMoveRows - 1) / (8 * kMoveRows);
    const int keys = (int)((c->Lmax + kEvThreads - 1) / kEvThreads);
    if (blocks > 0x7fffffffL) return nova_fail(ctx, NOVA_ERR_SHAPE, "nova_cache4_evict: too many rows");
    NOVA_DEVICE_GUARD(ctx, "nova_cache4_evict");
    cudaStream_t st = (cudaStream_t)stream;
    EvictParams p = {weight, c->kv_len, list, dst->kv_len, c->Lmax, budget, recent};
    {
        nova_launch_scope scope(ctx, NOVA_K_CACHE4, st);
        const dim3 grid((unsigned)c->B), block(kEvThreads);
        cudaError_t e;
        if (keys <= 1) e = nova_launch_pdl(cache4_evict_select<1>, grid, block, 0, st, 0, p);
        else if (keys <= 2) e = nova_launch_pdl(cache4_evict_select<2>, grid, block, 0, st, 0, p);
        else if (keys <= 4) e = nova_launch_pdl(cache4_evict_select<4>, grid, block, 0, st, 0, p);
        else if (keys <= 8) e = nova_launch_pdl(cache4_evict_select<8>, grid, block, 0, st, 0, p);
        else if (keys <= 16) e = nova_launch_pdl(cache4_evict_select<16>, grid, block, 0, st, 0, p);
        else if (keys <= 32) e = nova_launch_pdl(cache4_evict_select<32>, grid, block, 0, st, 0, p);
        else e = nova_launch_pdl(cache4_evict_select<0>, grid, block, 0, st, 0, p);
        NOVA_CUDA_CHECK(ctx, e);
    }
    if (blocks > 0) {
        nova_launch_scope scope(ctx, NOVA_K_CACHE4, st);
        NOVA_CUDA_CHECK(ctx, nova_launch_pdl(cache4_move_kernel, dim3((unsigned)blocks), dim3(256), 0, st, 0, m));
    }
    return NOVA_OK;
}

}  // extern "C"
