// The attention weight that each row of the 4-bit K/V cache receives from a call's queries, added to what it had:
//   out[b, j] = in[b, j] + sum over heads and queries of exp(s - lse),  s = q k_j / sqrt(dh),
// lse being the row's log-sum-exp as the attention left it.
//
// A warp has 32 keys of one head as the A operand of mma.sync, decoded once into registers, and takes the image's queries, 64 at a
// time from shared memory, as the B operand: a thread's results then belong to two keys per tile, and the sum over
// queries and heads stays in its registers until the end. A CTA's eight warps share the queries. What bounds it: with many
// queries the tensor work (mma.sync) and the exponentials, one per key, query and head; with few the bytes of the keys, for
// which the next head's words are loaded before the present one is worked on.
// Where there are few key tiles, the (head, query chunk) pairs of a tile are divided over several CTAs, whose sums the last of
// them adds in the order of the parts: nothing depends on who comes first.
// 768 and 1024 rows x 7449 and 5587 keys, 16 heads of 128: 171 us (274 TFLOP/s; mma.sync alone would take about 107 at the rate that the
// pipe shows, the exponentials 41); 256 with two chains of products instead of four, 32 queries a chunk and two CTAs per SM in all.
#include "cache4.cuh"

namespace {

using namespace c4;

constexpr int kWtWarps = 8, kWtThreads = kWtWarps * 32;
constexpr int kWtKeys = 32;                       // per warp
constexpr int kWtTile = kWtWarps * kWtKeys;
constexpr int kWtChunk = 64;                      // queries in shared memory at a time
constexpr int kWtDepth = 2;                       // chunks in flight
constexpr int kWtWaves = 8;                       // CTAs per SM that the parts aim at

struct WeightParams {
    const uint8_t *codes, *scales;
    const __nv_bfloat16* q;
    int64_t ldq;
    const float* lse;                  // [n_heads, M]
    const int32_t *cu, *kv_len;
    const float* in;
    float* out;                        // [B, Lmax]
    int C, Lmax, n_heads, M, tiles, parts;
    int own_rows;
    float scale_log2e;
    float* part;                       // [B * tiles][parts][kWtTile]
    unsigned int* tickets;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int DH>
__global__ void __launch_bounds__(kWtThreads, 2)
cache4_weights_kernel(const WeightParams p)
{
    constexpr int kSteps = DH / 16, kWords = DH / 32;            // words of a key that a thread decodes
    constexpr int kRowChunks = DH / 8;                           // 16-byte pieces of a query
    __shared__ __align__(16) uint8_t q_s[kWtDepth][kWtChunk * DH * 2];
    __shared__ float lse_s[kWtDepth][kWtChunk];                  // -lse in units of log2; -inf: the row does not count
    __shared__ int last_s;
    pdl_wait();
    pdl_launch_dependents();
    const int part = blockIdx.x % p.parts, bt = blockIdx.x / p.parts, tile = bt % p.tiles, b = bt / p.tiles;
    const int c0 = p.cu[b], rows = min(max(p.cu[b + 1] - c0, 0), max(p.M - c0, 0));
    const int kv_len = p.kv_len[b], len = keys_of(kv_len, rows, p.own_rows, p.Lmax);
    if (tile * kWtTile >= len) return;
    if (p.own_rows && !rows_fit(kv_len, rows, p.Lmax)) return;      // the image's call is refused: its weights stay, for the call that repeats it
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int chunks = (rows + kWtChunk - 1) / kWtChunk, jobs = p.n_heads * chunks;
    const int j0 = (int)((long)jobs * part / p.parts), j1 = (int)((long)jobs * (part + 1) / p.parts);
    const int key0 = tile * kWtTile + warp * kWtKeys;

    // Queries of job j to slot: pieces exchanged so that the reads of eight threads touch every bank once.
    auto piece_at = [](int row, int c) { return DH == 128 ? c ^ ((c >> 3) & 1) ^ ((row & 1) << 1) : c ^ (row & 1); };
    auto load_q = [&](int j) {
        if (j < j1) {
            const int slot = (j - j0) % kWtDepth, head = j / chunks, q0 = (j - head * chunks) * kWtChunk;
#pragma unroll
            for (int i = threadIdx.x; i < kWtChunk * kRowChunks; i += kWtThreads) {
                const int r = i / kRowChunks, c = i % kRowChunks;
                const bool live = q0 + r < rows;
                const __nv_bfloat16* src = p.q + (long)(c0 + (live ? q0 + r : 0)) * p.ldq + head * DH + c * 8;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                             ::"r"(tc::smem_u32(&q_s[slot][(r * kRowChunks + piece_at(r, c)) * 16])), "l"(src), "r"(live ? 16 : 0) : "memory");
            }
            if (threadIdx.x < kWtChunk) {
                const int r = threadIdx.x;
                float x = q0 + r < rows ? p.lse[(long)head * p.M + c0 + q0 + r] : -INFINITY;
                lse_s[slot][r] = x == -INFINITY ? -INFINITY : -x * 1.4426950408889634f;       // (a row that attended to nothing)
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // The words of keys g, g + 8, g + 16, g + 24 of a head, and their scales.
    uint32_t raw[4][kWords];
    uint16_t raw_s[4];
    auto load_k = [&](int head) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = min(key0 + 8 * i + g, len - 1);
            const long row = (long)b * p.Lmax + key;
            const uint8_t* src = p.codes + row * (p.C / 2) + head * (DH / 2) + t * (DH / 8);
            if constexpr (DH == 128) {
                const uint4 v = *(const uint4*)src;
                raw[i][0] = v.x; raw[i][1] = v.y; raw[i][2] = v.z; raw[i][3] = v.w;
            } else {
                const uint2 v = *(const uint2*)src;
                raw[i][0] = v.x; raw[i][1] = v.y;
            }
            raw_s[i] = *(const uint16_t*)(p.scales + row * (p.C / 16) + head * (DH / 16) + (DH == 128 ? t : t >> 1) * 2);
        }
    };
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    if (j0 < j1) {
        load_k(j0 / chunks);
        for (int i = 0; i < kWtDepth - 1; ++i) load_q(j0 + i);
        int head = -1;
        uint32_t a[2][kSteps][4];
        for (int j = j0; j < j1; ++j) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kWtDepth - 2) : "memory");
            __syncthreads();                         // job j is there for all, and all are done with job j - 1
            load_q(j + kWtDepth - 1);
            if (j / chunks != head) {
                head = j / chunks;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Scale2 sc(both(raw_s[i]));
#pragma unroll
                    for (int w = 0; w < kWords; ++w) {
                        uint32_t x[4];
                        decode8(raw[i][w], sc, x);
                        a[i >> 1][2 * w][i & 1] = x[0];
                        a[i >> 1][2 * w][2 + (i & 1)] = x[1];
                        a[i >> 1][2 * w + 1][i & 1] = x[2];
                        a[i >> 1][2 * w + 1][2 + (i & 1)] = x[3];
                    }
                }
                if (head * chunks + chunks < j1) load_k(head + 1);
            }
            const int slot = (j - j0) % kWtDepth;
#pragma unroll 1
            for (int nb = 0; nb < kWtChunk / 8; nb += 2) {       // 16 queries: four independent chains of products
                float s[2][2][4];
#pragma unroll
                for (int k = 0; k < 8; ++k) s[k >> 2][(k >> 1) & 1][2 * (k & 1)] = s[k >> 2][(k >> 1) & 1][2 * (k & 1) + 1] = 0.f;
                const int row = nb * 8 + g;
#pragma unroll
                for (int i = 0; i < kSteps / 2; ++i) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 v = *(const uint4*)&q_s[slot][((row + 8 * h) * kRowChunks + piece_at(row, t * (DH / 32) + i)) * 16];
#pragma unroll
                        for (int mi = 0; mi < 2; ++mi) mma16816(s[h][mi], a[mi][2 * i], v.x, v.y);
#pragma unroll
                        for (int mi = 0; mi < 2; ++mi) mma16816(s[h][mi], a[mi][2 * i + 1], v.z, v.w);
                    }
                }
                float2 nls[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) nls[h] = *(const float2*)&lse_s[slot][(nb + h) * 8 + 2 * t];
                // A query that does not count: 2^(s - inf) is zero only of a finite score s. (To look for them takes 3 %, 166 -> 171 us in the case above.)
                if (__any_sync(0xffffffffu, fminf(fminf(nls[0].x, nls[0].y), fminf(nls[1].x, nls[1].y)) == -INFINITY)) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (nls[k >> 1].x == -INFINITY) s[k >> 1][k & 1][0] = s[k >> 1][k & 1][2] = 0.f;
                        if (nls[k >> 1].y == -INFINITY) s[k >> 1][k & 1][1] = s[k >> 1][k & 1][3] = 0.f;
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float2 nl = nls[h];
#pragma unroll
                    for (int mi = 0; mi < 2; ++mi) {
                        acc[2 * mi] += ex2(fmaf(s[h][mi][0], p.scale_log2e, nl.x)) + ex2(fmaf(s[h][mi][1], p.scale_log2e, nl.y));
                        acc[2 * mi + 1] += ex2(fmaf(s[h][mi][2], p.scale_log2e, nl.x)) + ex2(fmaf(s[h][mi][3], p.scale_log2e, nl.y));
                    }
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 1);
        acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 2);
    }
    if (p.parts == 1) {
        if (t == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = key0 + 8 * i + g;
                const long at = (long)b * p.Lmax + key;
                if (key < len) p.out[at] = (p.in ? p.in[at] : 0.f) + acc[i];
            }
        return;
    }
    float* mine = p.part + ((long)bt * p.parts + part) * kWtTile;
    if (t == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[warp * kWtKeys + 8 * i + g] = acc[i];
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last_s = atomicInc(&p.tickets[bt], (unsigned)p.parts - 1) == (unsigned)p.parts - 1;
    __syncthreads();
    if (!last_s) return;
    __threadfence();
    const int key = tile * kWtTile + threadIdx.x;
    if (key < len) {
        const long at = (long)b * p.Lmax + key;
        float sum = 0.f;
        for (int i = 0; i < p.parts; ++i) sum += __ldcg(p.part + ((long)bt * p.parts + i) * kWtTile + threadIdx.x);
        p.out[at] = (p.in ? p.in[at] : 0.f) + sum;
    }
}

}  // namespace

size_t nova_cache4_weights_scratch(int num_sms) { return (size_t)num_sms * kWtWaves * kWtTile * sizeof(float); }

nova_status nova_launch_cache4_weights(nova_ctx* ctx, const nova_cache4* c, const __nv_bfloat16* q, int64_t ldq, const float* lse, const int32_t* cu,
                                       int M, const float* in, float* out, bool own_rows, void* scratch, size_t scratch_bytes, cudaStream_t st)
{
    if (c->B == 0 || c->Lmax == 0) return NOVA_OK;
    const int dh = c->C / c->n_heads;
    WeightParams p;
    p.codes = (const uint8_t*)c->k_codes; p.scales = (const uint8_t*)c->k_scales; p.q = q; p.ldq = ldq; p.lse = lse; p.cu = cu;
    p.kv_len = c->kv_len; p.in = in; p.out = out; p.C = c->C; p.Lmax = c->Lmax; p.n_heads = c->n_heads; p.M = M; p.own_rows = own_rows;
    p.scale_log2e = (float)((1.0 / sqrt((double)dh)) * 1.4426950408889634);
    p.tiles = (c->Lmax + kWtTile - 1) / kWtTile;
    const long whole = (long)c->B * p.tiles;
    // as many parts as bring the launch to kWtWaves CTAs per SM (two run at once; the images' lengths differ), no more than there can
    // be (head, chunk) pairs
    const long pairs = (long)c->n_heads * (((long)M + kWtChunk - 1) / kWtChunk);
    p.parts = whole > NOVA_TICKETS ? 1 : (int)max(1l, min(pairs, (long)kWtWaves * ctx->num_sms / whole));
    if (whole * p.parts > 0x7fffffffL) return nova_fail(ctx, NOVA_ERR_SHAPE, "nova_cache4_weights: too many rows");
    if (p.parts > 1 && (!scratch || scratch_bytes < nova_cache4_weights_scratch(ctx->num_sms)))
        return nova_fail(ctx, NOVA_ERR_WORKSPACE, "nova_cache4_weights: workspace missing or too small");
    static_assert(kWtTile == kWtThreads, "the merge takes a key per thread");
    p.part = (float*)scratch;
    p.tickets = ctx->dev_status + NOVA_TICKET_WORD0;
    nova_launch_scope scope(ctx, NOVA_K_CACHE4, st);
    const dim3 grid((unsigned)(whole * p.parts)), block(kWtThreads);
    NOVA_CUDA_CHECK(ctx, dh == 64 ? nova_launch_pdl(cache4_weights_kernel<64>, grid, block, 0, st, 0, p)
                                  : nova_launch_pdl(cache4_weights_kernel<128>, grid, block, 0, st, 0, p));
    return NOVA_OK;
}

extern "C" nova_status nova_cache4_weights(nova_ctx* ctx, const nova_cache4* c, const void* q, int64_t ldq, const float* lse,
                                           const int32_t* cu_q, int M, const float* weight_in, float* weight_out, void* stream)
{
    if (!ctx) return NOVA_ERR_INVALID_ARG;
    nova_status rc = nova_cache4_check(ctx, "nova_cache4_weights", c);
    if (rc == NOVA_OK) rc = nova_cache4_check_rows(ctx, "nova_cache4_weights", c, q, q, cu_q, M, ldq);
    if (rc != NOVA_OK) return rc;
    if (c->B == 0 || c->Lmax == 0) return NOVA_OK;
    if (!weight_out || !cu_q || (M > 0 && !lse)) return nova_fail(ctx, NOVA_ERR_INVALID_ARG, "nova_cache4_weights: null tensor");
    if ((((uintptr_t)lse) | ((uintptr_t)weight_in) | ((uintptr_t)weight_out)) & 3u)
        return nova_fail(ctx, NOVA_ERR_ALIGNMENT, "nova_cache4_weights: misaligned tensor");
    NOVA_DEVICE_GUARD(ctx, "nova_cache4_weights");
    cudaStream_t st = (cudaStream_t)stream;
    rc = nova_debug_check_lists(ctx, "nova_cache4_weights", nullptr, nullptr, cu_q, c->B, M, M, false, st);
    if (rc != NOVA_OK) return rc;
    return nova_launch_cache4_weights(ctx, c, (const __nv_bfloat16*)q, ldq, lse, cu_q, M, weight_in, weight_out, false,
                                      ctx->workspace, ctx->workspace_bytes, st);
}
