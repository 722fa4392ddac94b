// Attention of a few query rows per image over the 4-bit K/V cache.
//
// With few rows the keys and values are read once and hardly computed with, so the launch is a pass over the cache's bytes: 4.5
// bits a channel, 144 bytes for a row of one head of 128. The operands go from shared memory through registers, where they are
// decoded, straight into mma.sync: with 16 query rows to a tile the tensor work (2 x 16 x 128 x 128 multiply-adds per 128 keys and
// head) is small beside the decoding, and tcgen05 would want the decoded values written back to shared memory first.
//
// Work: units of (image, head, 16 query rows), each over the image's keys in tiles of 32 per warp. The launch's tiles, unit
// after unit, are divided evenly over the CTAs, so that a single query of one image keeps every SM busy and images of different
// length cost what they hold. A unit that several CTAs share is merged through memory by the one of them that finishes last (a
// ticket per unit says who that is), in the order of the CTAs: the same call gives the same bits.
// Each warp keeps its own running maximum and sum for the 16 rows; the maximum moves only when a tile exceeds it by more
// than 2^8, so the accumulators are rescaled a few times per unit instead of once per tile. Probabilities are at
// most 2^8, rounded to bf16 for the product with V (its operand type; a rounding of 2^-9 relative each, which averages out over
// keys), while the sum takes them in fp32.
// A fragment's channels and keys are permuted so that each thread decodes contiguous bytes: channels are the contraction of Q K^T,
// keys that of P V, and O's columns may lie anywhere, so only Q's loads and O's stores know of it.
// Up to kFewPerImage rows per image on average take this kernel, more the 128-row tiles of attention.cu: a second unit per head
// decodes everything once more, where those take 128 rows for one price. us for one image, 16 heads of 128, here and there: 10 rows
// x 512 keys 12.4 and 12.8, x 4096 16.3 and 29.9, x 29414 48 and 66; 64 rows x 29414 here (in four units) 123, there 64.
// What bounds it: at 29414 keys 1.2 us per SM for 128 keys of a head where the bytes would take 0.42, the decoding's integer and
// bf16 instructions and the products about 0.3 each if nothing else ran: latencies, at eight warps of 217 registers (twelve
// of 168 are 3 % slower there and 2 us slower in small calls, sixteen 20 %). With few keys the chain of
// lengths, keys, four steps of the warps' reduction, and, where a unit is shared, the merge (3 us).
#include "cache4.cuh"

namespace {

using namespace c4;

constexpr int kFewRows = 16;           // query rows of a unit
constexpr long kFewPerImage = 16;      // rows per image, on average, up to which the launch takes this kernel
constexpr int kWarpKeys = 32;          // keys of a warp's tile
constexpr float kRescale = 8.f;        // the maximum follows when it is exceeded by more than this (log2)

template <int DH>
struct FewCfg {
    static constexpr int kWarps = 8;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kTile = kWarps * kWarpKeys;         // keys of a CTA's tile
    static constexpr int kRowBytes = DH / 2, kScaleBytes = DH / 16;
    static constexpr int kStageBytes = kWarpKeys * 2 * (kRowBytes + kScaleBytes);
    static constexpr int kDepth = 3;
    static constexpr int kRedBytes = (kWarps + 1) / 2 * kFewRows * DH * 4;       // accumulators of half of the warps
    static constexpr int kRingOff = kRedBytes;
    static constexpr int kStatOff = kRingOff + kWarps * kDepth * kStageBytes;    // [kWarps][16] maxima and sums
    static constexpr int kQOff = kStatOff + kWarps * kFewRows * 8;               // Q as the lanes take it: [steps / 2][rows g, g + 8][lane] x 16 bytes
    static constexpr int kTotal = kQOff + DH / 32 * 2 * 32 * 16;
    static constexpr int kSlotFloats = kFewRows * (DH + 2);   // a partial result: O, maxima, sums
};

struct FewParams {
    const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
    const __nv_bfloat16* q;
    int64_t ldq;
    const int32_t *cu, *kv_len;
    __nv_bfloat16* o;
    float* lse;
    int B, C, Lmax, n_heads, M;
    int own_rows;
    float scale_log2e;
    float* part;                       // [gridDim.x][2][kSlotFloats]
    unsigned int* tickets;             // [gridDim.x], zero between launches
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&t);
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Copies to shared memory of which `live` = 0 writes zeros and reads nothing.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
template <int BYTES>
__device__ __forceinline__ void cp_async_small(uint32_t dst, const void* src, bool live)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(live ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// a / b of non-negative numbers. (Most fit in 32 bits, where it takes a fifth of the time; a CTA does six before its first tile.)
__device__ __forceinline__ long div_pos(long a, long b)
{
    if (((unsigned long long)a | (unsigned long long)b) >> 32) return a / b;
    return (long)((uint32_t)a / (uint32_t)b);
}

// A place in the launch's tiles: tile t of unit (b, head, block), of which the image has `units`, with T tiles each, the first of
// which (t = 0) has no keys: key tile t - 1 otherwise. It stands for what a unit costs besides its keys, about a tile's time, so
// that CTAs whose tiles are many units of few keys do not end last.
template <int DH>
struct FewWalk {
    int b, unit, units, t, T, rows, len;
    long row0;                         // first tile of the present unit, counted over the launch

    // (an image without keys has none: its rows are written by fill_empty)
    __device__ __forceinline__ static int image_units(const FewParams& p, int b)
    {
        return image_len(p, b) == 0 ? 0 : (max(min(p.cu[b + 1], p.M) - p.cu[b], 0) + kFewRows - 1) / kFewRows * p.n_heads;
    }
    __device__ __forceinline__ static int image_len(const FewParams& p, int b)
    {
        return keys_of(p.kv_len[b], p.own_rows ? max(min(p.cu[b + 1], p.M) - p.cu[b], 0) : 0, p.own_rows, p.Lmax);
    }
    // Tiles of a unit, and one more for what it costs to begin and to end one.
    __device__ __forceinline__ static int tiles(int len) { return (len + FewCfg<DH>::kTile - 1) / FewCfg<DH>::kTile + 1; }
    __device__ __forceinline__ static long image_work(const FewParams& p, int b) { return (long)image_units(p, b) * tiles(image_len(p, b)); }
    // Tiles of the launch; by a whole warp.
    __device__ __forceinline__ static long total(const FewParams& p)
    {
        const int lane = threadIdx.x & 31;
        long sum = 0;
        for (int b = lane; b < p.B; b += 32) sum += image_work(p, b);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        return sum;
    }
    __device__ __forceinline__ void enter(const FewParams& p)
    {
        units = image_units(p, b);
        rows = p.cu[b + 1] - p.cu[b];
        len = image_len(p, b);
        T = tiles(len);
    }
    // To tile `at` of the launch; by a whole warp.
    __device__ __forceinline__ void seek(const FewParams& p, long at)
    {
        const int lane = threadIdx.x & 31;
        long before = 0;
        for (int base = 0; base < p.B; base += 32) {
            const long mine = base + lane < p.B ? image_work(p, base + lane) : 0;
            long incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            const uint32_t past = __ballot_sync(0xffffffffu, before + incl > at);
            if (past) {
                const int l = __ffs((int)past) - 1;
                b = base + l;
                before += __shfl_sync(0xffffffffu, incl - mine, l);
                break;
            }
            before += __shfl_sync(0xffffffffu, incl, 31);
        }
        enter(p);
        unit = (int)div_pos(at - before, T);
        t = (int)((at - before) - (long)unit * T);
        row0 = at - t;
    }
    __device__ __forceinline__ void next(const FewParams& p, bool more)
    {
        if (++t < T) return;
        t = 0;
        row0 += T;
        if (++unit < units || !more) return;
        unit = 0;
        do ++b; while (image_units(p, b) == 0);        // (more: there is one)
        enter(p);
    }
};

// Rows of images without keys: o = 0, lse = -inf. By all warps of the launch.
template <int DH>
__device__ __forceinline__ void fill_empty(const FewParams& p)
{
    const int lane = threadIdx.x & 31, warps = gridDim.x * FewCfg<DH>::kWarps, me = blockIdx.x * FewCfg<DH>::kWarps + (threadIdx.x >> 5);
    for (int base = 0; base < p.B; base += 32) {
        uint32_t todo = __ballot_sync(0xffffffffu, base + lane < p.B && FewWalk<DH>::image_len(p, base + lane) == 0);
        for (; todo; todo &= todo - 1) {
            const int b = base + __ffs((int)todo) - 1;
            for (int r = p.cu[b] + me; r < min(p.cu[b + 1], p.M); r += warps) {
                for (int c = lane; c < p.C / 8; c += 32) ((uint4*)(p.o + (long)r * p.C))[c] = make_uint4(0, 0, 0, 0);
                for (int h = lane; p.lse && h < p.n_heads; h += 32) p.lse[(long)h * p.M + r] = -INFINITY;
            }
        }
    }
}

template <int DH>
__global__ void __launch_bounds__(FewCfg<DH>::kThreads, 1)
cache4_few_kernel(const FewParams p)
{
    using L = FewCfg<DH>;
    constexpr int kSteps = DH / 16, kBlocks = DH / 8, kWarps = L::kWarps;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int last_s;
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    fill_empty<DH>(p);
    const long W = FewWalk<DH>::total(p);
    const long G = min((long)gridDim.x, W);
    if ((long)blockIdx.x >= G) return;
    const long first = div_pos(W * blockIdx.x, G), end = div_pos(W * (blockIdx.x + 1), G);
    auto cta_of = [&](long tile) { return (int)div_pos((tile + 1) * G - 1, W); };     // the CTA whose range holds this tile

    uint8_t* ring = smem + L::kRingOff + warp * L::kDepth * L::kStageBytes;
    constexpr uint32_t kVOff = kWarpKeys * L::kRowBytes, kKsOff = 2 * kVOff, kVsOff = kKsOff + kWarpKeys * L::kScaleBytes;
    // Row of a V stage in which key n of the warp's tile lies, and the exchange of its 16-byte pieces: such that the 32
    // threads' reads of four rows touch every bank once.
    auto v_row = [](int n) { return (n & ~7) + 4 * (n & 1) + ((n >> 1) & 3); };
    auto v_swap = [](int row) { return DH == 128 ? (row & 2) : 0; };

    FewWalk<DH> pf;
    pf.seek(p, first);
    FewWalk<DH> at = pf;
    long issued = first;
    // Copies: a lane's pieces of a tile lie a constant number of rows apart; its place in the image and head is kept.
    constexpr int kPieces = L::kRowBytes / 16, kRowsApart = 32 / kPieces;
    const int code_row = p.C / 2, scale_row = p.C / 16, my_n = lane / kPieces;
    const long v_codes_at = p.v_codes - p.k_codes, v_scales_at = p.v_scales - p.k_scales;
    const uint8_t *code_at, *scale_at;
    uint32_t k_dst[kPieces], v_dst[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int n = i * kRowsApart + my_n, c = lane % kPieces, vr = v_row(n);
        k_dst[i] = (uint32_t)(n * L::kRowBytes + c * 16);
        v_dst[i] = kVOff + (uint32_t)(vr * L::kRowBytes + (c ^ v_swap(vr)) * 16);
    }
    const uint32_t ring_s = tc::smem_u32(ring);
    auto enter = [&]() {
        const int head = pf.unit % p.n_heads;
        const long row = (long)pf.b * p.Lmax + warp * kWarpKeys;
        code_at = p.k_codes + (row + my_n) * code_row + head * L::kRowBytes + lane % kPieces * 16;
        scale_at = p.k_scales + (row + lane) * scale_row + head * L::kScaleBytes;
    };
    enter();
    auto issue = [&](int slot) {
        if (issued < end) {
            const int tile0 = (pf.t - 1) * L::kTile, left = pf.t == 0 ? 0 : pf.len - tile0 - warp * kWarpKeys;       // keys from this warp's first on
            if (left > 0) {
                const uint32_t to = ring_s + (uint32_t)(slot * L::kStageBytes);
                const uint8_t* src = code_at + (long)tile0 * code_row;
                const uint8_t* sc = scale_at + (long)tile0 * scale_row;
                if (left >= kWarpKeys) {
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) {
                        cp_async16(to + k_dst[i], src, true);
                        cp_async16(to + v_dst[i], src + v_codes_at, true);
                        src += kRowsApart * code_row;
                    }
                    cp_async_small<L::kScaleBytes>(to + kKsOff + (uint32_t)(lane * L::kScaleBytes), sc, true);
                    cp_async_small<L::kScaleBytes>(to + kVsOff + (uint32_t)(lane * L::kScaleBytes), sc + v_scales_at, true);
                } else {
                    // (what lies past the last key reads as zeros; its address is that of row 0 of the tile)
#pragma unroll
                    for (int i = 0; i < kPieces; ++i) {
                        const bool live = i * kRowsApart + my_n < left;
                        const uint8_t* at = live ? src + (long)(i * kRowsApart) * code_row : src - (long)my_n * code_row;
                        cp_async16(to + k_dst[i], at, live);
                        cp_async16(to + v_dst[i], at + v_codes_at, live);
                    }
                    const bool live = lane < left;
                    if (!live) sc -= (long)lane * scale_row;
                    cp_async_small<L::kScaleBytes>(to + kKsOff + (uint32_t)(lane * L::kScaleBytes), sc, live);
                    cp_async_small<L::kScaleBytes>(to + kVsOff + (uint32_t)(lane * L::kScaleBytes), sc + v_scales_at, live);
                }
            }
            ++issued;
            const long unit_at = pf.row0;
            pf.next(p, issued < end);
            if (pf.row0 != unit_at) enter();
        }
        cp_commit();
    };
#pragma unroll 1
    for (int i = 0; i < L::kDepth - 1; ++i) issue(i);

    float* stat = (float*)(smem + L::kStatOff);
    uint4* q_s = (uint4*)(smem + L::kQOff);
    int slot = 0;
    for (long tile = first; tile < end;) {
        // ---- a piece: the tiles of one unit that are this CTA's
        const int head = at.unit % p.n_heads, q0 = at.unit / p.n_heads * kFewRows;
        const int row_base = p.cu[at.b] + q0, rows = min(at.rows - q0, kFewRows), len = at.len;
        const long row0 = at.row0;
        const int T = at.T;
        // Q: channels t * DH/4 .. of rows g and g + 8, for all warps
        if (threadIdx.x < kSteps / 2 * 64) {
            const int h = (threadIdx.x >> 5) & 1, i = threadIdx.x >> 6;
            const bool live = g + 8 * h < rows && row_base + g + 8 * h < p.M;
            const uint4* src = (const uint4*)(p.q + (long)(row_base + (live ? g + 8 * h : 0)) * p.ldq + head * DH + t * (DH / 4));
            q_s[threadIdx.x] = live ? src[i] : make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
        float acc[kBlocks][4];
#pragma unroll
        for (int j = 0; j < kBlocks; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
        float m[2] = {-1e30f, -1e30f}, l[2] = {0.f, 0.f};       // rows g and g + 8, log2 units; l of this thread's columns
        const long piece_end = min(end, row0 + T);
        for (; tile < piece_end; ++tile) {
            issue(slot == 0 ? L::kDepth - 1 : slot - 1);
            cp_wait<L::kDepth - 1>();
            __syncwarp();
            const int key0 = (int)(tile - row0 - 1) * L::kTile + warp * kWarpKeys;
            if (tile > row0 && key0 < len) {
                const uint8_t* s_at = ring + slot * L::kStageBytes;
                // 16 keys at a time, in a loop that is not unrolled: unrolled it is 2 % faster for ten rows x 29414 keys and no
                // faster for few keys, with 7 KB more code to fetch
#pragma unroll 1
                for (int kb = 0; kb < 2; ++kb) {
                    if (key0 + 16 * kb >= len) break;
                    float s[2][4];
                    uint32_t kw[2][4], ks[2];
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb) {
                        s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
                        const int n = 16 * kb + nb * 8 + g;
                        // dh 128: this thread's 32 channels are one group; dh 64: its 16 are half of one
                        ks[nb] = both(*(const uint16_t*)(s_at + kKsOff + n * L::kScaleBytes + (DH == 128 ? t : t >> 1) * 2));
                        if constexpr (DH == 128) {
                            const uint4 v = *(const uint4*)(s_at + n * L::kRowBytes + t * 16);
                            kw[nb][0] = v.x; kw[nb][1] = v.y; kw[nb][2] = v.z; kw[nb][3] = v.w;
                        } else {
                            const uint2 v = *(const uint2*)(s_at + n * L::kRowBytes + t * 8);
                            kw[nb][0] = v.x; kw[nb][1] = v.y;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kSteps / 2; ++i) {
                        const uint4 a = q_s[i * 64 + lane], b = q_s[i * 64 + 32 + lane];
#pragma unroll
                        for (int nb = 0; nb < 2; ++nb) {
                            uint32_t x[4];
                            decode8(kw[nb][i], Scale2(ks[nb]), x);
                            mma16816(s[nb], a.x, b.x, a.y, b.y, x[0], x[1]);
                            mma16816(s[nb], a.z, b.z, a.w, b.w, x[2], x[3]);
                        }
                    }
                    if (key0 + 16 * kb + 16 > len) {
#pragma unroll
                        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (key0 + 16 * kb + nb * 8 + 2 * t + (e & 1) >= len) s[nb][e] = -INFINITY;
                    }
                    float top[2];
                    top[0] = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])) * p.scale_log2e;
                    top[1] = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3])) * p.scale_log2e;
                    if (__any_sync(0xffffffffu, top[0] > m[0] + kRescale || top[1] > m[1] + kRescale)) {
                        float f[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
                            top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
                            const float m_new = top[h] > m[h] + kRescale ? top[h] : m[h];
                            f[h] = ex2(m[h] - m_new);
                            m[h] = m_new;
                            l[h] *= f[h];
                        }
#pragma unroll
                        for (int j = 0; j < kBlocks; ++j) {
                            acc[j][0] *= f[0]; acc[j][1] *= f[0];
                            acc[j][2] *= f[1]; acc[j][3] *= f[1];
                        }
                    }
                    uint32_t pa[4];
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb) {
                        float e[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[i] = ex2(fmaf(s[nb][i], p.scale_log2e, -m[i >> 1]));
                        l[0] += e[0] + e[1];
                        l[1] += e[2] + e[3];
                        pa[nb * 2] = pack_bf16(e[0], e[1]);
                        pa[nb * 2 + 1] = pack_bf16(e[2], e[3]);
                    }
                    // keys 16 kb + {2t, 2t+1} and {2t+8, 2t+9}; channels g * DH/8 ..
                    uint32_t lo[2][2], hi[2][2];          // [key pair][word]: even and odd channels of the pair's two keys
                    uint32_t s2[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t wv[2][2];
                        uint16_t sv[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int row = 16 * kb + 8 * h + 4 * e + t;         // v_row of key 16 kb + 8 h + 2 t + e
                            if constexpr (DH == 128) {
                                const uint2 v = *(const uint2*)(s_at + kVOff + row * L::kRowBytes + ((g >> 1) ^ v_swap(row)) * 16 + (g & 1) * 8);
                                wv[e][0] = v.x; wv[e][1] = v.y;
                            } else {
                                wv[e][0] = *(const uint32_t*)(s_at + kVOff + row * L::kRowBytes + g * 4);
                                wv[e][1] = 0;
                            }
                            const int n = 16 * kb + 8 * h + 2 * t + e;
                            sv[e] = *(const uint16_t*)(s_at + kVsOff + n * L::kScaleBytes + (DH == 128 ? g >> 1 : g >> 2) * 2);
                        }
#pragma unroll
                        for (int w = 0; w < kBlocks / 8; ++w) {
                            lo[h][w] = __byte_perm(wv[0][w], wv[1][w], 0x5410);
                            hi[h][w] = __byte_perm(wv[0][w], wv[1][w], 0x7632);
                        }
                        s2[h] = (uint32_t)sv[0] | (uint32_t)sv[1] << 16;
                    }
                    const Scale2 sa(s2[0]), sb(s2[1]);
#pragma unroll
                    for (int w = 0; w < kBlocks / 8; ++w) {
                        uint32_t xa[4], xb[4], ya[4], yb[4];
                        decode8(lo[0][w], sa, xa);
                        decode8(lo[1][w], sb, xb);
                        decode8(hi[0][w], sa, ya);
                        decode8(hi[1][w], sb, yb);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            mma16816(acc[8 * w + 2 * i], pa[0], pa[1], pa[2], pa[3], xa[i], xb[i]);
                            mma16816(acc[8 * w + 2 * i + 1], pa[0], pa[1], pa[2], pa[3], ya[i], yb[i]);
                        }
                    }
                }
            }
            __syncwarp();
            if (++slot == L::kDepth) slot = 0;
            at.next(p, tile + 1 < end);
        }
        if (piece_end == row0 + 1) continue;                  // this CTA's range ends with the unit's empty tile
        // ---- the warps' results become the CTA's
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            if (t == 0) {
                stat[(warp * kFewRows + g + 8 * h) * 2] = m[h];
                stat[(warp * kFewRows + g + 8 * h) * 2 + 1] = l[h];
            }
        }
        __syncthreads();
        float m_all[2], l_all[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            m_all[h] = -1e30f;
#pragma unroll 1
            for (int w = 0; w < kWarps; ++w) m_all[h] = fmaxf(m_all[h], stat[(w * kFewRows + g + 8 * h) * 2]);
            l_all[h] = 0.f;
#pragma unroll 1
            for (int w = 0; w < kWarps; ++w)
                l_all[h] = fmaf(stat[(w * kFewRows + g + 8 * h) * 2 + 1], ex2(stat[(w * kFewRows + g + 8 * h) * 2] - m_all[h]), l_all[h]);
            const float f = ex2(m[h] - m_all[h]);
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) { acc[j][2 * h] *= f; acc[j][2 * h + 1] *= f; }
        }
        // a tree over the warps: n -> ceil(n / 2), the upper ones hand over through shared memory
        float4* red = (float4*)smem;
#pragma unroll 1
        for (int n = kWarps; n > 1;) {
            const int half = (n + 1) / 2;
            if (warp >= half && warp < n)
#pragma unroll
                for (int j = 0; j < kBlocks; ++j) red[((warp - half) * kBlocks + j) * 32 + lane] = make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
            __syncthreads();
            if (warp < n - half)
#pragma unroll
                for (int j = 0; j < kBlocks; ++j) {
                    const float4 v = red[(warp * kBlocks + j) * 32 + lane];
                    acc[j][0] += v.x; acc[j][1] += v.y; acc[j][2] += v.z; acc[j][3] += v.w;
                }
            __syncthreads();
            n = half;
        }
        const bool shared_unit = row0 + 1 < first || row0 + T > end;
        if (!shared_unit) {
            if (warp == 0)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = g + 8 * h;
                    if (r < rows && row_base + r < p.M) {
                        const float inv = 1.f / l_all[h];
                        uint4* dst = (uint4*)(p.o + (long)(row_base + r) * p.C + head * DH + t * (DH / 4));
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int j = 0; j < kBlocks; j += 8)
                                dst[(e * kBlocks + j) / 8] = make_uint4(
                                    pack_bf16(acc[j][2 * h + e] * inv, acc[j + 1][2 * h + e] * inv), pack_bf16(acc[j + 2][2 * h + e] * inv, acc[j + 3][2 * h + e] * inv),
                                    pack_bf16(acc[j + 4][2 * h + e] * inv, acc[j + 5][2 * h + e] * inv), pack_bf16(acc[j + 6][2 * h + e] * inv, acc[j + 7][2 * h + e] * inv));
                        if (p.lse && t == 0)
                            p.lse[(long)head * p.M + row_base + r] = (m_all[h] + log2f(l_all[h])) * 0.69314718055994531f;
                    }
                }
            continue;
        }
        // ---- shared with other CTAs: leave the partial result, the last of them merges
        const int c0 = cta_of(row0 + 1), c1 = cta_of(row0 + T - 1);
        float* mine = p.part + ((long)blockIdx.x * 2 + ((int)blockIdx.x == c0 ? 1 : 0)) * L::kSlotFloats;
        if (warp == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = g + 8 * h;
                float4* dst = (float4*)(mine + r * DH + t * (DH / 4));
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < kBlocks; j += 4)
                        dst[(e * kBlocks + j) / 4] = make_float4(acc[j][2 * h + e], acc[j + 1][2 * h + e], acc[j + 2][2 * h + e], acc[j + 3][2 * h + e]);
                if (t == 0) {
                    mine[kFewRows * DH + r] = m_all[h];
                    mine[kFewRows * (DH + 1) + r] = l_all[h];
                }
            }
            __threadfence();
            __syncwarp();
            if (lane == 0) {
                const unsigned n = (unsigned)(c1 - c0 + 1);
                last_s = atomicInc(&p.tickets[c0], n - 1) == n - 1;          // back to zero with the last
            }
        }
        __syncthreads();
        if (last_s) {
            __threadfence();
            constexpr int kPer = DH / 16;                 // channels per thread: 16 threads to a row
            const int r = threadIdx.x >> 4, ch = (threadIdx.x & 15) * kPer;
            if (r < rows && r < kFewRows && row_base + r < p.M) {
                auto part = [&](int c) { return p.part + ((long)c * 2 + (c == c0 ? 1 : 0)) * L::kSlotFloats; };
                float top = -1e30f, sum = 0.f, o[kPer];
#pragma unroll 8
                for (int c = c0; c <= c1; ++c) top = fmaxf(top, __ldcg(part(c) + kFewRows * DH + r));
#pragma unroll
                for (int i = 0; i < kPer; ++i) o[i] = 0.f;
#pragma unroll 4
                for (int c = c0; c <= c1; ++c) {
                    const float* src = part(c);
                    const float f = ex2(__ldcg(src + kFewRows * DH + r) - top);
                    sum = fmaf(__ldcg(src + kFewRows * (DH + 1) + r), f, sum);
#pragma unroll
                    for (int i = 0; i < kPer; i += 4) {
                        const float4 v = __ldcg((const float4*)(src + r * DH + ch + i));
                        o[i] = fmaf(v.x, f, o[i]); o[i + 1] = fmaf(v.y, f, o[i + 1]);
                        o[i + 2] = fmaf(v.z, f, o[i + 2]); o[i + 3] = fmaf(v.w, f, o[i + 3]);
                    }
                }
                const float inv = 1.f / sum;
                uint32_t w[kPer / 2];
#pragma unroll
                for (int i = 0; i < kPer / 2; ++i) w[i] = pack_bf16(o[2 * i] * inv, o[2 * i + 1] * inv);
                __nv_bfloat16* dst = p.o + (long)(row_base + r) * p.C + head * DH + ch;
                if constexpr (kPer == 8) *(uint4*)dst = make_uint4(w[0], w[1], w[2], w[3]);
                else *(uint2*)dst = make_uint2(w[0], w[1]);
                if (p.lse && ch == 0) p.lse[(long)head * p.M + row_base + r] = (top + log2f(sum)) * 0.69314718055994531f;
            }
        }
        __syncthreads();                     // (last_s)
    }
    cp_wait<0>();
}

template <int DH>
nova_status launch_few(nova_ctx* ctx, const nova_cache4_attn_args& a, cudaStream_t st)
{
    using L = FewCfg<DH>;
    const nova_cache4& c = *a.cache;
    FewParams p;
    p.k_codes = (const uint8_t*)c.k_codes; p.v_codes = (const uint8_t*)c.v_codes;
    p.k_scales = (const uint8_t*)c.k_scales; p.v_scales = (const uint8_t*)c.v_scales;
    p.q = a.q; p.ldq = a.ldq; p.cu = a.cu; p.kv_len = c.kv_len; p.o = a.o; p.lse = a.lse;
    p.B = c.B; p.C = c.C; p.Lmax = c.Lmax; p.n_heads = c.n_heads; p.M = a.M; p.own_rows = a.own_rows;
    p.scale_log2e = (float)((1.0 / sqrt((double)DH)) * 1.4426950408889634);
    p.part = (float*)a.scratch;
    p.tickets = ctx->dev_status + NOVA_TICKET_WORD0;
    // an upper bound of the tiles: the counts per image live on the device
    const long units = (((long)a.M + (long)c.B * (kFewRows - 1)) / kFewRows) * c.n_heads;
    const long tiles = units * (c.Lmax / L::kTile + 2);
    const int ctas = (int)min(min((long)ctx->num_sms, (long)NOVA_TICKETS), tiles);
    static_assert(L::kTotal <= 227 * 1024, "shared memory");
    if (!ctx->attr_few) {
        NOVA_CUDA_CHECK(ctx, cudaFuncSetAttribute(cache4_few_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<64>::kTotal));
        NOVA_CUDA_CHECK(ctx, cudaFuncSetAttribute(cache4_few_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<128>::kTotal));
        ctx->attr_few = true;
    }
    nova_launch_scope scope(ctx, NOVA_K_CACHE4, st);
    NOVA_CUDA_CHECK(ctx, nova_launch_pdl(cache4_few_kernel<DH>, dim3(ctas), dim3(L::kThreads), L::kTotal, st, 0, p));
    return NOVA_OK;
}

}  // namespace

size_t nova_cache4_attention_scratch(int num_sms, int dh, int M)
{
    if (M <= 0) return 0;
    return max((size_t)num_sms * 2 * kFewRows * (dh + 2) * sizeof(float), nova_cache4_tiles_scratch(num_sms, dh));
}

nova_status nova_launch_cache4_attention(nova_ctx* ctx, const nova_cache4_attn_args& a, cudaStream_t st)
{
    if (a.M <= 0 || a.cache->B == 0) return NOVA_OK;
    const int dh = a.cache->C / a.cache->n_heads;
    if (!a.scratch || a.scratch_bytes < nova_cache4_attention_scratch(ctx->num_sms, dh, a.M))
        return nova_fail(ctx, NOVA_ERR_WORKSPACE, "nova_cache4_attention: workspace missing or too small");
    if (a.cache->Lmax > 0 && (long)a.M > kFewPerImage * (long)a.cache->B) return nova_launch_cache4_tiles(ctx, a, st);
    return dh == 64 ? launch_few<64>(ctx, a, st) : launch_few<128>(ctx, a, st);
}

extern "C" {

size_t nova_cache4_workspace_bytes(const nova_ctx* ctx, const nova_cache4* c, int M)
{
    if (!ctx || !c || c->n_heads < 1 || c->C < 1 || c->B < 0 || c->Lmax < 0 || M < 0) return 0;
    size_t need = nova_cache4_attention_scratch(ctx->num_sms, c->C / c->n_heads, M);
    need = max(need, nova_cache4_weights_scratch(ctx->num_sms));
    need = max(need, (size_t)c->B * c->Lmax * sizeof(int32_t));            // rows that an eviction keeps
    return (need + 255) / 256 * 256;
}

nova_status nova_cache4_attention(nova_ctx* ctx, const nova_cache4* c, const void* q, int64_t ldq, const int32_t* cu_q, int M,
                                  void* o, float* lse, void* stream)
{
    if (!ctx) return NOVA_ERR_INVALID_ARG;
    nova_status rc = nova_cache4_check(ctx, "nova_cache4_attention", c);
    if (rc == NOVA_OK) rc = nova_cache4_check_rows(ctx, "nova_cache4_attention", c, q, o, cu_q, M, ldq);
    if (rc != NOVA_OK) return rc;
    if (M == 0 || c->B == 0) return NOVA_OK;
    if (((uintptr_t)lse) & 3u) return nova_fail(ctx, NOVA_ERR_ALIGNMENT, "nova_cache4_attention: misaligned lse");
    if (o == q) return nova_fail(ctx, NOVA_ERR_INVALID_ARG, "nova_cache4_attention: o aliases q");
    NOVA_DEVICE_GUARD(ctx, "nova_cache4_attention");
    cudaStream_t st = (cudaStream_t)stream;
    rc = nova_debug_check_lists(ctx, "nova_cache4_attention", nullptr, nullptr, cu_q, c->B, M, M, false, st);
    if (rc != NOVA_OK) return rc;
    nova_cache4_attn_args a;
    a.cache = c; a.q = (const __nv_bfloat16*)q; a.ldq = ldq; a.cu = cu_q; a.M = M; a.o = (__nv_bfloat16*)o; a.lse = lse;
    a.own_rows = false; a.scratch = ctx->workspace; a.scratch_bytes = ctx->workspace_bytes;
    return nova_launch_cache4_attention(ctx, a, st);
}

}  // extern "C"
