// Reading keys and values back from the cache: the centres that the codes name.
//
// Nothing is computed; the values written bound it, 4 bytes a feature against a
// quarter of a byte to one that is read. A few tokens look their centres up in
// memory, one sub-vector to a thread. Many take them from LDS, where a workgroup
// keeps the centres of one head of the keys or the values (16 to 64 KB): looked up
// in the L2, each of 8 bytes moves a line of 128, and 65536 tokens of 8 heads of
// 128 features took 193 us instead of 48 (6.3 TB/s; stores alone of as much reach
// 6.8). The codes of a value sub-vector lie side by side for the tokens of a page,
// not for the token's other sub-vectors: read byte by byte they made it 79.
#include "kv_device.h"

namespace lloyd {

namespace {

constexpr int kThreads = 256;

// One sub-vector of one head of one token, key and value, to a thread.
template <int SUB>
__global__ __launch_bounds__(kThreads) void kv_read_few_kernel(KvCache c, KvTokens t, int64_t units)
{
    const int S = c.dim / SUB, kinds = c.heads * S;
    for (int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x; u < units;
         u += (int64_t)gridDim.x * kThreads) {
        const int64_t tok = u / kinds;
        const int kind = (int)(u - tok * kinds), h = kind / S, s = kind - h * S;
        uint32_t page, off;
        KvEntry<SUB> k{}, v{};
        if (kv_slot(c, t.slots[tok], &page, &off)) {
            const int64_t head = kv_head(c, page, h, S);
            const int kc = c.k_codes[head + off * S + s];
            const int vc = c.v_codes[head + ((unsigned)s << c.page_log2) + off];
            if (kc < c.K) k = kv_load<SUB>(c.k_centres + ((int64_t)kind * c.K + kc) * SUB);
            if (vc < c.K) v = kv_load<SUB>(c.v_centres + ((int64_t)kind * c.K + vc) * SUB);
        }
        *reinterpret_cast<KvEntry<SUB> *>(t.k + tok * t.k_token + h * t.k_head + s * SUB) = k;
        *reinterpret_cast<KvEntry<SUB> *>(t.v + tok * t.v_token + h * t.v_head + s * SUB) = v;
    }
}

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

constexpr int kWaves = 16;
constexpr int kTokens = 16;          // of a wave's step

// A workgroup takes one head of the keys or the values, of whose tokens the
// workgroups together go through one stretch after the other.
// A step of a wave is 16 tokens, their rows' runs of 16 bytes in order over its
// lanes: each store covers whole rows, and past the caches, for the rows are as
// large as those and not read here again.
template <int D, int SUB>
__global__ __launch_bounds__(kWaves * kWave) void kv_read_kernel(KvCache c, KvTokens t, int parts)
{
    constexpr int S = D / SUB, per = 8 / SUB;            // codes of a row, of a run
    constexpr int runs = D / 32;                         // of a lane
    constexpr int eights = 2 * S;                        // of codes, in a step of the values
    __shared__ KvEntry<SUB> book[S][256];
    __shared__ uint64_t turn[kWaves][eights];            // [sub-vector][token] of a step
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = (int)(blockIdx.x % c.heads);
    const bool values = blockIdx.x / c.heads % 2;
    const int64_t steps = (t.tokens + kTokens - 1) / kTokens, stride = (int64_t)parts * kWaves;
    const uint16_t *const centres = (values ? c.v_centres : c.k_centres) + (int64_t)h * S * c.K * SUB;
    if (c.K == 256) {
        uint4 *const dst = reinterpret_cast<uint4 *>(&book[0][0]);
        const uint4 *const src = reinterpret_cast<const uint4 *>(centres);
#pragma unroll
        for (int i = 0; i < D * 32 / (kWaves * kWave); ++i)
            dst[i * kWaves * kWave + tid] = src[i * kWaves * kWave + tid];
    } else {
        for (int i = tid; i < S * 256; i += kWaves * kWave) {
            KvEntry<SUB> e{};
            if ((i & 255) < c.K) e = kv_load<SUB>(centres + ((i >> 8) * c.K + (i & 255)) * SUB);
            book[i >> 8][i & 255] = e;
        }
    }
    __syncthreads();
    uint16_t *const out = values ? t.v + h * t.v_head : t.k + h * t.k_head;
    const int64_t out_stride = values ? t.v_token : t.k_token;
    // run i of the lane: of token (64 i + lane) / (D / 8) of the step
    const auto token_of = [&](int i) { return (i * kWave + lane) / (D / 8); };
    const auto run_of = [&](int i) { return (i * kWave + lane) % (D / 8); };
    // The slots of the next step's tokens are asked for a step ahead: keys, those of
    // the lane's runs; values, that of token lane % 16.
    int64_t next[runs];
    const auto ask = [&](int64_t step) {
#pragma unroll
        for (int i = 0; i < runs; ++i) {
            const int64_t tok = step * kTokens + (values ? lane & 15 : token_of(i));
            if (i && values) break;
            next[i] = tok < t.tokens ? t.slots[tok] : (int64_t)-1;
        }
    };
    const int64_t begin = (int64_t)(blockIdx.x / c.heads / 2) * kWaves + wave;
    ask(begin);
    for (int64_t step = begin; step < steps; step += stride) {
        uint32_t codes[runs];
        bool live[runs];
        uint32_t page, off;
        bool in_rows = false;
        if (values) {
            // do both eights of tokens lie side by side, on a page each?
            const int64_t first = __shfl(next[0], lane & 8);
            in_rows = __all(kv_slot(c, first, &page, &off) &&
                            off + 8 <= 1u << c.page_log2 && next[0] == first + (lane & 7));
        }
        if (in_rows) {
            // eight codes of a sub-vector to a load, turned in LDS
            kv_slot(c, __shfl(next[0], (lane & 1) * 8), &page, &off);
            const uint8_t *const v = c.v_codes + kv_head(c, page, h, S) + off;
#pragma unroll
            for (int i = 0; i < eights; i += kWave)
                if (i + lane < eights)
                    __builtin_memcpy(&turn[wave][i + lane],
                                     v + ((unsigned)((i + lane) >> 1) << c.page_log2), 8);
            kv_wave_order();
            const uint8_t *const turned = reinterpret_cast<const uint8_t *>(turn[wave]);
#pragma unroll
            for (int i = 0; i < runs; ++i) {
                live[i] = true;
                codes[i] = 0;
#pragma unroll
                for (int x = 0; x < per; ++x)
                    codes[i] |= (uint32_t)turned[(run_of(i) * per + x) * kTokens + token_of(i)] << (8 * x);
            }
            kv_wave_order();
        } else {
#pragma unroll
            for (int i = 0; i < runs; ++i) {
                live[i] = kv_slot(c, values ? __shfl(next[0], token_of(i)) : next[i], &page, &off);
                codes[i] = 0;
                if (!live[i]) continue;
                const int64_t head = kv_head(c, page, h, S);
                const int s = run_of(i) * per;
                if (values) {
                    const uint8_t *const v = c.v_codes + head + off + ((unsigned)s << c.page_log2);
#pragma unroll
                    for (int x = 0; x < per; ++x) codes[i] |= (uint32_t)v[x << c.page_log2] << (8 * x);
                } else {
                    __builtin_memcpy(&codes[i],
                                     __builtin_assume_aligned(c.k_codes + head + off * S + s, per), per);
                }
            }
        }
        ask(step + stride);
#pragma unroll
        for (int i = 0; i < runs; ++i) {
            KvEntry<8> row{};
            if (live[i])
#pragma unroll
                for (int x = 0; x < per; ++x) {
                    const KvEntry<SUB> e = book[run_of(i) * per + x][(codes[i] >> (8 * x)) & 255];
#pragma unroll
                    for (int w = 0; w < SUB / 2; ++w) row.w[x * (SUB / 2) + w] = e.w[w];
                }
            const int64_t tok = step * kTokens + token_of(i);
            if (tok < t.tokens)
                __builtin_nontemporal_store(
                    __builtin_bit_cast(u4v, row),
                    reinterpret_cast<u4v *>(out + tok * out_stride + run_of(i) * 8));
        }
    }
}

template <int SUB>
hipError_t launch(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    // Centres from LDS where their lookups in the L2 take longer than fetching them,
    // 512 bytes a feature to a workgroup, does. For sub-vectors of up to 32 a row (a
    // head of a token) that is from 2^18 of them on, above that, where a workgroup
    // also has more of them to place, from 2^13 rows. From the L2 and from LDS, us, at
    // half the limit and at it (dim in sub, heads): 128 in 4, 8 3.8 4.6, 5.2 4.8; 128
    // in 4, 1 3.6 4.7, 4.5 4.8; 96 in 4, 5 4.0 4.6, 5.0 4.8; 64 in 4, 8 4.0 3.7, 5.2
    // 4.2; 64 in 2, 8 3.6 4.1, 5.0 4.4; 128 in 8, 8 4.0 4.6, 5.8 5.4; 96 in 8, 8 4.1
    // 4.8, 5.8 5.4; 64 in 8, 3 3.7 4.2, 5.6 4.5; and with the second limit 128 in 2, 8
    // 5.0 6.3, 7.4 6.6; 128 in 2, 2 4.9 6.1, 6.9 6.4; 96 in 2, 8 (at 2^18 and 2^19
    // sub-vectors, 2^18.6 its limit) 5.1 5.6, 7.6 5.9. A workgroup has 128 tokens or
    // more, two to a CU at most.
    const int64_t kinds = 2 * c.heads, rows = t.tokens * c.heads, units = rows * (c.dim / SUB);
    if (units >= (int64_t)1 << 18 && rows >= (int64_t)1 << 13) {
        const int64_t most = (2 * kCUs + kinds - 1) / kinds, enough = (t.tokens + 127) / 128;
        const int parts = (int)(most < enough ? most : enough);
        const dim3 grid((unsigned)(parts * kinds)), block(kWaves * kWave);
        if (c.dim == 64)
            hipLaunchKernelGGL((kv_read_kernel<64, SUB>), grid, block, 0, s, c, t, parts);
        else if (c.dim == 96)
            hipLaunchKernelGGL((kv_read_kernel<96, SUB>), grid, block, 0, s, c, t, parts);
        else
            hipLaunchKernelGGL((kv_read_kernel<128, SUB>), grid, block, 0, s, c, t, parts);
        return hipGetLastError();
    }
    const int64_t groups = (units + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((kv_read_few_kernel<SUB>), dim3((unsigned)(groups < 65536 ? groups : 65536)),
                       dim3(kThreads), 0, s, c, t, units);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_read(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    return c.sub == 2 ? launch<2>(c, t, s) : c.sub == 4 ? launch<4>(c, t, s) : launch<8>(c, t, s);
}

}  // namespace lloyd
