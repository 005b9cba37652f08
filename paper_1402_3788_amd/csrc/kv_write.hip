// Encoding of keys and values into the cache: every sub-vector x gets the number
// of its nearest centre (Eq. (2), in the fp32 operations kmeans.h states).
//
// The matrix cores screen: score_j = T + x . c_j - |c_j|^2 / 2, the largest of
// which belongs to the nearest centre but for rounding. T, the same for all
// centres, is a little over M = |x|^2 + C^2, C the largest |c|, so that no score is
// negative and their bits compare as whole numbers do (a maximum of three needs
// no instruction to quiet its inputs then). What rounding can do is bounded:
//   products of 16-bit numbers are exact in fp32; up to 8 of them, the three parts
//   of |c|^2 / 2 and T are added, each addition off by at most 2^-23 of what it
//   adds up to, here below 2.1 M (no more than faithful rounding assumed), and
//   |c|^2 / 2 by 10 such units of itself: a score is off by E <= 31 * 2^-23 M;
//   the stated distance is off by 6.5 * 2^-24 of itself, itself <= 2 M.
// So the centre that the definition chooses scores at least the best score less
// 2 E + 6.5 * 2^-23 M < 2^-16 M. The groups of 8 centres whose best score is not
// below that are evaluated as the definition says, nearly always one group of the
// 32. Where a bound is not a finite number (overflow, NaN) every group is.
//
// A wave keeps the 256 centres of one sub-vector as matrix operands in its
// registers and takes 32 tokens a step. A lane then has 128 scores, at half an
// instruction each (the maximum of three), 16 groups at 2, and 4 distances at some
// 17: about 250 vector instructions and 8 matrix products a step. The former take
// 97 % of a SIMD's cycles and bound it, most of the latter run beside them. 4096
// tokens of 8 heads of 128 features in sub-vectors of 4, keys and values (2.1 million
// sub-vectors, 537 million distances): 36 us, 15 distances a picosecond, where all of
// them on the vector ALU took 153. A few tokens are better off with the latter (kFew
// below).
#include "kv_device.h"

#include <type_traits>

namespace lloyd {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kTokens = 32;          // tokens of a wave's step, columns of the product

// Sub-vectors up to which all distances are taken on the vector ALU: 8 heads of 128
// features in sub-vectors of 4, 1 token (512 of them) 2.9 us and 3.9 with the
// screen, 8 tokens (4096) 3.7 and 3.9, 12 4.4 and 4.1, 24 5.5 and 4.1; 8 of 128 in 8,
// 16 tokens (4096) 4.0 and 4.1, 24 4.8 and 4.4; 4 of 64 in 2, 16 tokens (4096) 3.6
// and 4.1, 24 4.1 and 4.0; 8 of 128 in 2, 4 tokens (4096) 3.5 and 3.9, 8 4.8 and 4.2;
// 1 of 128 in 4, 64 tokens (4096) 3.6 and 4.0, 128 5.0 and 4.1.
constexpr int kFew = 4096;

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef _Float16 h4v __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));

// What a lane holds of a matrix operand: 8 values for SUB = 8, else 4. A centre
// is padded to it with zeros; so is the record of -|c|^2 / 2 as three bf16
// numbers that add up to it.
template <int SUB>
struct alignas(SUB == 8 ? 16 : 8) Operand {
    uint32_t w[SUB == 8 ? 4 : 2];
};

template <int SUB>
__device__ inline f16v product(bool fp16, const Operand<SUB> &a, const Operand<SUB> &b, f16v c)
{
    if constexpr (SUB == 8)
        return fp16 ? __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8v, a),
                                                             __builtin_bit_cast(h8v, b), c, 0, 0, 0)
                    : __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8v, a),
                                                              __builtin_bit_cast(b8v, b), c, 0, 0, 0);
    else
        return fp16 ? __builtin_amdgcn_mfma_f32_32x32x8f16(__builtin_bit_cast(h4v, a),
                                                           __builtin_bit_cast(h4v, b), c, 0, 0, 0)
                    : __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(__builtin_bit_cast(s4v, a),
                                                               __builtin_bit_cast(s4v, b), c, 0, 0, 0);
}

__device__ inline uint32_t bf16_bits(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x); }

// Of two values of every lane: the lower lanes' x with their y in the upper lanes,
// and the upper lanes' x in the lower lanes with their y.
__device__ inline void halves(uint32_t x, uint32_t y, uint32_t *lower, uint32_t *upper)
{
    const auto both = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    *lower = both[0];
    *upper = both[1];
}

// The nearest of 4 centres from `row` on to x, if it is nearer than `near` or as
// near and lower in number.
template <bool FP16, int SUB>
__device__ inline void evaluate(const Operand<SUB> *centre, int row, const float (&x)[SUB],
                                float &near, int &code)
{
    float d[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Operand<SUB> o = centre[row + k];
        KvEntry<SUB> e;
#pragma unroll
        for (int i = 0; i < SUB / 2; ++i) e.w[i] = o.w[i];
        float y[SUB];
        kv_unpack<FP16>(e, y);
        d[k] = kv_distance(x, y);
    }
    const float least = fminf(fminf(d[0], d[1]), fminf(d[2], d[3]));
    int j = d[2] == least ? 2 : 3;
    j = d[1] == least ? 1 : j;
    j = row + (d[0] == least ? 0 : j);
    const bool nearer = (least < near) | ((least == near) & (j < code));     // not for a NaN
    near = nearer ? least : near;
    code = nearer ? j : code;
}

// A workgroup takes kWaves sub-vectors of one head of the keys or the values, one
// to a wave, and of the tokens the steps y, y + gridDim.y, ... The waves share
// nothing but the lines of memory their tokens lie on.
template <int SUB, bool FP16>
__global__ __launch_bounds__(kThreads, 4) void kv_write_kernel(KvCache c, KvTokens t)
{
    __shared__ Operand<SUB> centres_of[kWaves][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, up = lane >> 5;
    const int S = c.dim / SUB, groups = S / kWaves;
    const int s = (int)(blockIdx.x % groups) * kWaves + wave;
    const int h = (int)(blockIdx.x / groups) % c.heads;
    const bool values = (int)(blockIdx.x / groups) >= c.heads;
    const uint16_t *const centres = (values ? c.v_centres : c.k_centres) +
                                    ((int64_t)h * S + s) * c.K * SUB;
    Operand<SUB> *const centre = centres_of[wave];
    const uint32_t tokens = (uint32_t)t.tokens, stride = gridDim.y * kTokens;      // both below 2^31
    const uint32_t begin = blockIdx.y * kTokens;
    // Tokens of a step: the lane's sub-vector and slot. Past the end they stay
    // those before, and go nowhere.
    const int64_t row_stride = values ? t.v_token : t.k_token;
    const uint16_t *row = (values ? t.v + h * t.v_head : t.k + h * t.k_head) + s * SUB +
                          (int64_t)(begin + col) * row_stride;
    const int64_t *slots = t.slots + begin + col;
    const int64_t row_step = row_stride * stride;
    KvEntry<SUB> next{};
    int64_t next_slot = -1;
    const auto ask = [&](uint32_t first) {
        if (first + col < tokens) {
            next_slot = *slots;
            next = kv_load<SUB>(row);
        }
        slots += stride;
        row += row_step;
    };
    ask(begin);

    // Operands, tile n: centres 32 n + col. bf16: one product, the lower lanes'
    // values are the centre, the upper ones' the three parts of -|c|^2 / 2; fp16:
    // a product for each, the upper lanes' zeros. Places from K on: zeros and a norm
    // that never wins, and in LDS no number, whose distance never does. A lane
    // works one centre out for two tiles, those of the upper lanes the second's:
    // lanes and halves are swapped into place.
    Operand<SUB> a[8];
    Operand<4> norm_of[FP16 ? 8 : 1];
    float big = 0.f;
    KvEntry<SUB> given[4];                               // all asked for before one is waited for
#pragma unroll
    for (int p = 0; p < 4; ++p)
        given[p] = kv_load<SUB>(centres + min(p * kWave + lane, c.K - 1) * SUB);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const bool real = p * kWave + lane < c.K;
        float y[SUB], norm = 0.f;
        kv_unpack<FP16>(given[p], y);
#pragma unroll
        for (int i = 0; i < SUB; ++i) norm = __builtin_fmaf(y[i], y[i], norm);
        big = fmaxf(big, norm);
        const float n0 = -0.5f * norm;
        const uint32_t hi = bf16_bits(n0);
        const float n1 = n0 - __uint_as_float(hi << 16);
        const uint32_t mid = bf16_bits(n1);
        Operand<SUB> op{}, kept{};
        Operand<4> rec{};
        rec.w[0] = hi | mid << 16;
        rec.w[1] = bf16_bits(n1 - __uint_as_float(mid << 16)) | 0x3F800000u;
        const bool finite = norm < INFINITY;             // else every group is evaluated
        rec.w[0] = real ? finite ? rec.w[0] : 0u : 0xFF7Fu;      // bf16, as all of the record
        rec.w[1] = real && finite ? rec.w[1] : 0u;
#pragma unroll
        for (int i = 0; i < SUB / 2; ++i) {
            op.w[i] = real ? given[p].w[i] : 0u;
            kept.w[i] = real ? given[p].w[i] : 0x7FFF7FFFu;
        }
        centre[p * kWave + lane] = kept;
        constexpr int words = sizeof(op) / 4;
#pragma unroll
        for (int i = 0; i < words; ++i)
            halves(op.w[i], !FP16 && i < 2 ? rec.w[i] : 0u, &a[2 * p].w[i], &a[2 * p + 1].w[i]);
        if constexpr (FP16) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                halves(rec.w[i], 0u, &norm_of[2 * p].w[i], &norm_of[2 * p + 1].w[i]);
        }
    }
#pragma unroll
    for (int d = 32; d; d /= 2) big = fmaxf(big, __shfl_xor(big, d));
    const int tiles = (c.K + 31) >> 5;
    // columns of the norms' product: ones for the three parts, T for its 1
    const bool takes_norm = FP16 ? !up : up;
    kv_wave_order();

    uint8_t *const codes = values ? c.v_codes + ((uint32_t)s << c.page_log2) : c.k_codes + s;
    const uint32_t code_step = values ? 1 : S;           // from token to token of a page
    for (uint32_t first = begin; first < tokens; first += stride) {
        const KvEntry<SUB> e = next;
        const int64_t slot = next_slot;
        ask(first + stride);
        float x[SUB], norm = 0.f;
        kv_unpack<FP16>(e, x);
#pragma unroll
        for (int i = 0; i < SUB; ++i) norm = __builtin_fmaf(x[i], x[i], norm);
        const float total = norm + big;
        Operand<4> ones{};
        if (takes_norm) {
            ones.w[0] = 0x3F803F80u;
            ones.w[1] = 0x3F80u | bf16_bits(1.01f * total) << 16;
        }
        Operand<SUB> bx{};
#pragma unroll
        for (int i = 0; i < SUB / 2; ++i) bx.w[i] = up ? 0u : e.w[i];
        if (!FP16 && up) {
            bx.w[0] = ones.w[0];
            bx.w[1] = ones.w[1];
        }
        // top[2 n + u]: the bits of the best score of the lane's rows
        // 32 n + 16 u + 8 i + 4 up + 0..3, i = 0, 1
        int top[16];
        const auto score = [&](int n) {
            f16v d = {};
            if constexpr (FP16) d = product<4>(false, norm_of[n], ones, d);
            d = product<SUB>(FP16, a[n], bx, d);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                int m = max(__float_as_int(d[8 * u]), __float_as_int(d[8 * u + 1]));
#pragma unroll
                for (int i = 2; i < 8; ++i) m = max(m, __float_as_int(d[8 * u + i]));
                top[2 * n + u] = m;
            }
        };
        if (tiles == 8) {                                // without branches between the products
#pragma unroll
            for (int n = 0; n < 8; ++n) score(n);
        } else {
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                top[2 * n] = top[2 * n + 1] = (int)0x80000000;
                if (n < tiles) score(n);
            }
        }
        int best = top[0];
#pragma unroll
        for (int n = 1; n < 16; ++n) best = max(best, top[n]);
        best = max(best, __shfl_xor(best, 32));
        const float least = __int_as_float(best) - (0x1p-16f * total + 1e-30f);
        // bit 15 - n: group n is below the least that could be the nearest's
        uint32_t below = 0;
#pragma unroll
        for (int n = 0; n < 16; ++n)
            below = __builtin_amdgcn_alignbit(below, __float_as_uint(__int_as_float(top[n]) - least), 31);
        uint32_t open = least < INFINITY ? ~below & 0xFFFFu : 0xFFFFu;   // all for a NaN
        open &= 0xFFFFu << (16 - 2 * tiles);
        const uint32_t other = __shfl_xor(open, 32);
        open = up ? open << 16 | other : open | other << 16;
        // both lanes of a token evaluate half of a group's 8 centres each
        float near = INFINITY;
        int code = 0;
        do {                                             // a token has one at least
            const int bit = open ? __builtin_ctz(open) : 0;      // done: some group, not taken
            float there = near;
            int row = code;
            evaluate<FP16>(centre, (~bit & 15) * 16 + (bit >> 4) * 4 + up * 8, x, there, row);
            near = open ? there : near;
            code = open ? row : code;
            open &= open - 1;
        } while (__any(open));
        const float near2 = __shfl_xor(near, 32);
        const int code2 = __shfl_xor(code, 32);
        code = (near2 < near) | ((near2 == near) & (code2 < code)) ? code2 : code;
        uint32_t page, off;
        if (up || first + col >= tokens || !kv_slot(c, slot, &page, &off)) continue;
        codes[kv_head(c, page, h, S) + off * code_step] = (uint8_t)code;
    }
}

// The least of x over the wave (numbers that are none left out).
__device__ inline float wave_least(float x)
{
    const auto from = [](float v, auto ctrl, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(INFINITY), __float_as_int(v),
                                                          ctrl.value, rows.value, 0xF, false));
    };
    using std::integral_constant;
    x = fminf(x, from(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{}));
    x = fminf(x, from(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{}));
    x = fminf(x, from(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{}));
    x = fminf(x, from(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{}));
    x = fminf(x, from(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{}));
    x = fminf(x, from(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{}));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// A few tokens: all distances as the definition says, four centres to a lane of
// the wave that has the sub-vector. What counts is how little there is to load and
// run before the answer.
template <int SUB, bool FP16>
__global__ __launch_bounds__(kThreads) void kv_write_few_kernel(KvCache c, KvTokens t)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int S = c.dim / SUB, groups = S / kWaves;
    const int s = (int)(blockIdx.x % groups) * kWaves + wave;
    const int h = (int)(blockIdx.x / groups) % c.heads;
    const bool values = (int)(blockIdx.x / groups) >= c.heads;
    const uint16_t *const centres = (values ? c.v_centres : c.k_centres) +
                                    ((int64_t)h * S + s) * c.K * SUB;
    const uint16_t *const row = (values ? t.v + h * t.v_head : t.k + h * t.k_head) + s * SUB;
    const int64_t row_stride = values ? t.v_token : t.k_token;
    KvEntry<SUB> e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = kv_load<SUB>(centres + min(i * kWave + lane, c.K - 1) * SUB);
#pragma unroll 1
    for (int64_t tok = blockIdx.y; tok < t.tokens; tok += gridDim.y) {
        float x[SUB], d[4];
        kv_unpack<FP16>(kv_load<SUB>(row + tok * row_stride), x);
        const int64_t slot = t.slots[tok];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y[SUB];
            kv_unpack<FP16>(e[i], y);
            d[i] = kv_distance(x, y);
            if (i * kWave + lane >= c.K) d[i] = NAN;
        }
        const float least = wave_least(fminf(fminf(d[0], d[1]), fminf(d[2], d[3])));
        int code = 0;                                    // for distances that are no numbers
#pragma unroll
        for (int i = 3; i >= 0; --i)
            if (const uint64_t at = __ballot(d[i] == least)) code = i * kWave + __builtin_ctzll(at);
        uint32_t page, off;
        if (lane || !kv_slot(c, slot, &page, &off)) continue;
        const int64_t head = kv_head(c, page, h, S);
        if (values)
            c.v_codes[head + ((uint32_t)s << c.page_log2) + off] = (uint8_t)code;
        else
            c.k_codes[head + off * S + s] = (uint8_t)code;
    }
}

template <int SUB>
hipError_t launch(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    const unsigned kinds = 2 * c.heads * (c.dim / SUB / kWaves);
    if (t.tokens * (kinds * kWaves) <= kFew) {
        // a token to a workgroup while all fit the chip at once
        const int64_t most = (8 * kCUs + kinds - 1) / kinds;
        const dim3 grid(kinds, (unsigned)(t.tokens < most ? t.tokens : most));
        if (c.fp16)
            hipLaunchKernelGGL((kv_write_few_kernel<SUB, true>), grid, dim3(kThreads), 0, s, c, t);
        else
            hipLaunchKernelGGL((kv_write_few_kernel<SUB, false>), grid, dim3(kThreads), 0, s, c, t);
        return hipGetLastError();
    }
    const int64_t steps = (t.tokens + kTokens - 1) / kTokens;
    // Workgroups to a CU: a wave's start (256 centres read, eight operands made)
    // takes nearly as long as a step, so where each CU has few steps, three. 1021
    // tokens, 3 and 6: 8 heads of 128 in 8 (8 steps a CU) 9.0 and 9.8 us, 4 of 64 in 2
    // (8) 8.0 and 8.8, 8 of 128 in 4 (16) 13.4 and 13.0, in 2 (32) 21.1 and 20.0; 4096,
    // 1 of 128 in 4 (8) 6.7 and 7.9, 8 (64) 39.5 and 36.4.
    const int64_t each = steps * kinds <= 12 * kCUs ? 3 : 6;
    const int64_t most = (each * kCUs + kinds - 1) / kinds;
    const unsigned y = (unsigned)(steps < most ? steps : most);
    if (c.fp16)
        hipLaunchKernelGGL((kv_write_kernel<SUB, true>), dim3(kinds, y), dim3(kThreads), 0, s, c, t);
    else
        hipLaunchKernelGGL((kv_write_kernel<SUB, false>), dim3(kinds, y), dim3(kThreads), 0, s, c, t);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    return c.sub == 2 ? launch<2>(c, t, s) : c.sub == 4 ? launch<4>(c, t, s) : launch<8>(c, t, s);
}

}  // namespace lloyd
