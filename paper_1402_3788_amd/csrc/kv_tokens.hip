// Attention of many new tokens of every sequence over the cache of codes.
//
// A row is a query head of a new token: a sequence has tokens * group of them on
// each key-value head, and a unit is up to 256 of them and the positions that any of
// them sees. One pass over those keeps sum_i 2^(z_i - m) and sum_i 2^(z_i - m) v_i to a
// row, with the scores z to base 2, scaled when the reference m moves up; parts of a
// unit are joined by 2^(m - largest m).
//
// A workgroup keeps the centres of one head in LDS, a row of all features for each
// code, and turns the codes of 32 positions into a tile of keys and one of values
// there while it works on the tile before: so 256 rows share what a lookup costs, and
// no decoded copy of the cache passes through memory. Its 8 waves take 32 rows each.
// Keys are the rows of one operand of v_mfma_f32_32x32x16 and queries the columns of
// the other, so that a lane's 16 scores belong to one query, and their exponentials
// are an operand of the product with the values as they are (positions are numbered
// to that end: score register 8 s + j of lane half y is position 16 s + 8 y + j).
//
// The row of all units' tiles is shared evenly by the workgroups of a head; what is cut
// that way is joined by a second launch. A launch before says where units begin.
//
// Products bound long prompts, and beside them the exponentials: 4096 tokens of 64 heads on
// 16384 positions, 8 key heads of 128, bf16: 1.84 to 1.93 ms, 1000 to 1050 TFLOP/s, the vector ALU
// at work for 46 % of the time, the matrix cores for 46 %, LDS for 44 %, at a clock that falls to
// 2.1 GHz. A cap and slopes add 14 operations to a score, and the vector ALU bounds it (83 % of the
// time): 256 tokens on 65536 positions 0.82 to 0.87 ms, 640 to 670 TFLOP/s. Short prompts are three
// launches: 8 of 101 to 1000 tokens, 12 heads of 64, documents of 150, 5 us for the units, 25 for
// this, 9 for the joins. Every wave works on all tiles of its unit, also where none of its rows
// sees a position of one, and masks them where it has fewer than 32 rows.
#include "kv_few.h"

#include <type_traits>

#ifndef KV_SUB
#define KV_SUB 4
#endif

namespace lloyd {

// Geometry and workspace of a call (pure host code).
struct KvTokensPlan {
    int splits;                      // workgroups of a head
    int units;                       // at most
    KvUnits of;
    int2 *cut;                       // [heads][splits]: the unit that begins in a share and ends
                                     // in another's (-1: none), and how many have a part of it
    float *part_o, *part_ml;         // of a share's first and last unit, cut
    size_t total;
};

hipError_t launch_kv_tokens_2(const KvCache &, const KvNew &, const KvTokensOut &, const KvTokensPlan &, hipStream_t);
hipError_t launch_kv_tokens_4(const KvCache &, const KvNew &, const KvTokensOut &, const KvTokensPlan &, hipStream_t);
hipError_t launch_kv_tokens_8(const KvCache &, const KvNew &, const KvTokensOut &, const KvTokensPlan &, hipStream_t);

namespace {

constexpr int kRows = kKvRows;
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
// Tiles that are worth a workgroup of their own. bf16, 8 heads of 128: with 3, 8 and 24 in us
// 42, 38, 46 (256 new tokens behind 500), 47, 47, 52 (behind 2000), 34, 41, 81 (8 prompts of 100).
constexpr int kShare = 8;

// As in kv_attend.hip: a new reference lies kLift below the largest score and holds until
// a score is kLag above that one.
constexpr float kLag = 8.f;
template <bool FP16>
constexpr float kLift = FP16 ? 7.f : 0.f;

template <int D, int SUB>
struct Form {
    static constexpr int S = D / SUB;
    static constexpr int kRow = D * 2;                   // bytes of one code's centres
    static constexpr int kBook = 256 * kRow;
    static constexpr int kTile = 32 * D * 2;             // bytes of 32 keys, or values
    static constexpr int kLds = 2 * kBook + 4 * kTile;
    // Threads that look keys up (8 features of a position each) and that look values up
    // (VS features of NP positions); with D < 128 the first and the last ones.
    static constexpr int kTasks = 32 * D / 8;
    static constexpr int NC = D / 8;
    static constexpr int VS = SUB < 4 ? SUB : 4, NP = 8 / VS, NG = D / VS;
    static constexpr int F = D / 32;                     // accumulators, of 32 features
    static_assert(kLds <= kMaxLds && kTasks <= kThreads, "a workgroup");
};

__device__ inline int splits_used(int tiles, int splits)
{
    return min(splits, max(1, (tiles + kShare - 1) / kShare));
}

// Even shares of n things (the first n % k of k shares have one more).
__device__ inline int share_begin(int n, int i, int k)
{
    return (int)((unsigned)n / (unsigned)k) * i + min(i, (int)((unsigned)n % (unsigned)k));
}

__device__ inline int share_of(int n, int t, int k)
{
    const unsigned each = (unsigned)n / (unsigned)k, more = (unsigned)n % (unsigned)k;
    const unsigned long_end = more * (each + 1);
    return (int)((unsigned)t < long_end ? (unsigned)t / (each + 1) : more + ((unsigned)t - long_end) / each);
}

struct KvTokensArgs {
    KvCache c;
    KvNew a;
    KvTokensOut o;
    KvTokensPlan p;
};

// The kernel's arguments where they lie in memory: for what a loop needs seldom, read there
// each time, which would else be kept in scalar registers through it, more than there are.
__device__ inline const KvTokensArgs &seldom()
{
    auto p = (const __attribute__((address_space(4))) KvTokensArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const KvTokensArgs *)p;
}

// ONE_PAGE: pages of 32 tokens or more, so that a tile lies on one.
template <int D, int SUB, bool FP16, bool ONE_PAGE>
__global__ __launch_bounds__(kThreads) void kv_tokens_kernel(KvTokensArgs args)
{
    using F = Form<D, SUB>;
    const KvCache &c = args.c;
    const KvNew &a = args.a;
    const KvTokensPlan &p = args.p;
    // the kernel has no LDS but its dynamic one, which so begins at 0
    constexpr uint32_t kbook = 0, vbook = F::kBook, ktile = 2 * F::kBook, vtile = ktile + 2 * F::kTile;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int h = blockIdx.x % c.heads, j = blockIdx.x / c.heads;
    const int units = *p.of.count, tiles = p.of.first[units];
    const int used = splits_used(tiles, p.splits);

    // A row's token (among all) and query head.
    const auto row_of = [&](const KvUnit &u, int row, int *token, int *head) {
        const unsigned group = (unsigned)seldom().a.group, x = (unsigned)(u.row0 + row);
        *token = u.t0 + (int)(x / group);
        *head = h * group + (int)(x % group);
        return x < (unsigned)u.n * group;
    };
    // Units without positions.
    for (int u = j; u < units; u += p.splits) {
        if (p.of.first[u] != p.of.first[u + 1]) continue;
        const KvUnit x = p.of.unit[u];
        const KvTokensOut &o = args.o;
        for (int i = tid; i < kRows * (D / 8); i += kThreads) {
            int t, q;
            if (!row_of(x, i / (D / 8), &t, &q)) continue;
            *reinterpret_cast<u4v *>(o.out + t * o.out_token + q * o.out_head + i % (D / 8) * 8) = u4v{0, 0, 0, 0};
            if (o.lse && i % (D / 8) == 0) o.lse[(int64_t)t * c.heads * a.group + q] = -INFINITY;
        }
    }
    if (tid == 0) p.cut[(int64_t)h * p.splits + j] = make_int2(-1, 0);   // unless found below
    if (j >= used || tiles == 0) return;
    const int a0 = share_begin(tiles, j, used), a1 = share_begin(tiles, j + 1, used);

    // A place in the row of tiles: unit u, which has tiles [base, next), the first of which is
    // tile tile0 of its sequence; the entries of that one's row of the table that may be read.
    struct Cursor {
        int u, base, next, tile0, low, high;
        const int32_t *row;
    };
    const auto enter = [&](int u) {
        const KvUnits &of = seldom().p.of;
        const KvNew &n = seldom().a;
        Cursor y;
        y.u = __builtin_amdgcn_readfirstlane(u);
        y.base = __builtin_amdgcn_readfirstlane(of.first[y.u]);
        y.next = __builtin_amdgcn_readfirstlane(of.first[y.u + 1]);
        const KvUnit &x = of.unit[y.u];
        const int lo = __builtin_amdgcn_readfirstlane(x.lo), hi = __builtin_amdgcn_readfirstlane(x.hi);
        y.tile0 = lo >> 5;
        y.low = lo >> c.page_log2;
        y.high = (hi - 1) >> c.page_log2;
        y.row = n.table + __builtin_amdgcn_readfirstlane(x.b) * n.table_stride;
        return y;
    };
    const auto advance = [&](Cursor &y, int t) {
        if (t < y.next) return;
        const int32_t *const first = seldom().p.of.first;
        int u = y.u + 1;
        while (first[u + 1] <= t) ++u;
        y = enter(u);
    };
    Cursor cur;
    {
        // the last unit whose tiles begin at a0 or before: of 64 at a time
        int from = 0, n = units;
        while (n > 1) {
            const int step = (n + kWave - 1) / kWave, at = lane * step;
            const int before = __popcll(__ballot(at < n && p.of.first[from + at] <= a0));
            from += (before - 1) * step;
            n = min(step, n - (before - 1) * step);
        }
        cur = enter(from);
    }
    Cursor then = cur;

    // What a thread looks up of a tile: 8 features of key `key`, and VS of NP values.
    constexpr bool all_look = F::kTasks == kThreads;
    const bool looks_k = all_look || tid < F::kTasks, looks_v = all_look || tid >= kThreads - F::kTasks;
    const int xk = looks_k ? tid : 0, xv = looks_v ? tid - (kThreads - F::kTasks) : 0;
    const int key = xk % 4 + xk / (4 * F::NC) * 4, chunk = xk / 4 % F::NC;
    const int vpos = (xv % 4 + xv / (4 * F::NG) * 4) * F::NP, gran = xv / 4 % F::NG;
    struct Where {
        int pos, k_page, v_page;     // ONE_PAGE: k_page of both
    };
    struct Codes {
        uint32_t k, v;
    };
    const unsigned page_bytes = (unsigned)(c.heads * F::S) << c.page_log2;
    const unsigned last_page = (unsigned)min(c.pages - 1, (int64_t)0x7FFFFFFF);
    const unsigned pm = (1u << c.page_log2) - 1;
    const int64_t head_codes = ((int64_t)h * F::S) << c.page_log2;
    const uint8_t *const k_head = c.k_codes + head_codes, *const v_head = c.v_codes + head_codes;
    const unsigned k_lane = chunk * (8 / SUB), v_lane = (unsigned)(gran * F::VS / SUB) << c.page_log2;
    const unsigned k_whole = k_lane + key * F::S, v_whole = v_lane + vpos;
    const auto find = [&](int t) {
        advance(then, t);
        Where w;
        w.pos = (t - then.base + then.tile0) * 32;
        if constexpr (ONE_PAGE) {
            w.k_page = then.row[w.pos >> c.page_log2];
        } else {
            // positions that nobody sees: the nearest page of one that somebody does
            w.k_page = then.row[min(max((w.pos + key) >> c.page_log2, then.low), then.high)];
            w.v_page = then.row[min(max((w.pos + vpos) >> c.page_log2, then.low), then.high)];
        }
        return w;
    };
    const auto load = [&](const Where &w) {
        // a number that is no page's is some page's here, never followed out
        const auto page = [&](int n) { return (uint64_t)min((unsigned)n, last_page) * page_bytes; };
        Codes x{};
        const uint8_t *k, *v;
        if constexpr (ONE_PAGE) {
            const uint64_t at = page(__builtin_amdgcn_readfirstlane(w.k_page));
            const uint8_t *const k_tile = k_head + (at + ((unsigned)w.pos & pm) * F::S);
            const uint8_t *const v_tile = v_head + (at + ((unsigned)w.pos & pm));
            k = k_tile + k_whole;
            v = v_tile + v_whole;
        } else {
            k = k_head + page(w.k_page) + (((unsigned)w.pos + key) & pm) * F::S + k_lane;
            v = v_head + page(w.v_page) + (((unsigned)w.pos + vpos) & pm) + v_lane;
        }
        if (looks_k) {
            if constexpr (SUB == 2) x.k = *reinterpret_cast<const uint32_t *>(k);
            else if constexpr (SUB == 4) x.k = *reinterpret_cast<const uint16_t *>(k);
            else x.k = *k;
        }
        if (looks_v) {
            if constexpr (F::NP == 4) x.v = *reinterpret_cast<const uint32_t *>(v);
            else x.v = *reinterpret_cast<const uint16_t *>(v);
        }
        return x;
    };
    struct Found {
        KvEntry<8> k;
        KvEntry<F::VS> v[F::NP];
    };
    const auto look = [&](uint32_t k, uint32_t v) {
        Found f;
        if (looks_k) {
            KvEntry<SUB> e[8 / SUB];
#pragma unroll
            for (int i = 0; i < 8 / SUB; ++i)
                e[i] = lds_get<KvEntry<SUB>>((k >> (8 * i) & 255) * F::kRow + (kbook + chunk * 16), i * (SUB * 2));
            __builtin_memcpy(&f.k, e, 16);
        }
        if (looks_v) {
#pragma unroll
            for (int i = 0; i < F::NP; ++i)
                f.v[i] = lds_get<KvEntry<F::VS>>((v >> (8 * i) & 255) * F::kRow + (vbook + gran * (F::VS * 2)));
        }
        return f;
    };
    // Tiles in LDS: keys as runs of 16 bytes, run r of row m (position m with its bits 2
    // and 3 in each other's place) at 512 r + 16 m, bits 6 to 8 turned by r so that a wave
    // that writes reaches all banks; values as runs of 8 positions, run r of feature f at
    // 16 D r + 16 f, the feature's last two bits turned by the two above its fourth.
    const uint32_t k_to = ktile + chunk * 512 + ((((key & ~12) | (key & 4) << 1 | (key & 8) >> 1) * 16) ^ (chunk & 7) * 64);
    const auto v_slot = [](int f) { return (f ^ ((f >> 4) & 3)) * 16; };
    uint32_t v_to[F::VS];
#pragma unroll
    for (int e = 0; e < F::VS; ++e)
        v_to[e] = vtile + vpos / 8 * (D * 16) + (vpos & 7) * 2 + v_slot(gran * F::VS + e);
    const auto put_k = [&](const Found &f, int buf) {
        if (looks_k) lds_put(k_to, buf * F::kTile, f.k);
    };
    // feature e of the granule's
    const auto put_v = [&](const Found &f, int buf, int e) {
        if (!looks_v) return;
        KvEntry<F::NP> x;
#pragma unroll
        for (int i = 0; i < F::NP / 2; ++i)
            x.w[i] = __builtin_amdgcn_perm(f.v[2 * i + 1].w[e / 2], f.v[2 * i].w[e / 2],
                                           e % 2 ? 0x07060302u : 0x05040100u);
        lds_put(v_to[e], buf * F::kTile, x);
    };

    Where where = find(a0);
    // The centres of this head, entries from K up zeros.
    {
        const uint16_t *const books[2] = {c.k_centres + (int64_t)h * F::S * c.K * SUB,
                                          c.v_centres + (int64_t)h * F::S * c.K * SUB};
        constexpr int per16 = 8 / SUB, rounds = D * 32 / kThreads;
        static_assert(D * 32 % kThreads == 0, "whole rounds");
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            const uint32_t book = kind ? vbook : kbook;
            if (c.K == 256) {
                // 16 bytes to a load: 4 runs in each of 16 sub-vectors to a wave
                uint4 reg[rounds];
#pragma unroll
                for (int i = 0; i < rounds; ++i) {
                    const int n = i * kThreads + tid, s = (n >> 2) % F::S, code = ((n >> 2) / F::S * 4 + (n & 3)) * per16;
                    reg[i] = *reinterpret_cast<const uint4 *>(books[kind] + (s * 256 + code) * SUB);
                }
#pragma unroll
                for (int i = 0; i < rounds; ++i) {
                    const int n = i * kThreads + tid, s = (n >> 2) % F::S, code = ((n >> 2) / F::S * 4 + (n & 3)) * per16;
                    KvEntry<SUB> e[per16];
                    __builtin_memcpy(e, &reg[i], 16);
#pragma unroll
                    for (int x = 0; x < per16; ++x)
                        lds_put(book + (code + x) * F::kRow + s * (SUB * 2), 0, e[x]);
                }
            } else {
                for (int i = tid; i < F::S * 256; i += kThreads) {
                    const int s = i % F::S, code = i / F::S;
                    KvEntry<SUB> e{};
                    if (code < c.K) e = kv_load<SUB>(books[kind] + (s * c.K + code) * SUB);
                    lds_put(book + code * F::kRow + s * (SUB * 2), 0, e);
                }
            }
        }
    }
    // On its turn for tile t a wave looks up the keys of t + 2 and the values of t + 1. Codes
    // are asked for a tile before, numbers of pages two.
    int ahead = a0;                                      // the tile that `codes` are of
    uint32_t v_codes = 0;                                // of the tile before
    Codes codes = load(where);
    if (a0 + 1 < a1) where = find(a0 + 1);
    // Behind the share's last tile these go on with that one's, which nobody reads.
    const auto step = [&]() {
        v_codes = codes.v;
        codes = load(where);
        if (++ahead + 1 < a1) where = find(ahead + 1);
    };
    __syncthreads();
    put_k(look(codes.k, 0), 0);
    step();
    {
        const Found f = look(codes.k, v_codes);
        put_k(f, 1);
#pragma unroll
        for (int e = 0; e < F::VS; ++e) put_v(f, 0, e);
        step();
    }
    __syncthreads();

    // scores are more than products (times 0, -infinity in an unseen place would be NaN)
    const bool changed = a.cap_log2 > 0.f || a.slopes || a.scale_log2 == 0.f;
    const float scale = changed ? 1.f : fabsf(a.scale_log2);
    u4v q[D / 16];
    f16v acc[F::F];
    float m = 0.f, m0 = 0.f, l = 0.f, slope = 0.f;
    KvSeen seen{};
    const auto begin = [&]() {
        const KvTokensArgs &all = seldom();
        const KvNew &n = all.a;
        const KvUnit u = all.p.of.unit[cur.u];
        const uint32_t flip = !changed && n.scale_log2 < 0.f ? 0x80008000u : 0u;
        int t, hq;
        const bool there = row_of(u, wave * 32 + col, &t, &hq);
        const uint16_t *const src = n.q + t * n.q_token + hq * n.q_head + half * 8;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            q[s] = u4v{0, 0, 0, 0};
            if (there) q[s] = *reinterpret_cast<const u4v *>(src + s * 16) ^ flip;
        }
        seen = KvSeen{0, 0, 0};
        if (there) seen = kv_seen(n, KvSeq{u.t0, u.n, u.len, u.prefix}, t - u.t0);
        slope = there && n.slopes ? n.slopes[hq] * kLog2e : 0.f;
        m = -INFINITY;
        m0 = 0.f;
        l = 0.f;
#pragma unroll
        for (int n = 0; n < F::F; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
    };
    // The end of the unit, or of the share.
    const auto finish = [&]() {
        const KvTokensArgs &all = seldom();
        const KvTokensOut &o = all.o;
        const float sum = sum_halves(l);
        if (cur.base >= a0 && cur.next <= a1) {
            int t, hq;
            if (row_of(all.p.of.unit[cur.u], wave * 32 + col, &t, &hq)) {
                const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                uint16_t *const dst = o.out + t * o.out_token + hq * o.out_head + 4 * half;
#pragma unroll
                for (int n = 0; n < F::F; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<uint2 *>(dst + 32 * n + 8 * i) =
                            make_uint2(pack2<FP16>(acc[n][4 * i] * inv, acc[n][4 * i + 1] * inv),
                                       pack2<FP16>(acc[n][4 * i + 2] * inv, acc[n][4 * i + 3] * inv));
                if (o.lse && half == 0)
                    o.lse[(int64_t)t * all.c.heads * all.a.group + hq] =
                        sum > 0.f || sum != sum ? (m + __log2f(sum)) * kLn2 : -INFINITY;
            }
        } else {
            const int64_t wg = (int64_t)h * all.p.splits + j;
            const int slot = cur.base < a0 ? 0 : 1;
            float *const dst = all.p.part_o + (wg * 2 + slot) * (kRows * D) + tid;
#pragma unroll
            for (int n = 0; n < F::F; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) dst[(n * 16 + i) * kThreads] = acc[n][i];
            if (half == 0) {
                float *const ml = all.p.part_ml + (wg * 2 + slot) * (2 * kRows) + wave * 32 + col;
                ml[0] = m;
                ml[kRows] = sum;
            }
            if (slot == 1 && tid == 0) all.p.cut[wg] = make_int2(cur.u, share_of(tiles, cur.next - 1, used) - j + 1);
        }
    };

    // Operand n of the products: of a tile's keys, and of its values (a step of 16 positions
    // after the other, all features of each).
    uint32_t k_from[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) k_from[n] = ktile + half * 512 + ((col * 16) ^ (2 * n + half) * 64);
    const uint32_t v_even = vtile + v_slot(col) + half * (D * 16), v_odd = vtile + v_slot(32 + col) + half * (D * 16);
    const auto key_at = [&](int buf, int n) { return lds_get<u4v>(k_from[n % 4], buf * F::kTile + n * 1024); };
    const auto value_at = [&](int buf, int n) {
        const int s = n / F::F, f = n % F::F;
        return lds_get<u4v>(f % 2 ? v_odd : v_even, buf * F::kTile + s * (2 * D * 16) + f / 2 * 1024);
    };
    const auto scores = [&](int buf) {
        f16v z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) z = mfma32<FP16>(key_at(buf, n), q[n], z);
        return z;
    };

    // The scores of tile t + 1 are under way on the matrix cores while the vector ALU works
    // out the weights of tile t, and the product with its values while the next tiles are
    // written: one after the other a wave would wait for each. LDS is asked long before:
    // all keys, then a value for each key that is done with.
    // Tile t, whose keys' and values' buffer B is: the scores z of it, those of t + 1 in next.
    const auto turn = [&](auto B, int t, f16v &z, f16v &next) {
        constexpr int buf = decltype(B)::value;
        const bool same = t + 1 < min(cur.next, a1);     // the unit, and the share, go on
        // operands of the next tile's scores, then of this one's values, four of them ahead
        constexpr int N = D / 16, slots = 4;
        static_assert(N >= slots, "operands ahead");
        u4v kv[slots];
        const auto operand = [&](int n) { return n < N ? key_at(buf ^ 1, n) : value_at(buf, n - N); };
#pragma unroll
        for (int n = 0; n < slots; ++n) kv[n] = operand(n);
        const Found found = look(codes.k, v_codes);
        step();
        const int pos = (t - cur.base + cur.tile0) * 32;
        const int y0 = pos + 8 * half;                   // of the lane's scores 0 to 7
        const bool whole = __ballot(seen.lo <= pos && seen.hi >= pos + 32) == ~0ull;
        if (changed) {
            if (a.cap_log2 > 0.f) {
                kv_cap<16>(z, a);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] *= a.scale_log2;
            }
            if (a.slopes) {
                const float far = (float)(seen.at - y0);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    z[i] = __builtin_fmaf(-slope, fabsf(far - (float)(16 * (i / 8) + i % 8)), z[i]);
            }
        }
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = y0 + 16 * (i / 8) + i % 8;
                z[i] = at >= seen.lo && at < seen.hi ? z[i] : -INFINITY;
            }
        }
        float top = z[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, z[i]);
        top *= scale;
        if (__any(top > m + (kLag + kLift<FP16>))) {
            top = fmaxf(max_halves(top) - kLift<FP16>, m);
            m0 = top == -INFINITY ? 0.f : top;
            const float alpha = __builtin_amdgcn_exp2f(m - m0);
            m = top;
            l *= alpha;
#pragma unroll
            for (int n = 0; n < F::F; ++n) acc[n] *= alpha;
        }
        // One 16-bit number to a weight: rounded to nearest it leaves the output off as its
        // own last rounding does, and without the halves that a second number would double
        // the product by.
        u4v weight[2];
        float sum[2] = {0.f, 0.f};
        const auto weigh = [&](int i) {                  // scores i and i + 1
            float w[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                w[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i + k], scale, -m0));
                sum[k] += w[k];
            }
            weight[i / 8][i % 8 / 2] = pack2<FP16>(w[0], w[1]);
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) next[i] = 0.f;
        // the wave that has its products to give goes first
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            next = mfma32<FP16>(kv[n % slots], q[n], next);
            kv[n % slots] = operand(n + slots);
#pragma unroll
            for (int i = n * 8 / N; i < (n + 1) * 8 / N; ++i) weigh(2 * i);
            __builtin_amdgcn_sched_barrier(0);
        }
        l += sum[0] + sum[1];
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            acc[n % F::F] = mfma32<FP16>(kv[(N + n) % slots], weight[n / F::F], acc[n % F::F]);
            if (n + slots < N) kv[(N + n) % slots] = operand(N + n + slots);
            if (n == 0) put_k(found, buf);
            else if (n <= F::VS) put_v(found, buf ^ 1, n - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int e = N - 1; e < F::VS; ++e) put_v(found, buf ^ 1, e);
        if (!same) {
            finish();
            if (t + 1 < a1) {
                advance(cur, t + 1);
                begin();
                next = scores(buf ^ 1);
            }
        }
        lds_barrier();
    };
    begin();
    f16v z[2];
    z[0] = scores(0);
    lds_barrier();                                       // the keys of a0 make room for those of a0 + 2
    for (int t = a0;;) {
        turn(std::integral_constant<int, 0>{}, t, z[0], z[1]);
        if (++t == a1) break;
        turn(std::integral_constant<int, 1>{}, t, z[1], z[0]);
        if (++t == a1) break;
    }
}

// Joins the parts of units that several shares have. Share j's cut unit, if it has one,
// is its second part and the first ones of the shares after it; 8 features of every
// second lane's rows to a workgroup.
template <int D, bool FP16>
__global__ __launch_bounds__(kThreads) void kv_tokens_join_kernel(KvCache c, KvNew a, KvTokensOut o, KvTokensPlan p)
{
    constexpr int quads = D / 8;                         // of features, of a lane
    const int quad = blockIdx.x % quads, wg = blockIdx.x / quads;
    const int2 found = p.cut[wg];
    if (found.x < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int row = (tid >> 6) * 32 + col, h = wg / p.splits;
    const KvUnit u = p.of.unit[found.x];
    const unsigned at = (unsigned)(u.row0 + row);
    if (at >= (unsigned)u.n * (unsigned)a.group) return;
    const auto ml = [&](int i) { return p.part_ml + ((int64_t)(wg + i) * 2 + (i == 0)) * (2 * kRows) + row; };
    float top = -INFINITY;
    for (int i = 0; i < found.y; ++i) top = fmaxf(top, *ml(i));
    const float safe = top == -INFINITY ? 0.f : top;
    float sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < found.y; ++i) {
        const float w = __builtin_amdgcn_exp2f(*ml(i) - safe);
        sum += w * ml(i)[kRows];
        const float *const from = p.part_o + ((int64_t)(wg + i) * 2 + (i == 0)) * (kRows * D) + (quad * 4) * kThreads + tid;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += w * from[k * kThreads];
    }
    const int t = u.t0 + (int)(at / (unsigned)a.group), hq = h * a.group + (int)(at % (unsigned)a.group);
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    // accumulator n, registers 4 i to 4 i + 3
    uint16_t *const dst = o.out + t * o.out_token + hq * o.out_head + 32 * (quad / 4) + 8 * (quad % 4) + 4 * half;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2<FP16>(x[0] * inv, x[1] * inv), pack2<FP16>(x[2] * inv, x[3] * inv));
    if (o.lse && quad == 0 && half == 0)
        o.lse[(int64_t)t * c.heads * a.group + hq] = sum > 0.f || sum != sum ? (top + __log2f(sum)) * kLn2 : -INFINITY;
}

template <int D, int SUB, bool FP16>
hipError_t launch(const KvCache &c, const KvNew &a, const KvTokensOut &o, const KvTokensPlan &p, hipStream_t s)
{
    using F = Form<D, SUB>;
    const KvTokensArgs args{c, a, o, p};
    const auto kernel = c.page_log2 >= 5 ? kv_tokens_kernel<D, SUB, FP16, true> : kv_tokens_kernel<D, SUB, FP16, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(c.heads * p.splits)), dim3(kThreads), F::kLds, s, args);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL((kv_tokens_join_kernel<D, FP16>), dim3((unsigned)(c.heads * p.splits * (D / 8))),
                       dim3(kThreads), 0, s, c, a, o, p);
    return hipGetLastError();
}

template <int D>
hipError_t launch_type(const KvCache &c, const KvNew &a, const KvTokensOut &o, const KvTokensPlan &p, hipStream_t s)
{
    return c.fp16 ? launch<D, KV_SUB, true>(c, a, o, p, s) : launch<D, KV_SUB, false>(c, a, o, p, s);
}

}  // namespace

#define KV_CAT2(a, b) a##b
#define KV_CAT(a, b) KV_CAT2(a, b)
hipError_t KV_CAT(launch_kv_tokens_, KV_SUB)(const KvCache &c, const KvNew &a, const KvTokensOut &o,
                                             const KvTokensPlan &p, hipStream_t s)
{
    return c.dim == 64 ? launch_type<64>(c, a, o, p, s)
         : c.dim == 96 ? launch_type<96>(c, a, o, p, s) : launch_type<128>(c, a, o, p, s);
}

#if KV_SUB == 4
namespace {

// One workgroup: the units of all sequences and where their tiles begin.
__global__ __launch_bounds__(1024) void kv_units_kernel(KvCache c, KvNew a, KvUnits to, int rows)
{
    __shared__ int seq_first[kKvMaxSeqs + 1];
    __shared__ int wave_sum[16];
    __shared__ unsigned long long total;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // sum of x over the threads up to this one, and of all
    const auto scan = [&](int x, int *all) {
        x = scan_lanes(x);
        __syncthreads();
        if (lane == 63) wave_sum[wave] = x;
        __syncthreads();
        int before = 0, sum = 0;
        for (int i = 0; i < 16; ++i) {
            if (i == wave) before = sum;
            sum += wave_sum[i];
        }
        *all = sum;
        return x + before;
    };
    const int per = (a.seqs + 1023) / 1024;
    int n[(kKvMaxSeqs + 1023) / 1024] = {}, sum = 0, units;
    bool descend = false;
#pragma unroll
    for (int k = 0; k < (kKvMaxSeqs + 1023) / 1024; ++k) {
        const int b = tid * per + k;
        if (k < per && b < a.seqs) {
            n[k] = (kv_seq(c, a, b).n * a.group + rows - 1) / rows;
            descend |= a.bounds[b] > a.bounds[b + 1];
        }
        sum += n[k];
    }
    if (__syncthreads_or(descend)) {
        if (tid == 0) total = 0;
        __syncthreads();
        atomicAdd(&total, (unsigned long long)sum);
        __syncthreads();
        if (total > (unsigned long long)kv_most_units(a, rows)) {
            sum = 0;
#pragma unroll
            for (int k = 0; k < (kKvMaxSeqs + 1023) / 1024; ++k) n[k] = 0;
        }
    }
    int at = scan(sum, &units) - sum;
#pragma unroll
    for (int k = 0; k < (kKvMaxSeqs + 1023) / 1024; ++k) {
        const int b = tid * per + k;
        if (k < per && b < a.seqs) seq_first[b] = at;
        at += n[k];
    }
    if (tid == 0) seq_first[a.seqs] = units;
    __syncthreads();
    const auto seq_of = [&](int u) {
        int b = 0, end = a.seqs;                         // the last b with seq_first[b] <= u
        while (end - b > 1) {
            const int mid = (b + end) >> 1;
            if (seq_first[mid] <= u) b = mid;
            else end = mid;
        }
        return b;
    };
    if (a.starts) {
        // what a token sees says nothing of the next one's: a unit's over the lanes of a wave
        for (int u = wave; u < units; u += 16) {
            const int b = seq_of(u), row0 = (u - seq_first[b]) * rows;
            const KvSeq s = kv_seq(c, a, b);
            const int i1 = (min(row0 + rows, s.n * a.group) - 1) / a.group;
            int lo = INT32_MAX, hi = 0;
            for (int i = row0 / a.group + lane; i <= i1; i += kWave) {
                const KvSeen y = kv_seen(a, s, i);
                if (y.hi > 0) lo = min(lo, y.lo);
                hi = max(hi, y.hi);
            }
            for (int k = 1; k < kWave; k *= 2) {
                lo = min(lo, __shfl_xor(lo, k));
                hi = max(hi, __shfl_xor(hi, k));
            }
            if (lane == 0)
                to.unit[u] = KvUnit{b, row0, s.t0, s.n, s.len, s.prefix, lo < hi ? lo : 0, lo < hi ? hi : 0};
        }
        __syncthreads();
    }
    int tiles = 0;
    for (int u0 = 0; u0 < units; u0 += 1024) {
        const int u = u0 + tid;
        KvUnit x{};
        if (u < units) {
            if (a.starts) {
                x = to.unit[u];
            } else {
                const int b = seq_of(u);
                x = kv_unit(a, kv_seq(c, a, b), b, (u - seq_first[b]) * rows, rows);
                to.unit[u] = x;
            }
        }
        const int n1 = x.tiles();
        int all;
        const int upto = scan(n1, &all);
        if (u < units) to.first[u] = tiles + upto - n1;
        tiles += all;
    }
    if (tid == 0) {
        to.first[units] = tiles;
        *to.count = units;
    }
}

// Units of few rows (kv_attend.hip) read the cache once for every 16 rows; units of 256 take
// longer to begin and cost the same however few of their rows there are. bf16, 8 heads of 128,
// in us, units of few and of 256: 64 rows of each sequence 23 and 47 (8 of 2000 positions),
// 32 and 71 (one of 30000), 54 and 62 (64 of 500), 93 and 131 (256 of 300); 128 rows 42 and 48,
// 49 and 75, 144 and 164 (16 of 8000), but of many units 52 and 38 (32 of 500, 288 units), 88 and
// 69 (64 of 500, 576 units). More rows, by the tiles of units of few to a workgroup: with 22 of
// them 21 and 33 (128 tokens of 4 heads behind 500), 67: 38 and 48 (a prompt of 500), 134: 34
// and 57 (64 tokens behind 8000), 146: 45 and 48 (256 behind 2000), 259: 67 and 58 (a prompt of
// 1000), 280: 62 and 57 (8 of 64 behind 2000), 335: 57 and 42 (8 prompts to 1000, 12 heads of 64).
constexpr int kFewRows = 64;         // of a sequence on average, up to which units are of few;
constexpr int kFewUnits = 256;       // where that makes no more than those,
constexpr int kFewMore = 128;        // up to these, or
constexpr int kFewTiles = 192;       // where a workgroup has no more than these

KvTokensPlan plan_of(const KvCache &c, const KvNew &a, char *ws)
{
    KvTokensPlan p{};
    p.units = (int)kv_most_units(a, kRows);
    const int64_t span = ((int64_t)a.table_pages << c.page_log2) / 32 + 2;
    const int64_t most = (p.units * span + kShare - 1) / kShare;
    int64_t splits = kCUs / c.heads;                     // one workgroup to a CU: registers allow no more
    if (splits > most) splits = most;
    p.splits = splits < 1 ? 1 : (int)splits;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        char *const x = ws + at;
        at += (bytes + 255) / 256 * 256;
        return x;
    };
    const size_t shares = (size_t)c.heads * p.splits;
    p.of.count = reinterpret_cast<int32_t *>(take(4));
    p.of.first = reinterpret_cast<int32_t *>(take(4 * ((size_t)p.units + 1)));
    p.of.unit = reinterpret_cast<KvUnit *>(take(sizeof(KvUnit) * (size_t)p.units));
    p.cut = reinterpret_cast<int2 *>(take(sizeof(int2) * shares));
    p.part_ml = reinterpret_cast<float *>(take(shares * 2 * 2 * kRows * sizeof(float)));
    p.part_o = reinterpret_cast<float *>(take(shares * 2 * kRows * c.dim * sizeof(float)));
    p.total = at;
    return p;
}

}  // namespace

hipError_t launch_kv_units(const KvCache &c, const KvNew &n, const KvUnits &to, int rows, hipStream_t s)
{
    hipLaunchKernelGGL(kv_units_kernel, dim3(1), dim3(1024), 0, s, c, n, to, rows);
    return hipGetLastError();
}

// Whether a unit is of few rows: every sequence has few on average.
static bool few(const KvCache &c, const KvNew &a, const KvFewPlan &p)
{
    const int64_t rows = a.tokens * a.group, seqs = a.seqs;
    const int64_t span = ((int64_t)a.table_pages << c.page_log2) / kKvTile + 1;
    const int64_t workgroups = c.heads < kCUs ? kCUs / c.heads : 1;
    return (rows <= kFewRows * seqs && p.units <= kKvMaxFew) ||
           (p.units <= kFewUnits && (rows <= kFewMore * seqs || p.units * span <= kFewTiles * workgroups));
}

size_t kv_attend_tokens_bytes(const KvCache &c, const KvNew &a)
{
    const KvFewPlan p = plan_kv_few(c, a);
    return few(c, a, p) ? p.total : plan_of(c, a, nullptr).total;
}

hipError_t launch_kv_attend_tokens(const KvCache &c, const KvNew &a, const KvTokensOut &o, void *ws,
                                   hipStream_t s)
{
    const KvFewPlan f = plan_kv_few(c, a);
    if (few(c, a, f)) return launch_kv_few(c, a, o, f, ws, s);
    const KvTokensPlan p = plan_of(c, a, static_cast<char *>(ws));
    const hipError_t e = launch_kv_units(c, a, p.of, kRows, s);
    if (e != hipSuccess) return e;
    return c.sub == 2 ? launch_kv_tokens_2(c, a, o, p, s)
         : c.sub == 4 ? launch_kv_tokens_4(c, a, o, p, s) : launch_kv_tokens_8(c, a, o, p, s);
}
#endif

}  // namespace lloyd
