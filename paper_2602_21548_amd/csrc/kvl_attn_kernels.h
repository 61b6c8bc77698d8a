// Attention over a paged cache: kernels.
//
// For a query q and the keys t that it sees, with c = scale * log2(e):
//   m = max_t c <q, K_t>,  l = sum_t 2^(c <q, K_t> - m),  out = sum_t 2^(c <q, K_t> - m) V_t / l,  lse = ln 2 (m + log2 l),
// in one pass over the keys: m, l and the unnormalised output are kept for the keys so far, and what is there is multiplied by
// 2^(m - m') where a tile raises m to m'.  Results over different keys are joined by the same rule.
//
// The query heads that share a cache head are rows of one product: row = new token * group + head in group.
//
// Both kernels compute the scores' transpose, keys by rows of queries, S^T = K Q^T, and the outputs', O^T = V^T P^T.  In the
// registers that the first product leaves, a lane holds one query row's scores, so m and l need no exchange but between the two or
// four lanes that share a row; and what a lane holds of P^T is what the second product wants from it, if the keys of its contraction
// are taken in the order in which they lie there.  V^T is read in that order, by the transposing reads of the LDS.
#pragma once

#include <type_traits>

#include "kvl_attn_internal.h"
#include "kvl_attn_types.h"

namespace kvl {

struct AttnArgs {
    const AttnItem *items;
    const int32_t *tables;
    const char *k, *v;
    const float *scale_k, *scale_v;
    const char *q;
    char *out;
    float *lse;
    float *workspace;
    uint64_t q_stride, out_stride;      // elements
    uint32_t div_mul, div_shift, block_tokens;
    uint32_t kv_heads, group;
    uint32_t window, sinks;             // window: 2^31 where there is none
    float c;                            // scale * log2(e)
};

// A row's maximum is raised, and what it has so far multiplied, only where a score is beyond it by more than this (in powers of two): weights
// are then at most 2^8, which costs no bits, and most tiles raise nothing.
constexpr float kSlack = 8.f;
// Weights of fp16 are 2^6 times those of the formula: what is small beside the largest stays above fp16's least normal for longer.
template <typename T>
constexpr float kLift = 0.f;
template <>
constexpr float kLift<F16> = 6.f;

// The largest of the values of two lanes 32 apart, and of four lanes 16 apart.
__device__ __forceinline__ float max_halves(float x) {
    const u32x2 both = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}
__device__ __forceinline__ float max_quarters(float x) {
    const u32x2 both = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return max_halves(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
}

// 4 elements of a column out of the 16-lane group's 4 rows of 16: lane i of the group names 8 bytes, row i / 4, and gets column i.
__device__ __forceinline__ u32x2 read_columns16(const char *at) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 *ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(const_cast<char *>(at))));
}
// The same of bytes: 8 rows of 16, row i / 2.
__device__ __forceinline__ u32x2 read_columns8(const char *at) {
    typedef __attribute__((address_space(3))) i32x2 *ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((ptr)(const_cast<char *>(at))));
}

// The item and head of a workgroup.  Workgroups go to the 8 XCDs in turn.  `TOGETHER`: the heads of one item, which lie side by side in
// the rows of the pool, are taken by one XCD, one after the other.  That suits heads whose part of a row is short, and not 256 bytes of it, whatever
// the window (one new token, 64 + 8 heads; us together / apart; 32 requests of 16-64 K keys: 64 bytes 292 / 431, 128 of 8 bits 515 / 585, 128 of 16 bits 510 / 580,
// 256 (24 of them) 684 / 663; 128 requests under a window of 4096: 115 / 164, 207 / 221, 204 / 217, 387 / 379).
template <bool TOGETHER>
__device__ __forceinline__ void place_of(uint32_t group, uint32_t groups, uint32_t heads, uint32_t *item, uint32_t *head) {
    if (TOGETHER && group < groups / (8 * heads) * (8 * heads)) {
        *item = group / 8 / heads * 8 + group % 8;
        *head = group / 8 % heads;
    } else {
        *item = group / heads;
        *head = group % heads;
    }
}

// Where a key lies.  Its block's number is a load, and what is loaded by that number comes an iteration later: loads are waited for in
// their order, so one that needs another's result at once would wait for all keys and values on their way, too.
struct KeyPlace {
    uint32_t block, row_in_block;
};
__device__ __forceinline__ KeyPlace find_key(const AttnArgs &a, const AttnItem &it, uint32_t place) {
    const uint32_t v = min(place, it.end - 1), t = v < it.sinks ? v : v + it.gap;
    const uint32_t b = __umulhi(2 * t, a.div_mul) >> a.div_shift;
    return {(uint32_t)a.tables[it.table + b], t - b * a.block_tokens};
}
// What a block's codes are multiplied by.
struct Scales {
    float k, v;
};
__device__ __forceinline__ Scales load_scales(const AttnArgs &a, uint32_t block, uint32_t head) {
    const uint64_t at = (uint64_t)block * a.kv_heads + head;
    return {a.scale_k[at], a.scale_v[at]};
}

// Whether every query at positions [p0, p1] sees every key at places [v0, v1].
__device__ __forceinline__ bool all_seen(const AttnArgs &a, const AttnItem &it, uint32_t v0, uint32_t v1, uint32_t p0, uint32_t p1) {
    const uint32_t t0 = v0 < it.sinks ? v0 : v0 + it.gap, t1 = v1 < it.sinks ? v1 : v1 + it.gap;
    return v1 < it.end && t1 <= p0 && (t0 + a.window > p1 || t1 < a.sinks);
}

// The places that a query at `position` sees among those before `end`: v - first < count, and v < sinks.  (The first place whose token is t or a later
// one: t up to the first tokens' end, and t - gap beyond the gap.)
struct Seen {
    uint32_t first, count, sinks;
    __device__ __forceinline__ bool operator()(uint32_t v) const { return (v - first < count) | (v < sinks); }
};
__device__ __forceinline__ Seen seen_from(const AttnArgs &a, const AttnItem &it, uint32_t position) {
    auto place = [&](uint32_t t) { return t <= it.sinks ? t : max(t, it.sinks + it.gap) - it.gap; };
    const uint32_t end = min(place(position + 1), it.end), first = place(position + 1 > a.window ? position + 1 - a.window : 0);
    return {first, end > first ? end - first : 0, min(place(a.sinks), end)};
}

// Whether some of the elements in a word, two of T or four codes, are infinite or NaN; and the word with zeros for them.
template <typename T, bool E4M3>
__device__ __forceinline__ bool odd_word(uint32_t w) {
    if (E4M3) return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
    return (w & T::kExponent) == T::kExponent || ((w >> 16) & T::kExponent) == T::kExponent;
}
template <typename T, bool E4M3>
__device__ __forceinline__ uint32_t plain_word(uint32_t w) {
    if (E4M3) {
        for (int i = 0; i < 32; i += 8)
            if (((w >> i) & 0x7fu) == 0x7fu) w &= ~(0xffu << i);
        return w;
    }
    for (int i = 0; i < 32; i += 16)
        if (((w >> i) & T::kExponent) == T::kExponent) w &= ~(0xffffu << i);
    return w;
}
template <typename T, bool E4M3, int N>
__device__ __forceinline__ bool odd_pieces(const u32x4 (&x)[N]) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) odd = odd || odd_word<T, E4M3>(x[i][j]);
    return odd;
}
template <typename T, bool E4M3, int N>
__device__ __forceinline__ void make_plain(u32x4 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = plain_word<T, E4M3>(x[i][j]);
}

// The infinities and NaN among 4 values of row `row` from `dim` on, zeros for the rest.
template <typename T, bool E4M3, int D>
__device__ __forceinline__ f32x4 odd_values(const AttnArgs &a, uint32_t head, uint32_t row, uint32_t dim) {
    const char *at = a.v + (((uint64_t)row * a.kv_heads + head) * D + dim) * (E4M3 ? 1 : 2);
    f32x2 x, y;
    if (E4M3) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(at);
        x = widen_codes<0>(w);
        y = widen_codes<1>(w);
    } else {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(at);
        x = T::widen(w[0]);
        y = T::widen(w[1]);
    }
    f32x4 e{x[0], x[1], y[0], y[1]};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (fabsf(e[i]) < __builtin_inff()) e[i] = 0.f;
    return e;
}

// 2^(m - to), where neither may be there yet (-inf)
__device__ __forceinline__ float factor(float m, float to) { return m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - to); }

// Two floats as bf16 numbers, and what these leave.
struct TwoParts {
    uint32_t first, rest;
};
__device__ __forceinline__ TwoParts two_parts(float x, float y) {
    const uint32_t first = narrow<Bf16>(x, y);
    const f32x2 there = Bf16::widen(first);
    return {first, narrow<Bf16>(x - there[0], y - there[1])};
}

// The output of one row: its sum, maximum and E unnormalised elements from `dim` on.
template <typename T, int E>
__device__ __forceinline__ void write_row(const AttnArgs &a, uint32_t token0, uint32_t row, uint32_t head, uint32_t dim, int head_dim, float l, const float (&o)[E]) {
    const uint32_t token = token0 + row / a.group, h = head * a.group + row % a.group;
    const float over = l == 0.f ? 0.f : 1.f / l;
    uint32_t w[E / 2];
#pragma unroll
    for (int i = 0; i < E; i += 2) w[i / 2] = narrow<T>(o[i] * over, o[i + 1] * over);
    char *to = a.out + 2 * (token * a.out_stride + (uint64_t)h * head_dim + dim);
    __builtin_memcpy(__builtin_assume_aligned(to, 2 * E), w, 2 * E);
}
template <typename T>
__device__ __forceinline__ void write_lse(const AttnArgs &a, uint32_t token0, uint32_t row, uint32_t head, float m, float l) {
    if (!a.lse) return;
    const uint64_t token = token0 + row / a.group, h = head * a.group + row % a.group;
    a.lse[token * a.kv_heads * a.group + h] = l == 0.f ? -__builtin_inff() : 0.69314718055994531f * (m - kLift<T> + __log2f(l));
}

// Few rows -------------------------------------------------------------------------------------------------------------------------
//
// Up to 16 * RT * HALVES rows against pieces of their keys.  The keys' and values' bytes bound it: each is read once, by one wavefront, and used
// for all rows.  The wavefronts of a workgroup take tiles of keys in turn, each with its own maximum, sum and outputs, without a
// barrier until the end, so that at any time all but the tile in work is on its way; then they are joined in the LDS.  K goes from memory
// to the registers of the matrix instructions as it lies: lane (n, g) has key n's elements of four-lane group g, and the queries are laid out
// to match.  V goes through the wavefront's own part of the LDS, which turns it.  8-bit codes become T there and here, exactly; their
// scales multiply scores (K) and join the exponent (V: with x = c s_k <q, K_t> + log2 s_v, 2^(x - m) multiplies the codes, and 2^(x - m) / s_v
// is the term of l), in 32 bits, whatever T is.  These weights span as much as the values' scales do, which is more than fp16 holds: for fp16 queries
// values are bf16 there, exactly, and a weight is two bf16 numbers, as in the kernel for many rows (one token a request: no slower; 32 requests of 21 to 42 rows, heads
// of 128: 49 us, with weights in fp16 45).  A step of 64 requests of 16-64 K tokens, 64 + 8 heads, 8 bits: 5.3 GB at 5.6 TB/s; of 128 under a
// window of 4096, 16 bits: 2.0 GB at 5.6 TB/s.
//
// Beyond 32 rows the registers do not hold a wavefront's outputs beside what is on its way, and scratch memory's loads come in order behind those of
// the next keys: there HALVES = 2, and two wavefronts take the same tile of keys, half of the rows each; what the second one loads is in the caches.
// (32 requests of 21 to 42 rows, 8-bit heads of 128: 59 us with three tiles of rows a wavefront and five such loads for each of keys, 51 so.)
template <typename T, bool E4M3, int D, int RT, int HALVES>
__global__ void __launch_bounds__(256, 2) kvl_attn_few_kernel(const AttnArgs a) {
    constexpr int KT = few_rows_tile(D), NB = KT / 16;        // keys of a tile, blocks of 16
    constexpr int RB = D * (E4M3 ? 1 : 2);                          // bytes of a row
    constexpr int PR = RB / 16;                                     // pieces of 16 bytes in it
    constexpr int VP = KT * PR / 64;                                // a lane's pieces of V
    constexpr int KP = RB / 64;                                     // a lane's pieces of K for each block
    constexpr int CH = D / 32, DC = D / 16;                         // steps of the first product; blocks of the output
    constexpr int kSwizzle = DC - 1;                                // rows of V are turned by their number, for the LDS banks' sake
    constexpr int kWaveBytes = KT * RB + (E4M3 ? KT * 12 : 0);
    constexpr int OS = D + 4;                                       // floats of an output row in the LDS
    constexpr int kBytes = 4 * (kWaveBytes > 16 * OS * 4 ? kWaveBytes : 16 * OS * 4);
    __shared__ __attribute__((aligned(16))) char lds[kBytes];
    __shared__ f32x2 state[4][RT * 16];
    typedef typename T::x8 x8;
    // what values and weights are multiplied in
    constexpr bool kTwoParts = E4M3 && T::kExponent == F16::kExponent;
    typedef std::conditional_t<kTwoParts, Bf16, T> TV;
    typedef typename TV::x8 TV8;
    // where there are several tiles of rows: queries, in the order in which the matrix instructions take them, and what each row sees
    constexpr bool kStaged = RT > 1;
    constexpr int kTiles = RT * HALVES;
    __shared__ x8 staged[kStaged ? kTiles * CH : 1][64];
    __shared__ Seen seen_of[kStaged ? kTiles * 16 : 1];

    uint32_t item, head;
    place_of<(RB < 256)>(blockIdx.x, gridDim.x, a.kv_heads, &item, &head);
    const AttnItem it = a.items[item];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 16, g = lane / 16;
    constexpr uint32_t kStreams = 4 / HALVES;
    const uint32_t half = wave % HALVES, stream = wave / HALVES;     // (half: row tiles half, half + HALVES, ..)
    char *mine = lds + wave * kWaveBytes;
    float *key_c = reinterpret_cast<float *>(mine + KT * RB), *key_log = key_c + KT, *key_over = key_log + KT;
    const uint32_t row_pitch = a.kv_heads * RB;
    const char *k_head = a.k + head * RB, *v_head = a.v + head * RB;

    f32x4 o[RT][DC];
    float m[RT], l[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -__builtin_inff();
        l[r] = 0;
#pragma unroll
        for (int d = 0; d < DC; ++d) o[r][d] = f32x4{0, 0, 0, 0};
    }

    u32x4 kr[NB][KP], kn[NB][KP], vr[VP];
    Scales scales{};
    uint32_t rows = 0;                          // of the tile on its way, a lane each
    auto fetch = [&](const KeyPlace &at) {
        rows = at.block * a.block_tokens + at.row_in_block;
        if (E4M3) scales = load_scales(a, at.block, head);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const char *from = k_head + ((uint64_t)__shfl(rows, 16 * b + n) * row_pitch + g * 16);
#pragma unroll
            for (int i = 0; i < KP; ++i) kn[b][i] = *reinterpret_cast<const u32x4 *>(from + 64 * i);
        }
#pragma unroll
        for (int i = 0; i < VP; ++i) vr[i] = *reinterpret_cast<const u32x4 *>(v_head + ((uint64_t)__shfl(rows, (i * 64 + lane) / PR) * row_pitch + lane % PR * 16));
    };

    const uint32_t tiles = half * 16 < it.n_rows ? (it.end - it.begin + KT - 1) / KT : 0;
    KeyPlace next{};
    if (stream < tiles) {
        const KeyPlace first = find_key(a, it, it.begin + stream * KT + lane % KT);
        next = find_key(a, it, it.begin + (stream + kStreams) * KT + lane % KT);
        fetch(first);
    }
    x8 q[kStaged ? 1 : CH];
    const uint32_t p0 = it.hit + it.first_row / a.group, p1 = it.hit + (it.first_row + it.n_rows - 1) / a.group;
#pragma unroll
    for (int r = 0; r < kTiles; ++r) {
        const uint32_t i = min(r * 16 + n, it.n_rows - 1), row = it.first_row + i, token = row / a.group;
        const char *from = a.q + 2 * ((it.token0 + token) * a.q_stride + (head * a.group + row % a.group) * D);
#pragma unroll
        for (int s = 0; s < CH; ++s) {
            const uint32_t dim = E4M3 ? (g + 4 * (s / 2)) * 16 + s % 2 * 8 : s * 32 + g * 8;
            if (!kStaged) q[s] = *reinterpret_cast<const x8 *>(from + 2 * dim);
            else if (wave == (uint32_t)(r * CH + s) % 4) staged[r * CH + s][lane] = *reinterpret_cast<const x8 *>(from + 2 * dim);
        }
    }
    auto seen_by = [&](uint32_t i) { return seen_from(a, it, it.hit + (it.first_row + min(i, it.n_rows - 1)) / a.group); };
    Seen seen_here{};
    if (!kStaged) seen_here = seen_by(n);
    else if (threadIdx.x < kTiles * 16) seen_of[threadIdx.x] = seen_by(threadIdx.x);
    if (kStaged) __syncthreads();
    for (uint32_t tile = stream; tile < tiles; tile += kStreams) {
        const uint32_t v0 = it.begin + tile * KT;
        const bool whole = all_seen(a, it, v0, v0 + KT - 1, p0, p1);
        // Values that only some of the rows see must not reach the others: 0 * inf is NaN.  Infinities and NaN of such a tile are added
        // apart, to the rows that see them.
        const bool odd = !whole && __any(odd_pieces<T, E4M3>(vr));
        if (odd) make_plain<T, E4M3>(vr);
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            const uint32_t row = (i * 64 + lane) / PR, s = lane % PR;
            const uint32_t to = E4M3 ? row * RB + ((s ^ (row & kSwizzle)) << 4) : row * RB + (((s >> 1) ^ (row & kSwizzle)) << 5) + ((s & 1) << 4);
            *reinterpret_cast<u32x4 *>(mine + to) = vr[i];
        }
        if (E4M3) {
            if (lane < KT) {
                const float by = in_range(scales.v);
                key_c[lane] = a.c * in_range(scales.k);
                key_log[lane] = __log2f(by);
                key_over[lane] = __builtin_amdgcn_rcpf(by);        // (to a unit in the last place of 32 bits, as the sum it goes into)
            }
        }
        __builtin_amdgcn_wave_barrier();
        const uint32_t now_rows = rows;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < KP; ++i) kr[b][i] = kn[b][i];
        // the next tile comes while this one is worked on
        if (tile + kStreams < tiles) {
            fetch(next);
            if (tile + 2 * kStreams < tiles) next = find_key(a, it, it.begin + (tile + 2 * kStreams) * KT + lane % KT);
        }
        // Row tiles one after the other, but both together over an 8-bit cache: keys and values become T once for them.
        auto work = [&](auto first, auto count) {
            constexpr int R0 = decltype(first)::value, R = decltype(count)::value;
            // scores: lane (n, g) gets row n's of keys 16 b + 4 g + i
            f32x4 s[R][NB];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int b = 0; b < NB; ++b) s[r][b] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                x8 x[R];
#pragma unroll
                for (int r = 0; r < R; ++r) x[r] = kStaged ? staged[((R0 + r) * HALVES + half) * CH + j][lane] : q[kStaged ? 0 : j];
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    x8 k;
                    if (E4M3) {
                        const uint32_t w0 = kr[b][j / 2][j % 2 * 2], w1 = kr[b][j / 2][j % 2 * 2 + 1];
                        const u32x4 w{T::template from_codes<false>(w0, 1.f), T::template from_codes<true>(w0, 1.f), T::template from_codes<false>(w1, 1.f),
                                      T::template from_codes<true>(w1, 1.f)};
                        k = __builtin_bit_cast(x8, w);
                    } else {
                        k = __builtin_bit_cast(x8, kr[b][j]);
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) s[r][b] = T::mma16(k, x[r], s[r][b]);
                }
            }
            TV8 p[R][NB / 2], p_rest[R][NB / 2];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float top = -__builtin_inff();
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const int at_key = 16 * b + 4 * g;
                    const f32x4 kc = E4M3 ? *reinterpret_cast<const f32x4 *>(key_c + at_key) : f32x4{a.c, a.c, a.c, a.c};
                    const f32x4 kl = E4M3 ? *reinterpret_cast<const f32x4 *>(key_log + at_key) : f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[r][b][i] = E4M3 ? __builtin_fmaf(s[r][b][i], kc[i], kl[i]) : s[r][b][i] * kc[i];
                }
                if (!whole) {
                    const Seen seen = kStaged ? seen_of[((R0 + r) * HALVES + half) * 16 + n] : seen_here;
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!seen(v0 + 16 * b + 4 * g + i)) s[r][b][i] = -__builtin_inff();
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[r][b][i]);
                top = max_quarters(top);
                if (__any(top > m[R0 + r] + kSlack)) {
                    const float to = fmaxf(m[R0 + r], top), f = factor(m[R0 + r], to);
                    m[R0 + r] = to;
                    l[R0 + r] *= f;
#pragma unroll
                    for (int d = 0; d < DC; ++d) o[R0 + r][d] *= f;
                }
                const float from = m[R0 + r] == -__builtin_inff() ? 0.f : m[R0 + r] - kLift<T>;
#pragma unroll
                for (int b = 0; b < NB; b += 2) {
                    u32x4 w, rest;
#pragma unroll
                    for (int bb = b; bb < b + 2; ++bb) {
                        const f32x4 over = E4M3 ? *reinterpret_cast<const f32x4 *>(key_over + 16 * bb + 4 * g) : f32x4{1, 1, 1, 1};
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const float x = __builtin_amdgcn_exp2f(s[r][bb][i] - from), y = __builtin_amdgcn_exp2f(s[r][bb][i + 1] - from);
                            if (E4M3) l[R0 + r] = __builtin_fmaf(y, over[i + 1], __builtin_fmaf(x, over[i], l[R0 + r]));
                            else l[R0 + r] += x + y;
                            if (kTwoParts) {
                                const TwoParts parts = two_parts(x, y);
                                w[bb % 2 * 2 + i / 2] = parts.first;
                                rest[bb % 2 * 2 + i / 2] = parts.rest;
                            } else {
                                w[bb % 2 * 2 + i / 2] = narrow<T>(x, y);
                            }
                        }
                    }
                    p[r][b / 2] = __builtin_bit_cast(TV8, w);
                    if (kTwoParts) p_rest[r][b / 2] = __builtin_bit_cast(TV8, rest);
                }
            }
            // outputs: lane (n, g) gets row n's elements 16 d + 4 g + i; the contraction's keys of lane group g are 4 g .. + 3 and 16 + 4 g .. + 3
#pragma unroll
            for (int u = 0; u < NB / 2; ++u)
#pragma unroll
                for (int d = 0; d < DC; ++d) {
                    u32x4 w;
                    if (E4M3) {
                        const uint32_t j = n / 2, row = 32 * u + 4 * g + (j < 4 ? j : j + 12);
                        const u32x2 c = read_columns8(mine + row * RB + ((d ^ (row & kSwizzle)) << 4) + (n & 1) * 8);
                        w = u32x4{TV::template from_codes<false>(c[0], 1.f), TV::template from_codes<true>(c[0], 1.f), TV::template from_codes<false>(c[1], 1.f),
                                  TV::template from_codes<true>(c[1], 1.f)};
                    } else {
                        const uint32_t row = 32 * u + 4 * g + n / 4;
                        const u32x2 x = read_columns16(mine + row * RB + ((d ^ (row & kSwizzle)) << 5) + (n & 3) * 8);
                        const u32x2 y = read_columns16(mine + (row + 16) * RB + ((d ^ ((row + 16) & kSwizzle)) << 5) + (n & 3) * 8);
                        w = u32x4{x[0], x[1], y[0], y[1]};
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        o[R0 + r][d] = TV::mma16(__builtin_bit_cast(TV8, w), p[r][u], o[R0 + r][d]);
                        if (kTwoParts) o[R0 + r][d] = TV::mma16(__builtin_bit_cast(TV8, w), p_rest[r][u], o[R0 + r][d]);
                    }
                }
        };
        typedef std::integral_constant<int, 0> Zero;
        typedef std::integral_constant<int, 1> One;
        const bool second = RT > 1 && (HALVES + half) * 16 < it.n_rows;
        if (E4M3 && second) {
            work(Zero{}, std::integral_constant<int, RT>{});
        } else {
            work(Zero{}, One{});
            if (!E4M3 && second) work(std::integral_constant<int, RT - 1>{}, One{});
        }
        if (odd) {
            for (uint32_t j = 0; j < KT && v0 + j < it.end; ++j) {
                const uint32_t row = __shfl(now_rows, (int)j);
#pragma unroll
                for (int d = 0; d < DC; ++d) {
                    const f32x4 e = odd_values<T, E4M3, D>(a, head, row, 16 * d + 4 * g);
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        if ((kStaged ? seen_of[(r * HALVES + half) * 16 + n] : seen_here)(v0 + j)) o[r][d] += e;
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }

    // the wavefronts' results, joined
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        l[r] += __shfl_xor(l[r], 16);
        l[r] += __shfl_xor(l[r], 32);
        if (g == 0) state[wave][r * 16 + n] = f32x2{m[r], l[r]};
    }
    float *sums = reinterpret_cast<float *>(lds);
    const uint32_t row = threadIdx.x / 16;
    constexpr int E = D / 16;
    const uint32_t dim = threadIdx.x % 16 * E;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        __syncthreads();                        // (nobody reads V, or the rows before, any more; the states are there)
        float top = -__builtin_inff();
        for (uint32_t w = half; w < 4; w += HALVES) top = fmaxf(top, state[w][r * 16 + n][0]);
        const float f = factor(m[r], top);
#pragma unroll
        for (int d = 0; d < DC; ++d) *reinterpret_cast<f32x4 *>(sums + (wave * 16 + n) * OS + 16 * d + 4 * g) = o[r][d] * f;
        __syncthreads();
#pragma unroll
        for (uint32_t hh = 0; hh < HALVES; ++hh) {
            const uint32_t i = (r * HALVES + hh) * 16 + row;
            if (i >= it.n_rows) continue;
            float most = -__builtin_inff(), sum = 0, e[E] = {};
            for (uint32_t w = hh; w < 4; w += HALVES) most = fmaxf(most, state[w][r * 16 + row][0]);
            for (uint32_t w = hh; w < 4; w += HALVES) {
                const f32x2 at = state[w][r * 16 + row];
                sum += at[1] * factor(at[0], most);
#pragma unroll
                for (int j = 0; j < E; ++j) e[j] += sums[(w * 16 + row) * OS + dim + j];
            }
            if (it.pieces == 1) {
                write_row<T, E>(a, it.token0, it.first_row + i, head, dim, D, sum, e);
                if (dim == 0) write_lse<T>(a, it.token0, it.first_row + i, head, most, sum);
            } else {
                constexpr uint32_t kFloats = kTiles * 16 * (D + 2);
                float *to = a.workspace + it.partial + (uint64_t)head * kFloats;
#pragma unroll
                for (int j = 0; j < E; ++j) to[i * D + dim + j] = e[j];
                if (dim == 0) *reinterpret_cast<f32x2 *>(to + kTiles * 16 * D + 2 * i) = f32x2{most, sum};
            }
        }
    }
}

// Many rows ------------------------------------------------------------------------------------------------------------------------
//
// 128 rows, 32 for each wavefront, against pieces of their keys in tiles of 64 that the wavefronts share in the LDS.  A tile comes by way of
// registers, while the tile before is worked on; 8-bit codes become T there, once for all rows, with their scales: exactly where these are powers
// of two, else with one more rounding to T.  fp16 holds every code times 2^-15 to 2^7 and not much more: a tile with a scale outside of that has
// its codes alone there, keys' as fp16, values' as bf16; the keys' scales multiply scores, the values' the weights, in 32 bits, and a weight is two
// bf16 numbers, the second one what the first leaves (their products with codes are exact, and a weight keeps 16 bits).
//
// The matrix instructions (37 % of the time busy) and the vector unit (46 %, most of it the exponentials and what goes with them) bound it, which
// the two wavefronts that a SIMD has registers for do not overlap well: 810 to 850 TFLOP/s (by the card) in 8-bit tails over long prefixes, heads of 128; of 64,
// 26 % and 55 %, 610 to 630 under a window.
template <typename T, bool E4M3>
__device__ __forceinline__ void codes_to_half(u32x4 w, float scale, u32x4 *x, u32x4 *y) {
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[2 * i] = T::template from_codes<false>(w[i], scale);
        e[2 * i + 1] = T::template from_codes<true>(w[i], scale);
    }
    const uint32_t bits = __float_as_uint(scale);
    if (__any((bits & 0x7fffffu) != 0)) {
        const float rest = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2 v = T::widen(e[i]);
            e[i] = narrow<T>(v[0] * rest, v[1] * rest);
        }
    }
    *x = u32x4{e[0], e[1], e[2], e[3]};
    *y = u32x4{e[4], e[5], e[6], e[7]};
}

// Scales that leave codes in fp16's range.
__device__ __forceinline__ bool suits_f16(float scale) { return scale >= 0x1p-15f && scale <= 0x1p7f; }

template <typename T, bool E4M3, int D>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) kvl_attn_many_kernel(const AttnArgs a) {
    constexpr int KT = kManyRowsTile;
    constexpr int RB = 2 * D;                                       // bytes of a row in the LDS
    constexpr int PR = D * (E4M3 ? 1 : 2) / 16;                     // pieces of a row in memory
    constexpr int RP = 256 / PR;                                    // rows that the workgroup fetches at once
    constexpr int N = KT / RP;                                      // a lane's pieces of a tile
    constexpr int CH = D / 16, DB = D / 32;                         // steps of the first product; blocks of the output
    static_assert(KT % RP == 0 && KT == 64, "whole pieces; a key a lane");
    constexpr bool kNarrow = E4M3 && T::kExponent == F16::kExponent;    // some scales do not go into T
    // Pieces of 16 bytes are turned by their row's number so that the 16 rows that lanes read of K together, and the 4 rows by 64 bytes of V, lie in
    // different banks (256 bytes of them): rows of 128 bytes take half of these each.
    auto k_turn = [](uint32_t r) { return D == 128 ? r & 15 : r >> 1 & 7; };
    auto v_turn = [](uint32_t r) { return D == 128 ? (r & 3) << 2 | (r & 1) : (r >> 1 & 1) * 5; };
    __shared__ __attribute__((aligned(16))) char lds[2][2][KT * RB];
    __shared__ uint32_t odd_tile[3];
    typedef typename T::x8 x8;

    const AttnItem it = a.items[blockIdx.x / a.kv_heads];
    const uint32_t head = blockIdx.x % a.kv_heads;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane % 32, h = lane / 32;
    const uint32_t row_pitch = a.kv_heads * PR * 16;
    const char *k_head = a.k + head * PR * 16, *v_head = a.v + head * PR * 16;
    const uint32_t fetched = threadIdx.x / PR, piece = threadIdx.x % PR;

    const uint32_t rows_before = wave * 32;
    const bool works = rows_before < it.n_rows;
    const uint32_t row = it.first_row + min(rows_before + n, it.n_rows - 1);
    const uint32_t p0 = it.hit + it.first_row / a.group, p1 = it.hit + (it.first_row + it.n_rows - 1) / a.group;
    const uint32_t w0 = it.hit + (it.first_row + min(rows_before, it.n_rows - 1)) / a.group,
                   w1 = it.hit + (it.first_row + min(rows_before + 31, it.n_rows - 1)) / a.group;
    const Seen seen = seen_from(a, it, it.hit + row / a.group);
    x8 q[CH];
    {
        const char *from = a.q + 2 * ((it.token0 + row / a.group) * a.q_stride + (head * a.group + row % a.group) * D);
#pragma unroll
        for (int s = 0; s < CH; ++s) q[s] = *reinterpret_cast<const x8 *>(from + 2 * (16 * s + 8 * h));
    }
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0;
    float m = -__builtin_inff(), l = 0;

    u32x4 kr[N], vr[N];
    Scales scales{};
    uint32_t rows = 0;                          // of the tile on its way, a lane each
    auto fetch = [&](const KeyPlace &at) {
        rows = at.block * a.block_tokens + at.row_in_block;
        if (E4M3) scales = load_scales(a, at.block, head);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t from = (uint64_t)__shfl(rows, i * RP + fetched) * row_pitch + piece * 16;
            kr[i] = *reinterpret_cast<const u32x4 *>(k_head + from);
            vr[i] = *reinterpret_cast<const u32x4 *>(v_head + from);
        }
    };
    // Where a lane reads the first of its 16 bytes of K, and of its 8 of V, of a tile: the others are there with bits turned.
    uint32_t k_at = n * RB + ((h ^ k_turn(n)) << 4);
    uint32_t v_at = (4 * h + lane % 16 / 4) * RB + (((2 * (lane / 16 % 2) + lane % 4 / 2) ^ v_turn(lane % 16 / 4)) << 4) + lane % 2 * 8;
    if (threadIdx.x < 3) odd_tile[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t tiles = (it.end - it.begin + KT - 1) / KT;
    KeyPlace next{};
    if (tiles) {
        const KeyPlace first = find_key(a, it, it.begin + lane);
        next = find_key(a, it, it.begin + KT + lane);
        fetch(first);
    }
    for (uint32_t tile = 0; tile < tiles; ++tile) {
        const uint32_t v0 = it.begin + tile * KT;
        char *k_lds = lds[tile % 2][0], *v_lds = lds[tile % 2][1];
        // (infinities and NaN among values that not all rows see: as in the kernel above)
        if (!all_seen(a, it, v0, v0 + KT - 1, p0, p1) && odd_pieces<T, E4M3>(vr)) {
            odd_tile[tile % 3] = 1;
            make_plain<T, E4M3>(vr);
        }
        const Scales by{in_range(scales.k), in_range(scales.v)};
        // (the same in all wavefronts: each has every key's scales)
        const bool apart = kNarrow && __builtin_amdgcn_readfirstlane(__any(!suits_f16(by.k) || !suits_f16(by.v)));
        // (one branch around all of it: 32-K tails in fp16 784 us, one at each value 812, without the second form 768)
        auto convert = [&](auto key_type, auto value_type, Scales times) {
            typedef decltype(key_type) TK;
            typedef decltype(value_type) TV;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t r = i * RP + fetched;
                u32x4 x, y;
                codes_to_half<TK, E4M3>(kr[i], __shfl(times.k, (int)r), &x, &y);
                *reinterpret_cast<u32x4 *>(k_lds + r * RB + (((2 * piece) ^ k_turn(r)) << 4)) = x;
                *reinterpret_cast<u32x4 *>(k_lds + r * RB + (((2 * piece + 1) ^ k_turn(r)) << 4)) = y;
                codes_to_half<TV, E4M3>(vr[i], __shfl(times.v, (int)r), &x, &y);
                *reinterpret_cast<u32x4 *>(v_lds + r * RB + (((2 * piece) ^ v_turn(r)) << 4)) = x;
                *reinterpret_cast<u32x4 *>(v_lds + r * RB + (((2 * piece + 1) ^ v_turn(r)) << 4)) = y;
            }
        };
        if (!E4M3) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t r = i * RP + fetched;
                *reinterpret_cast<u32x4 *>(k_lds + r * RB + ((piece ^ k_turn(r)) << 4)) = kr[i];
                *reinterpret_cast<u32x4 *>(v_lds + r * RB + ((piece ^ v_turn(r)) << 4)) = vr[i];
            }
        } else if (apart) {
            convert(T{}, Bf16{}, Scales{1.f, 1.f});
        } else {
            convert(T{}, T{}, by);
        }
        if (tile + 1 < tiles) {
            fetch(next);
            if (tile + 2 < tiles) next = find_key(a, it, v0 + 2 * KT + lane);
        }
        __syncthreads();
        const bool odd = odd_tile[tile % 3] != 0;
        if (threadIdx.x == 0) odd_tile[(tile + 2) % 3] = 0;

        asm volatile("" : "+v"(k_at), "+v"(v_at));      // (the addresses made of them are made anew for each tile: registers are short)
        // a tile that none of the wavefront's rows sees
        const uint32_t v1 = min(v0 + KT, it.end) - 1;
        const uint32_t t0 = v0 < it.sinks ? v0 : v0 + it.gap, t1 = v1 < it.sinks ? v1 : v1 + it.gap;
        if (!works || t0 > w1 || (t1 + a.window <= w0 && t0 >= a.sinks)) continue;
        const bool whole = all_seen(a, it, v0, v0 + KT - 1, w0, w1);

        // scores: lane (n, h) gets row n's of keys 32 b + 8 (i / 4) + 4 h + i % 4
        f32x16 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const x8 k = *reinterpret_cast<const x8 *>(k_lds + 32 * b * RB + (k_at ^ j << 5));
                s[b] = T::mma32(k, q[j], s[b]);
            }
        }
        // what the lane of key `key` + 4 h has (its address made anew each time, too)
        auto of_key = [&](float x, int key) {
            int at = (int)(16 * h);
            asm volatile("" : "+v"(at));
            return __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(at + 4 * key, (int)__float_as_uint(x)));
        };
        if (apart) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] *= of_key(by.k, 32 * b + 8 * (i / 4) + i % 4);
        }
        if (!whole) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (!seen(v0 + 4 * h + 32 * b + 8 * (i / 4) + i % 4)) s[b][i] = -__builtin_inff();
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = max_halves(top) * a.c;
        if (__any(top > m + kSlack)) {
            const float to = fmaxf(m, top), f = factor(m, to);
            m = to;
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        const float from = m == -__builtin_inff() ? 0.f : kLift<T> - m;
        // the weights of keys 16 u + 8 (i / 4) + 4 h + i % 4 and the next, i even
        auto weights = [&](int u, int i) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u / 2][8 * (u % 2) + i], a.c, from));
            const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u / 2][8 * (u % 2) + i + 1], a.c, from));
            l += x + y;
            return f32x2{x, y};
        };
        auto values = [&](int u, int d) {
            const char *at = v_lds + 16 * u * RB + (v_at ^ d << 6);
            const u32x2 x = read_columns16(at), y = read_columns16(at + 8 * RB);
            return u32x4{x[0], x[1], y[0], y[1]};
        };
        // outputs: lane (n, h) gets row n's elements 32 d + 8 (i / 4) + 4 h + i % 4
        if (apart) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                u32x4 first, rest;
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const int key = 16 * u + 8 * (i / 4) + i % 4;
                    const f32x2 x = weights(u, i);
                    const TwoParts w = two_parts(x[0] * of_key(by.v, key), x[1] * of_key(by.v, key + 1));
                    first[i / 2] = w.first;
                    rest[i / 2] = w.rest;
                }
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const Bf16::x8 v = __builtin_bit_cast(Bf16::x8, values(u, d));
                    o[d] = Bf16::mma32(v, __builtin_bit_cast(Bf16::x8, first), o[d]);
                    o[d] = Bf16::mma32(v, __builtin_bit_cast(Bf16::x8, rest), o[d]);
                }
            }
        }
        if (kNarrow) {          // (a branch after the other: outputs of one stay where they are for the other)
#pragma unroll
            for (int d = 0; d < DB; ++d) asm volatile("" : "+v"(o[d]));
        }
        if (!apart) {
            x8 p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const f32x2 x = weights(u, i);
                    w[i / 2] = narrow<T>(x[0], x[1]);
                }
                p[u] = __builtin_bit_cast(x8, w);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] = T::mma32(__builtin_bit_cast(x8, values(u, d)), p[u], o[d]);
        }
        if (odd) {
            for (uint32_t j = 0; j < KT && v0 + j < it.end; ++j) {
                const KeyPlace place = find_key(a, it, v0 + j);
                const uint32_t pool_row = place.block * a.block_tokens + place.row_in_block;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f32x4 e = odd_values<T, E4M3, D>(a, head, pool_row, 32 * d + 2 * i + 4 * h);
                        if (seen(v0 + j))
#pragma unroll
                            for (int x = 0; x < 4; ++x) o[d][i + x] += e[x];
                    }
            }
        }
    }

    l += __shfl_xor(l, 32);
    const uint32_t i = rows_before + n;
    if (i >= it.n_rows) return;
    if (it.pieces == 1) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4) {
                const float e[4] = {o[d][x], o[d][x + 1], o[d][x + 2], o[d][x + 3]};
                write_row<T, 4>(a, it.token0, row, head, 32 * d + 2 * x + 4 * h, D, l, e);
            }
        if (h == 0) write_lse<T>(a, it.token0, row, head, m, l);
        return;
    }
    constexpr uint32_t kFloats = 128 * (D + 2);
    float *to = a.workspace + it.partial + (uint64_t)head * kFloats;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int x = 0; x < 16; x += 4) *reinterpret_cast<f32x4 *>(to + i * D + 32 * d + 2 * x + 4 * h) = f32x4{o[d][x], o[d][x + 1], o[d][x + 2], o[d][x + 3]};
    if (h == 0) *reinterpret_cast<f32x2 *>(to + 128 * D + 2 * i) = f32x2{m, l};
}

// Rows whose keys were cut ---------------------------------------------------------------------------------------------------------
//
// WAVES wavefronts a row, D / 64 elements a lane: one where there are few pieces, four, a quarter of the pieces each, where there are many
// (64 pieces for 32 rows, 8-bit step of one long request: 69 us with one and 8 pieces on their way).
template <typename T, int D, int WAVES>
__global__ void __launch_bounds__(256) kvl_attn_join_kernel(const AttnArgs a, const JoinItem *joins, uint32_t groups) {
    constexpr int E = D / 64, ROWS = 4 / WAVES;
    __shared__ float parts[4][64 * E + 2];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const JoinItem it = joins[blockIdx.x / groups / a.kv_heads];
    const uint32_t head = blockIdx.x / groups % a.kv_heads, i = blockIdx.x % groups * ROWS + wave / WAVES;
    if (i >= it.n_rows) return;                         // (all wavefronts of the row)
    const uint32_t floats = it.tile_rows * (D + 2);
    const uint64_t pitch = (uint64_t)a.kv_heads * floats;
    const float *from = a.workspace + it.partial + (uint64_t)head * floats;
    float m = -__builtin_inff(), l = 0, e[2] = {0, 0};
    for (uint32_t first = wave % WAVES; first < it.pieces; first += 64 * WAVES) {
        const uint32_t some = min(64u, (it.pieces - first + WAVES - 1) / WAVES);
        f32x2 state{-__builtin_inff(), 0};
        if (lane < some) state = *reinterpret_cast<const f32x2 *>(from + (first + lane * WAVES) * pitch + it.tile_rows * D + 2 * i);
        float top = state[0];
#pragma unroll
        for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float to = fmaxf(m, top), f = factor(m, to), mine = factor(state[0], to);
        m = to;
        float sum = state[1] * mine;
#pragma unroll
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        l = l * f + sum;
        e[0] *= f;
        e[1] *= f;
        const float *rows = from + first * pitch + i * D + lane * E;
        const uint64_t step = WAVES * pitch;
        for (uint32_t k = 0; k < some; k += 8) {
            float x[8][2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float *at = rows + min(k + j, some - 1) * step;
                x[j][0] = at[0];
                x[j][1] = at[E - 1];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float by = k + j < some ? __shfl(mine, (int)(k + j)) : 0.f;
                e[0] = __builtin_fmaf(x[j][0], by, e[0]);
                if (E == 2) e[1] = __builtin_fmaf(x[j][1], by, e[1]);
            }
        }
    }
    if (WAVES > 1) {
        parts[wave][lane * E] = e[0];
        if (E == 2) parts[wave][lane * E + E - 1] = e[1];
        if (lane == 0) {
            parts[wave][64 * E] = m;
            parts[wave][64 * E + 1] = l;
        }
        __syncthreads();
        if (wave) return;
        float top = m;
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, parts[w][64 * E]);
        const float f = factor(m, top);
        l *= f;
        e[0] *= f;
        e[1] *= f;
        for (int w = 1; w < WAVES; ++w) {
            const float by = factor(parts[w][64 * E], top);
            l += by * parts[w][64 * E + 1];
            e[0] = __builtin_fmaf(by, parts[w][lane * E], e[0]);
            if (E == 2) e[1] = __builtin_fmaf(by, parts[w][lane * E + E - 1], e[1]);
        }
        m = top;
    }
    const uint32_t row = it.first_row + i, token = it.token0 + row / a.group, h = head * a.group + row % a.group;
    const float over = l == 0.f ? 0.f : 1.f / l;
    const uint32_t w = narrow<T>(e[0] * over, e[1] * over);
    char *to = a.out + 2 * (token * a.out_stride + (uint64_t)h * D + lane * E);
    if (E == 2) *reinterpret_cast<uint32_t *>(to) = w;
    else *reinterpret_cast<uint16_t *>(to) = (uint16_t)w;
    if (lane == 0) write_lse<T>(a, it.token0, row, head, m, l);
}

}  // namespace kvl
