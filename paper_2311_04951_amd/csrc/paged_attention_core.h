// Attention of the new rows over the pages of a key-value cache: the kernel, and what it shares with the other kernels of such a cache
// (paged.hip).  Compiled for a storage type and head size at a time (paged_attention_*.hip).
//
// Positions of a sequence are numbered slots 0 .. n-1; slot s lives in page table[b][s / page] at s % page (page: a power of two >= 16).
// Within a page a position's keys (and values) of one head are contiguous; pages, heads and slots are `*_stride` elements apart.
#pragma once
#include "ss_device.h"
#include "ss_paged.h"
#include <algorithm>

namespace ss {

namespace {

constexpr float MINUS_INF = -__builtin_inff();

// A row of this running maximum and sum of weights has seen nothing, and is zero.  (Scores of NaN leave no maximum either, but a sum of NaN.)
__device__ __forceinline__ bool saw_nothing(float top, float l) { return top == MINUS_INF && l == 0.f; }

// The hardware's base-2 exponential: a weight below 2^-126 is zero
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// Weight of a score beside another one (a row's maximum)
__device__ __forceinline__ float weight_of(float score, float top, float scale_log2e) { return exp2_((score - top) * scale_log2e); }

__device__ __forceinline__ void flag(int32_t *status, int bit) {
    if (status) atomicOr(status, bit);
}

// Positions of sequence b, `pending` of them appended behind its length; never more than the table and the host's bound hold.
__device__ __forceinline__ int positions_of(const PagedArgs &kv, int b, int pending, int max_n) {
    const int len = kv.len[b];
    if (len < 0) return 0;
    const long long n = (long long)len + pending;
    const long long cap = min((long long)kv.max_pages << kv.page_bits, (long long)max_n);
    if (n > cap) {
        if (threadIdx.x == 0) flag(kv.status, PAGED_BAD_LENGTH);
        return (int)cap;
    }
    return (int)n;
}

// ------------------------------------------------------------------------------------------ attention
//
// Row x of a key head's GM = G * M query rows (x / M: query head of the group, x % M: new row) sees slots 0 .. n - M + x % M:
//   s_j = q . k_j,  p_j = exp2(c (s_j - max)) / sum with c = scale log2(e),  o = sum_j p_j v_j,  weight[j] += sum over x of p_j
// The difference is taken before it is scaled: the largest weight is exactly 1 and those that count are exact to a few units of 2^-24 however large the
// scores are.  (One fused multiply-add, c s_j less a rounded c max, leaves what was rounded off in every exponent: from scores of 2^34 on sums overflow.
// It saves a hundredth, us: 16 rows of 5 x 8 heads, 4 x 2999 positions, 41.2 | 41.7, 16 of 8 x 8 at 30000 62.5 | 63.2; its errors are the same.)  c is
// positive (of a negative scale the queries' signs are turned).
//
// A wavefront takes STEP positions at a time in tiles of 16 (a tile lies in one page).  S^T = K Q^T by MFMA with the keys as the A operand, 16
// query rows as B: lane (c, g) receives the scores of row c at positions 16 u + 4 g + r (u tile, r register).  P V takes the same lane's
// values as its B operand if contraction index (g, t = 4 u + r) stands for position 16 u + 4 g + r, so that nothing moves between lanes;
// its A operand is V^T: a lane loads VE consecutive elements of positions 16 u + 4 g + r and supplies element e of each as the row of
// output tile e, which therefore holds head elements VE * row + e.  Keys and values stay as they are appended, no transposed copy.
//
// Both go through the wavefront's own ring in LDS, a contiguous kilobyte to a load-to-LDS instruction where a page's slots are contiguous.
// Unit (16 bytes) p of row r of a tile holds unit p xor swizzle(r) of the key, so that sixteen rows are read from different banks.
template <typename T, int HD> struct PagedShape {
    static constexpr int E = Traits<T>::E, KB = 4 * E, NKC = HD / KB, NDT = HD / 16;
    static constexpr int VE = HD / 16 < E ? HD / 16 : E, NCG = NDT / VE; // elements of a value row that a lane reads at once, and how often
    static constexpr int VW = VE * (int)sizeof(T) / 4;                  // ... in words
    static constexpr int NU = sizeof(T) == 2 ? 2 : 1, STEP = 16 * NU;   // tiles and positions of a step
    static constexpr int ROW = HD * (int)sizeof(T), UPR = ROW / 16;     // bytes and 16-byte units of a row
    static constexpr int RPI = 64 / UPR, IPT = 16 / RPI;                // rows of a load instruction, instructions of a tile
    static constexpr int HALF = STEP * ROW;                             // bytes of a step's keys
    static constexpr int PER = HALF / 1024;                             // ... in load instructions
    static __device__ __forceinline__ int swizzle(int r) { return UPR >= 8 ? r & (UPR - 1) & 15 : (r >> 1) & 3; }
};
// One or two tiles of query rows to a wavefront, two wavefronts to a SIMD, a workgroup to a compute unit.  (Three tiles need more registers and so
// one wavefront to a SIMD, which waits for itself; us, three | two: 16 rows of 16 x 8 heads, 4 sequences of 3000 positions 118 | 80, in fp32
// 229 | 151; 16 of 8 x 8 at 30000 positions 128 | 106; 9 of 5 x 8 40.2 | 35.9; 16 of 5 x 8, where the sixth tile is empty, 51.2 | 52.5.)
constexpr int ATTN_WAVES = 8, ATTN_RING = 16384;
constexpr int attn_block(int dtype) { return ATTN_WAVES * (dtype ? 32 : 16); } // positions that a workgroup takes at a time

template <int W> __device__ __forceinline__ void lds_words(uint32_t (&d)[W], const unsigned char *p) {
    if constexpr (W == 1) {
        d[0] = *reinterpret_cast<const uint32_t *>(p);
    } else {
        typedef uint32_t vec __attribute__((ext_vector_type(W)));
        const vec x = *reinterpret_cast<const vec *>(p);
#pragma unroll
        for (int i = 0; i < W; ++i) d[i] = x[i];
    }
}

template <int QP> struct QueryChunk { u32x4 p[QP]; };
template <typename T, int QP> __device__ __forceinline__ f32x4 mma_q(f32x4 acc, u32x4 a, const QueryChunk<QP> &b) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < QP; ++i)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b.p[i]), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(a[j]), u2f(b.p[0][j]), acc, 0, 0, 0);
    }
    return acc;
}

// o += V^T P over the positions of a step
template <int HD> __device__ __forceinline__ void mma_pv(f32x4 (&o)[HD / 16], const uint32_t (&v)[8][PagedShape<bf16_t, HD>::NCG][PagedShape<bf16_t, HD>::VW],
                                                        const float (&p)[8], bf16_t) {
    typedef PagedShape<bf16_t, HD> S;
    const Act<bf16_t> P = pack_act(p, bf16_t{}); // hi + lo: a weight keeps 16 bits, so that the output's own rounding is what is left
#pragma unroll
    for (int cg = 0; cg < S::NCG; ++cg)
#pragma unroll
        for (int e = 0; e < S::VE; ++e) {
            u32x4 a;
#pragma unroll
            for (int j = 0; j < 4; ++j) // element e of positions t = 2j, 2j + 1
                a[j] = __builtin_amdgcn_perm(v[2 * j + 1][cg][e / 2], v[2 * j][cg][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
            o[cg * S::VE + e] = mma(o[cg * S::VE + e], a, P);
        }
}
template <int HD> __device__ __forceinline__ void mma_pv(f32x4 (&o)[HD / 16], const uint32_t (&v)[4][PagedShape<float, HD>::NCG][PagedShape<float, HD>::VW],
                                                        const float (&p)[4], float) {
    typedef PagedShape<float, HD> S;
#pragma unroll
    for (int cg = 0; cg < S::NCG; ++cg)
#pragma unroll
        for (int e = 0; e < S::VE; ++e)
#pragma unroll
            for (int t = 0; t < 4; ++t) o[cg * S::VE + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(u2f(v[t][cg][e]), p[t], o[cg * S::VE + e], 0, 0, 0);
}

// Whether a word of values holds an infinity or a NaN
__device__ __forceinline__ bool not_finite(uint32_t w, bf16_t) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool not_finite(uint32_t w, float) { return (w & 0x7f800000u) == 0x7f800000u; }

// ... and the word without them (nothing: without anything)
__device__ __forceinline__ uint32_t finite_part(uint32_t w, bool nothing, bf16_t) {
    const uint32_t low = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu, high = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
    return nothing ? 0u : low | high;
}
__device__ __forceinline__ uint32_t finite_part(uint32_t, bool, float) { return 0u; }

template <typename T, int VE> __device__ __forceinline__ void store_out(const PagedAttnArgs &a, size_t at, const float (&x)[VE]) {
    if constexpr (VE == 1) {
        ((T *)a.out)[at] = to_storage<T>(x[0]);
        if constexpr (sizeof(T) == 2) {
            if (a.out_lo) ((T *)a.out_lo)[at] = to_storage<T>(x[0] - to_f32(to_storage<T>(x[0])));
        }
    } else {
        store_cols((T *)a.out + at, x);
        if constexpr (sizeof(T) == 2) {
            if (a.out_lo) {
                float rest[VE];
#pragma unroll
                for (int e = 0; e < VE; ++e) rest[e] = x[e] - bf16_bits_to_f32(bf16_rne(x[e]));
                store_cols((T *)a.out_lo + at, rest);
            }
        }
    }
}

// 32-bit words that no kernel of this launch writes, by scalar loads (a vector load would be waited for behind all keys and values in flight)
__device__ __forceinline__ int ld_uniform(const int32_t *p) {
    typedef const int32_t __attribute__((address_space(4))) * cptr;
    return *(cptr)(uintptr_t)p;
}

template <typename T> __device__ __forceinline__ const T *uniform(const T *p) {
    const uint64_t x = (uint64_t)p;
    return (const T *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x));
}

// The positions of all sequences, each rounded up to blocks, times the key heads: one long row of blocks (fewer than 2^31: the host checks),
// sequence by sequence and head by head, of which every workgroup takes an equal part, wherever that begins and ends.  With several blocks of
// query rows a part has as many workgroups, eight apart and so on one XCD, which walk over the same keys and values at the same time and find
// them in its L2.
__device__ __forceinline__ int blocks_of(int n, int block) { return n > 0 ? (n + block - 1) / block : 1; } // (an idle place: one, which writes its zeros)
__device__ __forceinline__ int wave_scan(int x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int t = __shfl_up(x, d);
        if ((int)(threadIdx.x & 63) >= d) x += t;
    }
    return x;
}
// Blocks of one unit in all sequences; those in front of sequence `me`, where `me` is one.
__device__ __forceinline__ int count_blocks(const PagedAttnArgs &a, int block, int me, int &before) {
    before = 0;
    if (a.kv.B == 1) return blocks_of(positions_of(a.kv, 0, a.pending, a.max_n), block);
    int total = 0;
    for (int i = 0; i < a.kv.B; i += 64) {
        const int b = i + (threadIdx.x & 63);
        const int own = b < a.kv.B ? blocks_of(positions_of(a.kv, b, a.pending, a.max_n), block) : 0, upto = wave_scan(own);
        if (me >= i && me < i + 64) before = total + __shfl(upto - own, me - i);
        total += __shfl(upto, 63);
    }
    return total;
}
__device__ __forceinline__ int share_of(const PagedAttnArgs &a, int total) { return (total + a.workgroups - 1) / a.workgroups; }
// sequence that block t (of one unit) lies in, and the blocks in front of it
__device__ __forceinline__ int find_sequence(const PagedAttnArgs &a, int block, int t, int &before) {
    before = 0;
    int base = 0;
    for (int i = 0; i < a.kv.B && a.kv.B > 1; i += 64) {
        const int b = i + (threadIdx.x & 63);
        const int own = b < a.kv.B ? blocks_of(positions_of(a.kv, b, a.pending, a.max_n), block) : 0, upto = base + wave_scan(own);
        const unsigned long long behind = __ballot(b < a.kv.B && upto > t);
        if (behind) {
            const int l = __ffsll(behind) - 1;
            before = __shfl(upto - own, l);
            return i + l;
        }
        base = __shfl(upto, 63);
    }
    return 0;
}

// The scores that rows first, first + step, .. (at most 8 of the GM) gave four slots from s on, and what they make of them; the requests do not
// depend on the rows' statistics
struct SlotScores {
    f32x4 v[8];
};
__device__ __forceinline__ void load_scores(const PagedAttnArgs &a, int head, int s, int first, int step, SlotScores &t) {
    const float *sc = a.scores + (size_t)head * a.GM * a.ld_scores + s;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (first + j * step < a.GM) t.v[j] = *reinterpret_cast<const f32x4 *>(sc + (size_t)(first + j * step) * a.ld_scores);
}
__device__ __forceinline__ void sum_scores(const PagedAttnArgs &a, int first, int step, const float *m, const float *linv, const SlotScores &t, f32x4 &sum) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (first + j * step < a.GM) {
            const float top = m[first + j * step], l = linv[first + j * step];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += weight_of(t.v[j][i], top, a.scale_log2e) * l;
        }
}
// A row takes nothing from a slot that it does not see, a row of NaN neither, although a weight of zero times its reciprocal sum is NaN: where a sum
// of the newest slots is NaN, it is made again without what is hidden.
__device__ __forceinline__ void sum_seen(const PagedAttnArgs &a, int head, int s, int n, int first, int step, const float *m, const float *linv, f32x4 &sum) {
    const int over = s + 3 - (n - a.M); // slots of the four behind the last that every row sees
    if (over <= 0 || !(isnan(sum[0]) || isnan(sum[1]) || isnan(sum[2]) || isnan(sum[3]))) return;
    sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int x = first; x < a.GM; x += step) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(a.scores + ((size_t)head * a.GM + x) * a.ld_scores + s);
        const int last = 3 - over + x % a.M; // of the four, that the row sees
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i <= last) sum[i] += weight_of(v[i], m[x], a.scale_log2e) * linv[x];
    }
}
// Where slots s .. s + 3 keep their weights (they are in one page); -1: nowhere
__device__ __forceinline__ int64_t weights_at(const PagedArgs &kv, int b, int hk, int s) {
    const int page = kv.table[(size_t)b * kv.max_pages + (s >> kv.page_bits)];
    return (unsigned)page < (unsigned)kv.n_pages ? (((int64_t)page * kv.Hk + hk) << kv.page_bits) + (s & ((1 << kv.page_bits) - 1)) : -1;
}
__device__ __forceinline__ void add_weights(const PagedAttnArgs &a, int64_t at, int s, int n, f32x4 old, f32x4 sum) {
    if (at < 0) return;
    if (s + 4 <= n) {
        *reinterpret_cast<f32x4 *>(a.weight_out + at) = old + sum;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (s + i < n) a.weight_out[at + i] = old[i] + sum[i];
}

// Waits until at most N requests are in flight, or N and `scores` stores of scores
template <int N> __device__ __forceinline__ void wait_behind_at_most() { wait_vmcnt_at_most<(N < 63 ? N : 63)>(); }
template <int N, int ALL, int SOME> __device__ __forceinline__ void wait_behind(bool stored, bool all) {
    if (!stored) wait_behind_at_most<N>();
    else if (all) wait_behind_at_most<N + ALL>();
    else wait_behind_at_most<N + SOME>();
}

// WHOLE: a workgroup takes one unit of one sequence, and its result is the output.  Otherwise parts of equal size (above); what ends or begins
// inside a head goes to the partials, 2 w for a part's first piece and 2 w + 1 for a last one that starts its head, and paged_join_kernel joins.
//
// One token over 200000 positions of 8 key heads reads 819 MB in 124 us (6.6 TB/s, with the join 128): the memory bounds it, and so it does any call of
// one tile of rows over more than some ten megabytes.  With weights 8 x 9 rows at 4105 positions (548 MB) take 108 + 13 us, without 90.  Two tiles of
// rows are bound by vector instructions in bf16 and by the matrix instructions in fp32: 16 rows of 16 x 8 heads at 4 x 3000 positions 50 us without weights,
// 0.38 PFLOP/s of products (hi and lo), matrix units busy a sixth of the time; in fp32 129 us, 98 TFLOP/s, busy 70 % of the time.
template <typename T, int HD, int RT, int QP, bool WHOLE, bool W>
__global__ __launch_bounds__(ATTN_WAVES * 64) void paged_attn_kernel(PagedAttnArgs a) {
    typedef PagedShape<T, HD> S;
    constexpr int NW = ATTN_WAVES, RING = ATTN_RING, NDT = S::NDT, NKC = S::NKC, NT = 4 * S::NU, STAGES = RING / (2 * S::HALF), BLOCK = NW * S::STEP;
    static_assert(STAGES >= 1 && RING == STAGES * 2 * S::HALF && S::HALF == NDT * 4 * 64 * 4, "the merge of a row tile takes the last values' place");
    constexpr int STORES = W ? STAGES * S::NU : 0; // of scores, in STAGES steps and to a row tile
    __shared__ __align__(1024) unsigned char lds[NW * RING];
    __shared__ float sm_m[NW][RT][16], sm_l[NW][RT][16], fin_m[RT * 16], fin_l[RT * 16];
    const PagedArgs &kv = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int page_mask = (1 << kv.page_bits) - 1;
    const int part = blockIdx.x / 8 / a.rowblocks * 8 + blockIdx.x % 8, rowblock = WHOLE ? blockIdx.x / kv.Hk % a.rowblocks : blockIdx.x / 8 % a.rowblocks;
    unsigned char *ring = lds + wave * RING;
    const uint32_t ring_at = lds_address(ring);
    uint32_t request[S::IPT]; // bytes from a tile's first row to what this lane requests
#pragma unroll
    for (int i = 0; i < S::IPT; ++i) {
        const int r = i * S::RPI + lane / S::UPR;
        request[i] = (uint32_t)r * (uint32_t)kv.slot_stride * (uint32_t)sizeof(T) + (uint32_t)((lane % S::UPR) ^ S::swizzle(r)) * 16u;
    }

    int at_b = 0, t = 0, t_end = 0, before = 0;
    if (WHOLE) {
        at_b = blockIdx.x / kv.Hk / a.rowblocks;
    } else {
        int none;
        const int total = __builtin_amdgcn_readfirstlane(count_blocks(a, BLOCK, -1, none)) * kv.Hk, share = share_of(a, total);
        t = part * share;
        if (part >= (total + share - 1) / share) return;
        t_end = min(share, total - t) + t;
        at_b = __builtin_amdgcn_readfirstlane(find_sequence(a, BLOCK, t / kv.Hk, before)); // (t / Hk lies in the same sequence as t)
        before = __builtin_amdgcn_readfirstlane(before) * kv.Hk;
    }
    struct Piece { // blocks k0 .. k1 - 1 of the nb of sequence b's n positions, for a key head; the wavefront's first position, its steps
        int b, hk, n, nb, k0, k1, begin, end, first, steps;
    };
    auto piece_at = [&]() {
        Piece p;
        p.b = at_b;
        p.n = __builtin_amdgcn_readfirstlane(positions_of(kv, at_b, a.pending, a.max_n));
        p.nb = blocks_of(p.n, BLOCK);
        p.hk = WHOLE ? (int)blockIdx.x % kv.Hk : __builtin_amdgcn_readfirstlane((t - before) / p.nb);
        p.k0 = WHOLE ? 0 : t - before - p.hk * p.nb;
        p.k1 = WHOLE ? p.nb : min(p.nb, p.k0 + t_end - t);
        p.begin = p.k0 * BLOCK;
        p.end = min(p.k1 * BLOCK, p.n);
        p.first = p.begin + wave * S::STEP;
        p.steps = __builtin_amdgcn_readfirstlane(p.first < p.end ? (p.end - p.first + NW * S::STEP - 1) / (NW * S::STEP) : 0);
        return p;
    };
    auto page_of = [&](const Piece &p, int slot) { return ld_uniform(kv.table + (size_t)p.b * kv.max_pages + (min(slot, p.n - 1) >> kv.page_bits)); };
    struct Pages { // of a step's tiles
        int id[S::NU];
    };
    auto pages_at = [&](const Piece &p, int p0) {
        Pages g;
#pragma unroll
        for (int u = 0; u < S::NU; ++u) g.id[u] = page_of(p, p0 + 16 * u);
        return g;
    };
    auto missing = [&](const Pages &g) { // bit u: tile u lies in a page that does not exist
        unsigned bits = 0;
#pragma unroll
        for (int u = 0; u < S::NU; ++u) bits |= (unsigned)((unsigned)g.id[u] >= (unsigned)kv.n_pages) << u;
        return bits;
    };
    auto request_half = [&](const Piece &p, const void *pool, const Pages &g, int p0, uint32_t to) { // keys or values of a step
#pragma unroll
        for (int u = 0; u < S::NU; ++u) {
            const int page = (unsigned)g.id[u] >= (unsigned)kv.n_pages ? 0 : g.id[u]; // (masked below)
            const T *from = uniform((const T *)pool + p.hk * kv.head_stride + page * kv.page_stride + ((p0 + 16 * u) & page_mask) * kv.slot_stride);
            if (RT == 1 || a.stream) { // (a single tile of query rows is all there is)
#pragma unroll
                for (int i = 0; i < S::IPT; ++i) dma16<true>(from, request[i], to + (u * S::IPT + i) * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < S::IPT; ++i) dma16(from, request[i], to + (u * S::IPT + i) * 1024);
            }
        }
    };
    // The first steps of a piece, but the last of these values: their place is the merge's.  `bad`: what is missing, NU bits to a stage
    auto request_first = [&](const Piece &p, unsigned &bad, Pages &last) {
        bad = 0;
#pragma unroll
        for (int i = 0; i < STAGES; ++i)
            if (i < p.steps) {
                const int p0 = p.first + i * NW * S::STEP;
                last = pages_at(p, p0);
                bad |= missing(last) << i * S::NU;
                request_half(p, kv.k, last, p0, ring_at + i * 2 * S::HALF);
                if (i < STAGES - 1) request_half(p, kv.v, last, p0, ring_at + i * 2 * S::HALF + S::HALF);
            }
    };
    Piece piece = piece_at(), next = piece;
    unsigned bad, next_bad = 0;
    Pages pages{}, next_pages{};
    request_first(piece, bad, pages);
    bool first_piece = true, more = false;
    for (;;) {
        if (STAGES - 1 < piece.steps) request_half(piece, kv.v, pages, piece.first + (STAGES - 1) * NW * S::STEP, ring_at + (2 * STAGES - 1) * S::HALF);
        const int b = piece.b, hk = piece.hk, x0 = rowblock * (16 * RT), n = piece.n, begin = piece.begin, end = piece.end, first = piece.first, steps = piece.steps;
        const size_t row0 = (size_t)(b * kv.Hk + hk) * a.GM;

        QueryChunk<QP> q[RT][NKC];
        int limit[RT]; // last slot that row c of tile rt sees
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int x = min(x0 + rt * 16 + c, a.GM - 1), h = x / a.M, m = x - h * a.M;
            limit[rt] = n - a.M + m;
            const size_t at = (size_t)(b * a.M + m) * a.ldq + (size_t)(hk * a.G + h) * a.q_head + g * S::E;
#pragma unroll
            for (int kc = 0; kc < NKC; ++kc) {
                q[rt][kc].p[0] = ld16((const T *)a.q + at + kc * S::KB);
                if constexpr (QP == 2) q[rt][kc].p[1] = ld16((const T *)a.q_lo + at + kc * S::KB);
                if (a.turn)
#pragma unroll
                    for (int i = 0; i < QP; ++i) q[rt][kc].p[i] ^= sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
            }
        }
        f32x4 o[RT][NDT];
        float m_run[RT], l_run[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m_run[rt] = MINUS_INF;
            l_run[rt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const bool all_tiles = RT == 1 || x0 + 16 * (RT - 1) < a.GM;
        float *const scores = a.scores + (row0 + x0 + c) * a.ld_scores + 4 * g;
        if (STAGES < steps) pages = pages_at(piece, first + STAGES * NW * S::STEP); // (always a step before they are needed)
        int stage = 0;
        bool odd = false; // a value that only some rows see is no number
        for (int i = 0; i < steps; ++i) {
            const int p0 = first + i * NW * S::STEP;
            const unsigned char *keys = ring + stage * 2 * S::HALF, *values = keys + S::HALF;
            const uint32_t keys_at = ring_at + stage * 2 * S::HALF;
            const bool ahead = i + STAGES <= steps, again = i + STAGES < steps;
            // In flight behind these keys are this step's values, STAGES - 1 steps and the scores of STAGES steps (of all row tiles, or of one at least;
            // not counted, they would be waited for with half of the keys just asked for).  Everything comes back in order; near the end all is waited for.
            if (ahead) wait_behind<(2 * STAGES - 1) * S::PER, STORES * RT, STORES>(i >= STAGES, all_tiles);
            else wait_vmcnt_at_most<0>();
            asm volatile("" ::: "memory");
            u32x4 k[S::NU][NKC];
#pragma unroll
            for (int u = 0; u < S::NU; ++u)
#pragma unroll
                for (int kc = 0; kc < NKC; ++kc)
                    k[u][kc] = *reinterpret_cast<const u32x4 *>(keys + (16 * u + c) * S::ROW + ((kc * 4 + g) ^ S::swizzle(c)) * 16);
            if (again) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // the keys have been read
                request_half(piece, kv.k, pages, p0 + STAGES * NW * S::STEP, keys_at);
            }
            const unsigned hidden = bad >> stage * S::NU & ((1u << S::NU) - 1);
            const bool masked = hidden != 0 || p0 + S::STEP > n - a.M + 1; // not every row sees all of it
            float p[RT][NT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float top = MINUS_INF;
#pragma unroll
                for (int u = 0; u < S::NU; ++u) {
                    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kc = 0; kc < NKC; ++kc) s = mma_q<T>(s, k[u][kc], q[rt][kc]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float x = s[r];
                        if (masked && (p0 + 16 * u + 4 * g + r > limit[rt] || hidden >> u & 1)) x = MINUS_INF;
                        p[rt][4 * u + r] = x;
                        top = fmaxf(top, x);
                    }
                    if constexpr (W) {
                        const int x = x0 + rt * 16 + c;
                        if (x < a.GM)
                            *reinterpret_cast<f32x4 *>(scores + rt * 16 * a.ld_scores + p0 + 16 * u) = f32x4{p[rt][4 * u], p[rt][4 * u + 1], p[rt][4 * u + 2], p[rt][4 * u + 3]};
                    }
                }
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float m_new = fmaxf(m_run[rt], top), m_safe = m_new == MINUS_INF ? 0.f : m_new; // (nothing seen yet: all weights are exp2(-inf))
                const float alpha = weight_of(m_run[rt], m_safe, a.scale_log2e);
                m_run[rt] = m_new;
                l_run[rt] *= alpha;
#pragma unroll
                for (int e = 0; e < NT; ++e) {
                    p[rt][e] = weight_of(p[rt][e], m_safe, a.scale_log2e);
                    l_run[rt] += p[rt][e];
                }
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) o[rt][dt] *= alpha;
            }
            // ... behind these values: STAGES - 1 steps and the keys just asked for, and the scores
            if (again) wait_behind<(2 * STAGES - 1) * S::PER, STORES * RT, STORES>(i >= STAGES, all_tiles);
            else if (ahead) wait_behind<(2 * STAGES - 2) * S::PER, STORES * RT, STORES>(i >= STAGES, all_tiles);
            asm volatile("" ::: "memory");
            uint32_t v[NT][S::NCG][S::VW];
#pragma unroll
            for (int e = 0; e < NT; ++e) {
                const int r = 4 * g + (e & 3); // of its tile
#pragma unroll
                for (int cg = 0; cg < S::NCG; ++cg) {
                    const int byte = (cg * 16 + c) * S::VE * (int)sizeof(T);
                    lds_words<S::VW>(v[e][cg], values + (16 * (e >> 2) + r) * S::ROW + (((byte >> 4) ^ S::swizzle(r)) << 4) + (byte & 15));
                }
            }
            if (again) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // ... and the values
                request_half(piece, kv.v, pages, p0 + STAGES * NW * S::STEP, keys_at + S::HALF);
                bad = (bad & ~(((1u << S::NU) - 1) << stage * S::NU)) | missing(pages) << stage * S::NU;
                pages = pages_at(piece, p0 + (STAGES + 1) * NW * S::STEP);
            }
            if (masked) {
                if (hidden && lane == 0) flag(kv.status, PAGED_BAD_PAGE);
#pragma unroll
                for (int e = 0; e < NT; ++e) {
                    const int slot = p0 + 16 * (e >> 2) + 4 * g + (e & 3);
                    const bool nobody = slot >= n || (hidden >> (e >> 2) & 1), some = slot > n - a.M;
#pragma unroll
                    for (int cg = 0; cg < S::NCG; ++cg)
#pragma unroll
                        for (int w = 0; w < S::VW; ++w) {
                            // what is no number would reach the rows that do not see it through their weights of zero: added below
                            const bool out = some && not_finite(v[e][cg][w], T{});
                            odd |= out && !nobody;
                            if (nobody || out) v[e][cg][w] = finite_part(v[e][cg][w], nobody, T{});
                        }
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) mma_pv<HD>(o[rt], v, p[rt], T{});
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }

        if (__any(odd)) { // infinities and NaNs of the newest rows reach those that see them
#pragma unroll 1
            for (int slot = max(begin, n - a.M + 1); slot < end; ++slot) {
                if ((slot - begin) / S::STEP % NW != wave) continue;
                const int page = page_of(piece, slot);
                if ((unsigned)page >= (unsigned)kv.n_pages) continue;
                const T *V = (const T *)kv.v + hk * kv.head_stride + page * kv.page_stride + (slot & page_mask) * kv.slot_stride;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = to_f32(V[dt / S::VE * 16 * S::VE + S::VE * (4 * g + r) + dt % S::VE]);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
                            if (!(fabsf(x) < -MINUS_INF) && slot <= limit[rt]) o[rt][dt][r] += x;
                    }
            }
        }

        if constexpr (!WHOLE) { // the next piece's first steps are on their way during the merge
            t += piece.k1 - piece.k0;
            if (t - before >= piece.nb * kv.Hk) {
                before += piece.nb * kv.Hk;
                ++at_b;
            }
            more = t < t_end;
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // everything in the ring has been read
                next = piece_at();
                request_first(next, next_bad, next_pages);
            }
        }
        // The wavefronts' results, merged in a fixed order, in the place of their rings' last values
        const bool whole = WHOLE || (piece.k0 == 0 && piece.k1 == piece.nb);
        const size_t partial = ((size_t)(rowblock * a.workgroups + part) * 2 + (first_piece && piece.k0 ? 0 : 1)) * (16 * RT);
        auto merge_at = [&](int w, int dt, int r) -> float & { return reinterpret_cast<float *>(lds + (w + 1) * RING - S::HALF)[(dt * 4 + r) * 64 + lane]; };
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l_run[rt] += __shfl_xor(l_run[rt], 16);
            l_run[rt] += __shfl_xor(l_run[rt], 32);
            if (g == 0) {
                sm_m[wave][rt][c] = m_run[rt];
                sm_l[wave][rt][c] = l_run[rt];
            }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            __syncthreads();
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r) merge_at(wave, dt, r) = o[rt][dt][r];
            __syncthreads();
            float top = sm_m[0][rt][c], wt[NW], l = 0.f;
#pragma unroll
            for (int w = 1; w < NW; ++w) top = fmaxf(top, sm_m[w][rt][c]);
            const float safe = top == MINUS_INF ? 0.f : top;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                wt[w] = weight_of(sm_m[w][rt][c], safe, a.scale_log2e);
                l += sm_l[w][rt][c] * wt[w];
            }
            const int x = x0 + rt * 16 + c;
            const bool nothing = saw_nothing(top, l);
            const float linv = nothing ? 0.f : 1.f / l;
            if (wave == 0 && g == 0) {
                fin_m[rt * 16 + c] = safe;
                fin_l[rt * 16 + c] = linv;
                if (!whole) a.part_ml[partial + rt * 16 + c] = make_float2(top, l);
                else if (W && !WHOLE && x < a.GM) a.row_stats[row0 + x] = make_float2(safe, linv);
            }
            if (x < a.GM) {
                // this wavefront's share: output row 4 g + wave mod 4 of every tile, half of the consecutive elements
                constexpr int OE = S::VE * 4 / NW;
                const int r = wave & 3, e0 = wave / 4 * OE;
#pragma unroll
                for (int cg = 0; cg < S::NCG; ++cg) {
                    float y[OE];
#pragma unroll
                    for (int e = 0; e < OE; ++e) {
                        y[e] = 0.f;
#pragma unroll
                        for (int w = 0; w < NW; ++w) y[e] += merge_at(w, cg * S::VE + e0 + e, r) * wt[w];
                        if (whole) y[e] = nothing ? 0.f : y[e] * linv;
                    }
                    const int at = cg * 16 * S::VE + S::VE * (4 * g + r) + e0;
                    if (whole) {
                        const int h = x / a.M, m = x - h * a.M;
                        store_out<T, OE>(a, (size_t)(b * a.M + m) * a.ldo + (size_t)(hk * a.G + h) * a.o_head + at, y);
                    } else {
                        if constexpr (OE == 1) a.part_o[(partial + rt * 16 + c) * HD + at] = y[0];
                        else store_cols(a.part_o + (partial + rt * 16 + c) * HD + at, y);
                    }
                }
            }
        }
        __syncthreads();
        if constexpr (W && WHOLE) // (one block of query rows)
#pragma unroll 1
            for (int s = threadIdx.x * 4; s < n; s += NW * 64 * 4) {
                const int64_t at = weights_at(kv, b, hk, s);
                const f32x4 old = at < 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : *reinterpret_cast<const f32x4 *>(kv.weight + at);
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int x = 0; x < a.GM; x += 8) {
                    SlotScores t;
                    load_scores(a, b * kv.Hk + hk, s, x, 1, t);
                    sum_scores(a, x, 1, fin_m, fin_l, t, sum);
                }
                sum_seen(a, b * kv.Hk + hk, s, n, 0, 1, fin_m, fin_l, sum);
                add_weights(a, at, s, n, old, sum);
            }
        if (WHOLE || !more) return;
        first_piece = false;
        piece = next;
        bad = next_bad;
        pages = next_pages;
    }
}


template <typename T, int HD, int RT, int QP> void launch_attn(const PagedAttnArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(!a.workgroups ? (size_t)a.kv.B * a.kv.Hk * a.rowblocks : a.rowblocks == 1 ? (size_t)a.workgroups : (size_t)(a.workgroups + 7) / 8 * 8 * a.rowblocks));
    const bool w = a.weight_out != nullptr;
    if (a.workgroups == 0) {
        if (w) hipLaunchKernelGGL((paged_attn_kernel<T, HD, RT, QP, true, true>), grid, dim3(ATTN_WAVES * 64), 0, st, a);
        else hipLaunchKernelGGL((paged_attn_kernel<T, HD, RT, QP, true, false>), grid, dim3(ATTN_WAVES * 64), 0, st, a);
    } else {
        if (w) hipLaunchKernelGGL((paged_attn_kernel<T, HD, RT, QP, false, true>), grid, dim3(ATTN_WAVES * 64), 0, st, a);
        else hipLaunchKernelGGL((paged_attn_kernel<T, HD, RT, QP, false, false>), grid, dim3(ATTN_WAVES * 64), 0, st, a);
    }
}
} // namespace

// q_lo: two planes, of a model's rows, whose heads are not shared: at most 16 rows to a key head
template <typename T, int HD> void launch_paged_heads(const PagedAttnArgs &a, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (a.q_lo) return launch_attn<T, HD, 1, 2>(a, st);
    }
    if (a.row_tiles == 1) launch_attn<T, HD, 1, 1>(a, st);
    else launch_attn<T, HD, 2, 1>(a, st);
}

} // namespace ss
