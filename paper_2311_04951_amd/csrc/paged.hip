// A key-value cache in pages: append, the second launch of the attention (the first: paged_attention_core.h), eviction by accumulated
// attention weight.
#include "paged_attention_core.h"

namespace ss {

extern template void launch_paged_heads<bf16_t, 32>(const PagedAttnArgs &, hipStream_t); // paged_attention_*.hip
extern template void launch_paged_heads<bf16_t, 64>(const PagedAttnArgs &, hipStream_t);
extern template void launch_paged_heads<bf16_t, 128>(const PagedAttnArgs &, hipStream_t);
extern template void launch_paged_heads<float, 32>(const PagedAttnArgs &, hipStream_t);
extern template void launch_paged_heads<float, 64>(const PagedAttnArgs &, hipStream_t);
extern template void launch_paged_heads<float, 128>(const PagedAttnArgs &, hipStream_t);

namespace {

// What a launch writes to the pages takes the non-temporal bit where the L2s (32 MB) would not hold it.  us, without | with it: four prompts of 2001
// appended (131 MB written) 54.6 | 48.7, one of 30000 (61 MB a side) 48.7 | 40.4, a page of 32 layers x 8 sequences of 8 key heads evicted (67 MB) 53.6 | 51.5,
// of 32 key heads 199 | 166; one sequence's page (8 MB) 19.5 | 21.7.
constexpr size_t STREAMED = 32u << 20;
template <bool STREAM> __device__ __forceinline__ u32x4 ld_row(const void *p) { return STREAM ? __builtin_nontemporal_load((const u32x4 *)p) : ld16(p); }
template <bool STREAM> __device__ __forceinline__ void st_row(void *p, u32x4 x) {
    if constexpr (STREAM) __builtin_nontemporal_store(x, (u32x4 *)p);
    else *reinterpret_cast<u32x4 *>(p) = x;
}

// ------------------------------------------------------------------------------------------ append

// One workgroup to a new row of a sequence: 16 bytes a lane where everything is aligned (host: VEC elements), else an element a lane.
template <typename T, int VEC, bool STREAM>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
    const int r = blockIdx.x, b = r / a.M, m = r - b * a.M;
    const PagedArgs &kv = a.kv;
    const int len = kv.len[b];
    if (len < 0) return;
    const long long slot = (long long)len + m;
    if (slot >= ((long long)kv.max_pages << kv.page_bits)) {
        if (threadIdx.x == 0) flag(kv.status, PAGED_BAD_LENGTH);
        return;
    }
    const int at = (int)slot & ((1 << kv.page_bits) - 1);
    const int page = kv.table[(size_t)b * kv.max_pages + (slot >> kv.page_bits)];
    if ((unsigned)page >= (unsigned)kv.n_pages) {
        if (threadIdx.x == 0) flag(kv.status, PAGED_BAD_PAGE);
        return;
    }
    const int pos = a.next_pos ? a.next_pos[b] + m : (int)slot;
    T *k = (T *)kv.k + page * kv.page_stride + at * kv.slot_stride, *v = (T *)kv.v + page * kv.page_stride + at * kv.slot_stride;
    const T *kn = (const T *)a.k_new, *vn = (const T *)a.v_new;
    const int per = kv.hd / VEC;
    for (int i = threadIdx.x; i < kv.Hk * per; i += 256) {
        const int h = i / per, e = (i - h * per) * VEC;
        const size_t to = h * kv.head_stride + e;
        if (a.ring) {
            const int p = pos & (a.ring - 1);
            const size_t head = ((size_t)b * kv.Hk + h) * a.ring * kv.hd;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                k[to + j] = kn[head + (size_t)p * kv.hd + e + j];
                v[to + j] = vn[head + ((size_t)(p >> 6) * kv.hd + e + j) * 64 + (p & 63)];
            }
        } else if constexpr (VEC > 1) {
            st_row<STREAM>(k + to, ld16(kn + r * a.ld_k + h * a.head_k + e));
            st_row<STREAM>(v + to, ld16(vn + r * a.ld_v + h * a.head_v + e));
        } else {
            k[to] = kn[r * a.ld_k + h * a.head_k + e];
            v[to] = vn[r * a.ld_v + h * a.head_v + e];
        }
    }
    for (int h = threadIdx.x; h < kv.Hk; h += 256) {
        const size_t i = (((size_t)page * kv.Hk + h) << kv.page_bits) + at;
        if (kv.weight) kv.weight[i] = 0.f;
        if (kv.position) kv.position[i] = pos;
    }
}

__global__ void paged_positions_kernel(const int32_t *len, const int32_t *next_pos, int B, int last, int32_t *pos, int32_t *status) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= B) return;
    const int at = len[b] < 0 ? 0 : next_pos ? next_pos[b] : len[b];
    if (at < 0 || at > last) flag(status, PAGED_BAD_LENGTH);
    pos[b] = min(max(at, 0), last);
}

__global__ void paged_advance_kernel(int32_t *len, int32_t *next_pos, int B, int M) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= B || len[b] < 0) return;
    len[b] += M;
    if (next_pos) next_pos[b] += M;
}

// Joins the pieces: the first workgroups take `join_rows` query rows of a head each, every wavefront a quarter of a row's pieces; the others add the weights of `slots`
// positions of a key head, 1024 at a time, or, with more than 16 query rows, 256 at a time and every wavefront a quarter of the rows.  Either
// is a few loads that wait for one another and little else, so whatever does not depend on a load is asked for with it.
constexpr int MAX_GROUP_ROWS = 1024; // GM at most
template <typename T, bool BY_ROW>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, int block, int join_blocks, int join_rows, int slot_blocks, int slots) {
    __shared__ float sm[MAX_GROUP_ROWS], sl[MAX_GROUP_ROWS];
    __shared__ f32x4 quarter[3][64];
    const PagedArgs &kv = a.kv;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool weights = (int)blockIdx.x >= join_blocks;
    const int per_head = weights ? slot_blocks : (a.GM + join_rows - 1) / join_rows;
    const int i = blockIdx.x - (weights ? join_blocks : 0), head = i / per_head, part = i - head * per_head, b = head / kv.Hk, hk = head - b * kv.Hk;
    const int n = positions_of(kv, b, a.pending, a.max_n), nb = blocks_of(n, block), rows = 16 * a.row_tiles;
    if (weights && part * slots >= n) return;
    const int end = min(n, (part + 1) * slots);
    constexpr int STEP = BY_ROW ? 256 : 1024, FIRST_STEP = BY_ROW ? 4 : 1;
    const int x0 = BY_ROW ? wave : 0;
    int s = part * slots + (BY_ROW ? lane : (int)threadIdx.x) * 4;
    SlotScores t;
    int64_t at = -1;
    f32x4 old = {0.f, 0.f, 0.f, 0.f};
    if (weights && s < end) {
        load_scores(a, head, s, x0, FIRST_STEP, t);
        at = weights_at(kv, b, hk, s);
        if (at >= 0) old = *reinterpret_cast<const f32x4 *>(kv.weight + at);
    }
    int before;
    const int share = share_of(a, count_blocks(a, block, b, before) * kv.Hk);
    // a head's pieces: parts first .. first + count - 1; the first one's is its last piece
    const int from = before * kv.Hk + hk * nb, first = from / share, count = (from + nb - 1) / share - first + 1;
    auto row_at = [&](int j, int x) { return ((size_t)(x / rows * a.workgroups + first + j) * 2 + (j == 0 ? 1 : 0)) * rows + x % rows; };
    auto merge = [&](float &top, float &l, float other, float other_l) {
        const float now = fmaxf(top, other), safe = now == MINUS_INF ? 0.f : now;
        l = l * weight_of(top, safe, a.scale_log2e) + other_l * weight_of(other, safe, a.scale_log2e);
        top = now;
    };
    if (weights) {
        // maximum and reciprocal sum of every row: as many threads to a row as there are, up to a wavefront
        int per_row = 64;
        while (per_row > 1 && per_row * a.GM > 256) per_row >>= 1;
        for (int x = threadIdx.x / per_row; x < a.GM; x += 256 / per_row) {
            float top = MINUS_INF, l = 0.f;
            if (count == 1) {
                const float2 ml = a.row_stats[(size_t)head * a.GM + x];
                sm[x] = ml.x;
                sl[x] = ml.y;
                continue;
            }
            for (int j = threadIdx.x % per_row; j < count; j += per_row) {
                const float2 ml = a.part_ml[row_at(j, x)];
                merge(top, l, ml.x, ml.y);
            }
            for (int d = 1; d < per_row; d <<= 1) merge(top, l, __shfl_xor(top, d), __shfl_xor(l, d));
            sm[x] = top == MINUS_INF ? 0.f : top;
            sl[x] = saw_nothing(top, l) ? 0.f : 1.f / l;
        }
        __syncthreads();
#pragma unroll 1
        for (int s0 = part * slots; s0 < end; s0 += STEP) { // (every thread the same number of times)
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            if (s < end) {
                if (s0 != part * slots) {
                    load_scores(a, head, s, x0, FIRST_STEP, t);
                    at = weights_at(kv, b, hk, s);
                    if (at >= 0) old = *reinterpret_cast<const f32x4 *>(kv.weight + at);
                }
                sum_scores(a, x0, FIRST_STEP, sm, sl, t, sum);
#pragma unroll 1
                for (int x = x0 + 8 * FIRST_STEP; x < a.GM; x += 8 * FIRST_STEP) {
                    load_scores(a, head, s, x, FIRST_STEP, t);
                    sum_scores(a, x, FIRST_STEP, sm, sl, t, sum);
                }
                sum_seen(a, head, s, n, x0, FIRST_STEP, sm, sl, sum);
            }
            if constexpr (BY_ROW) {
                if (wave) quarter[wave - 1][lane] = sum;
                __syncthreads();
                if (wave == 0 && s < end) add_weights(a, at, s, n, old, sum + quarter[0][lane] + quarter[1][lane] + quarter[2][lane]);
                __syncthreads();
            } else {
                if (s < end) add_weights(a, at, s, n, old, sum);
            }
            s += STEP;
        }
        return;
    }
    __shared__ float sy[4][128], st[4][2];
    const int e = 2 * lane;
    for (int x = part * join_rows; x < min(a.GM, (part + 1) * join_rows); ++x) {
        if (count == 1) continue; // written where the unit was
        float y[2] = {0.f, 0.f}, top = MINUS_INF, l = 0.f;
        for (int j0 = wave; j0 < count; j0 += 32) { // eight pieces: lane i has the statistics of the i-th
            float2 v[8], ml = make_float2(MINUS_INF, 0.f);
            if (lane < 8 && j0 + 4 * lane < count) ml = a.part_ml[row_at(j0 + 4 * lane, x)];
    #pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = make_float2(0.f, 0.f);
                if (j0 + 4 * j < count && e < kv.hd) v[j] = *reinterpret_cast<const float2 *>(a.part_o + row_at(j0 + 4 * j, x) * kv.hd + e);
            }
            float now = ml.x;
    #pragma unroll
            for (int d = 1; d < 8; d <<= 1) now = fmaxf(now, __shfl_xor(now, d));
            now = fmaxf(top, __shfl(now, 0));
            const float safe = now == MINUS_INF ? 0.f : now, alpha = weight_of(top, safe, a.scale_log2e), f = weight_of(ml.x, safe, a.scale_log2e);
            top = now;
            y[0] *= alpha;
            y[1] *= alpha;
            l *= alpha;
    #pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = __shfl(f, j);
                l += w * __shfl(ml.y, j);
                y[0] += v[j].x * w;
                y[1] += v[j].y * w;
            }
        }
        sy[wave][e] = y[0];
        sy[wave][e + 1] = y[1];
        if (lane == 0) {
            st[wave][0] = top;
            st[wave][1] = l;
        }
        __syncthreads();
        if (wave == 0 && e < kv.hd) {
    #pragma unroll
        for (int w = 1; w < 4; ++w) {
            const float now = fmaxf(top, st[w][0]), safe = now == MINUS_INF ? 0.f : now, mine = weight_of(top, safe, a.scale_log2e), theirs = weight_of(st[w][0], safe, a.scale_log2e);
            l = l * mine + st[w][1] * theirs;
            y[0] = y[0] * mine + sy[w][e] * theirs;
            y[1] = y[1] * mine + sy[w][e + 1] * theirs;
            top = now;
        }
        const bool nothing = saw_nothing(top, l);
        const float linv = nothing ? 0.f : 1.f / l;
        y[0] = nothing ? 0.f : y[0] * linv;
        y[1] = nothing ? 0.f : y[1] * linv;
        const int h = x / a.M, m = x - h * a.M;
        const size_t to = (size_t)(b * a.M + m) * a.ldo + (size_t)(hk * a.G + h) * a.o_head + e;
        if constexpr (sizeof(T) == 2) store_out<T, 2>(a, to, y);
        else *reinterpret_cast<float2 *>((float *)a.out + to) = make_float2(y[0], y[1]);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------ eviction
//
// Of a head's n > budget positions stay the first `budget` in the order: kept anyway (position < keep_first or > newest - keep_recent),
// then larger weight, then lower slot.  Slots below the budget whose position goes (holes, ascending) take in turn the positions
// behind the budget that stay (movers, ascending): keys are rotated already, so order means nothing to the attention, and no more
// moves than positions go.

// Order of a position as an unsigned number: ANYWAY, or one more than its weight's bits (a weight that is not above zero, or not a number,
// counts as zero).  No position at all: 0.
constexpr uint32_t ANYWAY = 0xffffffffu, ZERO_WEIGHT = 1u;
__device__ __forceinline__ uint32_t keep_key(float w, int pos, int keep_first, long long oldest_recent) {
    return pos < keep_first || pos > oldest_recent ? ANYWAY : (w > 0.f ? f2u(w) : 0u) + 1u;
}

// A head to a workgroup.  Every wavefront has a contiguous part of the positions, 256 at a time and four to a lane, so that ranks in the order of the
// slots take counts within a wavefront and one exchange of sixteen numbers.  The budget's key comes from at most three radix passes over
// eleven bits (a pass that meets the budget exactly is the last); positions kept anyway and weights of zero are the hot bins and are
// counted without the histogram.  Keys of the first pass's bin go to a list in LDS if that holds them; of up to COMPARED the budget's is found by
// comparing each to all, else the other passes walk over the list.
// ITER > 0: all of a head's keys stay in registers (ITER * 4 a thread), else every pass over all of them reads them again.
// MOVES_TOO: the workgroup moves its head's rows as well (up to LISTED of them, listed in the histogram's place), which other workgroups' searches
// hide; else paged_move_kernel does.
constexpr int LISTED = 1024, COMPARED = 256;
enum : int { NO_MOVES, CACHED_MOVES, STREAMED_MOVES };
template <int NT, int ITER, int MOVES_TOO>
__global__ __launch_bounds__(NT, NT == 256 ? 8 : 4) // (2048 heads are all there at once: 62 -> 54 us)
void paged_select_kernel(PagedEvictArgs a) {
    constexpr int NW = NT / 64, BINS = 2048, PER_THREAD = BINS / NT;
    __shared__ __align__(16) unsigned hist[BINS];
    __shared__ int totals[3][NW];
    __shared__ __align__(16) uint32_t candidates[BINS + 4];
    __shared__ int sh_bin[2], sh_above[2], sh_own[2], sh_count;
    const PagedArgs &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hk = blockIdx.x % kv.Hk, b = blockIdx.x / kv.Hk % kv.B, layer = blockIdx.x / kv.Hk / kv.B;
    const int n = __builtin_amdgcn_readfirstlane(positions_of(kv, b, 0, a.max_n)), C = a.budget;
    const int32_t *table = kv.table + (size_t)b * kv.max_pages;
    const size_t layer_at = (size_t)layer * kv.n_pages * kv.Hk;
    const int part = ((n + NW - 1) / NW + 255) & ~255, begin = min(n, wave * part), end = min(n, begin + part);
    const bool apart = a.weight_out != kv.weight || a.position_out != kv.position;
    if (MOVES_TOO && a.len_out != kv.len && hk == 0 && layer == 0 && tid == 0) a.len_out[b] = min(kv.len[b], C);

    struct Four { // slots s .. s + 3 of a lane
        f32x4 w;
        int p[4];
        uint32_t place; // page and place in it of the first; all ones: nowhere
    };
    auto meta_at = [&](uint32_t place) { return ((layer_at + (size_t)(place >> kv.page_bits) * kv.Hk + hk) << kv.page_bits) + (place & ((1u << kv.page_bits) - 1)); };
    auto load = [&](int s, Four &f) {
        f.w = f32x4{0.f, 0.f, 0.f, 0.f};
        f.place = ~0u;
        if (s >= end) return;
        const int page = table[s >> kv.page_bits];
        if ((unsigned)page >= (unsigned)kv.n_pages) {
            flag(kv.status, PAGED_BAD_PAGE);
            return;
        }
        f.place = ((uint32_t)page << kv.page_bits) + (s & ((1 << kv.page_bits) - 1));
        const size_t i = meta_at(f.place);
        f.w = *reinterpret_cast<const f32x4 *>(kv.weight + i);
        const int4 p = *reinterpret_cast<const int4 *>(kv.position + i);
        f.p[0] = p.x; f.p[1] = p.y; f.p[2] = p.z; f.p[3] = p.w;
    };
    auto store = [&](const Four &f, unsigned which) { // the new state of those of the four that stay where they are
        const size_t i = meta_at(f.place);
        if (which == 15u) {
            *reinterpret_cast<f32x4 *>(a.weight_out + i) = f.w;
            *reinterpret_cast<int4 *>(a.position_out + i) = make_int4(f.p[0], f.p[1], f.p[2], f.p[3]);
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (which >> j & 1) {
                a.weight_out[i + j] = f.w[j];
                a.position_out[i + j] = f.p[j];
            }
    };
    if (n <= C) {
        for (int s = begin + 4 * lane; s < end && apart; s += 256) {
            Four f;
            load(s, f);
            if (f.place != ~0u) store(f, 15u >> max(0, s + 4 - n));
        }
        if (tid == 0 && !MOVES_TOO) a.n_moves[blockIdx.x] = 0;
        return;
    }
    struct Keys { // of the same slots
        uint32_t k[4], place;
    };
    Keys held[ITER ? ITER : 1];
    int newest = -0x7fffffff - 1;
    auto newer = [&](int s, const Four &f) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (f.place != ~0u && s + j < end) newest = max(newest, f.p[j]);
    };
    Four first[ITER ? ITER : 1];
    if constexpr (ITER > 0) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) load(begin + 256 * i + 4 * lane, first[i]);
#pragma unroll
        for (int i = 0; i < ITER; ++i) newer(begin + 256 * i + 4 * lane, first[i]);
    } else {
        for (int s = begin + 4 * lane; s < end; s += 256) {
            load(s, first[0]);
            newer(s, first[0]);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) newest = max(newest, __shfl_xor(newest, d));
    if (lane == 0) totals[0][wave] = newest;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) newest = max(newest, totals[0][w]);
    const long long oldest = (long long)newest - a.keep_recent;
    auto keys_of = [&](int s, const Four &f, Keys &t) {
        t.place = f.place;
#pragma unroll
        for (int j = 0; j < 4; ++j) t.k[j] = s + j >= end ? 0u : f.place == ~0u ? ZERO_WEIGHT : keep_key(f.w[j], f.p[j], a.keep_first, oldest);
    };
    if constexpr (ITER > 0) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) keys_of(begin + 256 * i + 4 * lane, first[i], held[i]);
    }
    // f(i, s, keys) for all of a wavefront's positions
    auto all = [&](auto f) {
        if constexpr (ITER > 0) {
#pragma unroll
            for (int i = 0; i < ITER; ++i)
                if (begin + 256 * i < end) f(i, begin + 256 * i + 4 * lane, held[i]);
        } else {
#pragma unroll 1
            for (int s = begin; s < end; s += 256) {
                Four four;
                Keys keys;
                load(s + 4 * lane, four);
                keys_of(s + 4 * lane, four, keys);
                f(0, s + 4 * lane, keys);
            }
        }
    };

    uint32_t prefix = 0, mask = 0;
    int want = C, listed = -1; // how many of the keys that match the prefix stay; how many of them are in the list (-1: it holds none)
    bool exact = false;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) hist[tid + i * NT] = 0;
    if (tid < 2) sh_bin[tid] = -1;
    if (tid == 0) sh_count = 0;
    __syncthreads(); // (and the maxima have been read)
    for (int pass = 0; mask != 0xffffffffu && !exact; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = shift ? 11 : 10, turn = pass & 1;
        int anyway = 0;
        auto add = [&](uint32_t key) { // (by lanes whose key counts)
            const uint32_t bin = key >> shift & ((1u << bits) - 1), one = __builtin_amdgcn_readfirstlane(bin);
            const unsigned long long who = __ballot(true);
            if (__ballot(bin != one) == 0) { // all in one bin
                if (lane == __ffsll(who) - 1) atomicAdd(&hist[one], (unsigned)__popcll(who));
            } else {
                atomicAdd(&hist[bin], 1u);
            }
        };
        if (listed >= 0) {
            for (int i = tid; i < listed; i += NT)
                if ((candidates[i] & mask) == prefix) add(candidates[i]);
        } else {
            all([&](int, int, const Keys &f) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t key = f.k[j];
                    if (pass == 0) anyway += __popcll(__ballot(key == ANYWAY));
                    if (key > ZERO_WEIGHT && key != ANYWAY && (key & mask) == prefix) add(key);
                }
            });
        }
        if (pass == 0 && lane == 0) totals[0][wave] = anyway;
        __syncthreads();
        // keys in the bins above each; thread 0 has the highest
        unsigned own[PER_THREAD], sum = 0;
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            sum += own[j] = hist[BINS - 1 - (PER_THREAD * tid + j)];
            hist[BINS - 1 - (PER_THREAD * tid + j)] = 0;
        }
        unsigned upto = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const unsigned t = __shfl_up(upto, d);
            if (lane >= d) upto += t;
        }
        if (lane == 63) totals[1][wave] = (int)upto;
        if (pass == 0) {
            anyway = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) anyway += totals[0][w];
            want -= anyway; // (nothing or less: no bin is found)
        }
        __syncthreads();
        unsigned before = upto - sum, counted = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            before += w < wave ? (unsigned)totals[1][w] : 0u;
            counted += (unsigned)totals[1][w];
        }
        if (want > 0) {
#pragma unroll
            for (int j = 0; j < PER_THREAD; ++j) {
                if ((int)before < want && (int)(before + own[j]) >= want) {
                    sh_bin[turn] = BINS - 1 - (PER_THREAD * tid + j);
                    sh_above[turn] = (int)before;
                    sh_own[turn] = (int)own[j];
                }
                before += own[j];
            }
        }
        if (tid == 0) sh_bin[turn ^ 1] = -1;
        __syncthreads();
        const int bin = sh_bin[turn];
        if (want <= 0) { // all that are kept anyway, or the first of them
            exact = want == 0;
            want = C;
            prefix = mask = ANYWAY;
        } else if (bin < 0) { // the rest of the budget goes to weights of zero
            want -= (int)counted;
            prefix = ZERO_WEIGHT;
            mask = 0xffffffffu;
        } else {
            prefix |= (uint32_t)bin << shift;
            mask |= ((1u << bits) - 1) << shift;
            want -= sh_above[turn];
            exact = sh_own[turn] == want; // everything with this prefix stays
            if (pass == 0 && !exact && sh_own[turn] <= BINS) {
                listed = sh_own[turn];
                all([&](int, int, const Keys &f) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (f.k[j] > ZERO_WEIGHT && (f.k[j] & mask) == prefix) candidates[atomicAdd(&sh_count, 1)] = f.k[j];
                });
                if (tid < 4) candidates[listed + tid] = 0u;
                __syncthreads();
                if (listed <= COMPARED) {
                    if (tid < listed) {
                        const uint32_t key = candidates[tid];
                        int above = 0, equal = 0;
                        for (int i = 0; i < listed; i += 4) {
                            const u32x4 other = *reinterpret_cast<const u32x4 *>(candidates + i);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                above += other[j] > key;
                                equal += other[j] == key;
                            }
                        }
                        if (above < want && above + equal >= want) { // (several threads, the same values)
                            sh_bin[0] = (int)key;
                            sh_above[1] = above;
                            sh_own[1] = equal;
                        }
                    }
                    __syncthreads();
                    prefix = (uint32_t)sh_bin[0];
                    mask = 0xffffffffu;
                    want -= sh_above[1];
                    exact = sh_own[1] == want;
                }
            }
        }
    }
    // Keys above the prefix stay, of those equal to it all (exact) or the first `want` in the order of the slots.
    int equal = 0;
    if (!exact) {
        all([&](int, int, const Keys &f) {
#pragma unroll
            for (int j = 0; j < 4; ++j) equal += __popcll(__ballot(f.k[j] == prefix));
        });
        __syncthreads(); // (totals have been read)
        if (lane == 0) totals[0][wave] = equal;
        __syncthreads();
        equal = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) equal += w < wave ? totals[0][w] : 0;
    }
    const unsigned long long lower = (1ull << lane) - 1;
    auto stays = [&](const Keys &f, int &equal_before) { // bit j: the lane's slot j stays
        unsigned is_equal = 0, above = 0;
        int mine = equal_before;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t key = f.k[j];
            const bool eq = (key & mask) == prefix && (key > ZERO_WEIGHT || mask == 0xffffffffu); // (zeros are not in the histogram)
            if (eq) is_equal |= 1u << j;
            if ((key & mask) > prefix) above |= 1u << j;
            if (!exact) {
                const unsigned long long vote = __ballot(eq);
                mine += __popcll(vote & lower);
                equal_before += __popcll(vote);
            }
        }
        if (exact) return above | is_equal;
        unsigned kept = above;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (is_equal >> j & 1) {
                if (mine < want) kept |= 1u << j;
                ++mine;
            }
        return kept;
    };
    // slots that change hands, below the budget (holes) and behind it (movers): counted, then listed
    int holes = 0, movers = 0, rank = equal;
    unsigned kept_bits[ITER ? ITER : 1];
    all([&](int i, int s, const Keys &f) {
        const unsigned kept = stays(f, rank);
        kept_bits[i] = kept;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (s - 4 * lane < C) holes += __popcll(__ballot(s + j < min(end, C) && !(kept >> j & 1)));
            if (s - 4 * lane + 256 > C) movers += __popcll(__ballot(s + j >= C && (kept >> j & 1)));
        }
    });
    __syncthreads(); // (totals have been read)
    if (lane == 0) {
        totals[1][wave] = holes;
        totals[2][wave] = movers;
    }
    __syncthreads();
    holes = movers = 0;
    int count = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        holes += w < wave ? totals[1][w] : 0;
        movers += w < wave ? totals[2][w] : 0;
        count += totals[1][w];
    }
    uint32_t *hole_list = a.moves + (size_t)blockIdx.x * 2 * a.list, *mover_list = hole_list + a.list;
    auto list = [&](int i, uint32_t *far, int which, uint32_t place) {
        if constexpr (MOVES_TOO) hist[which * LISTED + i] = place;
        else far[i] = place;
    };
    auto slots_of = [](int s, int limit) { return s >= limit ? 0u : 15u >> max(0, s + 4 - limit); }; // bit j: s + j is below it
    rank = equal;
    all([&](int i, int s, const Keys &f) {
        const unsigned kept = ITER > 0 ? kept_bits[i] : stays(f, rank);
        const unsigned in_range = slots_of(s, end), below = slots_of(s, C);
        const unsigned hole = ~kept & in_range & below, mover = kept & ~below;
        const uint32_t place = f.place;
        auto each = [&](unsigned which, int &before, uint32_t *far, int side) { // lists those of the four, behind `before` of the wavefront's
            if (!__any(which != 0)) return;
            int at = before;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned long long vote = __ballot(which >> j & 1);
                at += __popcll(vote & lower);
                before += __popcll(vote);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (which >> j & 1) list(at++, far, side, place == ~0u ? ~0u : place + j);
        };
        each(hole, holes, hole_list, 0);
        each(mover, movers, mover_list, 1);
        if (ITER == 0 && apart && place != ~0u && (kept & below & in_range)) {
            Four four;
            load(s, four);
            store(four, kept & below & in_range);
        }
    });
    if constexpr (ITER > 0) {
        if (apart) { // those below the budget that stay, read once more, all at a time
            Four again[ITER];
            auto which = [&](int i) { return kept_bits[i] & slots_of(begin + 256 * i + 4 * lane, min(end, C)); };
#pragma unroll
            for (int i = 0; i < ITER; ++i)
                if (begin + 256 * i < min(end, C)) load(begin + 256 * i + 4 * lane, again[i]);
#pragma unroll
            for (int i = 0; i < ITER; ++i)
                if (begin + 256 * i < min(end, C) && again[i].place != ~0u && which(i)) store(again[i], which(i));
        }
    }
    if constexpr (!MOVES_TOO) {
        if (tid == 0) a.n_moves[blockIdx.x] = count;
        return;
    }
    __syncthreads();
    // 16 bytes of a row of keys or values to a thread, BATCH of them asked for before the first is written
    constexpr int BATCH = 4;
    const int at_once = NT >> a.row_units, unit = tid & ((1 << a.row_units) - 1);
    const int64_t head_at = (layer * a.layer_stride + hk * kv.head_stride) * a.elem + unit * 16;
    const int page_mask = (1 << kv.page_bits) - 1;
    auto row = [&](uint32_t p) { return head_at + ((int64_t)(p >> kv.page_bits) * kv.page_stride + (int64_t)(p & page_mask) * kv.slot_stride) * a.elem; };
#pragma unroll 1
    for (int r0 = tid >> a.row_units; r0 < 2 * count; r0 += BATCH * at_once) {
        u32x4 data[BATCH];
        uint32_t to[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int r = r0 + i * at_once;
            to[i] = ~0u;
            if (r < 2 * count) {
                const uint32_t from = hist[LISTED + (r >> 1)];
                if (from != ~0u) {
                    to[i] = hist[r >> 1];
                    data[i] = ld_row<MOVES_TOO == STREAMED_MOVES>((const char *)(r & 1 ? kv.v : kv.k) + row(from));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
            if (to[i] != ~0u) st_row<MOVES_TOO == STREAMED_MOVES>((char *)((r0 + i * at_once) & 1 ? kv.v : kv.k) + row(to[i]), data[i]);
    }
    for (int i = tid; i < count; i += NT) {
        const uint32_t to = hist[i], from = hist[LISTED + i];
        if (to == ~0u || from == ~0u) continue;
        const size_t m_to = meta_at(to), m_from = meta_at(from);
        a.weight_out[m_to] = kv.weight[m_from];
        a.position_out[m_to] = kv.position[m_from];
    }
}

__global__ void paged_lengths_kernel(const int32_t *len, int B, int budget, int32_t *len_out) { // (in place: behind the searches, which read them)
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b < B) len_out[b] = min(len[b], budget);
}

// The listed moves: a workgroup takes 64 of a head's, with all rows of keys and values that it moves asked for before the first is written.
constexpr int MOVES = 64;
template <typename T, int HD, bool STREAM>
__global__ __launch_bounds__(256, 4) void paged_move_kernel(PagedEvictArgs a, int parts) {
    __shared__ uint32_t places[2][MOVES];
    const PagedArgs &kv = a.kv;
    const int head = blockIdx.x / parts, part = blockIdx.x - head * parts, hk = head % kv.Hk, b = head / kv.Hk % kv.B, layer = head / kv.Hk / kv.B;
    const int tid = threadIdx.x, page_mask = (1 << kv.page_bits) - 1;
    if (hk == 0 && layer == 0 && part == 0 && tid == 0) a.len_out[b] = min(kv.len[b], a.budget);
    constexpr int UNITS = HD * (int)sizeof(T) / 16, AT_ONCE = 256 / UNITS, PASSES = 2 * MOVES / AT_ONCE; // 16-byte units of a row; rows (of keys or values) at a time
    const int64_t head_at = layer * a.layer_stride + hk * kv.head_stride + tid % UNITS * (16 / (int)sizeof(T));
    auto row = [&](uint32_t p) { return head_at + (int64_t)(p >> kv.page_bits) * kv.page_stride + (int64_t)(p & page_mask) * kv.slot_stride; };
    constexpr int BATCH = PASSES < 8 ? PASSES : 8;
#pragma unroll 1
    for (int first = part * MOVES;; first += parts * MOVES) {
        const int count = min(a.n_moves[head] - first, MOVES);
        uint32_t place = ~0u;
        if (tid < 2 * MOVES && first + (tid & (MOVES - 1)) < a.list) place = a.moves[(size_t)head * 2 * a.list + (tid >= MOVES ? a.list : 0) + first + (tid & (MOVES - 1))];
        if (count <= 0) return;
        if (tid < 2 * MOVES) places[tid / MOVES][tid & (MOVES - 1)] = (tid & (MOVES - 1)) < count ? place : ~0u;
        __syncthreads();
#pragma unroll 1
        for (int i0 = 0; i0 < PASSES; i0 += BATCH) {
            u32x4 data[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int r = (i0 + i) * AT_ONCE + tid / UNITS, j = r >> 1;
                const uint32_t from = places[1][j];
                if (places[0][j] != ~0u && from != ~0u) data[i] = ld_row<STREAM>((const T *)(r & 1 ? kv.v : kv.k) + row(from));
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int r = (i0 + i) * AT_ONCE + tid / UNITS, j = r >> 1;
                const uint32_t to = places[0][j];
                if (to != ~0u && places[1][j] != ~0u) st_row<STREAM>((T *)(r & 1 ? kv.v : kv.k) + row(to), data[i]);
            }
        }
        if (tid < MOVES && places[0][tid] != ~0u && places[1][tid] != ~0u) {
            const size_t layer_at = (size_t)layer * kv.n_pages * kv.Hk;
            auto meta = [&](uint32_t p) { return ((layer_at + (size_t)(p >> kv.page_bits) * kv.Hk + hk) << kv.page_bits) + (p & page_mask); };
            const size_t from = meta(places[1][tid]), to = meta(places[0][tid]);
            const float w = kv.weight[from];
            const int p = kv.position[from];
            a.weight_out[to] = w;
            a.position_out[to] = p;
        }
        if (first >= a.list - parts * MOVES) return;
        __syncthreads(); // (the places have been read)
    }
}

// Blocks of query rows and their tiles of 16; parts of the positions, each of a workgroup for every block of rows, 0: a workgroup to a unit
struct AttnPlan {
    int rowblocks, row_tiles, workgroups;
};
AttnPlan attention_plan(int dtype, int B, int Hk, int GM, int max_n, bool weights) {
    AttnPlan p;
    const int tiles = (GM + 15) / 16;
    p.rowblocks = (tiles + 1) / 2;
    p.row_tiles = tiles == 1 ? 1 : 2;
    const long long block = attn_block(dtype);
    const long long heads = (long long)B * Hk * ((max_n + block - 1) / block), most = p.rowblocks == 1 ? 256 : std::max(1, 32 / p.rowblocks) * 8;
    p.workgroups = max_n <= 256 && (!weights || p.rowblocks == 1) ? 0 : (int)std::max(1ll, std::min(heads, most));
    return p;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

} // namespace

void launch_paged_append(int dtype, const PagedAppendArgs &a, hipStream_t st) {
    const dim3 grid(a.kv.B * a.M);
    const bool stream = (size_t)a.kv.B * a.M * a.kv.Hk * a.kv.hd * (dtype ? 4 : 8) >= STREAMED;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
    auto aligned = [&](int E) {
        auto ok = [&](const void *p) { return ((uintptr_t)p & 15) == 0; };
        return !a.ring && ok(a.k_new) && ok(a.v_new) && a.ld_k % E == 0 && a.ld_v % E == 0 && a.head_k % E == 0 && a.head_v % E == 0;
    };
    if (dtype) {
        if (!aligned(8)) go(paged_append_kernel<bf16_t, 1, false>);
        else stream ? go(paged_append_kernel<bf16_t, 8, true>) : go(paged_append_kernel<bf16_t, 8, false>);
    } else {
        if (!aligned(4)) go(paged_append_kernel<float, 1, false>);
        else stream ? go(paged_append_kernel<float, 4, true>) : go(paged_append_kernel<float, 4, false>);
    }
}

void launch_paged_positions(const int32_t *len, const int32_t *next_pos, int B, int last, int32_t *pos, int32_t *status, hipStream_t st) {
    hipLaunchKernelGGL(paged_positions_kernel, dim3((B + 255) / 256), dim3(256), 0, st, len, next_pos, B, last, pos, status);
}

void launch_paged_advance(int32_t *len, int32_t *next_pos, int B, int M, hipStream_t st) {
    hipLaunchKernelGGL(paged_advance_kernel, dim3((B + 255) / 256), dim3(256), 0, st, len, next_pos, B, M);
}

long long paged_attention_blocks(int dtype, int B, int Hk, int GM, int max_n, long long &units) {
    const AttnPlan p = attention_plan(dtype, B, Hk, GM, max_n, false);
    units = (long long)B * Hk * p.rowblocks;
    const int block = attn_block(dtype);
    return units * ((max_n + block - 1) / block);
}

size_t paged_attention_workspace(int dtype, int B, int Hk, int hd, int G, int M, int max_n, bool weights) {
    const int GM = G * M;
    const AttnPlan p = attention_plan(dtype, B, Hk, GM, max_n, weights);
    const size_t parts = (size_t)p.workgroups * p.rowblocks * 2 * 16 * p.row_tiles;
    return 256 + align256(parts * sizeof(float2)) + align256(parts * hd * sizeof(float)) +
           (weights ? align256((size_t)B * Hk * GM * sizeof(float2)) + (size_t)B * Hk * GM * (size_t)((max_n + 31) & ~31) * sizeof(float) : 0);
}

void launch_paged_attention(int dtype, PagedAttnArgs a, void *ws, hipStream_t st) {
    const AttnPlan p = attention_plan(dtype, a.kv.B, a.kv.Hk, a.GM, a.max_n, a.weight_out != nullptr);
    a.rowblocks = p.rowblocks;
    a.row_tiles = p.row_tiles;
    a.workgroups = p.workgroups;
    // Keys and values are used once in a pass over the layers, unless several blocks of query rows walk over them.  32 query heads over 8 of 128,
    // 8 sequences, us, without the non-temporal bit | with it: 33 MB 18.9 | 17.6, 66 MB 23.3 | 22.2, 131 MB 33.6 | 30.5, 393 MB 80.0 | 71.4; two blocks
    // of rows, 49 MB, 66.4 | 68.0.
    a.stream = p.rowblocks == 1;
    const size_t parts = (size_t)p.workgroups * p.rowblocks * 2 * 16 * p.row_tiles;
    a.part_ml = (float2 *)ws;
    a.part_o = (float *)((char *)ws + align256(parts * sizeof(float2)));
    a.row_stats = (float2 *)((char *)a.part_o + align256(parts * a.kv.hd * sizeof(float)));
    a.scores = (float *)((char *)a.row_stats + align256((size_t)a.kv.B * a.kv.Hk * a.GM * sizeof(float2)));
    a.ld_scores = (a.max_n + 31) & ~31;
    if (dtype) {
        if (a.kv.hd == 128) launch_paged_heads<bf16_t, 128>(a, st);
        else if (a.kv.hd == 64) launch_paged_heads<bf16_t, 64>(a, st);
        else launch_paged_heads<bf16_t, 32>(a, st);
    } else {
        if (a.kv.hd == 128) launch_paged_heads<float, 128>(a, st);
        else if (a.kv.hd == 64) launch_paged_heads<float, 64>(a, st);
        else launch_paged_heads<float, 32>(a, st);
    }
    if (p.workgroups == 0) return;
    // about 1536 workgroups for the weights, of 256 to 4096 positions each (more where a launch would not hold them)
    const int heads = a.kv.B * a.kv.Hk, join_rows = std::min(a.GM, (heads * a.GM + 1023) / 1024), join = heads * ((a.GM + join_rows - 1) / join_rows), least = a.GM <= 16 ? 1024 : 256;
    const long long positions = (long long)heads * a.max_n;
    auto round_up = [&](long long x) { return (int)std::min(1ll << 30, std::max(1ll, (x + least - 1) / least) * least); };
    const int slots = std::max(std::min(4096, round_up(positions / 1536)), round_up(positions >> 22)), slot_blocks = (a.max_n + slots - 1) / slots;
    const dim3 grid(join + (a.weight_out ? slot_blocks * heads : 0));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a, attn_block(dtype), join, join_rows, slot_blocks, slots); };
    if (a.GM <= 16) dtype ? go(paged_join_kernel<bf16_t, false>) : go(paged_join_kernel<float, false>);
    else dtype ? go(paged_join_kernel<bf16_t, true>) : go(paged_join_kernel<float, true>);
}

static int evict_list(int max_n, int budget) { return std::max(0, std::min(budget, max_n - budget)); }

size_t paged_evict_workspace(int n_layers, int B, int Hk, int max_n, int budget) {
    const size_t heads = (size_t)n_layers * B * Hk;
    return 256 + align256(heads * 4) + heads * 2 * evict_list(max_n, budget) * 4;
}

void launch_paged_evict(int dtype, PagedEvictArgs a, void *ws, hipStream_t st) {
    const unsigned heads = (unsigned)(a.n_layers * a.kv.B * a.kv.Hk);
    a.list = evict_list(a.max_n, a.budget);
    a.n_moves = (int32_t *)ws;
    a.moves = (uint32_t *)((char *)ws + align256((size_t)heads * 4));
    a.elem = dtype ? 2 : 4;
    a.row_units = __builtin_ctz((unsigned)(a.kv.hd * a.elem / 16));
    const bool stream = (size_t)heads * a.list * a.kv.hd * 2 * a.elem >= STREAMED;
    // The searching workgroup moves its head's rows where the heads alone fill the card, or a workgroup would be all that a head gets: a launch less.
    // us, apart | in one: 2048 heads of 1088 -> 1024 positions 64.7 | 53.6, 8192 of them 226 | 199, 256 of them 19.8 | 19.3.
    const bool moves_too = a.list <= LISTED && (heads >= 1024 || a.list <= MOVES);
    auto select = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(heads), dim3(threads), 0, st, a); };
    auto select_in = [&](auto mode) {
        constexpr int M = decltype(mode)::value;
        if (a.max_n <= 2048) select(paged_select_kernel<256, 2, M>, 256);
        else if (a.max_n <= 8192) select(paged_select_kernel<1024, 2, M>, 1024);
        else if (a.max_n <= 32768) select(paged_select_kernel<1024, 8, M>, 1024);
        else select(paged_select_kernel<1024, 0, M>, 1024);
    };
    if (!moves_too) select_in(std::integral_constant<int, NO_MOVES>{});
    else if (stream) select_in(std::integral_constant<int, STREAMED_MOVES>{});
    else select_in(std::integral_constant<int, CACHED_MOVES>{});
    if (moves_too) {
        if (a.len_out == a.kv.len) hipLaunchKernelGGL(paged_lengths_kernel, dim3((a.kv.B + 255) / 256), dim3(256), 0, st, a.kv.len, a.kv.B, a.budget, a.len_out);
        return;
    }
    const int parts = std::max(1, std::min((a.list + MOVES - 1) / MOVES, std::max(1, (int)((1u << 14) / heads)))); // (a launch holds fewer than 2^32 threads)
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(heads * (unsigned)parts), dim3(256), 0, st, a, parts); };
    auto move = [&](auto streamed) {
        constexpr bool S = decltype(streamed)::value;
        if (dtype) a.kv.hd == 128 ? go(paged_move_kernel<bf16_t, 128, S>) : a.kv.hd == 64 ? go(paged_move_kernel<bf16_t, 64, S>) : go(paged_move_kernel<bf16_t, 32, S>);
        else a.kv.hd == 128 ? go(paged_move_kernel<float, 128, S>) : a.kv.hd == 64 ? go(paged_move_kernel<float, 64, S>) : go(paged_move_kernel<float, 32, S>);
    };
    stream ? move(std::true_type{}) : move(std::false_type{});
}

} // namespace ss
