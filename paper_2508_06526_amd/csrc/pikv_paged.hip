// Writing a paged cache: the rows of whole prompts, and a step's entry.
//
//   fill_plan    : a block per shard gives the tokens that selected it their slots.  Every wave counts those of a run of tokens by
//                  ballots, the tokens in registers; one scan over the waves, and a second walk writes the slots.  Where the shard
//                  has too little room, a radix select over the weights (3 rounds of 11, 11 and 10 bits, counts in LDS: any order
//                  of its atomics gives the same) finds the cut first.  Bound by its chain of trips and barriers: 13 us for 4 x 777
//                  tokens over 32 full shards, 20 us for 16384 tokens over 16 with room.  (Tokens in LDS instead, in rolled loops
//                  with requests of whole selections: 15 us and 16 us.)
//   fill_rows    : lanes take the 16-byte pieces of a token's rows and write them to each of its slots: every row is read once.
//                  16384 tokens of 8 x 128 bf16 values into two slots each, 203 MB: 39 us, 5.2 TB/s.
//   paged_append : a block per (sequence, selected shard).  2.8 us, which are a launch and a chain of four trips to memory.  (Counts of
//                  all shards asked for beside the selection, a trip less: the same time.)
#include "pikv_paged_dev.h"

#include <math.h>

namespace pikv {
namespace {

struct FillParams {
    const char *K_new, *V_new;
    char *K_pool, *V_pool;
    const int32_t *cu, *topk, *positions;
    const float *weight;
    int32_t *entry_pos, *n_valid, *slots;
    float *utility;
    PageGeometry pages;
    int tokens, B, E, S, k, Hkv, row_bits;       // row_bits: log2 of a row's 16-byte pieces
};

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;
constexpr int kHeld = 16;                        // tokens of a lane that it asks for together, and keeps if the sequence has no more (16384)
constexpr int kBins = 2 * kPlanThreads;          // of a round of the select

// The place of expert e in a token's selection: the first of them, -1 if there is none.  (The first four are requested together.)
__device__ __forceinline__ int place_of(const int32_t *topk, int k, int e) {
    int listed[4], at = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) listed[j] = topk[min(j, k - 1)];
    for (int j = k - 1; j >= 4; --j) at = topk[j] == e ? j : at;
#pragma unroll
    for (int j = 3; j >= 0; --j) at = listed[j] == e && j < k ? j : at;
    return at;
}

__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0u : order_key(w); }

__global__ __launch_bounds__(kPlanThreads) void fill_plan(FillParams p) {
    __shared__ int hist[kBins];
    __shared__ int above[kPlanWaves], ties[kPlanWaves], sums[kPlanWaves], found[2], first_missing;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t be = blockIdx.x;
    const int b = blockIdx.x / p.E, e = blockIdx.x - b * p.E;
    const int lo = min(max(p.cu[b], 0), p.tokens), hi = min(max(p.cu[b + 1], lo), p.tokens);
    const int n = p.n_valid[be];
    hist[tid] = hist[tid + kPlanThreads] = 0;
    if (tid == 0) first_missing = p.pages.per_shard;
    // a wave's tokens: a run of whole steps
    const int steps = (hi - lo + kPlanThreads - 1) / kPlanThreads, from = lo + wave * steps * kWave, to = min(hi, from + steps * kWave);
    int place[kHeld], position[kHeld];
    float weight[kHeld];
    auto fetch = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (t0 + u * kWave < to) {           // (uniform)
                const int t = min(t0 + u * kWave + lane, to - 1);
                place[u] = place_of(p.topk + (int64_t)t * p.k, p.k, e);
                weight[u] = p.weight ? p.weight[t] : 0.0f;
                position[u] = p.entry_pos ? p.positions[t] : 0;
                if (t0 + u * kWave + lane >= to) place[u] = -1;
            } else {
                place[u] = -1;
            }
            if (u % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // (all addresses at once cost registers)
        }
    };
    const bool once = steps <= kHeld;
    if (once) fetch(from);
    // visit(token, place, weight, position) in the tokens' order, all lanes of the wave together
    auto walk = [&](auto visit) __attribute__((always_inline)) {
        for (int t0 = from; t0 < to; t0 += kHeld * kWave) {
            if (!once) fetch(t0);
#pragma unroll
            for (int u = 0; u < kHeld; ++u)
                if (t0 + u * kWave < to) visit(t0 + u * kWave + lane, place[u], weight[u], position[u]);
        }
    };
    __syncthreads();
    for (int i = (max(n, 0) >> p.pages.bits) + tid; i < p.pages.per_shard; i += kPlanThreads) {
        const int page = p.pages.table[be * p.pages.per_shard + i];
        if (page < 0 || page >= p.pages.n_pages) atomicMin(&first_missing, i);
    }
    int mine = 0;
    walk([&](int, int at, float, int) { mine += __popcll(__ballot(at >= 0)); });
    if (lane == 0) above[wave] = 0, ties[wave] = mine;
    __syncthreads();
    const int64_t room_end = min((int64_t)p.S, (int64_t)first_missing << p.pages.bits);
    const int room = n < 0 ? 0 : (int)max(room_end - n, (int64_t)0);
    int total = 0;
    for (int w = 0; w < kPlanWaves; ++w) total += ties[w];
    uint32_t cut = 0;                    // entries above it stay, of those at it the first `room - (those above)`
    const bool chosen = total > room && p.weight != nullptr;
    if (chosen) {
        int want = room;                 // the key that the want-th largest has, among those that share its upper bits
        uint32_t prefix = 0;
        if (room == 0) cut = 0xffffffffu;
        else {
            for (int round = 0; round < 3; ++round) {
                const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
                walk([&](int, int place, float weight, int) {
                    const uint32_t key = weight_key(weight);
                    const bool in = round == 0 || (key >> (shift + bits)) == prefix;
                    if (place >= 0 && in) atomicAdd(&hist[(key >> shift) & ((1 << bits) - 1)], 1);
                });
                __syncthreads();
                // bins from the top, two a thread; counts above them: of the lanes, then the waves, before
                const int top = kBins - 1 - 2 * tid, first = hist[top], both = first + hist[top - 1];
                hist[top] = hist[top - 1] = 0;
                int incl = both;
                for (int off = 1; off < kWave; off <<= 1) {
                    const int other = __shfl_up(incl, off, kWave);
                    if (lane >= off) incl += other;
                }
                if (lane == kWave - 1) sums[wave] = incl;
                __syncthreads();
                int before = incl - both;
                for (int w = 0; w < wave; ++w) before += sums[w];
                if (before < want && want <= before + both) {            // one thread
                    const bool second = want > before + first;
                    found[0] = second ? top - 1 : top;
                    found[1] = second ? before + first : before;
                }
                __syncthreads();
                prefix = (prefix << bits) | (uint32_t)found[0];
                want -= found[1];
            }
            cut = prefix;
        }
        int over = 0, at = 0;
        walk([&](int, int place, float weight, int) {
            const uint32_t key = weight_key(weight);
            over += __popcll(__ballot(place >= 0 && key > cut));
            at += __popcll(__ballot(place >= 0 && key == cut));
        });
        __syncthreads();                 // every wave has read the counts
        if (lane == 0) above[wave] = over, ties[wave] = at;
        __syncthreads();
    }
    int over = 0, at = 0, all_over = 0;          // before this wave's tokens; above the cut in all
    for (int w = 0; w < kPlanWaves; ++w) {
        all_over += above[w];
        if (w < wave) over += above[w], at += ties[w];
    }
    const int of_ties = room - all_over;         // at the cut: this many stay
    const uint64_t before_lane = (1ull << lane) - 1;
    walk([&](int t, int place, float weight, int position) {
        const uint32_t key = weight_key(weight);
        const bool is_over = chosen && place >= 0 && key > cut, is_at = place >= 0 && (!chosen || key == cut);
        const uint64_t over_votes = __ballot(is_over), at_votes = __ballot(is_at);
        const int my_over = over + __popcll(over_votes & before_lane), my_at = at + __popcll(at_votes & before_lane);
        over += __popcll(over_votes);
        at += __popcll(at_votes);
        if (place < 0) return;
        const bool stays = is_over || (is_at && my_at < of_ties);
        const int slot = stays ? n + my_over + min(my_at, of_ties) : -1;
        p.slots[(int64_t)t * p.k + place] = slot;
        if (!stays) return;
        p.utility[be * p.S + slot] = weight;
        if (p.entry_pos) p.entry_pos[be * p.S + slot] = position;
    });
    if (tid == 0 && min(total, room) > 0) p.n_valid[be] = n + min(total, room);
}

constexpr int kRowThreads = 256;

// Tokens of fewer than 64 pieces share a wave.
__global__ __launch_bounds__(kRowThreads) void fill_rows(FillParams p, int lane_bits) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const int lanes = 1 << lane_bits, sub = lane >> lane_bits, c = lane & (lanes - 1);
    const int64_t t64 = ((int64_t)blockIdx.x * (kRowThreads / kWave) + wave) * (kWave >> lane_bits) + sub;
    if (t64 >= p.tokens) return;
    const int t = (int)t64;
    int lo = 0, hi = p.B;                        // the sequence: the first that ends behind the token
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.cu[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    if (lo >= p.B || p.cu[lo] > t) return;
    const int64_t be0 = (int64_t)lo * p.E;
    const int pieces = p.Hkv << p.row_bits, row_mask = (1 << p.row_bits) - 1;
    const char *K = p.K_new + (int64_t)t * pieces * 16, *V = p.V_new + (int64_t)t * pieces * 16;
    const int32_t *topk = p.topk + (int64_t)t * p.k;
    int32_t *slots = p.slots + (int64_t)t * p.k;
    constexpr int U = 2;
    for (int i0 = c; i0 < pieces; i0 += U * lanes) {
        uint4 kv[U], vv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min(i0 + u * lanes, pieces - 1);
            kv[u] = load16_stream(K + (int64_t)i * 16);
            vv[u] = load16_stream(V + (int64_t)i * 16);
        }
        for (int j = 0; j < p.k; ++j) {
            const int e = topk[j];
            bool none = e < 0 || e >= p.E;       // no shard, or one that was listed before
            for (int i = 0; i < j; ++i) none |= topk[i] == e;
            if (none) {
                if (i0 == 0) slots[j] = -1;
                continue;
            }
            const int slot = slots[j];
            if (slot < 0) continue;
            const int64_t at = slot_offset(p.pages, be0 + e, slot);
            if (at < 0) continue;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * lanes;
                if (i >= pieces) break;
                const int64_t to = at + (i >> p.row_bits) * p.pages.stride_h + (i & row_mask) * 16;
                store16_stream(p.K_pool + to, kv[u]);
                store16_stream(p.V_pool + to, vv[u]);
            }
        }
    }
}

struct PagedAppendParams {
    const char *K_new, *V_new;
    char *K_pool, *V_pool;
    const int32_t *topk, *reuse_idx, *reuse_cnt, *positions;
    int32_t *entry_pos, *n_valid;
    float *utility;
    PageGeometry pages;
    FastDiv by_k;
    int E, S, k, Hkv, row_bits, max_evict;
};

constexpr int kAppendThreads = 256;

__global__ __launch_bounds__(kAppendThreads) void paged_append(PagedAppendParams p) {
    int j;
    const int b = fast_divide(p.by_k, blockIdx.x, &j);
    const int tid = threadIdx.x;
    const int pieces = p.Hkv << p.row_bits, row_mask = (1 << p.row_bits) - 1;
    const int32_t *topk = p.topk + (int64_t)b * p.k;
    const int e = topk[j];
    const int first = min(tid, pieces - 1);
    const char *K = p.K_new + (int64_t)b * pieces * 16, *V = p.V_new + (int64_t)b * pieces * 16;
    uint4 kv = load16(K + (int64_t)first * 16), vv = load16(V + (int64_t)first * 16);
    if (e < 0 || e >= p.E) return;               // (uniform, as every return here)
    for (int i = 0; i < j; ++i)
        if (topk[i] == e) return;
    const int64_t be = (int64_t)b * p.E + e;
    const int n = p.n_valid[be];
    int slot = n;
    if (p.reuse_cnt != nullptr && p.reuse_cnt[be] > 0) slot = p.reuse_idx[be * p.max_evict];
    __syncthreads();                             // every thread has read n before it changes
    if (n < 0 || n >= p.S || slot < 0 || slot >= p.S) return;    // full shard: the entry is dropped
    const int64_t at = slot_offset(p.pages, be, slot);
    if (at < 0) return;
    for (int i = tid; i < pieces; i += kAppendThreads) {
        if (i != tid) {
            kv = load16(K + (int64_t)i * 16);
            vv = load16(V + (int64_t)i * 16);
        }
        const int64_t to = at + (i >> p.row_bits) * p.pages.stride_h + (i & row_mask) * 16;
        store16(p.K_pool + to, kv);
        store16(p.V_pool + to, vv);
    }
    if (tid == 0) {
        p.utility[be * p.S + slot] = 0.0f;
        if (p.entry_pos) p.entry_pos[be * p.S + slot] = p.positions[b];
        p.n_valid[be] = n + 1;
    }
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace
}  // namespace pikv

using namespace pikv;

extern "C" int pikv_paged_fill(const pikv_desc *desc, const pikv_pages *pages, const void *K_new, const void *V_new, int32_t tokens,
                               const int32_t *cu_seqlens, const int32_t *topk_idx, int32_t k, const float *weight,
                               const int32_t *positions, void *K_pool, void *V_pool, const int32_t *page_table, int32_t *entry_pos,
                               float *utility, int32_t *n_valid, int32_t *slots, void *stream) {
    const int rc = check_paged(desc, pages);
    if (rc != PIKV_OK) return rc;
    if (tokens < 0 || k < 1 || k > desc->E) return PIKV_ERR_INVALID;
    if (desc->route_rows_per_seq != 1 || tokens > (1 << 23) || (int64_t)desc->B * desc->E >= (1 << 22)) return PIKV_ERR_UNSUPPORTED;
    if (tokens == 0 || desc->B == 0) return PIKV_OK;             // (tensors without elements have no address)
    if (!K_new || !V_new || !cu_seqlens || !topk_idx || !K_pool || !V_pool || !page_table || !utility || !n_valid || !slots) return PIKV_ERR_INVALID;
    if ((positions != nullptr) != (entry_pos != nullptr)) return PIKV_ERR_INVALID;
    if (!aligned16(K_new) || !aligned16(V_new) || !aligned16(K_pool) || !aligned16(V_pool)) return PIKV_ERR_INVALID;
    FillParams p;
    p.K_new = static_cast<const char *>(K_new);
    p.V_new = static_cast<const char *>(V_new);
    p.K_pool = static_cast<char *>(K_pool);
    p.V_pool = static_cast<char *>(V_pool);
    p.cu = cu_seqlens;
    p.topk = topk_idx;
    p.positions = positions;
    p.weight = weight;
    p.entry_pos = entry_pos;
    p.n_valid = n_valid;
    p.slots = slots;
    p.utility = utility;
    p.pages = page_geometry(desc, pages, page_table);
    p.tokens = tokens;
    p.B = desc->B;
    p.E = desc->E;
    p.S = desc->S;
    p.k = k;
    p.Hkv = desc->Hkv;
    p.row_bits = __builtin_ctz(desc->D * elem_bytes(desc->dtype) / 16);
    hipStream_t st = as_stream(stream);
    hipLaunchKernelGGL(fill_plan, dim3(desc->B * desc->E), dim3(kPlanThreads), 0, st, p);
    const int plan_rc = launch_status();
    if (plan_rc != PIKV_OK) return plan_rc;
    int lane_bits = 0;
    while (lane_bits < 6 && (1 << lane_bits) < desc->Hkv << p.row_bits) ++lane_bits;
    const int per_block = (kRowThreads / kWave) * (kWave >> lane_bits);
    hipLaunchKernelGGL(fill_rows, dim3((tokens + per_block - 1) / per_block), dim3(kRowThreads), 0, st, p, lane_bits);
    return launch_status();
}

extern "C" int pikv_paged_append(const pikv_desc *desc, const pikv_pages *pages, const void *K_new, const void *V_new,
                                 const int32_t *topk_idx, int32_t k, const int32_t *reuse_idx, const int32_t *reuse_cnt,
                                 int32_t max_evict, const int32_t *positions, void *K_pool, void *V_pool, const int32_t *page_table,
                                 int32_t *entry_pos, float *utility, int32_t *n_valid, void *stream) {
    const int rc = check_paged(desc, pages);
    if (rc != PIKV_OK) return rc;
    if (k < 1 || k > desc->E) return PIKV_ERR_INVALID;
    if (desc->route_rows_per_seq != 1) return PIKV_ERR_UNSUPPORTED;
    if ((reuse_idx != nullptr) != (reuse_cnt != nullptr) || (reuse_cnt && max_evict < 1)) return PIKV_ERR_INVALID;
    if ((int64_t)desc->B * k > (1 << 21)) return PIKV_ERR_UNSUPPORTED;
    if (desc->B == 0) return PIKV_OK;
    if (!K_new || !V_new || !topk_idx || !K_pool || !V_pool || !page_table || !utility || !n_valid) return PIKV_ERR_INVALID;
    if ((positions != nullptr) != (entry_pos != nullptr)) return PIKV_ERR_INVALID;
    if (!aligned16(K_new) || !aligned16(V_new) || !aligned16(K_pool) || !aligned16(V_pool)) return PIKV_ERR_INVALID;
    PagedAppendParams p;
    p.K_new = static_cast<const char *>(K_new);
    p.V_new = static_cast<const char *>(V_new);
    p.K_pool = static_cast<char *>(K_pool);
    p.V_pool = static_cast<char *>(V_pool);
    p.topk = topk_idx;
    p.reuse_idx = reuse_idx;
    p.reuse_cnt = reuse_cnt;
    p.positions = positions;
    p.entry_pos = entry_pos;
    p.n_valid = n_valid;
    p.utility = utility;
    p.pages = page_geometry(desc, pages, page_table);
    p.by_k = fast_div(k);
    p.E = desc->E;
    p.S = desc->S;
    p.k = k;
    p.Hkv = desc->Hkv;
    p.row_bits = __builtin_ctz(desc->D * elem_bytes(desc->dtype) / 16);
    p.max_evict = max_evict;
    hipLaunchKernelGGL(paged_append, dim3(desc->B * k), dim3(kAppendThreads), 0, as_stream(stream), p);
    return launch_status();
}
