// Eviction from a paged cache: the entries of a request that are kept, and their way together (spec_cache_evict).
//
// Selection (spec_evict_select_kernel).  Of the M entries between the first p and the last r, the m with the largest weights: the m-th largest is found by its bits (an
// order-preserving integer image of the weight, four passes of 256 counters), then one walk over the entries in order decides what stays (all above it, and the
// first of those equal to it) and where it goes.  The request's row of the table and its weights are on chip for all that, up to COLS and KEYS of them.
//
// Moves.  The i-th kept entry goes to entry i, in every cache.  It comes from an entry at or behind i, so a CTA that takes kept entries in order, so
// many at a time, reads all of a batch before it writes any of it, and may read the next batch before: what lies ahead of the last source is
// all that it writes.  No other CTA touches its bytes of the rows: each has a slice of them, in one cache.  So the move is in place, and every
// byte is read once and written once.
//
// What bounds it.  The moves: bytes (16 requests of up to 8192 entries to 4096, 16 caches of 1 KB a row: the first pass 333 us at 4.8 TB/s, floor 249).  One request:
// latency of the selection, one CTA's passes one after the other (1100 entries: 10 us of 11.4).
#pragma once
#include "cut.cuh"
#include "tree.cuh"

namespace specv {
namespace evict {

struct Params {
    int B, caches, budget, recent, num_blocks, block, width, free_size;
    unsigned char *cache;
    long long stride[3];
    float *weights;
    const int *table;
    long long table_stride;
    const int *lengths, *owned, *protect, *range;
    int *ring;
    int *lengths_out, *owned_out, *range_out, *status;
    int2 *moves;                                       // [B][row_moves] slots from and to, by the entry they go to
    long long row_moves;
    int2 *plan;                                        // [B] index of the first entry that moves (budget: none); blocks to free
    unsigned words, total;                             // of type W in a row's slice, and in a row
    int slices;
};

// ---- selection ----------------------------------------------------------------------------------------------------------------
constexpr int NT = 1024, WARPS = NT / 32, COLS = 4096, KEYS = 46 * 1024;         // 16 and 184 KB
constexpr int MOST = 0x7FFFFFFF - 65536;               // tokens of a request that is cut: KEYS, and a batch of the moves, may be added to an index
static_assert(KEYS + 8 * NT <= 65536, "an index and what is added to it");

__device__ __forceinline__ uint32_t weight_key(float w) { return w == w ? cut::key_of(w) : 0u; }

// Exclusive sums over the CTA of two counts of at most 1 a thread, and their totals.  part: of this call or of the one before last.
__device__ __forceinline__ void scan2(bool a, bool b, int *part, int &a_ahead, int &b_ahead, int &a_all, int &b_all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned below = (1u << lane) - 1u, all_a = __ballot_sync(0xffffffffu, a), all_b = __ballot_sync(0xffffffffu, b);
    if (lane == 0) part[warp] = __popc(all_a) | __popc(all_b) << 16;
    __syncthreads();
    static_assert(WARPS == 32, "a lane for a warp");
    int sum = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += t;
    }
    const int before = warp ? __shfl_sync(0xffffffffu, sum, warp - 1) : 0, total = __shfl_sync(0xffffffffu, sum, 31);
    a_ahead = (before & 0xFFFF) + __popc(all_a & below); b_ahead = (before >> 16) + __popc(all_b & below);
    a_all = total & 0xFFFF; b_all = total >> 16;
}

__global__ void __launch_bounds__(NT) spec_evict_select_kernel(const __grid_constant__ Params P)
{
    __shared__ int part[2][WARPS];
    __shared__ int count[256];
    __shared__ int s_digit, s_above, s_first;
    const int tid = threadIdx.x, lane = tid & 31, b = blockIdx.x;
    int *cols = (int *)dyn_smem;
    float *held = (float *)(cols + COLS);              // the weight of entry p + i
    grid_dependency_wait();
    grid_launch_dependents();                          // (the moving kernel waits by itself)
    const int len = __ldg(P.lengths + b), own = __ldg(P.owned + b), budget = P.budget;
    const int p = P.protect ? __ldg(P.protect + b) : 0;
    const int *table = P.table + (long long)b * P.table_stride;
    const bool idle = len <= budget;                   // (negative lengths too)
    bool page = false;
    if (!idle) {
        // (no more tokens than the cache has slots, nor so many that an index into them and a batch would pass 32 bits)
        page = own < 0 || own > P.width || (len - 1) / P.block >= own || len > min((long long)P.num_blocks * P.block, (long long)MOST);
        if (!page)
            for (int col = tid; col < own; col += NT) {
                const int id = __ldg(table + col);
                page |= id < 0 || id >= P.num_blocks;
                if (col < COLS) cols[col] = id;
            }
    }
    page = __syncthreads_or(page) != 0;
    const bool bad = !idle && (p < 0 || p > budget);
    if (idle || page || bad) {
        if (tid == 0) {
            P.lengths_out[b] = len;
            P.plan[b] = make_int2(budget, 0);
            P.status[b] = bad ? SPEC_DEV_TOPOLOGY : page ? SPEC_DEV_PAGE : SPEC_DEV_OK;
        }
        return;
    }
    const int r = min(P.recent, budget - p), end = len - r, m = budget - p - r;      // chosen: m of the entries [p, end)
    const auto slot_of = [&](int entry) {              // (entry < the owned columns' end)
        const unsigned col = (unsigned)entry / (unsigned)P.block;
        return (long long)(col < COLS ? cols[col] : __ldg(table + col)) * P.block + (entry - (int)col * P.block);
    };
    for (int j0 = p; j0 < min(len, p + KEYS); j0 += 8 * NT) {
        float w[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int j = j0 + x * NT + tid;
            w[x] = j < min(len, p + KEYS) ? __ldcg(P.weights + slot_of(j)) : 0.f;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int j = j0 + x * NT + tid;
            if (j < min(len, p + KEYS)) held[j - p] = w[x];
        }
    }
    const auto weight_of = [&](int j) { return j - p < KEYS ? held[j - p] : __ldcg(P.weights + slot_of(j)); };
    // the m-th largest key by its digits; `above`: entries with a larger one
    uint32_t key = 0u;
    int above = 0;
    if (m > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) count[tid] = 0;
            __syncthreads();
            // (whole warps go round, so that lanes with the same digit add up ahead of the counter: most weights share a few exponents)
            for (int j0 = p; j0 < end; j0 += NT) {
                const int j = j0 + tid;
                const uint32_t k = j < end ? weight_key(weight_of(j)) : 0u;
                const bool in = j < end && (shift == 24 || (k >> (shift + 8)) == key >> (shift + 8));
                const unsigned digit = in ? k >> shift & 255u : 256u;
                if (shift == 24) {
                    const unsigned same = __match_any_sync(0xffffffffu, digit);
                    if (in && lane == __ffs(same) - 1) atomicAdd(&count[digit], __popc(same));
                } else if (in) {
                    atomicAdd(&count[digit], 1);
                }
            }
            __syncthreads();
            if (tid < 32) {                            // the digit in which the count from above reaches m
                int c[8], sum = 0;
#pragma unroll
                for (int d = 0; d < 8; ++d) { c[d] = count[255 - (lane * 8 + d)]; sum += c[d]; }
                int incl = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int s = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += s;
                }
                int at = above + incl - sum;
#pragma unroll
                for (int d = 0; d < 8; ++d) {
                    if (at < m && at + c[d] >= m) { s_digit = 255 - (lane * 8 + d); s_above = at; }
                    at += c[d];
                }
            }
            __syncthreads();
            key |= (uint32_t)s_digit << shift;
            above = s_above;
            __syncthreads();
        }
    }
    // in order: what stays and where it goes
    const int equals = m - above;                      // of those with the key itself: the first so many
    if (tid == 0) s_first = budget;
    __syncthreads();
    int kept = p, same = 0;                            // entries kept, and entries with the key, so far
    int2 *moves = P.moves + (long long)b * P.row_moves;
    for (int j0 = p; j0 < len; j0 += NT) {
        const int j = j0 + tid;
        bool larger = false, equal = false;
        long long slot = 0;
        float w = 0.f;
        if (j < len) {
            slot = slot_of(j);
            w = weight_of(j);
            if (j >= end) larger = true;
            else if (m > 0) {
                const uint32_t k = weight_key(w);
                larger = k > key;
                equal = k == key;
            }
        }
        int a_ahead, e_ahead, a_all, e_all;
        scan2(larger, equal, part[(j0 - p) / NT & 1], a_ahead, e_ahead, a_all, e_all);
        // of the equal ones ahead in this batch, those that still count
        const int room = max(0, equals - same);
        const bool stays = larger || (equal && e_ahead < room);
        const int to = kept + a_ahead + min(e_ahead, room);
        if (stays) {
            const long long goal = slot_of(to);
            moves[to] = make_int2((int)slot, (int)goal);
            if (to != j) {
                atomicMin(&s_first, to);
                __stcg(P.weights + goal, w);           // (all of the batch have read theirs: the scan's barriers; later batches lie behind)
            }
        }
        kept += a_all + min(e_all, room);
        same += e_all;
    }
    __syncthreads();
    if (tid == 0) {
        P.lengths_out[b] = budget;
        P.plan[b] = make_int2(s_first, own - ((budget - 1) / P.block + 1));
        P.status[b] = SPEC_DEV_OK;
    }
}

// ---- moves --------------------------------------------------------------------------------------------------------------------
constexpr int MOVE_NT = 256;

// The last CTA: freed blocks behind the free ones of the ring, request by request.
__device__ void refill(const Params &P)
{
    __shared__ long long part[MOVE_NT / 32], from[MOVE_NT];
    __shared__ int many[MOVE_NT];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int begin = P.free_size ? __ldg(P.range) : 0, free_now = P.free_size ? __ldg(P.range + 1) : 0;
    const bool sound = begin >= 0 && begin < P.free_size && free_now >= 0 && free_now <= P.free_size;
    const long long room = sound ? P.free_size - free_now : 0;
    // requests in runs of MOVE_NT; one whose blocks find no room keeps them, and so do all behind it that have any
    long long ahead = 0, put = 0;
    for (int b0 = 0; b0 < P.B; b0 += MOVE_NT) {
        const int b = b0 + tid;
        const int n = b < P.B ? __ldcg(&P.plan[b]).y : 0;
        long long incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        if (lane == 31) part[warp] = incl;
        __syncthreads();
        long long at = ahead + incl - n, all = 0, fits_to;
        for (int w = 0; w < MOVE_NT / 32; ++w) {
            if (w < warp) at += part[w];
            all += part[w];
        }
        const bool fits = at + n <= room;
        if (b < P.B) {
            const int own = __ldg(P.owned + b);
            P.owned_out[b] = fits ? own - n : own;
            if (!fits && n > 0) P.status[b] = SPEC_DEV_BLOCKS;
        }
        from[tid] = begin + free_now + at;
        many[tid] = fits ? n : 0;
        fits_to = fits ? at + n : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) fits_to = max(fits_to, __shfl_xor_sync(0xffffffffu, fits_to, o));
        __syncthreads();
        if (lane == 0) part[warp] = fits_to;
        __syncthreads();
        for (int w = 0; w < MOVE_NT / 32; ++w) put = max(put, part[w]);
        ahead += all;
        for (int q = warp; q < min(MOVE_NT, P.B - b0); q += MOVE_NT / 32) {
            const int count = many[q];
            if (count == 0) continue;
            const int *row = P.table + (long long)(b0 + q) * P.table_stride + __ldg(P.owned + b0 + q) - count;
            for (int i = lane; i < count; i += 32) P.ring[(from[q] + i) % P.free_size] = __ldg(row + i);
        }
        __syncthreads();
    }
    if (tid == 0) {
        P.range_out[0] = P.free_size ? __ldg(P.range) : 0;
        P.range_out[1] = P.free_size ? (int)(__ldg(P.range + 1) + put) : 0;
    }
}

// DEPTH: rows of a thread on their way at once: 4 where there are many CTAs (six of them fit an SM), 16 where there are few, less than four an SM (one request of
// 13738 entries: 81 us with 4, 75 with 16; 16 requests 359 and 380).
template <typename W, int DEPTH> __global__ void __launch_bounds__(MOVE_NT) spec_evict_move_kernel(const __grid_constant__ Params P)
{
    grid_dependency_wait();
    if (blockIdx.x == gridDim.x - 1) {
        if (blockIdx.y == 0) refill(P);
        return;
    }
    const int tid = threadIdx.x, b = blockIdx.y, c = blockIdx.x / P.slices, s = blockIdx.x - c * P.slices;
    const int first = __ldcg(&P.plan[b]).x, budget = P.budget;
    if (first >= budget) return;
    const int2 *moves = P.moves + (long long)b * P.row_moves;
    unsigned char *base = P.cache + (long long)c * P.stride[0] + ((long long)s * P.words + tid % P.words) * (long long)sizeof(W);
    const int per = MOVE_NT / P.words, lane = (unsigned)s * P.words + tid % P.words < P.total ? tid / P.words : per;     // rows at a time; the thread's
    const auto offset = [&](int slot) {
        const unsigned id = (unsigned)slot / (unsigned)P.block;
        return (long long)id * P.stride[1] + (long long)(slot - (int)(id * P.block)) * P.stride[2];
    };
    W x[DEPTH];
    int2 way[DEPTH];
    for (int i0 = first; i0 < budget; i0 += per * DEPTH) {
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) {
            const int i = i0 + k * per + lane;
            way[k] = lane < per && i < budget ? __ldcg(moves + i) : make_int2(-1, -1);
        }
#pragma unroll
        for (int k = 0; k < DEPTH; ++k)
            if (way[k].x >= 0) x[k] = *(const W *)(base + offset(way[k].x));
        __syncthreads();                               // (all of the batch have their rows)
#pragma unroll
        for (int k = 0; k < DEPTH; ++k)
            if (way[k].x >= 0) *(W *)(base + offset(way[k].y)) = x[k];
    }
}

}  // namespace evict
}  // namespace specv
