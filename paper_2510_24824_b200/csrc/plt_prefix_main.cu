// The pass over shared prefixes: the queries of a whole group of sequences against the group's one prefix, on the 5th-generation
// tensor cores (tcgen05.mma, accumulators in tensor memory), and the plan that it walks.
//
// All sequences of a group, all loops, tokens and query heads of a KV head are rows of one matrix product:
//
//   S [128 rows x 128 keys] = Q . K_tile^T        A = packed query rows, B = K tile as TMA wrote it (K-major, 128-byte swizzle)
//   O [128 rows x d]       += P . V_tile          A = probabilities in tensor memory (written over S), B = V tile (MN-major)
//
// with an online softmax whose reference maximum is moved only when a score outruns it by more than a few powers of two. A unit
// is two such tiles of 128 rows, A and B, of one KV head. Where a unit has more than 128 rows, both tiles take every key tile, so
// that each K/V tile in shared memory serves 256 rows; where it has fewer, A and B are the same rows and take the key tiles in
// turn. Blocks are persistent, and leave unnormalised partials for the merge. Where the units can be cut into about as many equal
// pieces as there are blocks, each takes one piece; else each takes an equal range of a line on which the units' key tiles lie one behind
// the other.
//
// A tile's scores come in two halves of 64 keys, each with tensor memory and barriers of its own: while the warps work on one, the
// products of the other (P . V of these keys, then the next key tile's scores) run. With whole tiles a tile's softmax and its
// products took turns, 4600 cycles for a wide key tile of which the products alone are 2050; halves make the scores' products dearer
// (64 columns take 49 cycles for 16 elements of depth, 128 take 64: the rows of Q are read from shared memory for each) and the whole
// shorter: 128 sequences behind 32768 tokens 154 -> 144 us. A and B have an issuing warp each, since the issue of a half costs about
// as much in waits and commits as its products take.
//
// What bounds it: on long prefixes the 16 warps of the softmax, always busy with a latency chain of loads, maximum, exponentials and
// stores, next to the products (2600 cycles of some 3500 for a wide key tile), under the power limit: 1.04 PFLOP/s (128 sequences of
// two loops behind 32768 tokens, 133 us). On short ones the start: the plan, and code that a launch finds outside the instruction
// caches, so that what lies between the launch and the first product is kept short: 3 us of plan, 4 to the first scores.
//
// Warp roles: warp 0 loads K and V tiles by TMA into a ring (pages: their ids one tile ahead); warps 1 and 3 load query tiles and issue
// the products, warp 1 owns the tensor memory; warp 2 makes the plan; warps 2, 20, 21 and 22 turn E4M3 codes into f16 (exact) in a second ring; warps
// 4-11 and 12-19 are the softmax of A and of B, load their query rows and store the partials. A partial lies as [d / 4][128 rows][4].
//
// bf16 probabilities carry 8 bits, f16 ones (E4M3 caches) 11; their sum is taken before that rounding, in fp32. Where one key holds a
// large share of a row's weight, 8 bits show in the output (rows with a few dominant keys and large V came to 1.96 times the
// framework's bound of 2e-2), so there bf16 probabilities are multiplied with V in two terms, p = hi + lo, hi = bf16(p), lo = bf16(p -
// hi), as in the decode step's kernel. Scores above a limit, a share of the row's sum when it was last taken, send a warp the longer
// way, with the vote that lets a reference move: it takes the sum anew and, where a probability is above the share of it, leaves lo
// behind hi in tensor memory and sets a flag, by which the issuing warp adds a second product on the lanes of the warps that did (the
// others' lanes are masked off). That way costs 36.2 us instead of 34.0 (64 sequences of two loops behind 4096 tokens), 146 instead
// of 142 (128 behind 32768), 16.1 instead of 15.6 (two users): the first halves of a piece take it, and scores outrun the limit now
// and then until the sum has grown.
// Every wait is bounded and reports through the status word.
#include <cuda_bf16.h>

#include "plt_prefix.h"
#include "plt_seq_util.cuh"

namespace plt {
namespace {

constexpr int kNearGroups = 31;      // plans of up to this many groups are made by a warp of every block, without a kernel before

template <int D, bool FP8>
struct PCfg {
    static constexpr int TILE = kPrefixTile * D * 2;              // a tile of 16-bit elements
    static constexpr int RING = FP8 ? 3 : D == 64 ? 8 : 5;        // 16-bit tiles
    static constexpr int RAW = FP8 ? 4 : 0;                       // tiles of codes
    static constexpr int RAW_TILE = kPrefixTile * D;
    // mbarriers
    // (S, P and PV: of tile x and half h at 2 x + h)
    static constexpr int QFULL = 0, QRAW = 2, FULL = 4, EMPTY = FULL + RING, RFULL = EMPTY + RING, REMPTY = RFULL + RAW, SFULL = REMPTY + RAW,
                         PFULL = SFULL + 4, PVDONE = PFULL + 4, ODONE = PVDONE + 4, COUNT = ODONE + 2;
    // tiles, barriers, control words, the plan, the softmax's flags
    static constexpr size_t SMEM = 1024 + 2 * TILE + (size_t)RING * TILE + (size_t)RAW * RAW_TILE + COUNT * 8 + 64 + (5 * (kNearGroups + 1) + 4 + 8) * 4;
};

template <bool FP8>
constexpr int kPThreads = FP8 ? 736 : 640;

// Instruction descriptor: fp32 accumulate, A and B both bf16 or both f16, B majorness, N / 8, M / 16.
__host__ __device__ constexpr uint32_t p_instr_desc(int N, int b_mn_major, bool f16) {
    return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// ---- the walk over a block's range ------------------------------------------------------------------------------
struct PPiece {
    int g, slot, h, m;    // group, slot of the partial, KV head, 256-row block of the group
    int t0, t1;           // key tiles
    int len, rows;        // tokens of the prefix, packed rows of the group
    bool wide;            // both tiles have rows of their own
};
struct PWalk {
    int pos, hi, g;       // of the line; with chunks: piece pos = hi - 1, or none
    __device__ __forceinline__ static void fill(int h, int m, PPiece& pc) {
        pc.h = h;
        pc.m = m;
        pc.wide = pc.rows - m * kPrefixRows > 128;
    }
    __device__ __forceinline__ bool next(const PrefixParams& p, const PrefixPlan& plan, PPiece& pc) {
        for (;;) {
            if (pos >= hi) return false;
            const int chunk = *plan.chunk;
            if (chunk == 0)
                while (plan.line[g + 1] <= pos) ++g;
            pc.g = g;
            pc.len = plan.len[g];
            pc.rows = (plan.begin[g + 1] - plan.begin[g]) * p.R;
            const int tiles = (pc.len + kPrefixTile - 1) / kPrefixTile, nm = (pc.rows + kPrefixRows - 1) / kPrefixRows;
            if (chunk > 0) {
                // piece k of n: `each` tiles, one more in the first ones
                const int n = small_div(tiles + chunk - 1, chunk), o = pos - plan.piece[g], u = small_div(o, n), k = o - u * n;
                const int each = small_div(tiles, n), more = tiles - each * n;
                pc.slot = pos;
                pc.t0 = k * each + min(k, more);
                pc.t1 = pc.t0 + each + (k < more ? 1 : 0);
                pos = hi;
                const int h = small_div(u, nm);
                fill(h, u - h * nm, pc);
                return true;
            }
            const int per = tiles + kPrefixLead, o = pos - plan.line[g], u = o / per, v0 = o - u * per;
            const int end = min(pos + per - v0, hi), v1 = v0 + end - pos;
            pos = end;
            pc.t0 = max(v0 - kPrefixLead, 0);
            pc.t1 = max(v1 - kPrefixLead, 0);
            if (pc.t1 <= pc.t0) continue;
            pc.slot = plan.unit[g] + u + (int)blockIdx.x;
            fill(u / nm, u % nm, pc);
            return true;
        }
    }
};
__device__ __forceinline__ PWalk walk_of_block(const PrefixParams& p, const PrefixPlan& plan) {
    PWalk w;
    const int c = blockIdx.x;
    const int32_t* first = plan.line;       // of each group, on the scale that pos counts
    w.pos = w.hi = w.g = 0;
    if (*plan.chunk > 0) {
        first = plan.piece;
        if (c < first[p.groups]) {
            w.pos = c;
            w.hi = c + 1;
        }
    } else {
        const int T = first[p.groups], C = prefix_blocks(T, plan.chunk[1]);
        if (c < C && T > 0) {
            w.pos = prefix_range(T, c, C);
            w.hi = prefix_range(T, c + 1, C);
        }
    }
    if (w.pos < w.hi) {
        int lo = 0, hi = p.groups;          // first[lo] <= pos < first[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= w.pos) lo = mid; else hi = mid;
        }
        w.g = lo;
    }
    return w;
}

constexpr int kOwnStartNs = 7000;     // what starting and finishing the pass over the own caches takes, about
constexpr int kGapNs = 8000;          // what one pass behind the other loses between them, about (with less, large batches of 8-bit caches with
                                      // 16 packed rows took 71 us one behind the other instead of 61 side by side)
constexpr int kItemNs = 3000;         // what one of its items takes a block at least, about
constexpr int kMemoryRate = 5500;     // bytes a nanosecond that the device streams, about

// ---- making the plan ----------------------------------------------------------------------------------------------
__device__ __forceinline__ int warp_scan(int x, int lane) {     // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

constexpr int kLeavers = 512;        // threads of the last block that leave the sequences' lengths: the softmax's
constexpr int kBarLeft = 9, kBarGroups = 10;     // named barriers: the plan has been left; the groups and lengths are known

// The plan of up to kNearGroups groups, by one warp: lane g is group g. Everything but the sequences' lengths goes to `to`; where
// `leaves`, the threads that leave those are let go as soon as groups and lengths are known.
__device__ __forceinline__ void plan_by_warp(const PrefixParams& p, const PrefixPlan& to, int lane, bool leaves, uint32_t& flags) {
    const int given = lane <= p.groups ? p.group_begin[lane] : 0;
    int len = lane < p.groups ? p.prefix_lens[lane] : 0;
    int64_t tokens = 0;
    if (p.own_per_sm > 0)
#pragma unroll 4
        for (int b = lane; b < p.B; b += 32) tokens += max(p.seq_lens[b], 0);
    if (len < 0 || len > p.max_prefix_len) {
        flags |= kDevGroupClamped;
        len = len < 0 ? 0 : p.max_prefix_len;
    }
    // first sequences: the largest given so far, within [0, B]
    int begin = min(max(given, 0), p.B);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, begin, o);
        if (lane >= o) begin = max(begin, y);
    }
    if (lane <= p.groups && begin != given) flags |= kDevGroupClamped;
    const int next = __shfl_down_sync(0xffffffffu, begin, 1);
    const int rows = lane < p.groups ? (next - begin) * p.R : 0;
    if (rows == 0) len = 0;
    if (lane < p.groups) to.len[lane] = len;
    if (lane <= p.groups) to.begin[lane] = begin;
    if (leaves) named_barrier_sync(kBarGroups, kLeavers + 32);
    const int tiles = (len + kPrefixTile - 1) / kPrefixTile;
    const int units = tiles > 0 ? p.Hkv * ((rows + kPrefixRows - 1) / kPrefixRows) : 0;
    const int positions = units * (tiles + kPrefixLead);
    const int unit = warp_scan(units, lane), line = warp_scan(positions, lane);
    const int all_units = __shfl_sync(0xffffffffu, unit, 31), all = __shfl_sync(0xffffffffu, line, 31) - all_units * kPrefixLead;
    // How many blocks take part. What both passes take is estimated for sixteen ways of dividing the multiprocessors, a lane each (in
    // every block by the same instructions, so that all come to the same plan); none for the own caches means one pass behind the
    // other. Where the prefixes have so few tiles that half of the blocks stay idle, those are the own caches' anyway, and the
    // estimate (1.1 us, before the pass over the own caches can start) is left out.
    int blocks = p.blocks, own_blocks = 0x7fffffff;
    if (p.own_per_sm > 0 && all * 2 > p.blocks) {
        const bool wide = (rows - 1) % kPrefixRows >= 128;      // of a group's units all but the last are; that one may have half the work
        const int last = tiles > 0 && !wide ? p.Hkv * (tiles / 2) : 0;
        const int work = __reduce_add_sync(0xffffffffu, units * tiles - last);
        tokens -= (int64_t)(lane < p.groups ? next - begin : 0) * len;
        const float held = (float)__reduce_add_sync(0xffffffffu, (int)(tokens >> 24)) * 16777216.f + (float)__reduce_add_sync(0xffffffffu, (int)(tokens & 0xffffff));
        const float bytes = (fmaxf(held, 0.f) + (float)(p.B * (p.L - 1)) * (float)p.w) * (float)p.token_bytes;
        const int left = p.blocks * (lane & 15) / 16, mine = p.blocks - left, n_own = left > 0 ? left : p.blocks;
        const float prefix_ns = ceilf(__fdividef((float)work, (float)mine)) * (float)p.tile_ns;
        const float own_ns = (float)kOwnStartNs + fmaxf(__fdividef(bytes, (float)min(n_own * p.own_rate, kMemoryRate)),
                                                        __fdividef((float)p.own_items * (float)kItemNs, (float)(n_own * p.own_per_sm)));
        // side by side the longer one counts, and the shorter one a little: it takes its share of memory and of the L2
        const float ns = left > 0 ? fmaxf(prefix_ns, own_ns) + fminf(prefix_ns, own_ns) * 0.125f : prefix_ns + own_ns + (float)kGapNs;
        const uint32_t cost = (uint32_t)fminf(ns, 4e9f), best = __reduce_min_sync(0xffffffffu, cost);
        const int way = __ffs(__ballot_sync(0xffffffffu, cost == best)) - 1;
        if (way > 0) {
            blocks = __shfl_sync(0xffffffffu, mine, way);
            own_blocks = (p.blocks - blocks) * p.own_per_sm;
        }
    }
    // The shortest chunk that lets every piece have a block, tried in steps of an eighth from the average on, a lane each; not more
    // than a tenth and a tile above what the line's ranges hold.
    int chunk = 0, piece = 0;
    if (all_units > 0 && all_units <= blocks) {
        const int least = (all + blocks - 1) / blocks, step = (least + 7) / 8, s = least + lane * step;
        const int most = max((all + all_units * kPrefixLead) / blocks * 11 / 10 + 1, least);
        int n = 0;
        for (int g = 0; g < p.groups; ++g) {
            const int tg = __shfl_sync(0xffffffffu, tiles, g), ug = __shfl_sync(0xffffffffu, units, g);
            n += tg > 0 ? ug * small_div(tg + s - 1, s) : 0;
        }
        const uint32_t fits = __ballot_sync(0xffffffffu, s <= most && n <= blocks);
        if (fits != 0) {
            chunk = least + (__ffs(fits) - 1) * step;
            piece = warp_scan(tiles > 0 ? units * small_div(tiles + chunk - 1, chunk) : 0, lane);
        }
    }
    if (lane < p.groups) {
        to.line[lane + 1] = line;
        to.unit[lane + 1] = unit;
        to.piece[lane + 1] = piece;
    }
    if (lane == 0) {
        to.line[0] = to.unit[0] = to.piece[0] = 0;
        to.chunk[0] = chunk;
        to.chunk[1] = blocks;
        to.chunk[2] = own_blocks;
    }
}

// Leaves the plan `from` (in shared memory) where the kernels behind find it: here all but the lengths.
__device__ __forceinline__ void leave_plan(const PrefixParams& p, const PrefixPlan& from, int tid, int threads) {
    for (int g = tid; g <= p.groups; g += threads) {
        p.plan.begin[g] = from.begin[g];
        p.plan.line[g] = from.line[g];
        p.plan.unit[g] = from.unit[g];
        p.plan.piece[g] = from.piece[g];
        if (g < p.groups) p.plan.len[g] = from.len[g];
    }
    if (tid < 3) p.plan.chunk[tid] = from.chunk[tid];
}
// And what each sequence holds itself; `ahead` is the length of sequence `tid`.
__device__ __forceinline__ void leave_lens(const PrefixParams& p, const PrefixPlan& from, int tid, int threads, int ahead, uint32_t& flags) {
    for (int b = tid; b < p.B; b += threads) {
        // the group of sequence b, if any
        int len = 0;
        if (p.groups > 0 && b >= from.begin[0] && b < from.begin[p.groups]) {
            int lo = 0, hi = p.groups;             // begin[lo] <= b < begin[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (from.begin[mid] <= b) lo = mid; else hi = mid;
            }
            len = from.len[lo];
        }
        int n = b == tid ? ahead : p.seq_lens[b];
        if (n < 0 || n > (int64_t)len + p.max_seq_len) {
            flags |= kDevSeqLenClamped;
            n = n < 0 ? 0 : len + p.max_seq_len;
        }
        p.plan.own_lens[b] = max(0, n - len);
        for (int l = 1; l < p.L; ++l) {
            const int cut = max(0, n - p.delta[l]);
            int wl = min(cut, p.w);
            if (p.win_lens != nullptr && cut > 0) {
                wl = p.win_lens[b * (p.L - 1) + l - 1];
                if (wl < 0 || wl > p.w) {
                    flags |= kDevWinLenClamped;
                    wl = wl < 0 ? 0 : p.w;
                }
            }
            p.plan.win_lens[b * (p.L - 1) + l - 1] = wl;
        }
    }
}

// Key tiles of a piece that tile x takes: every one, or every second.
__device__ __forceinline__ int tiles_of(const PPiece& pc, int x) {
    const int n = pc.t1 - pc.t0;
    return pc.wide ? n : (n + 1 - x) >> 1;
}

// True in one thread of a converged warp, always the same. The compiler sees that a branch on it holds a single thread, and
// issues the products one behind the other; behind `lane == 0` it cannot know, and each took twice as long to issue.
__device__ __forceinline__ bool one_thread() {
    uint32_t y;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(y));
    return y != 0;
}

// A value that all lanes of a converged warp hold alike, in a form that the compiler keeps in uniform registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) { return __shfl_sync(0xffffffffu, x, 0); }
// umma_commit on a barrier's shared-memory address.
__device__ __forceinline__ void commit_to(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

template <int RING>
struct Ring {
    int slot = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void advance() {
        if (++slot == RING) {
            slot = 0;
            parity ^= 1u;
        }
    }
};

// ---- softmax ----------------------------------------------------------------------------------------------------------
// A warp takes 16 rows and the 64 keys of a half tile, four threads to a row, as the fragments of a tensor-memory load of 16 lanes lie:
// a thread has rows r and r + 8 (r = lane / 4 of the 16) and of each 8 keys the two at 2 (lane % 4): scores 4 g + {0, 1} are row r's at
// keys 8 g + 2 (lane % 4) + {0, 1}, 4 g + {2, 3} row r + 8's. A row's threads tell each other by shuffles; no warp waits for another.
//
// Powers of two above the reference that a score may reach before the reference moves. With f16 probabilities references lie 8
// below the maximum, so that the small ones do not fall under f16's range: up to 2^14 stays far from its end.
template <bool FP8>
constexpr float kAbove = FP8 ? 14.f : 8.f;
template <bool FP8>
constexpr float kBelow = FP8 ? 8.f : 0.f;
// Share of a row's sum, as 2^-kShareBits, from which on a bf16 probability has a second term. The largest error on sharply peaked
// rows is 0.88 of the bound (the result's rounding) for shares of 1/4, 0.35 and 1/2, and 1.43 for 0.66; 64 sequences of two loops behind
// 4096 tokens take 37.0, 36.5, 36.1 and 35.7 us.
constexpr float kShareBits = 1.5f;

// 64 columns of 16 lanes, as above.
__device__ __forceinline__ void tmem_ld_rows16(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
// 32 packed columns of 16 lanes: words 2 g + {0, 1} are rows r's and r + 8's pair of column 4 g + lane % 4.
__device__ __forceinline__ void tmem_st_pairs16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
                 "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
// Sum over a row's four threads.
__device__ __forceinline__ float row_sum(float y) {
    y += __shfl_xor_sync(0xffffffffu, y, 1);
    return y + __shfl_xor_sync(0xffffffffu, y, 2);
}
// D[tmem] += A[tmem] * B[smem] on the lanes whose bits in `off` are 0 (bit i of word w: lane 32 w + i).
__device__ __forceinline__ void umma_bf16_ts_lanes(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint4 off) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%4, %5, %6, %7}, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(off.x), "r"(off.y), "r"(off.z), "r"(off.w)
        : "memory");
}

// 16 columns of 16 lanes, to be scaled: row r's by f0, row r + 8's by f1.
__device__ __forceinline__ void tmem_scale_rows16(uint32_t taddr, float f0, float f1) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * ((i & 2) != 0 ? f1 : f0));
    asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

// Scores behind a row's last key become -inf; lim0, lim1: keys from the thread's first one to the end of its two rows.
__device__ __forceinline__ void p_mask(uint32_t (&r)[32], int lim0, int lim1) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (8 * (i >> 2) + (i & 1) >= ((i & 2) != 0 ? lim1 : lim0)) r[i] = 0xff800000u;
}
// Largest of a thread's scores of row r (K = 0) or r + 8 (K = 2).
template <int K>
__device__ __forceinline__ float p_max(const uint32_t (&r)[32]) {
    float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int g = 0; g < 8; ++g) m[g & 1] = fmaxf(fmaxf(m[g & 1], __uint_as_float(r[4 * g + K])), __uint_as_float(r[4 * g + K + 1]));
    return fmaxf(m[0], m[1]);
}
// Largest of a row's four threads.
__device__ __forceinline__ float row_max(float y) {
    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 1));
    return fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 2));
}

// 2^t of two numbers on the multiply-add units, which are less busy than the special-function unit (taken for an eighth of them: 128
// sequences behind 32768 tokens 141.4 us; for none 144.9, a quarter 142.3, half 147.8): t = n + f with n the nearest integer (Cody
// and Waite's split; n falls out of an addition of 1.5 * 2^23), 2^f on [-1/2, 1/2] by the cubic of least largest relative error
// (found by Lawson's iteration; 2^-13.7, a fiftieth of what rounding a probability to 8 bits costs), n added to the exponent. At
// 2^-125 and below, what the cubic gives there is taken off where EXACT0, so that a masked key weighs exactly 0 however large its
// value is (f16 probabilities lose so small a number anyway).
template <bool EXACT0>
__device__ __forceinline__ float2 exp2_by_fma(float2 t) {
    const float2 magic = make_float2(12582912.f, 12582912.f), minus = make_float2(-12582912.f, -12582912.f);
    t.x = fmaxf(t.x, -125.f);
    t.y = fmaxf(t.y, -125.f);
    const float2 z = __fadd2_rn(t, magic);
    const float2 n = __fadd2_rn(z, minus);
    const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), t);
    float2 e = __ffma2_rn(f, make_float2(0.05517167f, 0.05517167f), make_float2(0.24261113f, 0.24261113f));
    e = __ffma2_rn(f, e, make_float2(0.69326097f, 0.69326097f));
    e = __ffma2_rn(f, e, make_float2(0.99992806f, 0.99992806f));
    e = make_float2(__uint_as_float(__float_as_uint(e.x) + (__float_as_uint(z.x) << 23)), __uint_as_float(__float_as_uint(e.y) + (__float_as_uint(z.y) << 23)));
    constexpr float least = -0.99992806f * 0x1p-125f;
    return EXACT0 ? __fadd2_rn(e, make_float2(least, least)) : e;
}

// Scores -> probabilities, packed 16 bits wide, and their sums. KEEP: in fp32 they take the scores' place.
template <bool FP8, bool KEEP>
__device__ __forceinline__ void p_half(uint32_t (&r)[32], float scale, float m0, float m1, uint32_t (&pk)[16], float2& sum0, float2& sum1) {
    const float2 sc2 = make_float2(scale, scale), nm0 = make_float2(-m0, -m0), nm1 = make_float2(-m1, -m1);
#pragma unroll
    for (int g = 0; g < 8; ++g)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float2 t = __ffma2_rn(make_float2(__uint_as_float(r[4 * g + 2 * k]), __uint_as_float(r[4 * g + 2 * k + 1])), sc2, k == 0 ? nm0 : nm1);
            const float2 pr = (g & 3) == 3 && k == 1 ? exp2_by_fma<!FP8>(t) : make_float2(fast_exp2(t.x), fast_exp2(t.y));
            float2& s = k == 0 ? sum0 : sum1;
            s = __fadd2_rn(s, pr);
            pk[2 * g + k] = FP8 ? pack_f16x2(pr.x, pr.y) : pack_bf16x2(pr.x, pr.y);
            if (KEEP) {
                r[4 * g + 2 * k] = __float_as_uint(pr.x);
                r[4 * g + 2 * k + 1] = __float_as_uint(pr.y);
            }
        }
}
// What rounding the probabilities p to bf16 (pk) dropped, in the place of the first half of p.
__device__ __forceinline__ void p_second(uint32_t (&p)[32], const uint32_t (&pk)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
        p[i] = pack_bf16x2(__uint_as_float(p[2 * i]) - __uint_as_float(pk[i] << 16), __uint_as_float(p[2 * i + 1]) - __uint_as_float(pk[i] & 0xffff0000u));
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kPThreads<FP8>, 1)
plt_prefix_main(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmQ,
                const __grid_constant__ PrefixParams p) {
    using C = PCfg<D, FP8>;
    constexpr int HALVES = D / 64;
    extern __shared__ uint8_t prefix_smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)prefix_smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* q_smem = smem;                                        // [2][tile]
    uint8_t* ring = smem + 2 * C::TILE;                            // [RING][tile]
    uint8_t* raw = ring + (size_t)C::RING * C::TILE;               // [RAW][tile of codes]
    uint64_t* bars = (uint64_t*)(raw + (size_t)C::RAW * C::RAW_TILE);
    int32_t* s_ctl = (int32_t*)(bars + C::COUNT);                  // [0] abort flag, [1] tensor-memory base, [2] loads issued
    int32_t* s_plan = s_ctl + 16;                                  // begin, len, line, unit, piece: [kNearGroups + 1] each; chunk
    volatile uint8_t* s_lo = (uint8_t*)(s_plan + 5 * (kNearGroups + 1) + 4);       // [tile][half][warp]: 1: the warp has left second terms
    volatile int* abort_flag = (volatile int*)s_ctl;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;

    if (tid == 0) {
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
        if (p.q_tma) tma_prefetch_desc(&tmQ);
        s_ctl[0] = 0;
        s_ctl[2] = s_ctl[3] = s_ctl[4] = 0;
        for (int s = 0; s < C::RING; ++s) {
            mbar_init(&bars[C::FULL + s], FP8 ? 4 : 1);
            mbar_init(&bars[C::EMPTY + s], 2);
        }
        for (int s = 0; s < C::RAW; ++s) {
            mbar_init(&bars[C::RFULL + s], 1);
            mbar_init(&bars[C::REMPTY + s], 4);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&bars[C::QFULL + x], p.q_tma && !FP8 ? 1 : 8);
            mbar_init(&bars[C::QRAW + x], 1);
            mbar_init(&bars[C::ODONE + x], 1);
        }
        for (int s = 0; s < 4; ++s) {
            mbar_init(&bars[C::SFULL + s], 1);
            mbar_init(&bars[C::PFULL + s], 8);
            mbar_init(&bars[C::PVDONE + s], 1);
        }
        mbar_fence_init();
    }
    if (wid == 1) tmem_alloc((uint32_t*)&s_ctl[1], 512);
    if (wid == 3) s_lo[lane] = 0;
    // Few groups: this kernel is an ordinary launch, each block makes the plan for itself, and the last one leaves it for the kernels
    // behind. Many: it starts behind the plan kernel's start and waits for its end.
    const bool near = p.groups <= kNearGroups, leaves = near && blockIdx.x + 1 == gridDim.x;
    PrefixPlan plan = p.plan;
    uint32_t reported = 0;
    if (near) {
        constexpr int W = kNearGroups + 1;
        plan.begin = s_plan;
        plan.len = s_plan + W;
        plan.line = s_plan + 2 * W;
        plan.unit = s_plan + 3 * W;
        plan.piece = s_plan + 4 * W;
        plan.chunk = s_plan + 5 * W;
        if (!leaves) grid_launch_dependents();
        if (wid == 2) plan_by_warp(p, plan, lane, leaves, reported);
        if (leaves && wid >= 4 && wid < 20) {      // the warps of the softmax, which have nothing to do yet
            const int ahead = tid - 128 < p.B ? p.seq_lens[tid - 128] : 0;
            named_barrier_sync(kBarGroups, kLeavers + 32);
            leave_lens(p, plan, tid - 128, kLeavers, ahead, reported);
        }
    } else {
        grid_dependency_wait();
        grid_launch_dependents();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = (uint32_t)s_ctl[1];
    // columns: S_A 0..127 in halves of 64 (its P over the first 32 of each, once the scores have been read), S_B 128..255, O_A from
    // 256, O_B from 384
    if (leaves) {
        // The kernels behind acquire the plan: this one is let go once it has been released.
        if (wid >= 4 && wid < 20) {
            leave_plan(p, plan, tid - 128, kLeavers);
            named_barrier_sync(kBarLeft, kLeavers);
            if (tid == 128) {
                release_word(p.plan.ready);
                grid_launch_dependents();
            }
        }
        if (reported) atomicOr(p.status, reported);
    }
    PWalk walk = walk_of_block(p, plan);
    PPiece pc;
    bool ok = true;

    if (wid == 0) {
        // =========================== TMA producer ===========================================================
        constexpr int NRING = FP8 ? C::RAW : C::RING;
        constexpr int TILE_BYTES = FP8 ? C::RAW_TILE : C::TILE;
        constexpr int HB = kPrefixTile * 128;                      // bytes of a 128-byte wide half
        uint8_t* const to = FP8 ? raw : ring;
        uint64_t* const full = bars + (FP8 ? C::RFULL : C::FULL);
        uint64_t* const empty = bars + (FP8 ? C::REMPTY : C::EMPTY);
        const uint64_t keep = l2_evict_first_policy();
        const int box_bits = 31 - __clz(p.kbox), per_tile = kPrefixTile >> box_bits;     // boxes are of a power of two keys
        Ring<NRING> rg;
        uint32_t issued = 0, flags = 0;
        while (ok && walk.next(p, plan, pc)) {
            // lane j holds the page of the tile's j-th box, read one tile ahead
            auto page_of = [&](int t) {
                const int key = t * kPrefixTile + lane * p.kbox;
                if (p.page_size == 0 || lane >= per_tile || key >= pc.len) return 0;
                int page = p.page_table[(int64_t)pc.g * p.max_pages + key / p.page_size];
                if (page < 0 || page >= p.num_pool_pages) {
                    flags |= kDevPageIdClamped;
                    page = page < 0 ? 0 : p.num_pool_pages - 1;
                }
                return page;
            };
            int next_page = page_of(pc.t0);
            for (int t = pc.t0; t < pc.t1 && ok; ++t) {
                const int page = next_page;
                if (t + 1 < pc.t1) next_page = page_of(t + 1);
                const int boxes = min(per_tile, (pc.len - t * kPrefixTile + p.kbox - 1) >> box_bits);
                for (int which = 0; which < 2; ++which) {
                    if (issued >= (uint32_t)NRING) ok = seq_wait(&empty[rg.slot], rg.parity ^ 1u, abort_flag);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    uint8_t* dst = to + (size_t)rg.slot * TILE_BYTES;
                    if (lane == 0) mbar_expect_tx(&full[rg.slot], (uint32_t)(boxes * p.kbox) * (TILE_BYTES / kPrefixTile));
                    for (int j = 0; j < boxes; ++j) {
                        const int pg = __shfl_sync(0xffffffffu, page, j);
                        const int key = t * kPrefixTile + j * p.kbox;
                        const int row = p.page_size > 0 ? key % p.page_size : key, outer = p.page_size > 0 ? pg : pc.g;
                        if (lane == 0)
#pragma unroll
                            for (int hf = 0; hf < (FP8 ? 1 : HALVES); ++hf)
                                tma_load_4d(dst + hf * HB + j * p.kbox * 128, which == 0 ? &tmK : &tmV, &full[rg.slot], hf * 64, row, pc.h, outer, keep);
                    }
                    __syncwarp();
                    ++issued;
                    rg.advance();
                }
            }
        }
        if (lane == 0) s_ctl[2] = (int32_t)issued;
        if (flags) atomicOr(p.status, flags);
    } else if (wid == 1 || wid == 3) {
        // =========================== product issue (whole warps walk, one thread issues) =====================
        // A wide piece's tile A is warp 1's and its tile B warp 3's; a narrow piece is warp 1's.
        constexpr uint32_t idesc_qk = p_instr_desc(64, 0, FP8), idesc_pv = p_instr_desc(D, 1, FP8);
        constexpr int HB = kPrefixTile * 128;
        const uint32_t q_a = smem_u32(q_smem), ring_a = smem_u32(ring), bars_a = smem_u32(bars);
        const uint64_t keep = l2_evict_first_policy();
        uint32_t base = 0;                    // ring tiles before this piece: K of its i-th key tile is base + 2 i, V the next
        uint32_t q_parity[2] = {0, 0}, p_parity[2] = {0, 0}, o_parity[2] = {0, 0};
        while (ok && walk.next(p, plan, pc)) {
            const int n = pc.t1 - pc.t0;
            auto wait_for = [&](int bar, uint32_t parity) {
                const bool y = seq_wait(&bars[bar], parity, abort_flag);
                ok = __all_sync(0xffffffffu, y);
            };
            // S_x,h = Q_x . K(i)[64 h ..]^T. The K tile is free once the second half of the last tile that takes it has been issued
            // (two arrivals: one of each tile, or both of the one).
            auto issue_s = [&](int i, int x, int h) {
                const uint32_t cnt = base + 2u * (uint32_t)i, slot = cnt % C::RING;
                if (h == 0) wait_for(C::FULL + slot, (cnt / C::RING) & 1u);
                if (!ok) return;
                tc_fence_after_sync();
                const uint64_t k0 = uniform(seq_smem_desc(ring_a + slot * C::TILE + h * 8192, 16, 1024)), q0 = uniform(seq_smem_desc(q_a + (uint32_t)x * C::TILE, 16, 1024));
                const uint32_t to = uniform(tmem_base + x * 128 + h * 64), free_bar = uniform(bars_a + 8u * (C::EMPTY + slot)), full_bar = uniform(bars_a + 8u * (C::SFULL + 2 * x + h));
                if (one_thread()) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint64_t off = (uint64_t)(((kk >> 2) * HB + (kk & 3) * 32) >> 4);
                        umma_bf16(to, q0 + off, k0 + off, idesc_qk, kk == 0 ? 0u : 1u);
                    }
                    commit_to(full_bar);
                    if (h == 1) {
                        commit_to(free_bar);
                        if (!pc.wide) commit_to(free_bar);
                    }
                }
                __syncwarp();
            };
            auto finish = [&](int i, int x, int h, bool first, bool last) {       // O_x += P_x,h . V(i)[64 h ..]
                wait_for(C::PFULL + 2 * x + h, p_parity[x]);
                if (!ok) return;
                const uint32_t cnt = base + 2u * (uint32_t)i + 1u, slot = cnt % C::RING;
                if (h == 0) wait_for(C::FULL + slot, (cnt / C::RING) & 1u);
                if (!ok) return;
                // Rows of the V tile behind the prefix may hold anything: zero them, so that a probability of 0 times garbage
                // is 0. (Of a wide piece by both warps, each for its own products. E4M3: by the warps that convert.)
                const int held = pc.len - (pc.t0 + i) * kPrefixTile;
                if (!FP8 && held < kPrefixTile && h == 0) {
                    uint8_t* v = ring + (size_t)slot * C::TILE;
                    for (int idx = lane; idx < (kPrefixTile - held) * (D / 8); idx += 32) {
                        const int row = held + idx / (D / 8), ch = idx % (D / 8);
                        *(uint4*)(v + (ch >> 3) * HB + row * 128 + (ch & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                tc_fence_after_sync();
                const uint64_t v0 = uniform(seq_smem_desc(ring_a + slot * C::TILE + h * 8192, HB, 1024));
                const uint32_t from = uniform(tmem_base + x * 128 + h * 64), to = uniform(tmem_base + x * 128 + 256), more = uniform(first ? 0u : 1u);
                const uint32_t free_bar = uniform(bars_a + 8u * (C::EMPTY + slot)), done_bar = uniform(bars_a + 8u * (C::PVDONE + 2 * x + h)), all_bar = uniform(bars_a + 8u * (C::ODONE + x));
                if (one_thread()) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) umma_bf16_ts(to, from + kk * 8, v0 + (uint64_t)(kk * 2048 >> 4), idesc_pv, kk > 0 ? 1u : more);
                    // the flags are read while these products run
                    uint32_t low = 0, high = 0;        // of the warps with the lower and the upper 16 lanes of each quarter, a byte each
                    if (!FP8) {
                        low = *(volatile uint32_t*)(s_lo + (2 * x + h) * 8);
                        high = *(volatile uint32_t*)(s_lo + (2 * x + h) * 8 + 4);
                    }
                    if ((low | high) != 0) {
                        auto off = [&](int quarter) { return ~((low >> (8 * quarter) & 1u) * 0xffffu | (high >> (8 * quarter) & 1u) * 0xffff0000u); };
                        const uint4 mask = make_uint4(off(0), off(1), off(2), off(3));
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) umma_bf16_ts_lanes(to, from + 32 + kk * 8, v0 + (uint64_t)(kk * 2048 >> 4), idesc_pv, mask);
                    }
                    commit_to(done_bar);
                    if (h == 1) {
                        commit_to(free_bar);
                        if (!pc.wide) commit_to(free_bar);
                        if (last) commit_to(all_bar);
                    }
                }
                __syncwarp();
                if (h == 1) p_parity[x] ^= 1u;
            };
            // Tile x's query rows by TMA, behind the last product that reads the ones before (a tile without a key tile in this piece
            // has none). 128 / G tokens of the G heads: rows behind the group's belong to the next one or to nobody, and nobody reads
            // their results.
            auto load_q = [&](int x) {
                if (!p.q_tma) return;
                if (one_thread()) {
                    uint64_t* bar = &bars[(FP8 ? C::QRAW : C::QFULL) + x];
                    mbar_expect_tx(bar, C::TILE);
                    ++s_ctl[3 + x];
                    const int token = plan.begin[pc.g] * p.L * p.Qn + ((pc.m * kPrefixRows + (pc.wide ? x * 128 : 0)) >> (31 - __clz(p.G)));     // G is a power of two
#pragma unroll
                    for (int hf = 0; hf < HALVES; ++hf) tma_load_4d(q_smem + x * C::TILE + hf * HB, &tmQ, bar, hf * 64, pc.h * p.G, token, 0, keep);
                }
                __syncwarp();
            };
            auto start = [&](int i, int x) {
                wait_for(C::QFULL + x, q_parity[x]);
                if (ok) issue_s(i, x, 0);
                if (ok) issue_s(i, x, 1);
            };
            // Where the ring is short, K two tiles on waits for the V tile that is about to be used: its scores come behind both halves.
            auto step = [&](int i, int x, int by) {
                const bool next = i + by < n;
                finish(i, x, 0, i < by, false);
                if (ok && next && (C::RING > 3 || by == 1)) issue_s(i + by, x, 0);
                if (ok) finish(i, x, 1, false, !next);
                if (ok && next && C::RING <= 3 && by == 2) issue_s(i + by, x, 0);
                if (ok && next) issue_s(i + by, x, 1);
            };
            if (pc.wide) {
                const int x = wid >> 1;
                load_q(x);
                start(0, x);
                for (int i = 0; i < n && ok; ++i) step(i, x, 1);
                if (n & 1) p_parity[x ^ 1] ^= 1u;
            } else if (wid == 1) {
                load_q(0);
                if (n > 1) load_q(1);
                start(0, 0);
                if (ok && n > 1) start(1, 1);
                for (int i = 0; i < n && ok; ++i) step(i, i & 1, 2);
            } else {
                if (tiles_of(pc, 0) & 1) p_parity[0] ^= 1u;
                if (tiles_of(pc, 1) & 1) p_parity[1] ^= 1u;
            }
            q_parity[0] ^= 1u;
            if (tiles_of(pc, 1) > 0) q_parity[1] ^= 1u;
            base += 2u * (uint32_t)n;
            // On behind the piece's last products: then the query tiles are free, and all of the piece's ring tiles have landed, which
            // warp 3 does not see of a narrow piece (a barrier's parity says nothing about the phase before the last).
            for (int x = 0; x < 2 && ok; ++x)
                if (tiles_of(pc, x) > 0) {
                    wait_for(C::ODONE + x, o_parity[x]);
                    o_parity[x] ^= 1u;
                }
        }
    } else if (wid == 2 || wid >= 20) {
        // =========================== E4M3 codes to f16 =======================================================
        if constexpr (FP8) {
            constexpr int HB = kPrefixTile * 128;
            Ring<C::RAW> src;
            Ring<C::RING> dst;
            uint32_t done = 0;
            const int ct = (wid == 2 ? 0 : wid - 19) * 32 + lane;      // of 128
            while (ok && walk.next(p, plan, pc))
                for (int t = pc.t0; t < pc.t1 && ok; ++t)
                    for (int which = 0; which < 2 && ok; ++which) {
                        ok = seq_wait(&bars[C::RFULL + src.slot], src.parity, abort_flag);
                        if (ok && done >= (uint32_t)C::RING) ok = seq_wait(&bars[C::EMPTY + dst.slot], dst.parity ^ 1u, abort_flag);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        const uint8_t* a = raw + (size_t)src.slot * C::RAW_TILE;
                        uint8_t* o = ring + (size_t)dst.slot * C::TILE;
                        const int held = pc.len - t * kPrefixTile;       // rows from here on are zeroed
                        uint4 codes[8];
                        const int c = ct & 7;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int row = k * 16 + (ct >> 3);
                            codes[k] = *(const uint4*)(a + row * 128 + ((c ^ (row & 7)) << 4));
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int row = k * 16 + (ct >> 3);
                            uint4 v = codes[k];
                            if (row >= held) v = make_uint4(0, 0, 0, 0);
                            const uint4 lo = make_uint4(e4m3x2_to_f16x2(v.x & 0xffffu), e4m3x2_to_f16x2(v.x >> 16), e4m3x2_to_f16x2(v.y & 0xffffu),
                                                        e4m3x2_to_f16x2(v.y >> 16));
                            const uint4 hi = make_uint4(e4m3x2_to_f16x2(v.z & 0xffffu), e4m3x2_to_f16x2(v.z >> 16), e4m3x2_to_f16x2(v.w & 0xffffu),
                                                        e4m3x2_to_f16x2(v.w >> 16));
                            uint8_t* half = o + (c >> 2) * HB + row * 128;
                            const int c0 = (2 * (c & 3)) ^ (row & 7), c1 = (2 * (c & 3) + 1) ^ (row & 7);
                            // the two halves' threads store their pieces in opposite order: no two in one bank
                            const bool swap = c >= 4;
                            *(uint4*)(half + ((swap ? c1 : c0) << 4)) = swap ? hi : lo;
                            *(uint4*)(half + ((swap ? c0 : c1) << 4)) = swap ? lo : hi;
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(&bars[C::FULL + dst.slot]);
                            mbar_arrive(&bars[C::REMPTY + src.slot]);
                        }
                        ++done;
                        src.advance();
                        dst.advance();
                    }
        }
    } else {
        // =========================== softmax, query rows and partials ======================================
        constexpr int HB = kPrefixTile * 128;
        constexpr int PART = D / 2;                        // elements of a query row that a thread loads
        const int x = (wid - 4) >> 3, half = ((wid - 4) >> 2) & 1;
        const int wq = wid & 3, row = wq * 32 + lane;      // lane quarter of tensor memory; row of the tile whose query it loads
        const int row0 = wq * 32 + half * 16 + (lane >> 2);        // rows whose scores it has: this one and 8 on
        const uint32_t lane_off = (uint32_t)(wq * 32 + half * 16) << 16;
        const uint32_t tS = tmem_base + lane_off + x * 128, tO = tmem_base + lane_off + 256 + x * 128;
        uint32_t s_parity = 0, o_parity = 0, r_parity = 0, told = 0;       // told: bit h: the flag of half h is set
        while (ok && walk.next(p, plan, pc)) {
            // ---- a row's query, and how many tokens of the prefix the two rows see -----------------------------------
            const int first_row = pc.m * kPrefixRows + (pc.wide ? x * 128 : 0);
            const int mine = tiles_of(pc, x), step = pc.wide ? 1 : 2;
            auto sees_of = [&](int lr) {
                if (lr >= pc.rows) return 0;
                const int b = small_div(lr, p.R), lq = small_div(lr - b * p.R, p.G), l = small_div(lq, p.Qn);
                return min(pc.len, row_sees(p.seq_lens[plan.begin[pc.g] + b], (int64_t)pc.len + p.max_seq_len, p.delta[l], p.Qn - 1 - (lq - l * p.Qn)));
            };
            int sees0 = 0, sees1 = 0;
            if (mine > 0) {
                uint8_t* q = q_smem + x * C::TILE;
                if (FP8 || !p.q_tma) {
                    const int lr = first_row + row;
                    const bool in = lr < pc.rows;
                    const int bg = in ? small_div(lr, p.R) : 0, b = in ? plan.begin[pc.g] + bg : 0, r = in ? lr - bg * p.R : 0, lq = small_div(r, p.G);
                    uint4 v[PART / 8];
                    if (p.q_tma) {       // bf16 rows that TMA wrote become f16 in place
                        ok = seq_wait(&bars[C::QRAW + x], r_parity, abort_flag);
                        ok = __all_sync(0xffffffffu, ok);
                        r_parity ^= 1u;
                        if (!ok) break;
                    }
                    const uint4* src = (const uint4*)((const __nv_bfloat16*)p.q + (((int64_t)b * p.L * p.Qn + lq) * p.Hq + pc.h * p.G + (r - lq * p.G)) * D + half * PART);
#pragma unroll
                    for (int c = 0; c < PART / 8; ++c) {
                        const int ch = half * (PART / 8) + c;
                        if (p.q_tma) v[c] = *(const uint4*)(q + (ch >> 3) * HB + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
                        else v[c] = in ? src[c] : make_uint4(0, 0, 0, 0);
                    }
#pragma unroll
                    for (int c = 0; c < PART / 8; ++c) {
                        if (FP8) {
                            uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) w[i] = pack_f16x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
                            v[c] = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        const int ch = half * (PART / 8) + c;
                        *(uint4*)(q + (ch >> 3) * HB + row * 128 + (((ch & 7) ^ (row & 7)) << 4)) = v[c];
                    }
                    fence_proxy_async_smem();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars[C::QFULL + x]);
                }
                sees0 = sees_of(first_row + row0);
                sees1 = sees_of(first_row + row0 + 8);
            }
            const float scale = FP8 ? fmaxf(p.scale_log2 * p.k_scale[pc.h], 1e-30f) : p.scale_log2;     // above 0: -inf has to stay that
            float m0 = kSeqNoMax, m1 = kSeqNoMax, most0 = 0.f, most1 = 0.f;      // most (bf16): scores above it take a longer way
            float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
            const int all_see = __reduce_min_sync(0xffffffffu, min(sees0, sees1));
            for (int i = 0; i < mine; ++i) {
                const int t = pc.t0 + (pc.wide ? 0 : x) + i * step;
                auto half_tile = [&](int h) {
                    const bool first = i == 0 && h == 0;
                    ok = seq_wait(&bars[C::SFULL + 2 * x + h], s_parity, abort_flag);
                    ok = __all_sync(0xffffffffu, ok);      // the tensor-memory accesses below are collective over the warp
                    if (!ok) return;
                    tc_fence_after_sync();
                    uint32_t r[32];
                    tmem_ld_rows16(tS + h * 64, r);
                    const int key = t * kPrefixTile + h * 64;
                    tmem_wait_ld();
                    if (key + 64 > all_see) p_mask(r, sees0 - key - 2 * (lane & 3), sees1 - key - 2 * (lane & 3));
                    const float top0 = p_max<0>(r) * scale, top1 = p_max<2>(r) * scale;
                    const bool high = first || top0 > (FP8 ? m0 + kAbove<FP8> : most0) || top1 > (FP8 ? m1 + kAbove<FP8> : most1);
                    const bool slow = __any_sync(0xffffffffu, high || (!FP8 && (told >> h & 1u) != 0));
                    if (slow) {
                        if (FP8 || __any_sync(0xffffffffu, first || top0 > m0 + kAbove<FP8> || top1 > m1 + kAbove<FP8>)) {
                            const float n0 = fmaxf(m0, row_max(top0) - kBelow<FP8>), n1 = fmaxf(m1, row_max(top1) - kBelow<FP8>);
                            const float f0 = fast_exp2(m0 - n0), f1 = fast_exp2(m1 - n1);
                            m0 = n0;
                            m1 = n1;
                            sum0 = make_float2(sum0.x * f0, sum0.y * f0);
                            sum1 = make_float2(sum1.x * f1, sum1.y * f1);
                            if (!first) {
                                // O against the new reference, once the product of the half before has completed. (The one before that
                                // on the same barrier has: this warp has seen scores that were issued behind it.)
                                ok = seq_wait(&bars[C::PVDONE + 2 * x + (h ^ 1)], s_parity ^ (uint32_t)(h ^ 1), abort_flag);
                                ok = __all_sync(0xffffffffu, ok);
                                if (!ok) return;
                                tc_fence_after_sync();
#pragma unroll 1
                                for (int c = 0; c < D / 16; ++c) tmem_scale_rows16(tO + c * 16, f0, f1);
                            }
                        }
                        if (!FP8) {
                            uint32_t pk[16];          // (registers that both ways shared took 148.0 us instead of 145.5)
                            p_half<FP8, true>(r, scale, m0, m1, pk, sum0, sum1);
                            tmem_st_pairs16(tS + h * 64, pk);
                            const float all0 = row_sum(sum0.x + sum0.y) * exp2f(-kShareBits), all1 = row_sum(sum1.x + sum1.y) * exp2f(-kShareBits);
                            const bool second = __any_sync(0xffffffffu, fast_exp2(top0 - m0) > all0 || fast_exp2(top1 - m1) > all1);
                            most0 = m0 + fminf(__log2f(all0), kAbove<FP8>);
                            most1 = m1 + fminf(__log2f(all1), kAbove<FP8>);
                            if (second) {
                                p_second(r, pk);
                                tmem_st_pairs16(tS + h * 64 + 32, (const uint32_t(&)[16])r);
                            }
                            told = (told & ~(1u << h)) | (uint32_t)second << h;
                            if (lane == 0) s_lo[(2 * x + h) * 8 + half * 4 + wq] = second;
                        }
                    }
                    if (FP8 || !slow) {
                        uint32_t pk[16];
                        p_half<FP8, false>(r, scale, m0, m1, pk, sum0, sum1);
                        tmem_st_pairs16(tS + h * 64, pk);
                    }
                    tmem_wait_st();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars[C::PFULL + 2 * x + h]);
                };
                // a copy of the code for each half only where it is short enough: with second terms copies took 146.4 us against 145.5 (128
                // sequences behind 32768 tokens) and 36.9 against 36.2 (64 behind 4096); 8-bit caches 42.4 against 44.1
                if constexpr (FP8) {
                    half_tile(0);
                    if (ok) half_tile(1);
                } else {
#pragma unroll 1
                    for (int h = 0; h < 2 && ok; ++h) half_tile(h);
                }
                if (!ok) break;
                s_parity ^= 1u;
            }
            if (!ok) break;
            // ---- the partial ---------------------------------------------------------------------------------------
            const int64_t slot = pc.slot;
            float s0 = sum0.x + sum0.y, s1 = sum1.x + sum1.y;
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                s0 += __shfl_xor_sync(0xffffffffu, s0, o);
                s1 += __shfl_xor_sync(0xffffffffu, s1, o);
            }
            if ((lane & 3) < 2) {
                // by the count of keys, not by the reference, which scores that are not numbers leave alone
                const float m = (lane & 1) != 0 ? m1 : m0;
                const bool saw = mine > 0 && ((lane & 1) != 0 ? sees1 : sees0) > (pc.t0 + (pc.wide ? 0 : x)) * kPrefixTile;
                *(float2*)(p.ml + ((slot * 2 + x) * 128 + row0 + 8 * (lane & 1)) * 2) = make_float2(saw ? m : -INFINITY, !saw ? 0.f : (lane & 1) != 0 ? s1 : s0);
            }
            if (mine > 0) {
                ok = seq_wait(&bars[C::ODONE + x], o_parity, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                o_parity ^= 1u;
                if (!ok) break;
                tc_fence_after_sync();
                const float f = FP8 ? p.v_scale[pc.h] : 1.f;
                float* out = p.acc + (slot * 2 + x) * (128 * D) + ((lane & 3) >> 1) * 512 + row0 * 4 + 2 * (lane & 1);
#pragma unroll 1
                for (int c = 0; c < D / 64; ++c) {
                    uint32_t r[32];
                    tmem_ld_rows16(tO + c * 64, r);
                    tmem_wait_ld();
#pragma unroll
                    for (int g = 0; g < 8; ++g)
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            *(float2*)(out + (c * 16 + g * 2) * 512 + 32 * k) = make_float2(__uint_as_float(r[4 * g + 2 * k]) * f, __uint_as_float(r[4 * g + 2 * k + 1]) * f);
                }
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (tid == 0 && s_ctl[0] != 0) {
        atomicOr(p.status, kDevWaitTimeout);
        // give every copy that was issued a bounded chance to land before the block retires
        constexpr int NRING = FP8 ? C::RAW : C::RING;
        const uint32_t issued = (uint32_t)s_ctl[2], outstanding = issued < (uint32_t)NRING ? issued : (uint32_t)NRING;
        for (uint32_t k = 0; k < outstanding; ++k) {
            const uint32_t cnt = issued - 1 - k;
            mbar_wait_bounded(&bars[(FP8 ? C::RFULL : C::FULL) + cnt % NRING], (cnt / NRING) & 1u, kSeqWaitNs);
        }
        if (p.q_tma)        // the last query tiles: s_ctl[3 + x] counts the ones asked for
            for (int x = 0; x < 2; ++x)
                if (s_ctl[3 + x] > 0) mbar_wait_bounded(&bars[(FP8 ? C::QRAW : C::QFULL) + x], (uint32_t)(s_ctl[3 + x] - 1) & 1u, kSeqWaitNs);
    }
    __syncthreads();
    if (wid == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, 512);
    }
}

// ---- the plan of many groups, or of none ---------------------------------------------------------------------------------
// One block: clamped groups and lengths, the line of their units, and what each sequence holds itself.
constexpr int kPlanThreads = 512;

__global__ void __launch_bounds__(kPlanThreads) plt_prefix_plan(const __grid_constant__ PrefixParams p) {
    __shared__ int32_t s_begin[kMaxGroups + 1], s_len[kMaxGroups], s_line[kMaxGroups + 1], s_unit[kMaxGroups + 1], s_piece[kMaxGroups + 1], s_chunk[3];
    grid_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31;
    uint32_t flags = 0;
    for (int g = tid; g <= p.groups && p.groups > 0; g += kPlanThreads) s_begin[g] = p.group_begin[g];
    for (int g = tid; g < p.groups; g += kPlanThreads) {
        int n = p.prefix_lens[g];
        if (n < 0 || n > p.max_prefix_len) {
            flags |= kDevGroupClamped;
            n = n < 0 ? 0 : p.max_prefix_len;
        }
        s_len[g] = n;
    }
    if (tid == 0 && p.groups == 0) s_begin[0] = 0;
    __syncthreads();
    if (tid < 32) {
        // first sequences: running maximum of what the caller gave, within [0, B]; then the line and the units
        int last = 0, line = 0, unit = 0;
        for (int g0 = 0; g0 <= p.groups; g0 += 32) {
            const int g = g0 + lane;
            const int given = g <= p.groups ? s_begin[g] : 0;
            int v = min(max(given, 0), p.B);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v = max(v, y);
            }
            v = max(v, last);
            last = __shfl_sync(0xffffffffu, v, 31);
            if (g <= p.groups) {
                if (v != given) flags |= kDevGroupClamped;
                s_begin[g] = v;
            }
        }
        __syncwarp();
        for (int g0 = 0; g0 < p.groups; g0 += 32) {
            const int g = g0 + lane;
            int units = 0, positions = 0;
            if (g < p.groups) {
                const int rows = (s_begin[g + 1] - s_begin[g]) * p.R;
                if (rows == 0) s_len[g] = 0;
                const int tiles = (s_len[g] + kPrefixTile - 1) / kPrefixTile;
                units = tiles > 0 ? p.Hkv * ((rows + kPrefixRows - 1) / kPrefixRows) : 0;
                positions = units * (tiles + kPrefixLead);
            }
            const int u = warp_scan(units, lane), q = warp_scan(positions, lane);
            if (g < p.groups) {
                s_unit[g] = unit + u - units;
                s_line[g] = line + q - positions;
                s_piece[g] = 0;
            }
            unit += __shfl_sync(0xffffffffu, u, 31);
            line += __shfl_sync(0xffffffffu, q, 31);
        }
        if (lane == 0) {
            s_unit[p.groups] = unit;
            s_line[p.groups] = line;
            s_piece[p.groups] = 0;
            s_chunk[0] = 0;
            s_chunk[1] = p.blocks;
            s_chunk[2] = 0x7fffffff;
        }
    }
    __syncthreads();
    PrefixPlan from = p.plan;
    from.begin = s_begin;
    from.len = s_len;
    from.line = s_line;
    from.unit = s_unit;
    from.piece = s_piece;
    from.chunk = s_chunk;
    leave_plan(p, from, tid, kPlanThreads);
    leave_lens(p, from, tid, kPlanThreads, tid < p.B ? p.seq_lens[tid] : 0, flags);
    if (flags) atomicOr(p.status, flags);
    __syncthreads();
    if (tid == 0) release_word(p.plan.ready);
}

template <int D, bool FP8>
cudaError_t launch_one(const CUtensorMap maps[3], const PrefixParams& pp, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)pp.blocks);
    cfg.blockDim = dim3(kPThreads<FP8>);
    cfg.dynamicSmemBytes = PCfg<D, FP8>::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pp.groups <= kNearGroups ? 0 : 1;
    return cudaLaunchKernelEx(&cfg, plt_prefix_main<D, FP8>, maps[0], maps[1], maps[2], pp);
}

}  // namespace

cudaError_t prefix_prepare(int d, bool fp8) {
    return allow_max_dynamic_smem(fp8 ? (const void*)plt_prefix_main<128, true>
                                      : d == 128 ? (const void*)plt_prefix_main<128, false> : (const void*)plt_prefix_main<64, false>);
}

cudaError_t launch_prefix_plan(const PrefixParams& pp, cudaStream_t stream) {
    if (pp.groups > 0 && pp.groups <= kNearGroups) return cudaSuccess;       // the prefix kernel makes it
    plt_prefix_plan<<<1, kPlanThreads, 0, stream>>>(pp);
    return cudaGetLastError();
}

cudaError_t launch_prefix_main(const CUtensorMap maps[3], const PrefixParams& pp, bool fp8, cudaStream_t stream) {
    if (fp8) return launch_one<128, true>(maps, pp, stream);
    return pp.d == 128 ? launch_one<128, false>(maps, pp, stream) : launch_one<64, false>(maps, pp, stream);
}

}  // namespace plt
