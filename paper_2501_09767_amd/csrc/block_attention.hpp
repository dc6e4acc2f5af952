// Attention over listed key blocks: parameter blocks, the launchers, and what the forward and the gradient kernels share.
#pragma once
#include "lemo_common.hpp"

namespace lemo {

// A list names key blocks for the rows of one query block: R = bq * G rows of the G query heads that read one key head, row r being
// query r / G of the block in head r % G of the group.  Work on a list is cut into tiles of rows; keys come in subtiles of 32.
struct BlockAttnParams {
    const uint16_t *Q, *K, *V;
    uint16_t* O;
    float* lse2;         // [H, S_q] or null
    const int* blocks;   // [n_qb, H_kv, T]
    const int* lengths;  // single tokens: [n_qb] keys of every sequence, or null
    float* parts;        // where a list is shared by several workgroups: their results, see PART_ROW
    int S_q, S_k, H, H_kv, G, T, b, bq, n_qb;  // S_k: keys that any query may see; under the mask none behind the last query is touched
    int nb;                // key blocks, of all keys
    int R, n_rt, n_parts;  // rows of a query block, tiles of them, shares of a list
    int first;             // workgroup of the launch's first one
    int pack, n_lists;     // lists that are worked on together (bq, n_qb, R then count `pack` blocks as one), and all there are
    long long q_start;
    long long q_ts, q_hs, k_ts, k_hs, k_ss, v_ts, v_hs, v_ss, o_ts, o_hs;  // element strides: token, head, sequence
    float c2;
    unsigned flags;
    HeadOrder order;
};

struct BlockGradParams {
    BlockAttnParams a;   // (O: the forward result, read only; lse2: likewise)
    const uint16_t* dO;
    long long do_ts, do_hs;
    uint16_t *dQ, *dK, *dV;  // contiguous
    float scale;
    float* delta;        // [H, S_q]: sum over a row of dO O
    unsigned* bits;      // [H_kv][nb][words]: bit i of word w: query block 32 w + i lists key block n
    int* counts;         // [H_kv * nb] query blocks that list a key block
    int* first;          // [H_kv * nb] where their list starts in `lists`
    int* lists;          // query blocks, ascending, key block by key block
    int* slots;          // [H_kv * nb] first partial result of a key block that is shared, or -1
    int4* items;         // key block, where its query blocks start in `lists`, how many, partial result or -1
    int* totals;         // [0]: items
    float* partial;      // [slot][2][b][d]
    int nb, words, share;  // share: query blocks that a workgroup takes of a list
    int S_all;             // keys that have a gradient
    int max_items;
};

struct BlockGradLayout { size_t delta, bits, counts, first, lists, slots, items, totals, partial, bytes; int share, max_items; };

constexpr int MAX_LISTED_SUBTILES = 3840;  // subtiles of 32 keys that a list may name: they stand in LDS, 15 KB (two lists of them beside two stages)
constexpr int MAX_PACKED_SUBTILES = 2048;  // of the union of lists, with a word of bits each
constexpr int MAX_LISTED_BLOCKS = 16384;   // key blocks that a choice is made from: their scores stand in LDS, 128 KB

int block_attention_parts(long long tiles, long long subtiles);
int block_attention_tile_rows(int R, bool walk);
int block_attention_packed(BlockAttnParams& p);
int launch_block_attention(BlockAttnParams p, int d, hipStream_t st);
int prepare_block_attention_pipe();
int launch_block_attention_pipe(const BlockAttnParams& p, hipStream_t st);  // heads of 128; p filled in as for the others
BlockGradLayout block_grad_layout(long long S_q, long long S_k, int H, int H_kv, int d, int T, int b, int bq);
int launch_block_attention_grad(BlockGradParams p, int d, hipStream_t st);

struct BlockSelectParams {
    const void* Q;
    const float* means;   // [sequences][nb][H_kv][d]
    const int* lengths;   // single tokens, or null
    int* blocks;          // [n_qb, H_kv, T]
    int S_q, S_k, H, H_kv, G, d, T, b, bq, n_qb, nb;
    int first;            // workgroup of the launch's first one
    long long q_start, q_ts, q_hs, means_ss;
    unsigned flags;
};
int launch_block_means(const void* K, long long S, int H_kv, int d, lemo_dtype_t dt, long long k_ts, long long k_hs, int b, float* means, hipStream_t st);
int launch_block_means_step(const void* K, const int* lengths, int B, long long S_max, int H_kv, int d, lemo_dtype_t dt, long long k_ss, long long k_ts,
                            long long k_hs, int b, float* means, int nb, hipStream_t st);
int launch_select_blocks(const BlockSelectParams& p, lemo_dtype_t dt, hipStream_t st);

// floats of a row's partial result: D values relative to a reference, the reference, the normaliser, room to 16 bytes
template <int D> constexpr int PART_ROW = D + 4;

#ifdef __HIPCC__
typedef __attribute__((ext_vector_type(4))) short s16x4;

// A tile of head rows in LDS: rows of 16-byte pieces without padding, piece p of row r at position p ^ swz(r).  16 consecutive rows then
// have any one piece in 16 different bank groups (row fragments), and so have 4 consecutive rows any two neighbouring pieces
// (transposing reads): both kinds of read are free of conflicts.
template <int D> struct HeadTile {
    static constexpr int ROWB = D * 2, PIECES = D / 8, CHUNKS = D / 16, COLS = D / 32;
    __device__ static constexpr int swz(int r) { return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3); }
    // this lane's 16 bytes of chunk c of row l32 of a subtile (an MFMA operand that has the subtile's rows as its own)
    __device__ static u32x4 row_fragment(const char* sub, int c, int lane) {
        const int r = lane & 31;
        return *reinterpret_cast<const u32x4*>(sub + r * ROWB + (((2 * c + (lane >> 5)) ^ swz(r)) << 4));
    }
    // operand that has columns 32 col + l32 as its rows and, as its contraction, rows 16 c + 4 half + {0..3} and 16 c + 8 + 4 half + {0..3}
    // of the subtile: the rows that registers 8 c .. 8 c + 7 of an accumulator belong to
    __device__ static u32x4 column_fragment(const char* sub, int col, int c, int lane) {
        const int half = lane >> 5, l32 = lane & 31, r = 16 * c + 4 * half + ((l32 & 15) >> 2);
        const int piece = col * 4 + (l32 >> 4) * 2 + ((l32 & 3) >> 1), low = (l32 & 1) * 8;
        const char* at0 = sub + r * ROWB + ((piece ^ swz(r)) << 4) + low;
        const char* at1 = sub + (r + 8) * ROWB + ((piece ^ swz(r + 8)) << 4) + low;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(at0));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(at1));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        return u32x4{l2.x, l2.y, h2.x, h2.y};
    }
};

// The same reads from addresses that differ by constants alone: a lane's place in a subtile once, then an exclusive or and an offset
// in the instruction for each fragment, so that no kernel has to keep (or spill) an address for every one.  Subtiles must begin at
// multiples of 256 bytes of LDS: workgroup memory that is dynamic only begins at 0.
template <typename T> __device__ __forceinline__ T __attribute__((address_space(3)))* lds_pointer(unsigned at) {
    return (T __attribute__((address_space(3)))*)(uintptr_t)at;
}
template <int D> struct TilePlace {
    using Tile = HeadTile<D>;
    unsigned row, col;
    __device__ explicit TilePlace(int lane) {
        const int half = lane >> 5, l32 = lane & 31, r = 4 * half + ((l32 & 15) >> 2);
        row = l32 * Tile::ROWB + ((half ^ Tile::swz(l32)) << 4);
        col = r * Tile::ROWB + ((((l32 >> 4) * 2 + ((l32 & 3) >> 1)) ^ Tile::swz(r)) << 4) + (l32 & 1) * 8;
    }
    // chunk c of row l32 of the subtile at `sub` (bytes of LDS)
    __device__ u32x4 row_fragment(unsigned sub, int c) const {
        return *lds_pointer<const u32x4>((sub + row) ^ (unsigned)(c << 5));
    }
    // columns 32 t + l32, rows 16 c + 4 half + {0..3} and 16 c + 8 + 4 half + {0..3}: 8 rows on, the exchange of pieces differs by 2
    __device__ u32x4 column_fragment(unsigned sub, int t, int c) const {
        const unsigned at = (sub + col) ^ (unsigned)(t << 6);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_pointer<s16x4>(at + 16 * c * Tile::ROWB));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_pointer<s16x4>((at ^ 32u) + (16 * c + 8) * Tile::ROWB));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        return u32x4{l2.x, l2.y, h2.x, h2.y};
    }
};

// Descriptor of the rows of a subtile from key `key` on, as many of the 32 as there are (none: S == key): what lies behind them arrives as
// zeros.  32-bit scalar arithmetic and no branch: 64-bit selections would put one beside every load.
template <int D> __device__ __forceinline__ u32x4 subtile_rsrc(const char* base, int key, int S, int pitch) {
    const unsigned long long a = reinterpret_cast<unsigned long long>(base) + (unsigned long long)(unsigned)key * (unsigned)pitch;
    u32x4 r;
    r[0] = (unsigned)a;
    r[1] = (unsigned)(a >> 32) & 0xffffu;
    r[2] = (unsigned)max((min(S - key, 32) - 1) * pitch + HeadTile<D>::ROWB, 0);  // (a pitch below a row's bytes: the row before ends where this does)
    r[3] = 0x00020000u;
    return r;
}

// The list of a query block as the rule for it says: an entry counts if it names a block, [0, nb), and lies above every such entry
// before it.  One wave; `take(entry, counts)` is called for 64 entries at a time, by all lanes.  `head`: this lane's entry of the
// first 64 (what lies past the list is -1).
__device__ __forceinline__ int list_head(const int* list, int T, int lane) { return lane < T ? list[lane] : -1; }
template <typename F> __device__ __forceinline__ void walk_list(const int* list, int T, int nb, int lane, int head, F&& take) {
    int top = -1;  // highest block so far
    for (int e0 = 0; e0 < T; e0 += 64) {
        const int raw = e0 == 0 ? head : e0 + lane < T ? list[e0 + lane] : -1, n = raw >= 0 && raw < nb ? raw : -1;
        int high = n;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int other = __shfl_up(high, s);
            if (lane >= s) high = max(high, other);
        }
        const int before = __shfl_up(high, 1);
        take(n, n > max(top, lane > 0 ? before : -1));
        top = max(top, __shfl(high, 63));
    }
}
template <typename F> __device__ __forceinline__ void walk_list(const int* list, int T, int nb, int lane, F&& take) {
    walk_list(list, T, nb, lane, list_head(list, T, lane), take);
}

// The subtiles of a list up to key `limit`, as first keys in `keys` (LDS); returns how many.  One wave.
__device__ __forceinline__ int list_subtiles(const int* list, int T, int b, int nb, int limit, int* keys, int lane, int head) {
    int count = 0;
    const int most = b / 32;
    walk_list(list, T, nb, lane, head, [&](int n, bool counts) {
        const int first = n * b;
        const int mine = counts && first <= limit ? min(most, (limit - first) / 32 + 1) : 0;
        int sum = mine;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int other = __shfl_up(sum, s);
            if (lane >= s) sum += other;
        }
        const int at = count + sum - mine;
        for (int i = 0; i < mine; ++i) keys[at + i] = first + 32 * i;
        count += __shfl(sum, 63);
    });
    return count;
}

__device__ __forceinline__ int list_subtiles(const int* list, int T, int b, int nb, int limit, int* keys, int lane) {
    return list_subtiles(list, T, b, nb, limit, keys, lane, list_head(list, T, lane));
}

// Several lists of few rows as one: the subtiles of all blocks that any of `lists` consecutive lists names, with a bit for each list that
// does.  Work on 32 rows costs the matrix cores the same whether one list fills 4 of them or eight lists fill all, so the union is
// never more than the lists one by one, and less by what they share.  All of the workgroup's waves; `marks` has room for nb words, `at`
// for the result: first keys, and `room` behind them the bits.  The count is written to *count.
template <int WAVES>
__device__ __forceinline__ void union_subtiles(const int* list, long long pitch, int lists, int T, int b, int nb, int limit, unsigned* marks, int* at, int room,
                                               int* count, int wave, int lane) {
    const int reach = min(nb, limit / b + 1);  // blocks that begin at or before the limit
    for (int n = threadIdx.x; n < reach; n += WAVES * 64) marks[n] = 0;
    __syncthreads();
    if (T <= 16) {  // four lists at a time, each in 16 lanes
        const int e = lane & 15;
        for (int m0 = wave * 4; m0 < lists; m0 += WAVES * 4) {
            const int m = m0 + (lane >> 4), raw = m < lists && e < T ? list[m * pitch + e] : -1, n = raw >= 0 && raw < nb ? raw : -1;
            int high = n;
#pragma unroll
            for (int s = 1; s < 16; s <<= 1) {
                const int other = __shfl_up(high, s, 16);
                if (e >= s) high = max(high, other);
            }
            const int before = __shfl_up(high, 1, 16);
            if (n > (e > 0 ? before : -1) && n < reach) atomicOr(marks + n, 1u << m);
        }
    } else {
        for (int m = wave; m < lists; m += WAVES)
            walk_list(list + m * pitch, T, nb, lane, [&](int n, bool counts) {
                if (counts && n < reach) atomicOr(marks + n, 1u << m);
            });
    }
    __syncthreads();
    if (wave == 0) {
        int total = 0;
        const int most = b / 32;
        for (int n0 = 0; n0 < reach; n0 += 64) {
            const int n = n0 + lane;
            const unsigned bits = n < reach ? marks[n] : 0;
            const int mine = bits ? min(most, (limit - n * b) / 32 + 1) : 0;
            int sum = mine;
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) {
                const int other = __shfl_up(sum, s);
                if (lane >= s) sum += other;
            }
            for (int i = 0; i < mine; ++i) {
                at[total + sum - mine + i] = n * b + 32 * i;
                at[room + total + sum - mine + i] = (int)bits;
            }
            total += __shfl(sum, 63);
        }
        if (lane == 0) *count = total;
    }
    __syncthreads();
}

// before a barrier that hands a stage over: this wave's LDS-direct loads have landed, its LDS reads have returned
__device__ __forceinline__ void settle_stage() {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __builtin_amdgcn_s_waitcnt(LGKMCNT0);
}
__device__ __forceinline__ float half_waves_max(float v) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
#endif

}  // namespace lemo
