// Attention over a tree of drafted tokens and the gathered context, and the accepted tokens' way into the contexts.
#include "en_tree_lane.h"

// ---------------------------------------------------------------------------
// tree_attn (bf16)
//
// All r * n rows of a KV head attend over the same L_c + done keys of the context, so the context is read once for all of
// them: 4 D bytes a key against 4 D flops a key and row. Up to 64 rows a KV head the step is bound by that read (64 agents x
// 16 K tokens x 4 nodes 766 us, 5.6 TB/s, as fast as a kernel that only reads), at 256 and more by feeding the matrix
// instructions (64 nodes of 56 heads over 8 K tokens 27.8 us, 15.1 GFLOP: 5 us of start, then 1.8 us a tile of 64 keys), and a
// short one by its start: arguments, the agent's header and counts, rows and angles are trips to memory one behind the other
// (8 nodes over 1.5 K tokens 9.0 us). A workgroup takes up to 8 row blocks of 32 rows (a wave each) of a KV head and a split
// of its keys; 64-key tiles of K and V^T go straight into LDS, NST of them in turn, and every wave reads all of them there.
//
// The tree's own keys are one more tile, the last split's first: the workgroup rotates them and lays them out in LDS as a
// tile of the context would be. Its mask is a row's way, a word whose bit m is node m.
//
// S^T = K Q^T and O^T += V^T P^T with 32 x 32 x 16 products as in attn_decode_kernel: a lane's column is a query row, its
// scores of 16 keys of a 32-key block are the operand of the second product as they are (that is what the exchanged bits
// 2 and 3 of a value's column are for). Scores are in log2 units, taken against a reference that is the maximum of the
// first keys a row sees and changes only where a score is 2^59 above it. The drafted keys, the probabilities and the output
// are rounded to bf16 once each (what the products take); sums, references and what the splits leave for the merge are
// float32. A query is the sum of two bf16 numbers (see cut_off) where up to four blocks of rows share a tile, and is rounded
// once, as in the other bf16 attention calls, where eight do: the second product of its scores would be half as much again of
// what those steps are bound by. (Outputs' error against 64 bits, 2-norm, 0.0021 - 0.0023 / 0.0029, of which the output's own
// rounding is 0.0017. Two parts / one, us: 8 nodes over 1.5 K tokens 9.0 / 8.2, 16 agents with 13 nodes over 2 K 32.4 / 30.6,
// 64 agents over 16 K 772 / 771, 4 agents with 32 nodes over 4 K 26.1 / 24.1. Eight blocks of 128 values in two parts spill, four
// blocks by eight waves do not; these / eight blocks in one part, with the merge: 64 nodes of 56 heads over 8 K 39.7 / 34.0, 64
// agents' 64 nodes over 2 K 257 / 179.)
//
// 16-byte chunks of a row lie in LDS exchanged by XOR with its number, so that 16 consecutive rows' reads of the same
// chunk meet distinct banks; the loads bring them there by reading their source in that order.
// ---------------------------------------------------------------------------
// Values that may be infinite or NaN are looked at, left out and added as bits: this library is built without NaN compares,
// and a NaN may be taken not to occur wherever a floating-point operation sees it.
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bool no_number(unsigned short bf16) { return (bf16 & 0x7f80) == 0x7f80; }

// A query's two parts have one sign and neither is zero, unless the query is: against a key that is infinite both products
// are the same infinity, and a score of minus infinity is no weight, where an infinity times zero, or two of different signs,
// were NaN. So the first part is cut off, not rounded (what is left is below 2^-7 of it, and its rounding below 2^-15), and the
// second is the smallest normal number where nothing is left.
__device__ __forceinline__ float cut_off(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ __forceinline__ bf16x8 with_sign_of(bf16x8 v, bf16x8 of)
{
    const u16x8 a = __builtin_bit_cast(u16x8, v) & (unsigned short)0x7fff, least = (unsigned short)0x0080;
    return __builtin_bit_cast(bf16x8, __builtin_elementwise_max(a, least) | (__builtin_bit_cast(u16x8, of) & (unsigned short)0x8000));
}

// Operands that are read ahead of the products. (64 nodes of 56 heads over 8 K tokens: 31.5 us in the compiler's own order,
// which reads an operand and waits for it, 29.3 so; eight spill.)
constexpr int EN_TREE_AHEAD = 6;
// KW = 2: two waves share a row block, a 32-key block of every tile each, and meet at the end.
template <int D, int RW, int KW, int NST>
__global__ __launch_bounds__(64 * RW * KW, RW * KW == 2 ? 1 : 2) __attribute__((amdgpu_num_vgpr(256))) void tree_attn_kernel(EnTreeArgs a)
{
    constexpr int W = RW * KW;
    constexpr bool TWO_PARTS = W < 8;            // of the queries, see above
    constexpr int NT = 64 * W;                   // threads
    constexpr int KB = 32;                       // keys per matrix-instruction block
    constexpr int LB = EN_KEY_TILE;              // keys per tile
    constexpr int NUW = LB / KB / KW;            // blocks of a tile per wave
    constexpr int NKS = D / 16;
    constexpr int NDB = D / 32;
    constexpr int ROWB = 2 * D;                  // bytes per K row
    constexpr int KBYTES = LB * ROWB;
    constexpr int VROWB = 2 * LB;                // bytes per V^T row of a tile
    constexpr int VBYTES = D * VROWB;
    constexpr int STAGE = KBYTES + VBYTES;
    constexpr int NBK = KBYTES / 1024, NBV = VBYTES / 1024;      // loader blocks
    constexpr int PER = (NBK + NBV) / W;         // loads per wave and tile
    static_assert(NBK % W == 0 && NBV % W == 0 && NST >= 2, "whole loader blocks per wave");
    __shared__ __attribute__((aligned(1024))) char smem[NST * STAGE];
    __shared__ int s_no_number;                  // a value of the tree is infinite or NaN
    typedef __bf16 pair_t __attribute__((ext_vector_type(2)));

    // (the arguments in one batch, and no integer divisions: see attn_bf16_kernel)
    asm volatile("" ::"s"(a.q), "s"(a.k_rows), "s"(a.kc), "s"(a.vt), "s"(a.cos_tab), "s"(a.hdr), "s"(a.parent), "s"(a.B), "s"(a.n), "s"(a.n_units),
                 "s"(a.by_ptiles.mul), "s"(a.by_splits.mul), "s"(a.by_hkv.mul), "s"(a.by_n.mul), "s"(a.by_r.n), "s"(a.ws_ml));
    // Neighbours in this order share a split's keys, and an XCD takes a run of them.
    const unsigned per_xcd = gridDim.x / EN_XCDS;
    const unsigned unit = (blockIdx.x % EN_XCDS) * per_xcd + blockIdx.x / EN_XCDS;
    if (unit >= a.n_units)
        return;
    unsigned t = divided(unit, a.by_ptiles);
    const int ptile = unit - t * a.n_ptiles;
    unsigned t2 = divided(t, a.by_splits);
    const int sp = a.n_splits - 1 - (t - t2 * a.n_splits);       // the last split, which has the tree, starts first
    const int b = divided(t2, a.by_hkv);
    const int kvh = t2 - b * a.Hkv;

    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int lane = tid % 64;
    const int col = lane % 32, half = lane / 32;
    const int rw = wave % RW, kw = wave / RW;
    const int r = a.by_r.n, n = a.n;
    const int block = ptile * a.tile_blocks + rw;        // the wave's 32 rows
    const bool idle = rw >= a.tile_blocks || block * 32 >= r * n;        // none: it loads, and keeps the barriers
    const int c_row = block * 32 + col;
    const bool row_there = !idle && c_row < r * n;
    const int hl = row_there ? divided(c_row, a.by_n) : 0;
    const int i_row = row_there ? c_row - hl * n : 0;
    const int hq = kvh * r + hl;

    // ---- what does not wait for anything, asked for first ----
    const int done = as_table(a.done)[b];
    const int Lc = as_table(a.hdr)[4 * b + 1];
    const int my_parent = tree_parent(a.parent + (size_t)b * n, n);
    bf16x8 qraw[NKS];
    {
        const bf16_t *qp = (const bf16_t *)a.q + (((size_t)b * n + i_row) * a.Hq + hq) * D + 8 * half;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
            qraw[ks] = *reinterpret_cast<const bf16x8 *>(qp + 16 * ks);
    }
    // the tree's keys and values: a thread takes 8 dimensions and their partners of a node, then of others NT / PAIRS on
    constexpr int PAIRS = D / 16;
    const bool last_split = sp == a.n_splits - 1;
    const int t_m = tid / PAIRS, t_c = tid % PAIRS;
    bf16x8 k1, k2;
    u16x8 v1, v2;
    auto tree_load = [&](int m) __attribute__((always_inline)) {
        const size_t from = (((size_t)b * n + min(m, n - 1)) * a.Hkv + kvh) * D + 8 * t_c;
        const bf16_t *kr = (const bf16_t *)a.k_rows + from, *vr = (const bf16_t *)a.v_rows + from;
        k1 = *reinterpret_cast<const bf16x8 *>(kr);
        k2 = *reinterpret_cast<const bf16x8 *>(kr + D / 2);
        v1 = *reinterpret_cast<const u16x8 *>(vr);
        v2 = *reinterpret_cast<const u16x8 *>(vr + D / 2);
    };
    if (last_split)
        tree_load(t_m);

    const int room = tree_room(done, a.Nq);
    const unsigned blocks_before = (b * a.Hkv + kvh) * a.head_blocks;
    auto nothing = [&]() {                       // of this split's keys a row sees none
        if (row_there && half == 0 && kw == 0) {
            if (a.n_splits > 1) {
                f32x2 none = {EN_NEG_INF, 0.f};
                *reinterpret_cast<f32x2 *>(a.ws_ml + (((size_t)sp * a.n_blocks + blocks_before + block) * 32 + col) * 2) = none;
            } else {
                bf16_t *op = (bf16_t *)a.out + (((size_t)b * n + i_row) * a.Hq + hq) * D;
                for (int d = 0; d < D; d += 8)
                    *reinterpret_cast<bf16x8 *>(op + d) = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
        }
    };
    const int L = Lc + done;                     // keys of the context (an idle agent's is not used)
    const int n_ctx = room > 0 ? (L + LB - 1) / LB : 0;
    // (split_first_tile; the tree's tile counts as tree_tiles of them)
    const int n_all = n_ctx + a.tree_tiles;
    const int t_begin = min((int)divided(sp * n_all + a.n_splits - 1, a.by_splits), n_ctx);
    const int t_end = min((int)divided((sp + 1) * n_all + a.n_splits - 1, a.by_splits), n_ctx);
    const int n_it = max(t_end - t_begin, 0) + (last_split ? 1 : 0);
    if (n_it == 0 || room == 0) {                // an agent with fewer tiles than splits, or an idle one
        nothing();
        return;
    }

    // ---- loader ----
    const char *kg = (const char *)a.kc + ((size_t)b * a.Hkv + kvh) * (size_t)a.T * ROWB;
    const char *vg = (const char *)a.vt + ((size_t)b * a.Hkv + kvh) * (size_t)a.T * ROWB;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    // chunk c of K row `row` lies at c ^ k_pattern(row), chunk c of V^T row d at c ^ v_pattern(d)
    auto k_pattern = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
    auto v_pattern = [](int d) { return (d >> 1) & 7; };
    // A wave's loads are every W-th kilobyte of the tile: 1024 / ROWB rows of K, 8 of V^T. Which chunk of its row a lane asks
    // for is the same in all of them, but for K with D = 128 and two waves, where every other one has bit 3 exchanged.
    constexpr bool ALTERNATES = D == 128 && W == 2;
    const unsigned ul = lane, uw = wave;
    const unsigned k_row = ul / (ROWB / 16), k_at = D == 128 ? k_row ^ (uw % 4) * 4 : (ul / 16) ^ (uw % 2) * 4;
    const uint32_t koff = k_row * ROWB + ((ul % (ROWB / 16)) ^ k_at) * 16;
    const uint32_t voff = ul / 8 * (uint32_t)a.T * 2u + ((ul % 8) ^ (ul / 16) ^ (uw % 2) * 4) * 16;
    const unsigned v_step = 16u * (unsigned)a.T;         // bytes of 8 rows of V^T
    auto issue = [&](int tile, int stage) __attribute__((always_inline)) {
        const char *kt = kg + (size_t)tile * KBYTES + uw * 1024;
        const char *vt = vg + (size_t)tile * VROWB + (size_t)uw * v_step;
        const uint32_t dst = lds0 + stage * STAGE + uw * 1024;
#pragma unroll
        for (int j = 0; j < NBK / W; ++j)
            dma16(kt + W * j * 1024, ALTERNATES && j % 2 ? koff ^ 128 : koff, dst + W * j * 1024);
#pragma unroll
        for (int j = 0; j < NBV / W; ++j)
            dma16(vt + (size_t)(W * j) * v_step, voff, dst + KBYTES + W * j * 1024);
    };
    const int ctx0 = t_begin - (last_split ? 1 : 0);     // iteration it takes tile ctx0 + it of the context
    const EnTreeLane tree = tree_lane(my_parent, n, room);
    const unsigned long long present = __ballot(tree.present());
    if (!present) {
        nothing();
        return;
    }

    // ---- Q: rotate at the node's position, scale, round to bf16 ----
    const unsigned long long way = __shfl(tree.way, i_row, 64);
    const int depth = __shfl(tree.depth, i_row, 64);
    const bool row_valid = row_there && way != 0;
    bf16x8 qf[NKS], ql[TWO_PARTS ? NKS : 1];         // the query, and what its rounding left
    f32x8 t_cs, t_sn;                            // of the tree's keys
    auto tree_angles = [&](int m) __attribute__((always_inline)) {
        const int d_m = __popcll(__shfl(tree.way, m, 64)) - 1;
        const size_t at = (size_t)(L + max(d_m, 0)) * (D / 2) + 8 * t_c;
        t_cs = *reinterpret_cast<const f32x8 *>(a.cos_tab + at);
        t_sn = *reinterpret_cast<const f32x8 *>(a.sin_tab + at);
    };
    if (last_split)
        tree_angles(t_m & 63);
    {
        const size_t pos = L + (row_valid ? depth : 0);
        const float *ct = a.cos_tab + pos * (D / 2) + 8 * half, *st = a.sin_tab + pos * (D / 2) + 8 * half;
        f32x8 cs[NKS / 2], sn[NKS / 2];
#pragma unroll
        for (int ks = 0; ks < NKS / 2; ++ks) {
            cs[ks] = *reinterpret_cast<const f32x8 *>(ct + 16 * ks);
            sn[ks] = *reinterpret_cast<const f32x8 *>(st + 16 * ks);
        }
        // Here they have come, and the tiles are asked for, which come while the queries are turned. (Loads come in the order
        // in which they were asked for, and the compiler does not see these: asked for before the cosines and sines they
        // would be waited for with them.)
#pragma unroll
        for (int ks = 0; ks < NKS / 2; ++ks)
            asm volatile("" : "+v"(cs[ks]), "+v"(sn[ks]));
        if (last_split)
            asm volatile("" : "+v"(t_cs), "+v"(t_sn));
#pragma unroll
        for (int it = 0; it < (W < 8 ? NST - 1 : 2); ++it)
            if (it >= (last_split ? 1 : 0) && it < n_it)
                issue(ctx0 + it, it);
        // (two stages: the tree's tile has no other to wait for)
        if (NST == 2 && last_split && n_it > 1)
            issue(ctx0 + 1, 1);
        const float scale = row_valid ? a.scale_log2e : 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS / 2; ++ks)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x1 = (float)qraw[ks][j], x2 = (float)qraw[ks + NKS / 2][j];
                const float c = cs[ks][j] * scale, s = sn[ks][j] * scale;
                const float y1 = x1 * c - x2 * s, y2 = x2 * c + x1 * s;
                if constexpr (TWO_PARTS) {
                    ql[ks][j] = (bf16_t)(y1 - cut_off(y1));
                    ql[ks + NKS / 2][j] = (bf16_t)(y2 - cut_off(y2));
                    qf[ks][j] = (bf16_t)cut_off(y1);
                    qf[ks + NKS / 2][j] = (bf16_t)cut_off(y2);
                } else {
                    qf[ks][j] = (bf16_t)y1;
                    qf[ks + NKS / 2][j] = (bf16_t)y2;
                }
            }
        if constexpr (TWO_PARTS)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                ql[ks] = with_sign_of(ql[ks], qf[ks]);
        if (!row_valid)                          // (what such a row holds may be no number)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                qf[ks] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
                if constexpr (TWO_PARTS)
                    ql[ks] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
    }

    // ---- the tree's tile into stage 0. Keys of absent nodes may stay what they are (nobody sees their scores), their
    // values have to be 0. ----
    if (last_split) {
        for (int x = tid; x < VBYTES / 16; x += NT)
            *reinterpret_cast<f32x4 *>(smem + KBYTES + x * 16) = f32x4{0.f, 0.f, 0.f, 0.f};
        if (tid == 0)
            s_no_number = 0;
        __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        lds_data_ready();
        bool odd = false;
#pragma unroll 1
        for (int m0 = 0; m0 < n; m0 += NT / PAIRS) {
            const int m = m0 + t_m;
            if (m0 > 0) {
                tree_load(m);
                tree_angles(m & 63);
            }
            if (m < n && (present >> m & 1)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float y1, y2;
                    rope_key_pair((float)k1[j], (float)k2[j], t_cs[j], t_sn[j], y1, y2);
                    k1[j] = (bf16_t)y1;
                    k2[j] = (bf16_t)y2;
                }
                const int pat = k_pattern(m);
                *reinterpret_cast<bf16x8 *>(smem + m * ROWB + (t_c ^ pat) * 16) = k1;
                *reinterpret_cast<bf16x8 *>(smem + m * ROWB + ((t_c + PAIRS) ^ pat) * 16) = k2;
                const int vc = (m & ~0xC) | ((m & 4) << 1) | ((m & 8) >> 1);
                // (dimension d of a column lies at chunk (column / 8) ^ v_pattern(d) of row d; v_pattern(d + D / 2) is
                // v_pattern(d))
                char *const at = smem + KBYTES + 8 * t_c * VROWB + vc % 8 * 2;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    // no number has no place in a product with weights of 0: it joins the sums of the rows that see it
                    // behind the loop
                    const bool n1 = no_number(v1[j]), n2 = no_number(v2[j]);
                    odd = odd || n1 || n2;
                    char *const to = at + j * VROWB + (((unsigned)vc / 8) ^ v_pattern(8 * t_c + j)) * 16;
                    *reinterpret_cast<unsigned short *>(to) = n1 ? 0 : v1[j];
                    *reinterpret_cast<unsigned short *>(to + D / 2 * VROWB) = n2 ? 0 : v2[j];
                }
            }
        }
        if (__any(odd) && lane == 0)
            s_no_number = 1;
    }

    // ---- state ----
    f32x16 o[NDB];
#pragma unroll
    for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            o[d][e] = 0.f;
    float m_ref = 0.f, l = 0.f;                  // l: this lane's share
    f32x16 negm;                                 // -m_ref
#pragma unroll
    for (int e = 0; e < 16; ++e)
        negm[e] = 0.f;
    bool has_ref = !row_valid;                   // (rows that are not there need none)
    // byte offsets of a lane's chunk in its rows, of the first k-step; the others' are these with bits exchanged
    const int kchunk = (half ^ k_pattern(col)) * 16, vchunk = (half ^ v_pattern(col)) * 16;
    const int u0 = kw * NUW;

    // The order of N products and the reads of their operands.
    auto feed = [](auto n_tag) __attribute__((always_inline)) {
        constexpr int N = decltype(n_tag)::value, A = N < EN_TREE_AHEAD ? N : EN_TREE_AHEAD, EACH = TWO_PARTS ? 2 : 1;
        __builtin_amdgcn_sched_group_barrier(0x100, A, 0);
        static_for<N - A>([](auto) {
            __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        });
        __builtin_amdgcn_sched_group_barrier(0x008, A * EACH, 0);
    };

    // ---- a tile in three pieces: scores, probabilities, values; iteration `it` of the workgroup's ----
    f32x16 sv[NUW];
    bf16x8 pf[NUW][2];
    auto stage_of = [&](int it) { return smem + it % NST * STAGE; };
    auto is_tree = [&](int it) { return last_split && it == 0; };
    auto left_of = [&](int it) { return L - (ctx0 + it) * LB; };         // keys of a context tile from its first on
    auto score_blocks = [&](const char *stg) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
            for (int u = 0; u < NUW; ++u) {
                const bf16x8 fr = *reinterpret_cast<const bf16x8 *>(stg + ((u0 + u) * KB + col) * ROWB + (kchunk ^ (32 * ks)));
                sv[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr, qf[ks], ks == 0 ? negm : sv[u], 0, 0, 0);
                if constexpr (TWO_PARTS)
                    sv[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr, ql[ks], sv[u], 0, 0, 0);
            }
    };
    auto probability_block = [&](int u) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            pf[u][e / 8][e % 8] = (bf16_t)fast_exp2(sv[u][e]);
    };
    // HIDES: the tile has columns behind the context's last token. Whatever they hold has no weight, but 0 times infinity
    // is no 0: they become zero on their way, two columns a word.
    auto value_block = [&](const char *stg, auto hides_tag, int left, int u) __attribute__((always_inline)) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u32x4 keep;
            if constexpr (decltype(hides_tag)::value)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int key = KB * (u0 + u) + 16 * kk + 4 * half + 8 * (w / 2) + 2 * (w % 2);
                    keep[w] = key + 1 < left ? ~0u : key < left ? 0xffffu : 0u;
                }
#pragma unroll
            for (int d = 0; d < NDB; ++d) {
                bf16x8 v = *reinterpret_cast<const bf16x8 *>(stg + KBYTES + (32 * d + col) * VROWB + (vchunk ^ (16 * (4 * (u0 + u) + 2 * kk))));
                if constexpr (decltype(hides_tag)::value)
                    v = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, v) & keep);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[u][kk], o[d], 0, 0, 0);
            }
        }
    };
    // Hidden keys, and a reference for rows that have none or whose scores have outgrown it. Returns whether scores have
    // changed.
    auto settle_scores = [&](int it) __attribute__((always_inline)) {
        float mx = sv[0][0];
#pragma unroll
        for (int u = 0; u < NUW; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                mx = fmaxf(mx, sv[u][e]);
        const bool hides = is_tree(it) || left_of(it) < LB;
        if (!hides && !__any(!has_ref || mx > 59.f))
            return false;
        if (hides) {
            // Element e of block u is key 32 u + 8 (e / 4) + e % 4 + 4 half of the tile. (Masks by arithmetic: as comparisons
            // they would take two scalar registers each.)
            const unsigned long long keys = is_tree(it) ? way : (1ull << left_of(it)) - 1;
            mx = EN_NEG_INF;
#pragma unroll
            for (int u = 0; u < NUW; ++u) {
                const uint32_t sees = (uint32_t)(keys >> (KB * (u0 + u))) >> (4 * half);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t on = (uint32_t)((int32_t)(sees << (31 - (8 * (e / 4) + e % 4))) >> 31);
                    sv[u][e] = __uint_as_float((__float_as_uint(sv[u][e]) & on) | (0xff800000u & ~on));
                    mx = fmaxf(mx, sv[u][e]);
                }
            }
        }
        mx = pair_max(mx);
        const bool fix = (!has_ref || mx > 59.f) && mx > EN_NEG_INF;
        const float delta = fix ? mx : 0.f;
        const float alpha = fix ? (has_ref ? fast_exp2(-delta) : 0.f) : 1.f;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                o[d][e] *= alpha;
        l *= alpha;
        has_ref = has_ref || fix;
        m_ref += delta;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            negm[e] = -m_ref;
#pragma unroll
        for (int u = 0; u < NUW; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                sv[u][e] -= delta;
        return true;
    };
    auto add_weights = [&]() __attribute__((always_inline)) {    // (the rounded probabilities, like the products)
#pragma unroll
        for (int u = 0; u < NUW; ++u)
#pragma unroll
            for (int e = 0; e < 16; e += 2)
                l = __builtin_amdgcn_fdot2_f32_bf16(pair_t{pf[u][e / 8][e % 8], pf[u][e / 8][e % 8 + 1]}, pair_t{(bf16_t)1.f, (bf16_t)1.f}, l,
                                                    false);
    };

    if constexpr (W < 8) {
        for (int it = 0; it < n_it; ++it) {
            // this tile's loads have landed when at most those of the later tiles are outstanding; all of them near the end
            if (it + NST - 2 < n_it)
                __builtin_amdgcn_s_waitcnt((((NST - 2) * PER) & 15) | ((((NST - 2) * PER) >> 4) << 14) | 0x0f70);
            else
                __builtin_amdgcn_s_waitcnt(0x0f70);
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the previous tile has been read, the tree's written
            __builtin_amdgcn_s_barrier();
            if (it + NST - 1 < n_it && !(NST == 2 && last_split && it == 0))
                issue(ctx0 + it + NST - 1, (it + NST - 1) % NST);
            lds_data_ready();
            if (idle)
                continue;
            // The first block's exponentials are taken beside the second block's scores, against the reference as it is, and
            // once more where that has changed; the second's beside the first block's values.
            const char *stg = stage_of(it);
            score_blocks(stg);
            feed(std::integral_constant<int, NUW * NKS>{});
            probability_block(0);
            if (settle_scores(it))
                probability_block(0);
            const int left = is_tree(it) ? LB : left_of(it);
            auto values = [&](auto hides_tag) __attribute__((always_inline)) {
#pragma unroll
                for (int u = 0; u < NUW; ++u) {
                    if (u + 1 < NUW)
                        probability_block(u + 1);
                    value_block(stg, hides_tag, left, u);
                }
            };
            if (left < LB)
                values(std::true_type{});
            else
                values(std::false_type{});
            add_weights();
        }
    } else {
        // Two waves share a SIMD, and in step they would ask for its matrix core together and then for its vector ALU
        // together. So the second four waves are half a tile behind: while
        // one half of the waves has its products (the values of a tile and the scores of the next), the other has its
        // exponentials. (64 nodes, us, in step / like this: 56 heads over 8 K tokens 28.7 / 28.0, 32 heads over 8 K 22.9 /
        // 22.2, 4 agents over 12 K 66.0 / 62.3; over 2 K no difference.) A tile's values are read until one and a half tiles
        // behind its scores: of the four stages one is being read, one still, two are on their way.
        static_assert(W != 8 || NST == 4, "two tiles are read at a time");
        auto half_done = [&]() __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            lds_data_ready();
        };
        auto tile_done = [&](int it) __attribute__((always_inline)) {
            // the next tile has landed when the one behind it is all that is outstanding
            if (it + 2 < n_it)
                __builtin_amdgcn_s_waitcnt((PER & 15) | ((PER >> 4) << 14) | 0x0f70);
            else
                __builtin_amdgcn_s_waitcnt(0x0f70);
            half_done();
        };
        auto ahead = [&](int it) __attribute__((always_inline)) {
            if (it + 2 < n_it)
                issue(ctx0 + it + 2, (it + 2) % NST);
        };
        auto probabilities = [&](int it) __attribute__((always_inline)) {
            settle_scores(it);
            probability_block(0);
            probability_block(1);
            add_weights();
        };
        auto values = [&](int it, auto hides_tag) __attribute__((always_inline)) {
            value_block(stage_of(it), hides_tag, left_of(it), 0);
            value_block(stage_of(it), hides_tag, left_of(it), 1);
        };
        auto last_values = [&]() __attribute__((always_inline)) {
            if (!is_tree(n_it - 1) && left_of(n_it - 1) < LB)
                values(n_it - 1, std::true_type{});
            else
                values(n_it - 1, std::false_type{});
        };
        tile_done(-1);
        if (idle) {
            for (int it = 0; it < n_it; ++it) {
                ahead(it);
                half_done();
                tile_done(it);
            }
            half_done();
        } else if (wave < 4) {
            for (int it = 0; it < n_it; ++it) {
                ahead(it);
                if (it > 0) {
                    values(it - 1, std::false_type{});
                    score_blocks(stage_of(it));
                    feed(std::integral_constant<int, 2 * (NKS + 2 * NDB)>{});
                } else {
                    score_blocks(stage_of(it));
                    feed(std::integral_constant<int, 2 * NKS>{});
                }
                half_done();
                probabilities(it);
                tile_done(it);
            }
            last_values();
            half_done();
        } else {
            for (int it = 0; it < n_it; ++it) {
                ahead(it);
                if (it > 0)
                    probabilities(it - 1);
                half_done();
                if (it > 0) {
                    values(it - 1, std::false_type{});
                    score_blocks(stage_of(it));
                    feed(std::integral_constant<int, 2 * (NKS + 2 * NDB)>{});
                } else {
                    score_blocks(stage_of(it));
                    feed(std::integral_constant<int, 2 * NKS>{});
                }
                tile_done(it);
            }
            probabilities(n_it - 1);
            half_done();
            last_values();
        }
    }

    l += xor32(l);
    // ---- two waves of a row block meet: the second leaves its state in LDS, the first takes it up ----
    if constexpr (KW == 2) {
        __builtin_amdgcn_s_waitcnt(0xc07f);
        __builtin_amdgcn_s_barrier();            // everybody is done with the tiles
        lds_data_ready();
        // [row block][register][lane], four registers at a time
        f32x4 *so = reinterpret_cast<f32x4 *>(smem) + rw * (NDB * 4 + 1) * 64;
        static_assert(RW * (NDB * 4 + 1) * 1024 <= NST * STAGE, "the waves' sums fit the stages");
        if (kw == 1) {
#pragma unroll
            for (int d = 0; d < NDB; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    so[(4 * d + g) * 64 + lane] = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
            so[NDB * 4 * 64 + lane] = f32x4{m_ref, l, 0.f, 0.f};
        }
        __syncthreads();
        if (kw == 1)
            return;
        const f32x4 other = so[NDB * 4 * 64 + lane];
        // (a sum is 0, by the bits, where the wave had no key that the row sees: one of NaN is not. The sums of values are 0
        // then, too.)
        const bool mine = __float_as_uint(l) != 0u, its = __float_as_uint(other[1]) != 0u;
        const float m = mine && its ? fmaxf(m_ref, other[0]) : mine ? m_ref : other[0];
        const float wm = mine ? fast_exp2(m_ref - m) : 0.f, wo = its ? fast_exp2(other[0] - m) : 0.f;
        l = l * wm + other[1] * wo;
        m_ref = m;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 x = so[(4 * d + g) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[d][4 * g + e] = o[d][4 * g + e] * wm + x[e] * wo;
            }
    }
    if (!row_there)
        return;
    if (!row_valid)
        l = 0.f;
    if (last_split && s_no_number) {
        // what the tree's tile left out: infinite with any weight, or NaN
#pragma unroll 1
        for (int m = 0; m < n; ++m) {
            const bf16_t *vr = (const bf16_t *)a.v_rows + (((size_t)b * n + m) * a.Hkv + kvh) * D + 4 * half;
            if (way >> m & 1)
#pragma unroll
                for (int d = 0; d < NDB; ++d)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const u16x4 v = *reinterpret_cast<const u16x4 *>(vr + 32 * d + 8 * g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[d][4 * g + e] += __uint_as_float(no_number(v[e]) ? (uint32_t)v[e] << 16 : 0u);
                    }
        }
    }
    if (a.n_splits > 1) {
        const size_t part = (size_t)sp * a.n_blocks + blocks_before + block;
        if (half == 0) {
            f32x2 v = {m_ref, l};
            *reinterpret_cast<f32x2 *>(a.ws_ml + (part * 32 + col) * 2) = v;
        }
        if (!row_valid)
            return;                              // (a sum of 0: nobody reads the rest)
        // as the registers lie: a kilobyte a store, where rows would be 32 bytes here and there
        f32x4 *op = reinterpret_cast<f32x4 *>(a.ws_opart + part * (32 * D)) + lane;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                op[(4 * d + g) * 64] = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    } else {
        // (zero where no key has a weight, as a merge leaves it; by the bits: a sum of NaN stays one)
        const float inv = row_valid && __float_as_uint(l) ? 1.f / l : 0.f;
        bf16_t *op = (bf16_t *)a.out + (((size_t)b * n + i_row) * a.Hq + hq) * D + 4 * half;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = row_valid ? (bf16_t)(o[d][4 * g + e] * inv) : (bf16_t)0.f;
                *reinterpret_cast<bf16x4 *>(op + 32 * d + 8 * g) = v;
            }
    }
}

// ---------------------------------------------------------------------------
// tree_merge: out = sum_sp 2^(m_sp - m) O_sp / sum_sp 2^(m_sp - m) l_sp. What the splits left lies as their waves' registers
// lay: per block of rows, groups of four values per lane. The four waves of a workgroup share a group's splits and meet in
// LDS (SHARE = 4), or take a group each, where these fill the chip. A split that a row saw nothing of left a sum of 0 and no
// values; a row without any is zero. grid: blocks * groups * SHARE / 4. Bound by latency (8 nodes of 32 heads in 25 splits 3.9
// us) and by its read (3584 rows in 16 splits, 29 MB, 6.7 us, 4.4 TB/s).
// ---------------------------------------------------------------------------
// Blocks of 32 rows, a lane's row is lane % 32, group x is dimensions 8 x + 4 (lane / 32) on
template <typename T, int D, int SHARE>
__global__ __launch_bounds__(256) void tree_merge_kernel(EnTreeArgs a)
{
    constexpr int GROUPS = D / 8, ROWS = 32, NB = SHARE == 4 ? 4 : 8;
    __shared__ f32x4 s_acc[SHARE == 4 ? 256 : 1];
    __shared__ f32x2 s_ml[SHARE == 4 ? 256 : 1];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    // an XCD takes a run of them, as it took one of the units that left them: part of that is in its L2 still
    const unsigned wg = (blockIdx.x % EN_XCDS) * (gridDim.x / EN_XCDS) + blockIdx.x / EN_XCDS;
    const unsigned item = SHARE == 4 ? wg : wg * 4 + wave;
    if (item >= a.n_blocks * GROUPS)
        return;
    const unsigned blk = item / GROUPS;
    const int x = item % GROUPS, first = SHARE == 4 ? wave : 0;
    const unsigned bh = divided(blk, a.by_blocks);       // (agent, KV head)
    const int c_row = (blk - bh * a.head_blocks) * ROWS + lane % ROWS;
    const bool there = c_row < (int)a.by_r.n * a.n;
    float M = EN_NEG_INF, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (there)
        for (int sp0 = first; sp0 < a.n_splits; sp0 += SHARE * NB) {
            f32x2 ml[NB];
            f32x4 v[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const bool on = sp0 + SHARE * j < a.n_splits;
                const size_t part = (size_t)(on ? sp0 + SHARE * j : sp0) * a.n_blocks + blk;
                ml[j] = *reinterpret_cast<const f32x2 *>(a.ws_ml + (part * ROWS + lane % ROWS) * 2);
                v[j] = reinterpret_cast<const f32x4 *>(a.ws_opart + part * (ROWS * D))[x * 64 + lane];
                if (!on)
                    ml[j][1] = 0.f;
            }
            float Mb = M;
#pragma unroll
            for (int j = 0; j < NB; ++j)
                Mb = __float_as_uint(ml[j][1]) ? fmaxf(Mb, ml[j][0]) : Mb;
            const float keep = M == EN_NEG_INF ? 0.f : fast_exp2(M - Mb);
            l *= keep;
            acc *= keep;
            M = Mb;
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (__float_as_uint(ml[j][1])) {
                    const float w = fast_exp2(ml[j][0] - M);
                    l += w * ml[j][1];
                    acc += w * v[j];
                }
        }
    if constexpr (SHARE == 4) {
        s_acc[tid] = acc;
        s_ml[tid] = f32x2{M, l};
        __syncthreads();
        if (wave != 0)
            return;
        f32x2 ml[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            ml[k] = s_ml[lane + 64 * k];
            M = __float_as_uint(ml[k][1]) ? fmaxf(M, ml[k][0]) : M;
        }
        l = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (__float_as_uint(ml[k][1])) {
                const float w = fast_exp2(ml[k][0] - M);
                l += w * ml[k][1];
                acc += w * s_acc[lane + 64 * k];
            }
    }
    if (!there)
        return;
    const float inv = __float_as_uint(l) ? 1.f / l : 0.f;
    const unsigned hl = divided(c_row, a.by_n), i = c_row - hl * a.n;
    const unsigned b = divided(bh, a.by_hkv), hq = (bh - b * a.Hkv) * a.by_r.n + hl;
    typedef T tvec __attribute__((ext_vector_type(4)));
    *reinterpret_cast<tvec *>((T *)a.out + (((size_t)b * a.n + i) * a.Hq + hq) * D + 8 * x + 4 * (lane / ROWS)) =
        __builtin_convertvector(acc * inv, tvec);
}

template <typename T, int D>
static void launch_merge(const EnTreeArgs &a, hipStream_t st)
{
    // Four waves to a group / one, us: 128 groups of 25 splits 3.9 / 5.8, 512 of 32 5.0 / 6.9, 1792 of 16 6.8 / 6.8, 2048 of 8
    // 5.4 / 5.3, 4096 of 8 7.9 / 7.6, 4096 of 4 8.4 / 6.3, 8192 of 4 14.9 / 12.0.
    const unsigned items = a.n_blocks * (D / 8);
    if (items < 2048)
        hipLaunchKernelGGL((tree_merge_kernel<T, D, 4>), dim3((items + EN_XCDS - 1) / EN_XCDS * EN_XCDS), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((tree_merge_kernel<T, D, 1>), dim3((items / 4 + EN_XCDS - 1) / EN_XCDS * EN_XCDS), dim3(256), 0, st, a);
}

template <int D>
static int launch_tree_bf16(const EnTreeArgs &a, int blocks, hipStream_t st)
{
    const dim3 grid((a.n_units + EN_XCDS - 1) / EN_XCDS * EN_XCDS);
    if (blocks == 1)
        hipLaunchKernelGGL((tree_attn_kernel<D, 1, 2, 2>), grid, dim3(128), 0, st, a);
    else if (blocks == 2)
        hipLaunchKernelGGL((tree_attn_kernel<D, 2, 2, 2>), grid, dim3(256), 0, st, a);
    else if (blocks == 4)
        hipLaunchKernelGGL((tree_attn_kernel<D, 4, 1, 2>), grid, dim3(256), 0, st, a);
    else if (blocks == 8)
        hipLaunchKernelGGL((tree_attn_kernel<D, 8, 1, 4>), grid, dim3(512), 0, st, a);
    else
        return (int)hipErrorInvalidValue;
    return (int)hipGetLastError();
}
// ---------------------------------------------------------------------------
// tree_f32: the same in single precision on the fp32 matrix instruction (16 x 16 x 4), for small layers, which are bound by
// latency. As in attn_f32_kernel a workgroup takes 16 rows of a KV head, its eight waves share a split's keys 16 at a time
// and meet in LDS; no operand goes through LDS. The blocks of the tree's own keys follow those of the context: a lane holds
// both halves of the pairs of its key, so it turns them in its registers. 7 nodes of 4 heads over 128 tokens 7.6 us;
// one wave a row with a softmax of its own a lane 13.4.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(512) void tree_f32_kernel(EnTreeArgs a)
{
    constexpr int WAVES = 8, ROWS = EN_F32_ROWS, KEYS = 16;
    constexpr int NJ = D / 16;                   // 16-byte loads per key row and lane; blocks of O^T
    constexpr int NV = D / 64;                   // 16-byte loads per value row and lane
    constexpr int OSTR = D + 4;                  // floats per merged row in LDS
    __shared__ __attribute__((aligned(16))) float so[WAVES][ROWS][OSTR];
    __shared__ f32x2 sml[WAVES][ROWS];           // (reference, sum) of a wave's rows

    // (arguments and divisions: see attn_bf16_kernel)
    asm volatile("" ::"s"(a.q), "s"(a.k_rows), "s"(a.kc), "s"(a.vt), "s"(a.cos_tab), "s"(a.hdr), "s"(a.parent), "s"(a.B), "s"(a.n),
                 "s"(a.by_ptiles.mul), "s"(a.by_splits.mul), "s"(a.by_hkv.mul), "s"(a.by_n.mul), "s"(a.by_r.n), "s"(a.ws_ml));
    const unsigned t = divided(blockIdx.x, a.by_ptiles);
    const int rg = blockIdx.x - t * a.n_ptiles;
    const unsigned t2 = divided(t, a.by_splits);
    const int sp = t - t2 * a.n_splits;
    const int b = divided(t2, a.by_hkv);
    const int kvh = t2 - b * a.Hkv;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int lane = tid % 64;
    const int col = lane % 16, grp = lane / 16;
    const int r = a.by_r.n, n = a.n;

    const int done = as_table(a.done)[b];
    const int Lc = as_table(a.hdr)[4 * b + 1];
    const int my_parent = tree_parent(a.parent + (size_t)b * n, n);
    const int n_rows = r * n;
    const int r0 = rg * ROWS, r1 = min(r0 + ROWS, n_rows) - 1;
    const int rr = min(r0 + col, r1);
    const int hl = divided(rr, a.by_n), i_row = rr - hl * n;
    f32x4 qf[NJ];
    {
        const float *qp = (const float *)a.q + (((size_t)b * n + i_row) * a.Hq + kvh * r + hl) * D + 4 * grp;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            qf[j] = *reinterpret_cast<const f32x4 *>(qp + 16 * j);
    }
    const int room = tree_room(done, a.Nq);
    const int L = Lc + done;                     // keys of the context (an idle agent's is not used)
    const int n_ctx = room > 0 ? (L + KEYS - 1) / KEYS : 0, n_blk = room > 0 ? n_ctx + (n + KEYS - 1) / KEYS : 0;
    const int first = divided(sp * n_blk + a.n_splits - 1, a.by_splits), last = divided((sp + 1) * n_blk + a.n_splits - 1, a.by_splits);
    const int per = (last - first + WAVES - 1) / WAVES;
    const int wb = min(first + wave * per, last), we = min(first + (wave + 1) * per, last);      // this wave's blocks
    const float *const K = (const float *)a.kc + ((size_t)b * a.Hkv + kvh) * (size_t)a.T * D;
    const float *const V = (const float *)a.vt + ((size_t)b * a.Hkv + kvh) * (size_t)a.T * D;
    const size_t own = ((size_t)b * n * a.Hkv + kvh) * D;
    const float *const Kt = (const float *)a.k_rows + own, *const Vt = (const float *)a.v_rows + own;
    // (context rows reach up to a multiple of 64 keys: whole blocks can be read)
    f32x4 kf[NJ], vf[4][NV];
    auto load_block = [&](int blk) {
        const bool tree = blk >= n_ctx;
        const int k0 = (blk - (tree ? n_ctx : 0)) * KEYS;
        const float *const kb = tree ? Kt : K, *const vb = tree ? Vt : V;
        const size_t stride = tree ? (size_t)a.Hkv * D : D;
        const int most = tree ? n - 1 : 0x7fffffff;
        const float *kr = kb + min(k0 + col, most) * stride + 4 * grp;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            kf[j] = *reinterpret_cast<const f32x4 *>(kr + 16 * j);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float *vr = vb + min(k0 + 4 * grp + e, most) * stride + col * NJ;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                vf[e][v] = *reinterpret_cast<const f32x4 *>(vr + 4 * v);
        }
    };
    if (wb < we)
        load_block(wb);

    const EnTreeLane tree = tree_lane(my_parent, n, room);
    const unsigned long long row_way = __shfl(tree.way, i_row, 64);      // (all lanes exchange)
    const unsigned long long way = r0 + col <= r1 ? row_way : 0ull;
    const bool row_valid = way != 0;
    // ---- the query, rotated at its node's position and scaled ----
    {
        const int depth = __shfl(tree.depth, i_row, 64);
        const size_t at = (size_t)(room > 0 ? L + (row_valid ? depth : 0) : 0) * (D / 2) + 4 * grp;
#pragma unroll
        for (int j = 0; j < NJ / 2; ++j) {
            const f32x4 cs = *reinterpret_cast<const f32x4 *>(a.cos_tab + at + 16 * j);
            const f32x4 sn = *reinterpret_cast<const f32x4 *>(a.sin_tab + at + 16 * j);
            const f32x4 x1 = qf[j], x2 = qf[j + NJ / 2];
            qf[j] = (x1 * cs - x2 * sn) * a.scale_log2e;
            qf[j + NJ / 2] = (x2 * cs + x1 * sn) * a.scale_log2e;
        }
        if (!row_valid)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                qf[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    f32x4 o[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
        o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = EN_NEG_INF, l = 0.f;                       // l: this lane's share
    auto row_sum = [](float v) {                         // over the four lanes of a row
        v += __shfl_xor(v, 16, 64);
        return v + xor32(v);
    };
    for (int blk = wb; blk < we; ++blk) {
        const bool of_tree = blk >= n_ctx;
        const int k0 = (blk - (of_tree ? n_ctx : 0)) * KEYS;
        if (of_tree) {
            const int node = min(k0 + col, n - 1);
            const int depth = __popcll(__shfl(tree.way, node, 64)) - 1;
            const size_t at = (size_t)(L + max(depth, 0)) * (D / 2) + 4 * grp;
#pragma unroll
            for (int j = 0; j < NJ / 2; ++j) {
                const f32x4 cs = *reinterpret_cast<const f32x4 *>(a.cos_tab + at + 16 * j);
                const f32x4 sn = *reinterpret_cast<const f32x4 *>(a.sin_tab + at + 16 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float y1, y2;
                    rope_key_pair(kf[j][e], kf[j + NJ / 2][e], cs[e], sn[e], y1, y2);
                    kf[j][e] = y1;
                    kf[j + NJ / 2][e] = y2;
                }
            }
        }
        // ---- scores; eight chains of products, whose sums meet in a tree (see attn_f32_kernel) ----
        f32x4 s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int i = (e * NJ + j) % 8;
                s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][e], qf[j][e], s[i], 0, 0, 0);
            }
        // the lane's keys are 4 grp + e of the block
        const uint32_t sees = of_tree ? (uint32_t)(way >> k0) >> (4 * grp) : L - k0 >= KEYS ? 0xfu : ((1u << (L - k0)) - 1u) >> (4 * grp);
        const uint32_t there = of_tree ? 0xfu : sees;
        f32x4 vc[4][NV];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int x = 0; x < 4; ++x)      // (what lies behind the context's last token counts as zero)
                    vc[e][v][x] = __uint_as_float(there >> e & 1 ? __float_as_uint(vf[e][v][x]) : 0u);
        if (blk + 1 < we)
            load_block(blk + 1);
        f32x4 p = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(sees >> e & 1))
                p[e] = EN_NEG_INF;
        float mn = fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3]));
        mn = fmaxf(mn, __shfl_xor(mn, 16, 64));
        mn = fmaxf(m, pair_max(mn));
        const float ref = mn == EN_NEG_INF ? 0.f : mn;   // nothing seen yet: all exponentials are 0
        const float alpha = fast_exp2(m - ref);
        m = mn;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            p[e] = fast_exp2(p[e] - ref);
        l = l * alpha + ((p[0] + p[1]) + (p[2] + p[3]));
        // ---- O^T += V^T P^T (the block's products by themselves: one rounding per block of a sum that grows). A hidden
        // key's value that is infinite or NaN has no place in a product with 0: then the keys go one by one, and a row
        // keeps its sums where it does not see the key. ----
        f32x4 ob[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            ob[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        bool by_key = false;
        if (of_tree) {
            uint32_t top = 0;                            // (by the bits: this library is built without NaN compares)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    top = max(top, __float_as_uint(vc[e][j / 4][j % 4]) & 0x7f800000u);
            by_key = __any(top == 0x7f800000u);
        }
        if (!by_key) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    ob[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vc[e][j / 4][j % 4], p[e], ob[j], 0, 0, 0);
        } else {
#pragma unroll 1
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const f32x4 with = __builtin_amdgcn_mfma_f32_16x16x4f32(
                            grp == g ? vc[e][j / 4][j % 4] : 0.f, grp == g ? p[e] : 0.f, ob[j], 0, 0, 0);
                        ob[j] = way >> (k0 + 4 * g + e) & 1 ? with : ob[j];
                    }
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            o[j] = o[j] * alpha + ob[j];
    }

    // ---- the waves meet ----
    {
        const float lt = row_sum(l);
        if (grp == 0)
            sml[wave][col] = f32x2{m, row_valid ? lt : 0.f};     // (a sum of 0: no key that the row sees)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                f32x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    x[j] = o[4 * v + j][e];
                *reinterpret_cast<f32x4 *>(&so[wave][col][(4 * grp + e) * NJ + 4 * v]) = x;
            }
    }
    __syncthreads();
    // ---- the output, a 16-byte piece per thread at a time ----
    constexpr int CPR = D / 4;
    static_assert(ROWS * CPR % 256 == 0, "whole waves");
    for (int x = tid; x < ROWS * CPR; x += 64 * WAVES) {
        const int row = x / CPR, c4 = x % CPR * 4, c_row = r0 + row;
        if (c_row > r1)
            break;
        float M = EN_NEG_INF, sum = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        f32x2 ml[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            ml[w] = sml[w][row];
            M = __float_as_uint(ml[w][1]) ? fmaxf(M, ml[w][0]) : M;
        }
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const f32x4 part = *reinterpret_cast<const f32x4 *>(&so[w][row][c4]);
            if (__float_as_uint(ml[w][1])) {
                const float wt = fast_exp2(ml[w][0] - M);
                sum += ml[w][1] * wt;
                acc += part * wt;
            }
        }
        if (a.n_splits > 1) {
            // as tree_merge_kernel reads it
            const size_t part = (size_t)sp * a.n_blocks + ((unsigned)b * a.Hkv + kvh) * a.head_blocks + c_row / 32;
            if (c4 == 0) {
                f32x2 v = {M, sum};
                *reinterpret_cast<f32x2 *>(a.ws_ml + (part * 32 + c_row % 32) * 2) = v;
            }
            reinterpret_cast<f32x4 *>(a.ws_opart + part * (32 * D))[c4 / 8 * 64 + c_row % 32 + c4 / 4 % 2 * 32] = acc;
        } else {
            const int ho = divided(c_row, a.by_n), i = c_row - ho * n;
            const float inv = __float_as_uint(sum) ? 1.f / sum : 0.f;
            *reinterpret_cast<f32x4 *>((float *)a.out + (((size_t)b * n + i) * a.Hq + kvh * r + ho) * D + c4) = acc * inv;
        }
    }
}

int en_launch_tree_attention(const en_pool *pool, const EnTreeArgs &a, int blocks, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const int D = pool->d.head_dim;
    if (pool->d.dtype != EN_F32)
        return D == 64 ? launch_tree_bf16<64>(a, blocks, st) : launch_tree_bf16<128>(a, blocks, st);
    const dim3 grid(a.n_units), blk(512);
    if (D == 64)
        hipLaunchKernelGGL((tree_f32_kernel<64>), grid, blk, 0, st, a);
    else
        hipLaunchKernelGGL((tree_f32_kernel<128>), grid, blk, 0, st, a);
    return (int)hipGetLastError();
}

int en_launch_tree_merge(const en_pool *pool, const EnTreeArgs &a, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    if (pool->d.dtype == EN_F32) {
        if (pool->d.head_dim == 64)
            launch_merge<float, 64>(a, st);
        else
            launch_merge<float, 128>(a, st);
    } else {
        if (pool->d.head_dim == 64)
            launch_merge<bf16_t, 64>(a, st);
        else
            launch_merge<bf16_t, 128>(a, st);
    }
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------------------
// tree_commit: entry j of an agent's path goes to context row L_c + (done - accepted) + j, the key rotated there. A workgroup
// takes a KV head of a layer and agent, all of its tokens: four tokens at positions 4 x to 4 x + 3 are eight bytes side by
// side in a row of the transposed values, and a store of two bytes costs the memory as much as one of eight. Bound by those
// rows: D lines per (layer, agent, KV head), read and written back whatever the tokens are. 16 agents x 40 layers x 8 KV heads of
// 128: 84 MB of such lines, 31 us; one agent's 40 layers 5.0. grid: (Hkv * layers, B).
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(D) void tree_commit_kernel(EnTreeCommitArgs a)
{
    constexpr int HALF = D / 2;
    const int b = blockIdx.y, layer = divided(blockIdx.x, a.by_hkv), h = blockIdx.x - layer * a.Hkv;
    const int tid = threadIdx.x, lane = tid % 64;
    const int most = min(as_table(a.accepted)[b], a.n);
    const int row0 = (int)((unsigned)as_table(a.done)[b] - (unsigned)as_table(a.accepted)[b]);       // of the plan's new tokens
    const int Lc = as_table(a.hdr)[4 * b + 1];
    const int my_node = lane < most ? a.path[(size_t)b * a.n + lane] : -1;
    // entries that are a node and have a place
    const unsigned long long valid = __ballot((unsigned)my_node < (unsigned)a.n && row0 + lane >= 0 && row0 + lane < a.Nq && row0 >= -64);
    if (valid == 0)
        return;
    const size_t slab = (size_t)b * a.Hkv + h;
    const size_t step = (size_t)a.Hkv * D, from = (size_t)b * a.n * step + h * D;
    const T *const kr = (const T *)a.k_rows[layer] + from, *const vr = (const T *)a.v_rows[layer] + from;
    T *const kd = (T *)a.kc[layer] + slab * a.T * D, *const vd = (T *)a.vt[layer] + slab * a.T * D;
    const int pos0 = Lc + row0;
    auto node_of = [&](int j) { return __builtin_amdgcn_readlane(my_node, j); };
    // keys, two tokens at a time: thread c and c + D/2 own the pair (c, c + D/2) of one each
    const int c = tid % HALF, second = tid / HALF;
    for (unsigned long long todo = valid; todo;) {
        const int j1 = __builtin_ctzll(todo);
        todo &= todo - 1;
        const int j2 = todo ? __builtin_ctzll(todo) : j1;
        todo &= todo - 1;
        const int j = second ? j2 : j1, node = second ? node_of(j2) : node_of(j1);
        const size_t pos = (size_t)(pos0 + j);
        float y1, y2;
        rope_key_pair((float)kr[node * step + c], (float)kr[node * step + c + HALF], a.cos_tab[pos * HALF + c], a.sin_tab[pos * HALF + c], y1, y2);
        kd[pos * D + c] = (T)y1;
        kd[pos * D + c + HALF] = (T)y2;
    }
    if constexpr (sizeof(T) == 4) {
        for (unsigned long long todo = valid; todo; todo &= todo - 1) {
            const int j = __builtin_ctzll(todo);
            vd[(size_t)(pos0 + j) * D + tid] = vr[node_of(j) * step + tid];
        }
    } else {
        // values: thread d owns row d of the transposed layout, token t in column t with bits 2 and 3 exchanged
        typedef unsigned short u16;
        const u16 *const v_in = (const u16 *)vr + tid;
        u16 *const v_out = (u16 *)vd + (size_t)tid * a.T;
        const int j_first = __builtin_ctzll(valid), j_last = 63 - __builtin_clzll(valid);
        for (int t0 = (pos0 + j_first) & ~3; t0 <= pos0 + j_last; t0 += 4) {
            const int j0 = t0 - pos0;                    // entry of token t0; -3 at least
            const unsigned there = (unsigned)(j0 >= 0 ? valid >> j0 : valid << -j0) & 15u;
            u16 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] = there >> k & 1 ? v_in[node_of(j0 + k) * step] : 0;
            u16 *const to = v_out + ((t0 & ~0xC) | ((t0 & 4) << 1) | ((t0 & 8) >> 1));
            if (there == 15u) {
                *reinterpret_cast<u16x4 *>(to) = u16x4{v[0], v[1], v[2], v[3]};
            } else {
#pragma unroll
                for (int k = 0; k < 4; k += 2) {
                    const unsigned pair = there >> k & 3u;
                    if (pair == 3u)
                        *reinterpret_cast<uint32_t *>(to + k) = (uint32_t)v[k] | (uint32_t)v[k + 1] << 16;
                    else if (pair == 1u)
                        to[k] = v[k];
                    else if (pair == 2u)
                        to[k + 1] = v[k + 1];
                }
            }
        }
    }
}

int en_launch_tree_commit(const en_pool *pool, const EnTreeCommitArgs &a, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const int D = pool->d.head_dim;
    const dim3 grid(a.Hkv * a.layers, a.B), blk(D);
    if (pool->d.dtype == EN_F32) {
        if (D == 64)
            hipLaunchKernelGGL((tree_commit_kernel<float, 64>), grid, blk, 0, st, a);
        else
            hipLaunchKernelGGL((tree_commit_kernel<float, 128>), grid, blk, 0, st, a);
    } else {
        if (D == 64)
            hipLaunchKernelGGL((tree_commit_kernel<bf16_t, 64>), grid, blk, 0, st, a);
        else
            hipLaunchKernelGGL((tree_commit_kernel<bf16_t, 128>), grid, blk, 0, st, a);
    }
    return (int)hipGetLastError();
}
