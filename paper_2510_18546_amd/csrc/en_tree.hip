// Attention over a tree of drafted tokens and the gathered context, and the accepted tokens' way into the contexts.
#include "en_tree_lane.h"

// ---------------------------------------------------------------------------
// tree_attn (bf16)
//
// All r * n rows of a KV head attend over the same L_c + done keys of the context, so the context is read once for all of
// them: 32 bytes of it per key and dimension pair against 4 D flops a row. Up to 64 rows a KV head the step is bound by
// that read, at 256 and more by the matrix instructions too. A workgroup takes up to 8 row blocks of 32 rows (a wave each)
// of a KV head and a split of its keys; 64-key tiles of K and V^T go straight into LDS, NST of them in turn, and every
// wave reads all of them there.
//
// The tree's own keys are one more tile, the last split's first: the workgroup rotates them and lays them out in LDS as a
// tile of the context would be. Its mask is a row's way, a word whose bit m is node m.
//
// S^T = K Q^T and O^T += V^T P^T with 32 x 32 x 16 products as in attn_decode_kernel: a lane's column is a query row, its
// scores of 16 keys of a 32-key block are the operand of the second product as they are (that is what the exchanged bits
// 2 and 3 of a value's column are for). Scores are in log2 units, taken against a reference that is the maximum of the
// first keys a row sees and changes only where a score is 2^59 above it. The queries, the drafted keys, the probabilities
// and the output are rounded to bf16 once each (what the products take); sums, references and what the splits leave for
// the merge are float32.
//
// 16-byte chunks of a row lie in LDS exchanged by XOR with its number, so that 16 consecutive rows' reads of the same
// chunk meet distinct banks; the loads bring them there by reading their source in that order.
// ---------------------------------------------------------------------------
// Values that may be infinite or NaN are looked at, left out and added as bits: this library is built without NaN compares,
// and a NaN may be taken not to occur wherever a floating-point operation sees it.
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bool no_number(unsigned short bf16) { return (bf16 & 0x7f80) == 0x7f80; }

#ifndef EN_TREE_AHEAD
#define EN_TREE_AHEAD 6
#endif
// KW = 2: two waves share a row block, a 32-key block of every tile each, and meet at the end.
template <int D, int RW, int KW, int NST>
__global__ __launch_bounds__(64 * RW * KW, RW * KW == 2 ? 1 : 2) __attribute__((amdgpu_num_vgpr(256))) void tree_attn_kernel(EnTreeArgs a)
{
    constexpr int W = RW * KW;
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
    bf16x8 qf[NKS];
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
                qf[ks][j] = (bf16_t)(x1 * c - x2 * s);
                qf[ks + NKS / 2][j] = (bf16_t)(x2 * c + x1 * s);
            }
        if (!row_valid)                          // (what such a row holds may be no number)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                qf[ks] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
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

    // The order of N products and the reads of their operands: EN_TREE_AHEAD reads ahead. (Left to itself the compiler
    // reads an operand and waits for it.)
    auto feed = [](auto n_tag) __attribute__((always_inline)) {
        constexpr int N = decltype(n_tag)::value, A = N < EN_TREE_AHEAD ? N : EN_TREE_AHEAD;
        __builtin_amdgcn_sched_group_barrier(0x100, A, 0);
        static_for<N - A>([](auto) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        });
        __builtin_amdgcn_sched_group_barrier(0x008, A, 0);
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
        // together: 3850 cycles a tile of 64 keys, the sum of both. So the second four waves are half a tile behind: while
        // one half of the waves has its products (the values of a tile and the scores of the next), the other has its
        // exponentials. A tile's values are read until one and a half tiles behind its scores: of the four stages one is
        // being read, one still, two are on their way.
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
        const float inv = row_valid ? 1.f / l : 0.f;
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
// values; a row without any is zero. grid: blocks * groups * SHARE / 4.
// ---------------------------------------------------------------------------
// bf16: blocks of 32 rows, a lane's row is lane % 32, group x is dimensions 8 x + 4 (lane / 32) on
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
// tree_attention: one workgroup per (agent, query head, node), 256 keys at a time: a thread takes the score of a key,
// the workgroup their maximum and sum, then a thread one dimension of a part of the keys.
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_attention_kernel(EnTreeArgs a)
{
    __shared__ float sq[D], sp[256], sred[4], sacc[256];
    const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, kvh = hq / (a.Hq / a.Hkv);
    const int done = a.done[b];
    const EnTreeLane mine = tree_lane(tree_parent(a.parent + (size_t)b * a.n, a.n), a.n, tree_room(done, a.Nq));
    const unsigned long long way = readlane64(mine.way, i);
    T *out = (T *)a.out + (((size_t)b * a.n + i) * a.Hq + hq) * D;
    if (way == 0) {
        if (tid < D)
            out[tid] = (T)0.f;
        return;
    }
    const int L = a.hdr[4 * b + 1] + done;
    const int pos = L + __builtin_amdgcn_readlane(mine.depth, i);
    if (tid < D / 2) {
        const T *q = (const T *)a.q + (((size_t)b * a.n + i) * a.Hq + hq) * D;
        const float c = a.cos_tab[(size_t)pos * (D / 2) + tid], s = a.sin_tab[(size_t)pos * (D / 2) + tid];
        rope_scale_pair((float)q[tid], (float)q[tid + D / 2], c, s, a.scale_log2e, sq[tid], sq[tid + D / 2]);
    }
    __syncthreads();
    const size_t slab = (size_t)b * a.Hkv + kvh;
    float m = EN_NEG_INF, l = 0.f, acc = 0.f;
    const int d = tid % D, part = tid / D;
    constexpr int PARTS = 256 / D;
    for (int k0 = 0; k0 < L + 64; k0 += 256) {
        // keys 0 .. L - 1: the context; L .. L + 63: the nodes
        const int key = k0 + tid, node = key - L;
        float s = EN_NEG_INF;
        if (node < 0) {
            const T *k = (const T *)a.kc + (slab * a.T + key) * D;
            s = 0.f;
            for (int c = 0; c < D; ++c)
                s += sq[c] * (float)k[c];
        } else if (node < 64 && (way >> node & 1)) {
            const T *k = (const T *)a.k_rows + (((size_t)b * a.n + node) * a.Hkv + kvh) * D;
            const size_t p = L + __popcll(way & ((1ull << node) - 1));
            s = 0.f;
            for (int c = 0; c < D / 2; ++c) {
                float y1, y2;
                rope_key_pair((float)k[c], (float)k[c + D / 2], a.cos_tab[p * (D / 2) + c], a.sin_tab[p * (D / 2) + c], y1, y2);
                s += sq[c] * (float)(T)y1 + sq[c + D / 2] * (float)(T)y2;
            }
        }
        float mx = wave_max(s);
        __syncthreads();
        if (tid % 64 == 0)
            sred[tid / 64] = mx;
        __syncthreads();
        mx = fmaxf(fmaxf(sred[0], sred[1]), fmaxf(sred[2], sred[3]));
        const float now = fmaxf(m, mx), ref = now == EN_NEG_INF ? 0.f : now, keep = fast_exp2(m - ref);
        m = now;
        const float p = s == EN_NEG_INF ? 0.f : fast_exp2(s - ref);
        sp[tid] = p;
        const float ps = wave_sum(p);
        __syncthreads();
        if (tid % 64 == 0)
            sred[tid / 64] = ps;
        __syncthreads();
        l = l * keep + ((sred[0] + sred[1]) + (sred[2] + sred[3]));
        acc *= keep;
        for (int j = part; j < 256; j += PARTS) {
            const int kj = k0 + j, nj = kj - L;
            if (nj < 0) {
                float v;
                if constexpr (sizeof(T) == 4)
                    v = ((const float *)a.vt)[(slab * a.T + kj) * D + d];
                else
                    v = (float)((const T *)a.vt)[(slab * D + d) * a.T + ((kj & ~0xC) | ((kj & 4) << 1) | ((kj & 8) >> 1))];
                acc += sp[j] * v;
            } else if (nj < 64 && (way >> nj & 1)) {
                acc += sp[j] * (float)((const T *)a.v_rows)[(((size_t)b * a.n + nj) * a.Hkv + kvh) * D + d];
            }
        }
    }
    sacc[tid] = acc;
    __syncthreads();
    if (tid < D) {
        float sum = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
            sum += sacc[p * D + tid];
        out[tid] = (T)(sum / l);
    }
}

int en_launch_tree_attention(const en_pool *pool, const EnTreeArgs &a, int blocks, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const int D = pool->d.head_dim;
    if (pool->d.dtype != EN_F32)
        return D == 64 ? launch_tree_bf16<64>(a, blocks, st) : launch_tree_bf16<128>(a, blocks, st);
    const dim3 grid(a.n, a.Hq, a.B), blk(256);
    if (D == 64)
        hipLaunchKernelGGL((tree_attention_kernel<float, 64>), grid, blk, 0, st, a);
    else
        hipLaunchKernelGGL((tree_attention_kernel<float, 128>), grid, blk, 0, st, a);
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
// tree_commit: entry j of an agent's path goes to context row L_c + (done - accepted) + j, the key rotated there. grid:
// (n, Hkv * layers, B), D/2 threads: thread c owns the rotary pair (c, c + D/2).
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(D / 2) void tree_commit_kernel(EnTreeCommitArgs a)
{
    const int j = blockIdx.x, layer = blockIdx.y / a.Hkv, h = blockIdx.y - layer * a.Hkv, b = blockIdx.z;
    const int c = threadIdx.x;
    const int accepted = a.accepted[b], row = a.done[b] - accepted + j;
    const int node = a.path[(size_t)b * a.n + j];
    if (j >= accepted || (unsigned)node >= (unsigned)a.n || (unsigned)row >= (unsigned)a.Nq)
        return;
    const size_t pos = (size_t)a.hdr[4 * b + 1] + row;
    const size_t from = (((size_t)b * a.n + node) * a.Hkv + h) * D, slab = (size_t)b * a.Hkv + h;
    const T *kr = (const T *)a.k_rows[layer] + from, *vr = (const T *)a.v_rows[layer] + from;
    float y1, y2;
    rope_key_pair((float)kr[c], (float)kr[c + D / 2], a.cos_tab[pos * (D / 2) + c], a.sin_tab[pos * (D / 2) + c], y1, y2);
    T *kd = (T *)a.kc[layer] + (slab * a.T + pos) * D;
    kd[c] = (T)y1;
    kd[c + D / 2] = (T)y2;
    if constexpr (sizeof(T) == 4) {
        T *vd = (T *)a.vt[layer] + (slab * a.T + pos) * D;
        vd[c] = vr[c];
        vd[c + D / 2] = vr[c + D / 2];
    } else {
        // transposed layout [D][T], token j in column j with bits 2 and 3 exchanged
        T *vd = (T *)a.vt[layer] + slab * D * a.T + ((pos & ~(size_t)0xC) | ((pos & 4) << 1) | ((pos & 8) >> 1));
        vd[(size_t)c * a.T] = vr[c];
        vd[(size_t)(c + D / 2) * a.T] = vr[c + D / 2];
    }
}

int en_launch_tree_commit(const en_pool *pool, const EnTreeCommitArgs &a, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const int D = pool->d.head_dim;
    const dim3 grid(a.n, a.Hkv * a.layers, a.B), blk(D / 2);
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
