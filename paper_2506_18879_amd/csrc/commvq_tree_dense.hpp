// k_tree_decode and k_tree_dense: many rows over long contexts.  Included by commvq_tree.hip.
#pragma once

namespace {

constexpr int kDecodeWaves = 16;
constexpr int kDecodeThreads = 64 * kDecodeWaves;
constexpr int kDecodeSetTokens = 32 * kDecodeWaves;                  // tokens of a tile for each set of 32 of a wavefront: 64 fine positions x 8 coarse rows
constexpr int kDecodeMaxSets = 4;                                    // tiles of 2048 tokens, or of 1024 (two sets)
constexpr int kStageBytes = 64 * 1024;                               // 16 codebooks x 256 codewords x 8 elements
constexpr int kStepBytes = 32 * kD * 2;                              // 32 decoded keys (values)
// LDS behind the two stages: coarse phase factors of the tile (keys), or a set's values on their way to columns, 1 KiB a wavefront
constexpr int kAuxAt = 2 * kStageBytes;
constexpr int kDecodeLds = kAuxAt + (8 * kDecodeMaxSets + 1) * kJ * 8;
static_assert(kDecodeWaves * 1024 <= kDecodeLds - kAuxAt, "values' exchange fits");

// What one pass of the two kernels has: tiles tile0 .. tile0 + tiles - 1 of the batch's (sequence by sequence), decoded into
// keys / vals [tile][head][step][kStepBytes], seen [tile][head][step]: bit i, token i of the step counts.
struct DensePass {
    char *keys, *vals;
    unsigned *seen;
    floatx4_t *phases;   // explicit positions: [tile][step][slice][lane], E of the lane's two sub-spaces
    uint4_t *queries;    // [head][row tile of 16][k-step][lane], see turn_rows
    float *query_scales; // [head][row tile of 16][16], their powers of two
    int tiles_per_head;  // row tiles of a head, of all sequences
    int tile0, tiles;
    int sets, tile_tokens, steps;  // of a tile: sets of a wavefront, tokens, sets
    int turn_wgs, turn_tiles;  // workgroups of k_tree_decode that turn queries instead (first pass), row tiles of the largest tree
};

// where the row tiles of sequence b begin among those of a KV head
__host__ __device__ __forceinline__ int first_tile(int n0, int G, int b) { return n0 * G / 16 + b; }

// The sequence and the place in it of tile t of the batch, by one wavefront; false if there are not so many.  (A sequence without nodes has none:
// nothing reads its tiles, and a first node's position is not there.)
__device__ __forceinline__ bool find_tile(const TreeArgs &a, int tile_tokens, int t, int lane, int &b, int &at)
{
    if (a.batch == 1) {
        b = 0;
        at = t;
        const Span s = span_of(a, 0);
        return s.n > 0 && (long long)t * tile_tokens < s.L;
    }
    int before = 0;
    for (int c = 0; c < a.batch; c += 64) {
        const Span s = span_of(a, min(c + lane, a.batch - 1));
        const int own = c + lane < a.batch && s.n > 0 ? (s.L + tile_tokens - 1) / tile_tokens : 0;
        int incl = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(incl, d);
            if (lane >= d) incl += x;
        }
        const int first = before + incl - own;
        const unsigned long long hit = __ballot(t >= first && t < first + own);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            b = c + l;
            at = t - __builtin_amdgcn_readlane(first, l);
            return true;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

typedef __attribute__((address_space(3))) const uint4_t *tree_u4_ptr;
typedef __attribute__((address_space(3))) uint4_t *tree_u4_out;
typedef __attribute__((address_space(3))) const floatx4_t *tree_f4_ptr;
__device__ __forceinline__ void order() { asm volatile("" ::: "memory"); }

// element that lane 16 gk + n has in place e (of 4) of the operands of a pair of slices
__device__ __forceinline__ int slice_dim(int pair, int gk, int e) { return 16 * pair + 8 * (gk >> 1) + 4 * (gk & 1) + e; }

// Decodes the keys (turned) or values of a tile of 2048 (1024) tokens of one head into the operands of k_tree_dense.
// All codebooks of the head pass through LDS once per tile, 8 elements of 16 codebooks (64 KiB, a stage) at a time, in two buffers.
//
// Tokens.  A tile is 64 fine positions x 32 (16) coarse rows of 64; wavefront w has fine positions 4 w .. + 3 of all rows, in four (two) sets of 32 tokens:
// token n of a set's first (second) half is fine position n % 4, coarse row 8 set + n / 4 (+ 4).  A lane's tokens then are whole coarse rows apart
// and share the fine phase factor.  Per stage and set: the codes (registers for the whole tile) name 16-byte pieces in LDS, the matrix
// cores add them (selection operand and order of the codebooks as in k_score_stream: no bank conflicts, whatever the codes), a lane gets four
// elements of one token.  Keys: it turns its two sub-spaces; the wavefront's halves of two slices are exchanged, so that a lane has 4 elements of
// each half's token n, and leaves them four slices at a time.  Values: two slices of a set go through 1 KiB of LDS, written by token and read by columns (ds_read_b64_tr_b16).
// Times the head's power of two, rounded to fp16.
// Measured: a pass of 16 large tiles of 8 heads with 16 codebooks 50 us (32: 63 to 75), a workgroup a compute unit; without the stores (134 MB) 38, without
// the turn as well 31; LDS reads take 38 % of the cycles, vector instructions 32 %.
// EXPLICIT: positions from the pool, or of several axes; the phase factors are k_tree_phases' then.
template <int NB, int kSets, bool KEYS, bool EXPLICIT>
__device__ __forceinline__ void decode_tile(const TreeArgs &a, const DensePass &d, const char *src, int g, int tile)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int kTile = kSets * kDecodeSetTokens, kSteps = kSets * kDecodeWaves;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto send = [&](const char *from, int buf, int j) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     : : "s"((unsigned)(buf * kStageBytes + j * (kDecodeThreads * 16) + wave * 1024)), "v"((unsigned)tid * 16u), "s"(from + j * (kDecodeThreads * 16)));
    };
    constexpr int SENDS = kStageBytes / (kDecodeThreads * 16);       // 4 per thread and stage
#pragma unroll
    for (int j = 0; j < SENDS; ++j) send(src, 0, j);
    int b = 0, at = 0;
    if (!find_tile(a, d.tile_tokens, d.tile0 + tile, lane, b, at)) {                // (the same for the whole workgroup)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        return;
    }
    const Span s = span_of(a, b);
    const float scale = a.scales[2 * g + (KEYS ? 0 : 1)];
    const int n = lane & 15, gk = lane >> 4, par = gk & 1, second = gk >> 1;
    const int c0 = at * kTile;

    uint4_t sel;
    unsigned sidx;
    selection(lane, sel, sidx);
    const bf16x8_t selv = __builtin_bit_cast(bf16x8_t, sel);
    unsigned xreg[4], rsel = 0u;
#pragma unroll
    for (int st = 0; st < 4; ++st) xreg[st] = (unsigned)(8 * par + ((n + st + 4 * second) & 7)) * 16u | 1u << 24;
#pragma unroll
    for (int x = 0; x < 4; ++x) rsel |= (unsigned)((x + n + 4 * second) & 7) << (8 * x);

    // pages and codes of the lane's tokens, halves A and B of every set; of the codes bytes 8 par .. + 7 of every block of 16
    const int32_t *table = a.tables + (size_t)b * a.max_blocks;
    const int in_page = (1 << a.block_bits) - 1;
    const int tok0 = c0 + 4 * wave + (n & 3) + kLo * (n >> 2);
    unsigned long long seen[kSets];                                  // bit l: the token that lane l ends up with counts
    unsigned cc[kSets][2][NB];
    {
        int page[kSets][2];
#pragma unroll
        for (int ts = 0; ts < kSets; ++ts)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int tok = tok0 + kLo * (8 * ts + 4 * h);
                const int pg = table[min(tok, s.L - 1) >> a.block_bits];   // (no branches: all loads are asked for at once)
                page[ts][h] = tok < s.L && pg >= 0 && pg < a.n_blocks ? pg : -1;
            }
#pragma unroll
        for (int ts = 0; ts < kSets; ++ts) {
            const int own = page[ts][0] ^ ((page[ts][0] ^ page[ts][1]) & -second);   // (a selection would index the array by lane, in memory)
            seen[ts] = __ballot(own >= 0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // (a token that does not count takes the other half's codes: its pieces meet that token's in a matrix instruction, times zero)
                const bool stand_in = page[ts][h] < 0;
                const int tok = tok0 + kLo * (8 * ts + (stand_in ? 4 * (1 - h) : 4 * h)), pg = max(stand_in ? page[ts][1 - h] : page[ts][h], 0);
                const size_t rec = (((size_t)pg * a.Hkv + g) << a.block_bits) + (tok & in_page);
                const uint8_t *codes = (KEYS ? a.key_pages : a.val_pages) + rec * (16 * NB) + 8 * par;
#pragma unroll
                for (int k = 0; k < NB; ++k) {
                    const uint2_t c = *reinterpret_cast<const uint2_t *>(codes + 16 * k);
                    cc[ts][h][k] = __builtin_amdgcn_perm(c[1], c[0], rsel);
                }
            }
        }
    }
    const size_t step0 = ((size_t)tile * a.Hkv + g) * kSteps + wave * kSets;
    if (KEYS && lane == 0) {
#pragma unroll
        for (int ts = 0; ts < kSets; ++ts) d.seen[step0 + ts] = (unsigned)(seen[ts] & 0xffffu) | (unsigned)(seen[ts] >> 32 & 0xffffu) << 16;
    }

    // Phase factors of implicit positions: distances 64 H + lo from the first node; H's factors of the tile's rows wait in LDS, lo is the same for
    // all sets.
    const int t0 = KEYS && !EXPLICIT && a.turn ? a.node_pos[(size_t)s.n0 * a.n_axes] : 0;
    const int dist0 = c0 - t0, H0 = dist0 >> kLoBits;
    const int lane_dist = dist0 + 4 * wave + (n & 3) + kLo * (n >> 2) + 4 * kLo * second;
    const int lo = lane_dist & (kLo - 1);
    const unsigned hi_at = kAuxAt + (unsigned)((lane_dist >> kLoBits) - H0) * (kJ * 8) + par * 16;
    if (KEYS && !EXPLICIT) {
        for (int x = tid; x < (8 * kSets + 1) * kJ; x += kDecodeThreads) {
            const int H = H0 + x / kJ;
            float2 e = a.turn ? a.tbl_hi[(size_t)min((unsigned)(H < 0 ? -H : H), (unsigned)(a.n_hi - 1)) * kJ + (x & (kJ - 1))] : make_float2(1.f, 0.f);
            if (H < 0) e.y = -e.y;
            *reinterpret_cast<float2 *>(lds + kAuxAt + x * 8) = e;
        }
    }

    char *out = (KEYS ? d.keys : d.vals) + step0 * kStepBytes;
    const floatx4_t *phases = d.phases + ((size_t)tile * kSteps + wave * kSets) * 16 * 64 + lane;
    const unsigned wave_at = kAuxAt + (unsigned)wave * 1024u;
    constexpr int kAhead = 3;
    auto fine = [&](int sl) { return *reinterpret_cast<const floatx4_t *>(a.tbl_lo + (size_t)lo * kJ + 4 * sl + 2 * par); };
    constexpr bool FINE = KEYS && !EXPLICIT;
    floatx4_t e_next = {1.f, 0.f, 1.f, 0.f};
    if (FINE && a.turn) e_next = fine(0);
#pragma unroll 1
    for (int ks = 0; ks < 4; ++ks) {
        uint2_t kw[kSets], ka[kSets], kb[kSets];                     // (keys: of the first two slices, halves A and B)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int sl = 4 * ks + i;
            floatx4_t e_lo, e_hi, acc[kSets];
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) {
                const int buf = (NB * i + blk) & 1;
                // this stage's transfers have landed; the results of the last one, sent off after them, may still be on their way
                if (blk == 0 && ((i == 0 && ks > 0) || (i == 2 && !KEYS))) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(KEYS ? 2 * kSets : kSets) : "memory");
                else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                order();
                if (blk == 0) {
                    e_lo = e_next * scale;
                    asm volatile("" : "+v"(e_lo));
                    if (FINE && a.turn) e_next = fine((sl + 1) & 15);
                }
                // (behind the last stage the transfer is for nothing: one of 16, and no branch around every send)
                const char *next = src + (size_t)((NB * sl + blk + 1) & (16 * NB - 1)) * kStageBytes;
                // what is done with the sums of a pair of sets, in eight slots between the steps of the next one
                auto work = [&](int p, int slot) __attribute__((always_inline)) {
                    if (blk != NB - 1) return;
                    if constexpr (KEYS) {
                        if (EXPLICIT && (slot == 0 || slot == 3)) e_hi = phases[((2 * p + slot / 3) * 16 + sl) * 64];
                        if (!EXPLICIT && (slot == 0 || slot == 3)) e_hi = *reinterpret_cast<tree_f4_ptr>(hi_at + (unsigned)(8 * (2 * p + slot / 3) * kJ * 8 + sl * 32));
                        if (slot != 2 && slot != 5) return;
                        const int ts = 2 * p + slot / 5;
                        const floatx4_t z = acc[ts];
                        float w[4];
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            float ex, ey;
                            if constexpr (EXPLICIT) {
                                ex = e_hi[2 * u] * scale;
                                ey = e_hi[2 * u + 1] * scale;
                            } else {
                                ex = e_hi[2 * u] * e_lo[2 * u] - e_hi[2 * u + 1] * e_lo[2 * u + 1];
                                ey = e_hi[2 * u] * e_lo[2 * u + 1] + e_hi[2 * u + 1] * e_lo[2 * u];
                            }
                            w[2 * u] = z[2 * u] * ex + z[2 * u + 1] * ey;
                            w[2 * u + 1] = z[2 * u + 1] * ex - z[2 * u] * ey;
                        }
                        const uint2_t k = {pack_f16(w[0], w[1]), pack_f16(w[2], w[3])};
                        if (i % 2 == 0) {
                            kw[ts] = k;
                            return;
                        }
                        uint2_t xa, xb;                              // tokens of halves A and B
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            auto x = __builtin_amdgcn_permlane32_swap(kw[ts][r], k[r], false, false);
                            xa[r] = x[0];
                            xb[r] = x[1];
                        }
                        if (i == 1) {
                            ka[ts] = xa;
                            kb[ts] = xb;
                            return;
                        }
                        char *to = out + ts * kStepBytes + ks * 1024 + lane * 16;
                        *reinterpret_cast<uint4_t *>(to) = uint4_t{ka[ts][0], ka[ts][1], xa[0], xa[1]};
                        *reinterpret_cast<uint4_t *>(to + 4096) = uint4_t{kb[ts][0], kb[ts][1], xb[0], xb[1]};
                    } else {
                        if (slot != 1 && slot != 4) return;
                        const int ts = 2 * p + slot / 4;
                        const floatx4_t z = acc[ts] * scale;
                        uint2_t v = {pack_f16(z[0], z[1]), pack_f16(z[2], z[3])};
                        // (a weight of zero does not hide an infinity: tokens that do not count are cleared)
                        asm("v_cndmask_b32 %0, 0, %0, %1" : "+v"(v[0]) : "s"(seen[ts]));
                        asm("v_cndmask_b32 %0, 0, %0, %1" : "+v"(v[1]) : "s"(seen[ts]));
                        if (i % 2 == 0) {
                            kw[ts] = v;
                            return;
                        }
                        // by token: 16 bytes at 32 token + 16 par; back by columns: element slots 4 (lane / 16) ..
                        *reinterpret_cast<tree_u4_out>(wave_at + (unsigned)(n + 16 * second) * 32u + par * 16u) = uint4_t{kw[ts][0], kw[ts][1], v[0], v[1]};
                        order();
                        const unsigned from = wave_at + (unsigned)(4 * gk + n / 4) * 32u + 8u * (n & 3);
                        const uint2_t x0 = __builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(from)));
                        const uint2_t x1 = __builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(from + 512u)));
                        order();
                        *reinterpret_cast<uint4_t *>(out + ts * kStepBytes + (2 * ks + i / 2) * 1024 + lane * 16) = uint4_t{x0[0], x0[1], x1[0], x1[1]};
                    }
                };
                // The gather sums: steps of one read for each half of a set, sets two by two so that no matrix instruction waits for the one before
                // it, reads kAhead steps ahead.
                uint4_t v[kAhead][2];
                auto issue = [&](int x) __attribute__((always_inline)) {
                    const int ts = 2 * (x / 8) + (x & 1), st = x / 2 % 4;
                    const unsigned psel = 0x0c000000u | (unsigned)(2 + buf) << 16 | (unsigned)(4 + st) << 8;
#pragma unroll
                    for (int h = 0; h < 2; ++h) v[x % kAhead][h] = *reinterpret_cast<tree_u4_ptr>(__builtin_amdgcn_perm(cc[ts][h][blk], xreg[st], psel));
                };
#pragma unroll
                for (int ts = 0; ts < kSets; ++ts)                   // (opaque copies: addresses must not be kept from stage to stage, they would take all registers)
#pragma unroll
                    for (int h = 0; h < 2; ++h) asm volatile("" : "+v"(cc[ts][h][blk]));
#pragma unroll
                for (int x = 0; x < kAhead; ++x) issue(x);
#pragma unroll
                for (int x = 0; x < 4 * kSets; ++x) {
                    const int ts = 2 * (x / 8) + (x & 1);
                    const uint4_t pa = v[x % kAhead][0], pb = v[x % kAhead][1];
                    const uint8v_t both = {pa[0], pa[1], pa[2], pa[3], pb[0], pb[1], pb[2], pb[3]};
                    if (blk == 0 && x % 8 < 2) acc[ts] = floatx4_t{0.f, 0.f, 0.f, 0.f};
                    acc[ts] = __builtin_amdgcn_smfmac_f32_16x16x64_bf16(selv, __builtin_bit_cast(bf16x16_t, both), acc[ts], (int)sidx, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (x + kAhead < 4 * kSets) issue(x + kAhead);
                    __builtin_amdgcn_sched_barrier(0);
                    if (x < SENDS) send(next, buf ^ 1, x);           // (before this stage's results: see the wait above)
                    if (x >= 8) work(x / 8 - 1, x % 8);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int slot = 0; slot < 8; ++slot) work(kSets / 2 - 1, slot);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // the transfer behind the last stage has landed
}

// Queries of row tile id of the launch's [sequence][row tile][head], turned, times a power of two of the row and rounded to fp16, by a wavefront: the
// second operand of the logits, 8 elements of row lane % 16 in the order in which the decoded keys have them.
__device__ __forceinline__ void turn_rows(const TreeArgs &a, const DensePass &d, int id, int lane)
{
    const int g = id % a.Hkv;
    id /= a.Hkv;
    const int rt = id % d.turn_tiles, b = id / d.turn_tiles;
    if (b >= a.batch) return;
    const Span s = span_of(a, b);
    const int R = s.n * a.G;
    if (rt * 16 >= R) return;
    const int n = lane & 15, gk = lane >> 4, r = rt * 16 + n;
    const bool there = r < R;
    const int node = s.n0 + (there ? r / a.G : 0);
    const uint16_t *row = static_cast<const uint16_t *>(a.q) + (size_t)node * a.q_stride + (size_t)(g * a.G + r % a.G) * kD;
    const size_t tile = (size_t)g * d.tiles_per_head + first_tile(s.n0, a.G, b) + rt;
    unsigned raw[4][4];
    float top = 0.f;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            raw[ks][u] = *reinterpret_cast<const unsigned *>(row + slice_dim(2 * ks + u / 2, gk, 2 * (u & 1)));
            top = fmaxf(top, fmaxf(fabsf(bf16_lo(raw[ks][u])), fabsf(bf16_hi(raw[ks][u]))));
        }
    const float scale = half_scale(quads_max(top));
    if (gk == 0) d.query_scales[tile * 16 + n] = scale;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
        uint4_t w;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = slice_dim(2 * ks + u / 2, gk, 2 * (u & 1)) / 2, ax = axis_of(a, j);
            float2 z = make_float2(bf16_lo(raw[ks][u]) * scale, bf16_hi(raw[ks][u]) * scale);
            if (a.turn) z = times(z, turned_by(a, a.node_pos[(size_t)node * a.n_axes + ax] - a.node_pos[(size_t)s.n0 * a.n_axes + ax], j));
            w[u] = there ? pack_f16(z.x, z.y) : 0u;
        }
        d.queries[tile * 256 + 64 * ks + lane] = w;
    }
}

// Phase factors of the tokens of a pass's tiles, for all heads; a thread has the two sub-spaces that the lane of k_tree_decode turns.
__global__ __launch_bounds__(256) void k_tree_phases(const TreeArgs a, const DensePass d)
{
    const int step = blockIdx.x % d.steps, tile = blockIdx.x / d.steps, lane = threadIdx.x & 63;
    int b = 0, at = 0;
    if (!find_tile(a, d.tile_tokens, d.tile0 + tile, lane, b, at)) return;
    const Span s = span_of(a, b);
    const int n = lane & 15, par = lane >> 4 & 1, second = lane >> 5;
    const int tok = at * d.tile_tokens + 4 * (step / d.sets) + (n & 3) + kLo * (n >> 2) + kLo * (8 * (step % d.sets) + 4 * second);
    const int page = tok < s.L ? a.tables[(size_t)b * a.max_blocks + (tok >> a.block_bits)] : -1;
    const bool there = page >= 0 && page < a.n_blocks;
    const int32_t *own = a.key_pos && there ? a.key_pos + (((size_t)page << a.block_bits) + (tok & ((1 << a.block_bits) - 1))) * a.n_axes : nullptr;
    const int32_t *origin = a.node_pos + (size_t)s.n0 * a.n_axes;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int sl = 4 * k + (threadIdx.x >> 6);
        floatx4_t e;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int j = 4 * sl + 2 * par + u, ax = axis_of(a, j);
            const float2 c = turned_by(a, (own ? own[ax] : tok) - origin[ax], j);
            e[2 * u] = c.x;
            e[2 * u + 1] = -c.y;
        }
        d.phases[((size_t)blockIdx.x * 16 + sl) * 64 + lane] = e;
    }
}

// Workgroups: some that turn queries (first pass), then keys and values of every (tile, head); neighbours in the grid have different heads, so
// that with 8 of them an XCD's L2 serves one.
template <int NBK, int NBV, int SETS, bool EXPLICIT>
__global__ __launch_bounds__(kDecodeThreads) void k_tree_decode(const TreeArgs a, const DensePass d, const char *__restrict__ packed)
{
    int id = blockIdx.x;
    if (id < d.turn_wgs) {
        turn_rows(a, d, id * kDecodeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), threadIdx.x & 63);
        return;
    }
    id -= d.turn_wgs;
    const int g = id % a.Hkv;
    id /= a.Hkv;
    const int tile = id % d.tiles;
    if (id < d.tiles) decode_tile<NBK, SETS, true, EXPLICIT>(a, d, packed + (size_t)g * 16 * NBK * kStageBytes, g, tile);
    else decode_tile<NBV, SETS, false, false>(a, d, packed + (size_t)(a.Hkv * NBK + g * NBV) * 16 * kStageBytes, g, tile);
}

// ------------------------------------------------------------------ k_tree_dense
// Attention over decoded tiles: a workgroup has 32 steps of 32 tokens of one head, half of a large tile, and 32 WR rows, WR of its wavefronts different rows,
// 8 / WR of them different steps.  Operands need no exchange: logits = K Q^T with tokens as rows, whose weights are the operand of V^T P^T.
// With up to 64 rows they come from memory as they are (keys of the next step travel during the second product, values during the first); with more, four
// or eight wavefronts need the same step, which then goes from memory into one of three buffers in LDS, two rounds ahead.
// Parts of a sequence's tiles that are a whole pass apart are added up where the first of them left its own.
// Measured: a pass of 134 MB of decoded tiles: 27 us with up to 32 rows, 37 with 128, 12 of which are start and end: the rest is 5.5 TB/s out of the
// last-level cache.  256 rows: 52, by exponentials and matrix instructions.
constexpr int kDenseWaves = 8;
constexpr int kDenseRows = 2;                                        // row tiles of a wavefront
constexpr int kDenseSteps = 32;
constexpr int kDenseBuffers = 3;
constexpr int kMeet = 36;                                            // floats of a lane's row tile on its way to another wavefront: 32 sums, maximum, sum
constexpr bool dense_shared(int wr) { return wr >= 4; }
constexpr int dense_lds(int wr)
{
    const int meet = wr < 8 ? wr * kDenseRows * 64 * kMeet * 4 : 0, steps = dense_shared(wr) ? kDenseBuffers * (kDenseWaves / wr) * 2 * kStepBytes : 0;
    return meet > steps ? meet : steps;
}
template <int WR>
__global__ __launch_bounds__(64 * kDenseWaves) void k_tree_dense(const TreeArgs a, const DensePass d)
{
    constexpr int WT = kDenseWaves / WR, RT = kDenseRows, STEPS = kDenseSteps;
    constexpr bool SHARED = dense_shared(WR);
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, gk = lane >> 4;
    int id = blockIdx.x;
    const int g = id % a.Hkv;
    id /= a.Hkv;
    const int halves = d.steps / STEPS, half = id % halves;
    id /= halves;
    const int tile = id % d.tiles, rt0 = id / d.tiles;
    const int wr = wave % WR, wt = wave / WR;
    const size_t step0 = ((size_t)tile * a.Hkv + g) * d.steps + half * STEPS;

    // SHARED: round i's steps WT i .. + WT - 1 into buffer i % 3, in pieces of 1 KiB; behind the last round it once more, for nothing
    constexpr int PIECES = WT * 2 * kStepBytes / 1024 / kDenseWaves; // of a wavefront and round
    auto send_round = [&](int i) __attribute__((always_inline)) {
        const int st = min(i, STEPS / WT - 1) * WT;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const int piece = k * kDenseWaves + wave, which = piece / (2 * kStepBytes / 1024), part = piece % (2 * kStepBytes / 1024);
            const char *from = (part < kStepBytes / 1024 ? d.keys : d.vals) + (step0 + st + which) * kStepBytes + part % (kStepBytes / 1024) * 1024;
            lds_dma16(from, (unsigned)lane * 16u, (unsigned)(i % kDenseBuffers * (WT * 2 * kStepBytes) + piece * 1024));
        }
    };
    if constexpr (SHARED) {                                          // (the scratch is there, whether the tile is or not)
        send_round(0);
        send_round(1);
    }
    int b = 0, at = 0;
    const bool found = find_tile(a, d.tile_tokens, d.tile0 + tile, lane, b, at);
    const Span s = span_of(a, b);
    const int R = s.n * a.G, rows0 = rt0 * WR * 16 * RT, r0 = rows0 + wr * 16 * RT;
    if (!found || rows0 >= R) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        return;
    }
    const int tiles16 = (R + 15) / 16;
    const float head_unit = a.scale2 / a.scales[2 * g], undo = 1.f / a.scales[2 * g + 1];   // of the logits (and of a row's), of the values
    float unit[RT];

    uint4_t qv[RT][4];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const size_t tile16 = (size_t)g * d.tiles_per_head + first_tile(s.n0, a.G, b) + min(r0 / 16 + rt, tiles16 - 1);
        const uint4_t *from = d.queries + tile16 * 256 + lane;
        unit[rt] = head_unit / d.query_scales[tile16 * 16 + n];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qv[rt][ks] = from[64 * ks];   // (rows past the last take the last tile's and are not written)
    }
    floatx4_t o[RT][8];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x) o[rt][x] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    }
    const char *kp = d.keys + step0 * kStepBytes + lane * 16, *vp = d.vals + step0 * kStepBytes + lane * 16;
    uint4_t kv[2][4];
    auto load_keys = [&](const char *from) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) kv[h][ks] = *reinterpret_cast<const uint4_t *>(from + h * 4096 + ks * 1024);
    };
    if constexpr (!SHARED) load_keys(kp + (size_t)wt * kStepBytes);
    unsigned seen = d.seen[step0 + wt];
    if constexpr (SHARED) {                                          // (from here on the transfers are all that is counted)
        asm volatile("" ::"v"(qv[0][0]), "v"(qv[RT - 1][3]), "v"(unit[0]), "v"(unit[RT - 1]), "s"(seen));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    for (int st = wt, round = 0; st < STEPS; st += WT, ++round) {
        uint4_t vv[8];
        if constexpr (SHARED) {
            if (round > 0) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(PIECES) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            send_round(round + 2);
            const char *step = lds + round % kDenseBuffers * (WT * 2 * kStepBytes) + wt * 2 * kStepBytes;
            load_keys(step + lane * 16);
#pragma unroll
            for (int x = 0; x < 8; ++x) vv[x] = *reinterpret_cast<const uint4_t *>(step + kStepBytes + x * 1024 + lane * 16);
        } else {
#pragma unroll
            for (int x = 0; x < 8; ++x) vv[x] = *reinterpret_cast<const uint4_t *>(vp + (size_t)st * kStepBytes + x * 1024);
            __builtin_amdgcn_sched_barrier(0);
        }
        floatx4_t sc[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) sc[rt][0] = sc[rt][1] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    sc[rt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, kv[h][ks]), __builtin_bit_cast(f16x8_t, qv[rt][ks]), sc[rt][h], 0, 0, 0);
            }
        const unsigned now_seen = seen;
        const int next = min(st + WT, STEPS - 1);                    // (behind the last step: once more, not used)
        if constexpr (!SHARED) {
            __builtin_amdgcn_sched_barrier(0);
            load_keys(kp + (size_t)next * kStepBytes);
        }
        seen = d.seen[step0 + next];
        if constexpr (!SHARED) __builtin_amdgcn_sched_barrier(0);
        if (now_seen != 0xffffffffu) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool counts = now_seen >> (16 * h + 4 * gk + i) & 1u;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) sc[rt][h][i] = counts ? sc[rt][h][i] : -INFINITY;
                }
        }
        uint4_t pv[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            // Weights are relative to a number that is raised, to 2^7 below the maximum, only when a logit is more than 2^15 above it: rarely after
            // the first steps.  They stay below fp16's 65504, and its smallest number is 2^-31 of the largest weight or less.
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[rt][h][i]);
            top *= unit[rt];
            if (__ballot(top > m[rt] + 15.f)) {
                const float now = fmaxf(m[rt], quads_max(top) - 7.f);
                const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[rt] - now);
                m[rt] = now;
                l[rt] *= f;
#pragma unroll
                for (int x = 0; x < 8; ++x) o[rt][x] *= f;
            }
            const float base = m[rt] == -INFINITY ? 0.f : m[rt];
            float w[8], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[rt][i / 4][i & 3], unit[rt], -base));
                sum += w[i];
            }
            l[rt] += sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) pv[rt][i] = pack_f16(w[2 * i], w[2 * i + 1]);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                o[rt][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, vv[x]), __builtin_bit_cast(f16x8_t, pv[rt]), o[rt][x], 0, 0, 0);
    }
    if constexpr (SHARED) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the transfers behind the last round have landed
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16);
        l[rt] += __shfl_xor(l[rt], 32);
#pragma unroll
        for (int x = 0; x < 8; ++x) o[rt][x] *= undo;
    }
    // where the rows' parts go; what a pass before has left there is asked for before the wavefronts meet
    float *to[RT];
    size_t part_row[RT];
    floatx4_t was[RT][8];
    float2 was_stat[RT];
    const bool again = at >= d.tiles;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = min(r0 + 16 * rt + n, R - 1);
        part_row[rt] = ((size_t)(s.n0 + r / a.G) * a.Hq + g * a.G + r % a.G) * a.splits + at % d.tiles * halves + half;
        to[rt] = a.part + part_row[rt] * kD + 8 * (gk & 1) + 4 * (gk >> 1);   // (slot 4 gk + i of slices 2 x, 2 x + 1: see decode_tile's columns)
        if (again && wt == 0) {
            was_stat[rt] = a.stat[part_row[rt]];
#pragma unroll
            for (int x = 0; x < 8; ++x) was[rt][x] = *reinterpret_cast<const floatx4_t *>(to[rt] + 16 * x);
        }
    }
    auto add = [&](int rt, float mo, float lo, auto other) __attribute__((always_inline)) {
        const float now = fmaxf(m[rt], mo), base = now == -INFINITY ? 0.f : now;
        const float fa = __builtin_amdgcn_exp2f(m[rt] - base), fb = __builtin_amdgcn_exp2f(mo - base);
        m[rt] = now;
        l[rt] = l[rt] * fa + lo * fb;
#pragma unroll
        for (int x = 0; x < 8; ++x) o[rt][x] = o[rt][x] * fa + other(x) * fb;
    };
    // the steps' wavefronts meet, one after the other, in LDS
    if constexpr (WT > 1) {
        float *meet = reinterpret_cast<float *>(lds);
        for (int w = 1; w < WT; ++w) {
            __syncthreads();
            if (wt == w) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    float *to = meet + ((wr * RT + rt) * 64 + lane) * kMeet;
#pragma unroll
                    for (int x = 0; x < 8; ++x) *reinterpret_cast<floatx4_t *>(to + 4 * x) = o[rt][x];
                    to[32] = m[rt];
                    to[33] = l[rt];
                }
            }
            __syncthreads();
            if (wt == 0) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float *from = meet + ((wr * RT + rt) * 64 + lane) * kMeet;
                    add(rt, from[32], from[33], [&](int x) { return *reinterpret_cast<const floatx4_t *>(from + 4 * x); });
                }
            }
        }
        if (wt) return;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + 16 * rt + n;
        if (r >= R) continue;
        if (again) add(rt, was_stat[rt].x, was_stat[rt].y, [&](int x) { return was[rt][x]; });
#pragma unroll
        for (int x = 0; x < 8; ++x) *reinterpret_cast<floatx4_t *>(to[rt] + 16 * x) = o[rt][x];
        if (gk == 0) a.stat[part_row[rt]] = make_float2(m[rt], l[rt]);
    }
}

}  // namespace
