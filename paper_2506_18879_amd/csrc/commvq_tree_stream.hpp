// k_tree_stream: few rows over long contexts, codebooks streamed through LDS.  Included by commvq_tree.hip.
#pragma once

namespace {

constexpr int kStreamWaves = 8;
constexpr int kStreamThreads = 64 * kStreamWaves;
constexpr int kStreamRows = 16;
constexpr int kStreamMaxSets = 8;                                    // sets of 32 tokens of a wavefront: 8, 4 or 2
constexpr int stream_tile(int sets) { return 32 * kStreamWaves * sets; }   // 64 fine positions x 4 coarse rows a set
constexpr int kStreamMaxTile = stream_tile(kStreamMaxSets);
// LDS behind the two stages.  Key stages: coarse phase factors of the tile [33 rows][64], row maxima [8 wavefronts][16], slots [set][wavefront][32];
// value stages, over the phase factors: per wavefront 1 KiB for one set's values on their way to columns, then for its sums of 16 elements [lane][4].
// All stages: the queries [pair of slices][lane][4 fp16].
constexpr int kMaxAt = kAuxAt + (kStreamMaxTile / kLo + 1) * kJ * 8;
constexpr int kSlotAt = kMaxAt + kStreamWaves * kStreamRows * 4;
constexpr int kQueryAt = kSlotAt + kStreamMaxTile * 4;
constexpr int kTreeLds = kQueryAt + 8 * 64 * 8;
static_assert(kTreeLds <= kLdsBytes && kStreamWaves * 1024 <= kMaxAt - kAuxAt, "fits a compute unit");

constexpr float kShift = 14.f;                                       // largest weight: 2^14

typedef __attribute__((address_space(3))) const uint2_t *tree_u2_ptr;
typedef __attribute__((address_space(3))) floatx4_t *tree_f4_out;

// The long form of k_tree_rows: a codeword row is not fetched through the L1 for every code, but all codebooks of a head pass
// through LDS, 8 elements of 16 codebooks (64 KiB, a stage) at a time, once per tile of 2048, 1024 or 512 tokens, in two buffers.
//
// Tokens.  A tile is 64 fine positions x 32 (16, 8) coarse rows of 64; wavefront w has fine positions 8 w .. + 7 of all rows, in eight (four, two) sets
// of 32 tokens: token n of a set's first (second) half is fine position n % 8, coarse row 4 set + n / 8 (+ 2).  A lane's tokens then are whole coarse rows
// apart and share the fine phase factor.
// Keys, per stage and set: the codes (registers for the whole tile) name 16-byte pieces in LDS, the matrix cores add them
// (selection operand as in k_score_stream, whose rule for the order of the codebooks keeps the reads free of bank conflicts), the lane turns its two
// sub-spaces, times the head's power of two, and rounds to fp16.  After two slices, an exchange of the wavefront's halves makes them the operand of
// logits (tokens as rows) += K Q^T (16x16x16: the faster 16x16x32 would keep four slices in registers).
// Softmax: the workgroup's maxima meet in LDS, so that all wavefronts' weights are relative to the same number; weights stay in
// registers as fp16 operands for all value stages (2^14 for the largest: below 65504, and the smallest number is 2^-38 of it).
// Values, per pair of slices: the sums of a set go through 1 KiB of LDS, written by token and read by columns
// (ds_read_b64_tr_b16), into sums for 16 elements += V^T P^T; these meet in LDS across the wavefronts and are added to the rows' parts
// in memory (the range's earlier tiles, scaled to the new maximum).
// Measured: 8 heads, 4 rows each, 128K tokens, 16 codebooks 156 us: two tiles of 32 stages a compute unit, 2.3 a stage.  Of its cycles the gather's LDS
// reads take 49 %, vector instructions 41 %, matrix instructions 22 %; the arrival of a stage's codebooks is hidden, the barrier at its end is not.
// NBK, NBV: stages of a slice of keys and of values (codebooks / 16).
template <int NBK, int NBV, int SETS>
__global__ __launch_bounds__(kStreamThreads) void k_tree_stream(const TreeArgs a, const char *__restrict__ packed)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int id = blockIdx.x;
    const int g = id % a.Hkv;
    id /= a.Hkv;
    const int split = id % a.splits, b = id / a.splits;
    const Span s = span_of(a, b);
    const int R = s.n * a.G, t_begin = split * a.split_len, t_end = min(s.L, t_begin + a.split_len);
    if (R < 1 || t_begin >= t_end) return;
    const int n = lane & 15, gk = lane >> 4, par = gk & 1, second = gk >> 1;
    const float scale = a.scales[2 * g], head_unit = a.scale2 / scale, val_scale = a.scales[2 * g + 1], undo = 1.f / val_scale;
    const int t0 = a.turn ? a.node_pos[(size_t)s.n0 * a.n_axes] : 0;

    const char *ksrc = packed + (size_t)g * 16 * NBK * kStageBytes;
    const char *vsrc = packed + (size_t)a.Hkv * 16 * NBK * kStageBytes + (size_t)g * 16 * NBV * kStageBytes;
    // (not a barrier to the compiler: it writes the buffer that nobody reads until the next stage begins, which is one)
    auto send = [&](const char *src, int buf, int j) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     : : "s"((unsigned)(buf * kStageBytes + j * (kStreamThreads * 16) + wave * 1024)), "v"((unsigned)tid * 16u), "s"(src + j * (kStreamThreads * 16)));
    };
    constexpr int kSets = SETS, kTile = stream_tile(SETS), kCoarse = kTile / kLo;
    constexpr int SENDS = kStageBytes / (kStreamThreads * 16);    // 8 per thread and stage
#pragma unroll
    for (int j = 0; j < SENDS; ++j) send(ksrc, 0, j);

    uint4_t sel;
    unsigned sidx;
    selection(lane, sel, sidx);
    const bf16x8_t selv = __builtin_bit_cast(bf16x8_t, sel);
    unsigned xreg[4], rsel = 0u;
#pragma unroll
    for (int st = 0; st < 4; ++st) xreg[st] = (unsigned)(8 * par + ((n + st + 4 * second) & 7)) * 16u | 1u << 24;
#pragma unroll
    for (int x = 0; x < 4; ++x) rsel |= (unsigned)((x + n + 4 * second) & 7) << (8 * x);

    const int32_t *table = a.tables + (size_t)b * a.max_blocks;
    const int in_page = (1 << a.block_bits) - 1;
    float m = -INFINITY, l = 0.f;
    // queries, turned, times a power of two and rounded to fp16: wavefront w those of pair of slices w, 4 elements of row n in the order of the keys
    float unit;                                               // of row n's logits
    {
        const bool there = n < R;
        const int node = s.n0 + (there ? n / a.G : 0);
        const int e = slice_dim(wave, gk, 0);
        const uint2_t raw = *reinterpret_cast<const uint2_t *>(static_cast<const uint16_t *>(a.q) + (size_t)node * a.q_stride + (size_t)(g * a.G + n % a.G) * kD + e);
        // (the power of two is the row's: the wavefronts' maxima meet)
        float *maxima = reinterpret_cast<float *>(lds + kMaxAt);
        const float top = quads_max(fmaxf(fmaxf(fabsf(bf16_lo(raw[0])), fabsf(bf16_hi(raw[0]))), fmaxf(fabsf(bf16_lo(raw[1])), fabsf(bf16_hi(raw[1])))));
        if (gk == 0) maxima[wave * 16 + n] = top;
        __syncthreads();
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < kStreamWaves; ++w) all = fmaxf(all, maxima[w * 16 + n]);
        const float q_scale = half_scale(all);
        unit = head_unit / q_scale;
        uint2_t w;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float2 z = make_float2(bf16_lo(raw[u]) * q_scale, bf16_hi(raw[u]) * q_scale);
            if (a.turn) z = times(z, turned_by(a, a.node_pos[(size_t)node * a.n_axes] - t0, e / 2 + u));
            w[u] = there ? pack_f16(z.x, z.y) : 0u;
        }
        *reinterpret_cast<uint2_t *>(lds + kQueryAt + (wave * 64 + lane) * 8) = w;
    }
    // the sums that this thread joins: two elements of row jl % 16, for 16 elements at a time
    const int jl = tid >> 1 & 63, qr = jl & 15;
    const bool joins = tid < 128 && qr < R;
    const size_t out_row = ((size_t)(s.n0 + (joins ? qr / a.G : 0)) * a.Hq + g * a.G + (joins ? qr % a.G : 0)) * a.splits + split;
    float *mine = a.part + out_row * kD + 8 * (jl >> 4 & 1) + 4 * (jl >> 5) + 2 * (tid & 1);
    float m_row = -INFINITY;

    for (int c0 = t_begin; c0 < t_end; c0 += kTile) {
        // (made anew in every tile: what depends on it would else be kept in registers, or spilled, through all of them)
        const int lane = fresh_lane(), n = lane & 15, gk = lane >> 4, par = gk & 1, second = gk >> 1;
        // slots and key codes of the lane's tokens, halves A and B of every set; of the codes bytes 8 par .. + 7 of every block of 16
        unsigned long long seen[kSets];                           // bits 0..15: half A, 32..47: half B
        unsigned cc[kSets][2][NBK > NBV ? NBK : NBV];
        const int tok0 = c0 + 8 * wave + (n & 7) + kLo * (n >> 3);
        auto code_of = [&](const uint8_t *pages, int NB, int at, int k) {
            const size_t rec = (((size_t)(at >> a.block_bits) * a.Hkv + g) << a.block_bits) + (at & in_page);
            const uint2_t c = *reinterpret_cast<const uint2_t *>(pages + rec * (16 * NB) + 16 * k + 8 * par);
            return __builtin_amdgcn_perm(c[1], c[0], rsel);
        };
        bool whole = true;
        {
            int page[kSets][2];
#pragma unroll
            for (int ts = 0; ts < kSets; ++ts)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int tok = tok0 + kLo * (4 * ts + 2 * h);
                    const int pg = table[min(tok, t_end - 1) >> a.block_bits];   // (no branches: all loads are asked for at once)
                    page[ts][h] = tok < t_end && pg >= 0 && pg < a.n_blocks ? pg : -1;
                }
#pragma unroll
            for (int ts = 0; ts < kSets; ++ts) {
                const int own = page[ts][0] ^ ((page[ts][0] ^ page[ts][1]) & -second);   // (a selection would index the array by lane, in memory)
                seen[ts] = __ballot(own >= 0);
                whole = whole && seen[ts] == ~0ull;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // (a token that does not count takes the other half's codes: its pieces meet that token's in a matrix instruction, times zero)
                    const bool stand_in = page[ts][h] < 0;
                    const int pg = max(stand_in ? page[ts][1 - h] : page[ts][h], 0);
                    const int at = (pg << a.block_bits) + ((tok0 + kLo * (4 * ts + (stand_in ? 2 * (1 - h) : 2 * h))) & in_page);
                    if (gk == 2 * h) *reinterpret_cast<int *>(lds + kSlotAt + ((ts * kStreamWaves + wave) * 32 + 16 * h + n) * 4) = at;
#pragma unroll
                    for (int k = 0; k < NBK; ++k) cc[ts][h][k] = code_of(a.key_pages, NBK, at, k);
                }
            }
        }
        // coarse phase factors of the tile's rows: distances 64 H + lo from the first node, H from the first token's on
        const int dist0 = c0 - t0, H0 = dist0 >> kLoBits;
        for (int x = tid; x < (kCoarse + 1) * kJ; x += kStreamThreads) {
            const int H = H0 + x / kJ;
            float2 e = a.turn ? a.tbl_hi[(size_t)min((unsigned)(H < 0 ? -H : H), (unsigned)(a.n_hi - 1)) * kJ + (x & (kJ - 1))] : make_float2(1.f, 0.f);
            if (H < 0) e.y = -e.y;
            *reinterpret_cast<float2 *>(lds + kAuxAt + x * 8) = e;
        }
        const int lane_dist = dist0 + 8 * wave + (n & 7) + kLo * (n >> 3) + 2 * kLo * second;
        const int lo = lane_dist & (kLo - 1);
        const unsigned hi_at = kAuxAt + (unsigned)((lane_dist >> kLoBits) - H0) * (kJ * 8) + par * 16;

        // The gather sums of a stage: steps of one read for each half of a set, sets two by two so that no matrix instruction waits for the one
        // before it, reads kAhead steps ahead.  send_part(j): the next stage's transfers; work(pair, slot): what is done with the sums of a pair, in
        // eight slots between the steps of the next one.
        constexpr int kAhead = 5;
        auto stage = [&](int blk, int buf, floatx4_t (&acc)[kSets], auto send_part, auto work) __attribute__((always_inline)) {
            uint4_t v[kAhead][2];
            auto issue = [&](int x) __attribute__((always_inline)) {
                const int ts = 2 * (x / 8) + (x & 1), st = x / 2 % 4;
                const unsigned psel = 0x0c000000u | (unsigned)(2 + buf) << 16 | (unsigned)(4 + st) << 8;
#pragma unroll
                for (int h = 0; h < 2; ++h) v[x % kAhead][h] = *reinterpret_cast<tree_u4_ptr>(__builtin_amdgcn_perm(cc[ts][h][blk], xreg[st], psel));
            };
#pragma unroll
            for (int ts = 0; ts < kSets; ++ts)                    // (opaque copies: addresses must not be kept from stage to stage, they would take all registers)
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
                if (x % (kSets / 2) == 0) send_part(x / (kSets / 2));
                if (x >= 8) work(x / 8 - 1, x % 8);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int slot = 0; slot < 8; ++slot) work(kSets / 2 - 1, slot);
        };
        auto stage_begin = [&]() {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            order();
        };

        floatx4_t sc[kSets][2];
#pragma unroll
        for (int ts = 0; ts < kSets; ++ts) sc[ts][0] = sc[ts][1] = floatx4_t{0.f, 0.f, 0.f, 0.f};

        // ---- keys
        auto fine = [&](int sl) { return *reinterpret_cast<const floatx4_t *>(a.tbl_lo + (size_t)lo * kJ + 4 * sl + 2 * par); };
        floatx4_t e_next = {1.f, 0.f, 1.f, 0.f};                  // a stage ahead
        if (a.turn) e_next = fine(0);
#pragma unroll 1
        for (int pr = 0; pr < 8; ++pr) {
            uint2_t kw[kSets], qv;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int sl = 2 * pr + i;
                floatx4_t acc[kSets], e_hi, e_lo;
#pragma unroll
                for (int blk = 0; blk < NBK; ++blk) {
                    const int buf = (NBK * i + blk) & 1;
                    stage_begin();
                    if (blk == 0) {
                        e_lo = e_next * scale;
                        asm volatile("" : "+v"(e_lo));            // (has arrived: the next stage's transfers are not to be waited for)
                        if (a.turn) e_next = fine((sl + 1) & 15);
                        if (i == 1) qv = *reinterpret_cast<tree_u2_ptr>(kQueryAt + (pr * 64 + lane) * 8);
                    }
                    const int next = NBK * sl + blk + 1;
                    const char *src = next < 16 * NBK ? ksrc + (size_t)next * kStageBytes : vsrc;
                    stage(blk, buf, acc, [&](int j) { send(src, buf ^ 1, j); },
                          [&](int p, int slot) __attribute__((always_inline)) {
                              if (blk != NBK - 1) return;
                              if (slot == 0 || slot == 3) e_hi = *reinterpret_cast<tree_f4_ptr>(hi_at + (unsigned)(4 * (2 * p + slot / 3) * kJ * 8 + sl * 32));
                              if (slot != 2 && slot != 5) return;
                              const int ts = 2 * p + slot / 5;
                              const floatx4_t z = acc[ts], eh = e_hi;
                              float w[4];
#pragma unroll
                              for (int u = 0; u < 2; ++u) {
                                  const float ex = eh[2 * u] * e_lo[2 * u] - eh[2 * u + 1] * e_lo[2 * u + 1];
                                  const float ey = eh[2 * u] * e_lo[2 * u + 1] + eh[2 * u + 1] * e_lo[2 * u];
                                  w[2 * u] = z[2 * u] * ex + z[2 * u + 1] * ey;
                                  w[2 * u + 1] = z[2 * u + 1] * ex - z[2 * u] * ey;
                              }
                              const uint2_t k = {pack_f16(w[0], w[1]), pack_f16(w[2], w[3])};
                              if (i == 0) {
                                  kw[ts] = k;
                                  return;
                              }
                              uint2_t ka, kb;                     // tokens of halves A and B as first operand
#pragma unroll
                              for (int r = 0; r < 2; ++r) {
                                  auto x = __builtin_amdgcn_permlane32_swap(kw[ts][r], k[r], false, false);
                                  ka[r] = x[0];
                                  kb[r] = x[1];
                              }
                              sc[ts][0] = __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4_t, ka), __builtin_bit_cast(f16x4_t, qv), sc[ts][0], 0, 0, 0);
                              sc[ts][1] = __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4_t, kb), __builtin_bit_cast(f16x4_t, qv), sc[ts][1], 0, 0, 0);
                          });
                }
            }
        }

        // value codes, from the slots that wait in LDS
#pragma unroll
        for (int ts = 0; ts < kSets; ++ts)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = *reinterpret_cast<const int *>(lds + kSlotAt + ((ts * kStreamWaves + wave) * 32 + 16 * h + n) * 4);
#pragma unroll
                for (int k = 0; k < NBV; ++k) cc[ts][h][k] = code_of(a.val_pages, NBV, at, k);
            }

        // ---- weights
        if (!whole) {
#pragma unroll
            for (int ts = 0; ts < kSets; ++ts) {
                const unsigned long long bits = seen[ts] >> (4 * gk);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[ts][h][i] = bits >> (32 * h + i) & 1 ? sc[ts][h][i] : -INFINITY;
            }
        }
        float *maxima = reinterpret_cast<float *>(lds + kMaxAt);
        {
            float top = -INFINITY;
#pragma unroll
            for (int ts = 0; ts < kSets; ++ts)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[ts][h][i]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (gk == 0) maxima[wave * 16 + n] = top * unit;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        order();
        uint4_t pv[kSets];
        {
            float now = m;
#pragma unroll
            for (int w = 0; w < kStreamWaves; ++w) now = fmaxf(now, maxima[w * 16 + n]);
            const float base = now == -INFINITY ? 0.f : now, ref = base - kShift;
            l *= __builtin_amdgcn_exp2f(m - base);
            m = now;
#pragma unroll
            for (int ts = 0; ts < kSets; ++ts)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[ts][h][i], unit, -ref));
                        l += w[i];
                    }
                    pv[ts][2 * h] = pack_f16(w[0], w[1]);
                    pv[ts][2 * h + 1] = pack_f16(w[2], w[3]);
                }
        }
        float old = 0.f;                                          // factor of the row's earlier tiles
        if (joins) {
            float now = m_row;
#pragma unroll
            for (int w = 0; w < kStreamWaves; ++w) now = fmaxf(now, maxima[w * 16 + qr]);
            old = __builtin_amdgcn_exp2f(m_row - (now == -INFINITY ? 0.f : now));
            m_row = now;
        }

        // ---- values
        const unsigned wave_at = kAuxAt + (unsigned)wave * 1024u;
        auto join = [&](int sp) __attribute__((always_inline)) {
            if (!joins) return;
            float2 t = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kStreamWaves; ++w) {
                const float2 x = *reinterpret_cast<const float2 *>(lds + kAuxAt + w * 1024 + jl * 16 + (tid & 1) * 8);
                t.x += x.x;
                t.y += x.y;
            }
            t.x *= undo;
            t.y *= undo;
            float2 *to = reinterpret_cast<float2 *>(mine + 16 * sp);
            if (c0 > t_begin) { const float2 was = *to; t.x += was.x * old; t.y += was.y * old; }
            *to = t;
        };
#pragma unroll 1
        for (int sp = 0; sp < 8; ++sp) {
            uint2_t vw[kSets];
            floatx4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                floatx4_t acc[kSets];
                uint4_t vv[2];
#pragma unroll
                for (int blk = 0; blk < NBV; ++blk) {
                    const int buf = (NBV * i + blk) & 1;
                    stage_begin();
                    const int next = NBV * (2 * sp + i) + blk + 1;
                    // (behind the last tile the transfer is for nothing: one in 64, and no branch around every send)
                    const char *src = next < 16 * NBV ? vsrc + (size_t)next * kStageBytes : ksrc;
                    if (i == 0 && blk == 0 && sp > 0) join(sp - 1);   // all wavefronts' sums of the pair before are there
                    stage(blk, buf, acc, [&](int j) { send(src, buf ^ 1, j); },
                          [&](int p, int slot) __attribute__((always_inline)) {
                              if (blk != NBV - 1) return;
                              if (slot == 1 || slot == 3) {
                                  const int y = slot == 3, ts = 2 * p + y;
                                  const floatx4_t z = acc[ts] * val_scale;
                                  uint2_t v = {pack_f16(z[0], z[1]), pack_f16(z[2], z[3])};
                                  // (a weight of zero does not hide an infinity: tokens that do not count are cleared)
                                  asm("v_cndmask_b32 %0, 0, %0, %1" : "+v"(v[0]) : "s"(seen[ts]));
                                  asm("v_cndmask_b32 %0, 0, %0, %1" : "+v"(v[1]) : "s"(seen[ts]));
                                  if (i == 0) {
                                      vw[ts] = v;
                                      return;
                                  }
                                  // by token: 16 bytes at 32 token + 16 par; back by columns: element slots 4 (lane / 16) ..
                                  *reinterpret_cast<tree_u4_out>(wave_at + (unsigned)(n + 16 * second) * 32u + par * 16u) = uint4_t{vw[ts][0], vw[ts][1], v[0], v[1]};
                                  order();
                                  const unsigned at = wave_at + (unsigned)(4 * gk + n / 4) * 32u + 8u * (n & 3);
                                  const uint2_t x0 = __builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(at)));
                                  const uint2_t x1 = __builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(at + 512u)));
                                  order();
                                  vv[y] = uint4_t{x0[0], x0[1], x1[0], x1[1]};
                              }
                              if (i == 1 && (slot == 4 || slot == 6)) {
                                  const int y = slot == 6, ts = 2 * p + y;
                                  o = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, vv[y]), __builtin_bit_cast(f16x8_t, pv[ts]), o, 0, 0, 0);
                              }
                          });
                }
            }
            order();
            *reinterpret_cast<tree_f4_out>(wave_at + lane * 16) = o;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        order();
        join(7);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                             // the next tile's coarse factors go where the sums were
        order();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");              // the transfers behind the last tile have landed
    // sums of the weights: lanes, then wavefronts
    float *sums = reinterpret_cast<float *>(lds + kMaxAt);
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (gk == 0) sums[wave * 16 + n] = l;
    __syncthreads();
    if (joins && (tid & 1) == 0 && jl < 16) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kStreamWaves; ++w) t += sums[w * 16 + qr];
        a.stat[out_row] = make_float2(m_row - kShift, t);
    }
}

}  // namespace
